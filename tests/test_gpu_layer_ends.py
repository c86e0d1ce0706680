"""Nothing is read behind an operand's last value (marker gpu)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows, n_in, n_out, ld", [(70, 96, 71, 72), (300, 130, 257, 264), (1, 64, 33, 33), (65, 40, 1, 8)])
def test_odd_rows_of_gradients_are_copied_first(rows, n_in, n_out, ld):
    """Loads are of whole words, so an odd row's last one would reach behind the matrix: dw reads such rows of dy from a copy in the
    workspace whose rows are padded with zeros, although they lie at multiples of 16 bytes."""
    import torch
    from paper_2204_10562_amd import layer as pp
    g = torch.Generator(device="cuda").manual_seed(91)
    room = torch.full((rows, ld), float("nan"), dtype=torch.bfloat16, device="cuda")
    dy = room[:, :n_out]
    dy.copy_(torch.randint(-3, 4, (rows, n_out), generator=g, device="cuda"))
    x = torch.randint(-4, 5, (rows, n_in), generator=g, device="cuda").float()
    x[:, ::32] = 4.0
    kept = pp.empty_packed(pp.PP_PACK_INT8, rows, n_in)
    pp.pp_pack(pp.PP_PACK_INT8, x, kept)
    ws = torch.full((pp.pp_linear_workspace_bytes(pp.PP_LINEAR_BACKWARD_WEIGHT, torch.bfloat16, rows, n_in, n_out),), 255, dtype=torch.uint8, device="cuda")
    dw, db = torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
    pp.pp_linear_backward_weight(dy, kept, None, dw, db, ws)
    d = dy.double().t().contiguous()
    assert torch.equal(dw.double(), d @ x.double()) and torch.equal(db.double(), d.sum(1))
    padded = -(-n_out // 8) * 8
    copy = ws[:rows * padded * 2].view(torch.bfloat16).view(rows, padded)
    assert torch.equal(copy[:, :n_out], dy) and not copy[:, n_out:].any()
