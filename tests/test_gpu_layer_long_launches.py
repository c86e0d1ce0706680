"""Rows and features so many that a call takes more than one launch of a kernel (marker gpu)."""
import pytest

pytestmark = pytest.mark.gpu

ROWS = (1 << 27) + 77     # 2^31 threads of packing are 2^27 rows of one group, 2^20 tiles of 128 rows as well
AT = [0, (1 << 26) - 9, (1 << 27) - 2048, ROWS - 2000]


@pytest.fixture(scope="module")
def pp():
    import torch
    from paper_2204_10562_amd import layer
    yield layer
    torch.cuda.empty_cache()


def whole(rows, cols, most, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, (rows, cols), generator=g, device="cuda", dtype=torch.int8).bfloat16()


def test_pack_and_activations(pp):
    import torch
    print("[case] pack, act", ROWS, flush=True)
    x = whole(ROWS, 2, 60, 1)
    x4, out = pp.empty_packed(pp.PP_PACK_FP4, ROWS, 2), torch.full_like(x, float("nan"))
    pp.pp_pack(pp.PP_PACK_FP4, x, x4)
    pp.pp_unpack(pp.PP_PACK_FP4, x4, out)
    assert not out.isnan().any()
    for r in AT:
        part, want = pp.empty_packed(pp.PP_PACK_FP4, 2000, 2), torch.empty(2000, 2, dtype=x.dtype, device="cuda")
        pp.pp_pack(pp.PP_PACK_FP4, x[r:r + 2000], part)
        pp.pp_unpack(pp.PP_PACK_FP4, part, want)
        assert torch.equal(out[r:r + 2000], want) and torch.equal(x4[0][r:r + 2000], part[0]) and torch.equal(x4[1][r:r + 2000], part[1])
    del x4
    x8 = pp.empty_packed(pp.PP_PACK_INT8, ROWS, 2)
    pp.pp_act_forward(pp.PP_ACT_SILU, x, None, out, x8)
    back = torch.full_like(x, float("nan"))
    pp.pp_act_backward(pp.PP_ACT_SILU, out, x8, None, back)
    assert not out.isnan().any() and not back.isnan().any()
    for r in AT:
        part, y, d = pp.empty_packed(pp.PP_PACK_INT8, 2000, 2), torch.empty(2000, 2, dtype=x.dtype, device="cuda"), torch.empty(2000, 2, dtype=x.dtype, device="cuda")
        pp.pp_act_forward(pp.PP_ACT_SILU, x[r:r + 2000], None, y, part)
        pp.pp_act_backward(pp.PP_ACT_SILU, y, part, None, d)
        assert torch.equal(out[r:r + 2000], y) and torch.equal(back[r:r + 2000], d)
        assert torch.equal(x8[0][r:r + 2000], part[0]) and torch.equal(x8[1][r:r + 2000], part[1])


def test_forward_and_input_gradient(pp):
    import torch
    print("[case] forward, backward_input", ROWS, flush=True)
    n_in, n_out = 2, 8
    x, dy = whole(ROWS, n_in, 4, 2), whole(ROWS, n_out, 3, 3)
    x[:, 0] = 4
    wv = whole(n_out, n_in, 4, 4).float()
    wv[:, 0] = 4
    w = pp.empty_packed(pp.PP_PACK_FP4, n_out, n_in)
    pp.pp_pack(pp.PP_PACK_FP4, wv, w)
    y, dx = torch.full((ROWS, n_out), float("nan"), dtype=x.dtype, device="cuda"), torch.full((ROWS, n_in), float("nan"), dtype=x.dtype, device="cuda")
    ws = torch.empty(max(pp.pp_linear_workspace_bytes(c, x.dtype, ROWS, n_in, n_out) for c in (0, 1)), dtype=torch.uint8, device="cuda")
    pp.pp_linear_forward(x, w, None, y, None, ws)
    pp.pp_linear_backward_input(dy, w, dx, ws)
    assert not y.isnan().any() and not dx.isnan().any()
    for r in AT:
        assert torch.equal(y[r:r + 2000], (x[r:r + 2000].double() @ wv.double().t().contiguous()).to(y.dtype))
        assert torch.equal(dx[r:r + 2000], (dy[r:r + 2000].double() @ wv.double()).to(dx.dtype))


def test_weight_gradient(pp):
    """33 x 32768 tiles of 128 x 128; dw is 69 GB."""
    import torch
    n_in, n_out = 4100, 1 << 22
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GiB of the GPU's memory")
    print("[case] backward_weight", n_in, n_out, flush=True)
    x, dy = whole(1, n_in, 4, 5), whole(1, n_out, 3, 6)
    x[:, ::32] = 4
    kept = pp.empty_packed(pp.PP_PACK_INT8, 1, n_in)
    pp.pp_pack(pp.PP_PACK_INT8, x, kept)
    dw, db = torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
    dw[:, -1] = float("nan")
    ws = torch.empty(pp.pp_linear_workspace_bytes(pp.PP_LINEAR_BACKWARD_WEIGHT, x.dtype, 1, n_in, n_out), dtype=torch.uint8, device="cuda")
    pp.pp_linear_backward_weight(dy, kept, None, dw, db, ws)
    assert torch.equal(db, dy[0].float()) and torch.equal(dw[:, -1], dy[0].float() * x[0, -1].float())
    first = (1 << 20) // 33 * 128        # rows of the first launch
    for r in (0, first - 1000, n_out - 2000):
        assert torch.equal(dw[r:r + 2000], dy[0, r:r + 2000, None].float() * x.float())
