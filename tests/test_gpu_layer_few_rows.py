"""The forward product of few rows on both sides of where one way takes over from another (marker gpu)."""
import pytest

from layer_helpers import TYPES, torch_type
from test_gpu_layer_tiles import close, sum_bound, values, workspace

pytestmark = pytest.mark.gpu

# rows that pack x in place or not (64 groups of 128 values), one or two blocks of 16, small weights and large ones
CASES = [(1, 8192, 40), (1, 8193, 40), (2, 4096, 100), (2, 4100, 100), (16, 512, 33), (16, 520, 33), (15, 640, 257), (17, 512, 2000), (31, 300, 4099),
         (32, 4096, 4096), (33, 4096, 512), (32, 4096, 8192), (32, 4096, 8200), (17, 8300, 4100), (5, 20000, 17), (30, 16500, 65), (1, 100, 40000)]


@pytest.fixture(scope="module")
def pp():
    from paper_2204_10562_amd import layer
    return layer


@pytest.mark.parametrize("t", TYPES)
def test_few_rows(pp, t):
    import torch
    g = torch.Generator(device="cuda").manual_seed(71)
    for i, (rows, n_in, n_out) in enumerate(CASES):
        print("[case] few rows", t, rows, n_in, n_out, flush=True)
        room = torch.full((rows, n_in + 3), float("nan"), dtype=torch_type(t), device="cuda")
        x = room[:, :n_in]
        x.copy_(torch.randn(rows, n_in, generator=g, device="cuda"))
        w, x4, kept, again = pp.empty_packed(1, n_out, n_in), pp.empty_packed(1, rows, n_in), pp.empty_packed(0, rows, n_in), pp.empty_packed(0, rows, n_in)
        pp.pp_pack(1, torch.randn(n_out, n_in, generator=g, device="cuda"), w)
        pp.pp_pack(1, x, x4)
        pp.pp_pack(0, x, again)
        b = torch.randn(n_out, generator=g, device="cuda") if i % 2 else None
        out = torch.full((rows, n_out + 5), 77.0, dtype=x.dtype, device="cuda")
        pp.pp_linear_forward(x, w, b, out[:, :n_out], kept, workspace(pp, 0, t, rows, n_in, n_out))
        xv, wv = values(pp, 1, x4, n_in), values(pp, 1, w, n_in).t().contiguous()
        want = xv @ wv
        if b is not None:
            want += b.double()
        close(out[:, :n_out], want, sum_bound(xv, wv, n_in) + 2.0 ** -22 * want.abs(), t)
        assert (out[:, n_out:] == 77).all()
        assert torch.equal(kept[0], again[0]) and torch.equal(kept[1], again[1])


@pytest.mark.parametrize("rows, n_in, n_out", [(3, 300, 50), (16, 1000, 70), (20, 600, 100), (32, 4096, 8200)])
def test_missing_values_stay_in_their_row_and_column(pp, rows, n_in, n_out):
    import torch
    g = torch.Generator(device="cuda").manual_seed(72)
    x, wv = torch.randn(rows, n_in, generator=g, device="cuda"), torch.randn(n_out, n_in, generator=g, device="cuda")
    x[rows - 1, n_in - 1] = float("inf")
    wv[7, 5] = float("nan")
    w, y = pp.empty_packed(1, n_out, n_in), torch.empty(rows, n_out, device="cuda")
    pp.pp_pack(1, wv, w)
    pp.pp_linear_forward(x, w, None, y, None, workspace(pp, 0, "f32", rows, n_in, n_out))
    lost = torch.zeros(rows, n_out, dtype=torch.bool, device="cuda")
    lost[rows - 1] = True
    lost[:, 7] = True
    assert torch.equal(y.isnan(), lost)
