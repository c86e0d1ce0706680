"""Every tile shape of the products, whole and in pieces, at sizes that choose it (marker gpu).

The reference is in 64 bits on the GPU, from packed values that other tests compare with the oracle's;
a second one checks that small whole numbers come out exactly."""
import numpy as np
import pytest

from layer_helpers import TYPES, torch_type

pytestmark = pytest.mark.gpu

# (rows, n_in, n_out): the large tile with and without ends in every direction, pieces of long sums in
# the large, the middle and the flat tile, more than one round of each
FORWARD = [(4096, 512, 4096), (4097, 300, 4100), (2050, 1000, 8192), (33, 16384, 256), (64, 4096, 4096), (700, 2000, 1500), (100, 257, 9000)]
INPUT = [(4096, 4096, 512), (4099, 4100, 264), (8200, 2056, 72), (300, 256, 8192), (40, 4096, 2048), (2048, 4096, 1000), (16, 520, 5000)]
WEIGHT = [(512, 4096, 4096), (200, 4100, 4104), (70, 2056, 8200), (9000, 256, 250), (16390, 520, 300), (33, 3000, 2000), (2048, 1030, 700)]


@pytest.fixture(scope="module")
def pp():
    from paper_2204_10562_amd import layer
    return layer


def values(pp, fmt, pair, cols):
    """A packed matrix's values, which 32 bits hold."""
    import torch
    out = torch.empty(pair[0].shape[0], cols, device="cuda")
    pp.pp_unpack(fmt, pair, out)
    return out.double()


def close(got, want, bound, t):
    """As layer_helpers.assert_within, on the GPU; bound: a matrix that is used up."""
    import torch
    eps = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[t]
    bound += eps * (want.abs() + bound) + 2.0 ** -25
    far = ~((got.double() - want).abs() <= bound)
    assert not far.any(), (int(far.sum()), torch.nonzero(far)[:4].tolist(), got[far][:4].tolist(), want[far][:4].tolist())


def sum_bound(a, b, n):
    """n products added in 32 bits in any order, each addition off by a unit of the last place at most; in practice they grow with the root of n."""
    return (a.abs() @ b.abs()) * ((n + 8) * 2.0 ** -23)


def workspace(pp, call, t, rows, n_in, n_out):
    import torch
    return torch.full((pp.pp_linear_workspace_bytes(call, torch_type(t), rows, n_in, n_out),), 255, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("t", TYPES)
def test_forward(pp, t):
    import torch
    g = torch.Generator(device="cuda").manual_seed(31)
    for rows, n_in, n_out in FORWARD:
        print("[case] forward", t, rows, n_in, n_out, flush=True)
        x = torch.randn(rows, n_in, generator=g, device="cuda").to(torch_type(t))
        w, x4 = pp.empty_packed(1, n_out, n_in), pp.empty_packed(1, rows, n_in)
        pp.pp_pack(1, torch.randn(n_out, n_in, generator=g, device="cuda"), w)
        pp.pp_pack(1, x, x4)
        b = torch.randn(n_out, generator=g, device="cuda")
        y, kept, again = torch.empty(rows, n_out, dtype=x.dtype, device="cuda"), pp.empty_packed(0, rows, n_in), pp.empty_packed(0, rows, n_in)
        pp.pp_linear_forward(x, w, b, y, kept, workspace(pp, 0, t, rows, n_in, n_out))
        xv, wv = values(pp, 1, x4, n_in), values(pp, 1, w, n_in).t().contiguous()
        want = xv @ wv + b.double()
        close(y, want, sum_bound(xv, wv, n_in) + 2.0 ** -22 * want.abs(), t)
        pp.pp_pack(0, x, again)
        assert torch.equal(kept[0], again[0]) and torch.equal(kept[1], again[1])


@pytest.mark.parametrize("t", TYPES)
def test_backward_input(pp, t):
    import torch
    g = torch.Generator(device="cuda").manual_seed(32)
    for rows, n_in, n_out in INPUT:
        print("[case] backward_input", t, rows, n_in, n_out, flush=True)
        dy = torch.randn(rows, n_out, generator=g, device="cuda").to(torch_type(t))
        w = pp.empty_packed(1, n_out, n_in)
        pp.pp_pack(1, torch.randn(n_out, n_in, generator=g, device="cuda"), w)
        dx = torch.empty(rows, n_in, dtype=dy.dtype, device="cuda")
        pp.pp_linear_backward_input(dy, w, dx, workspace(pp, 1, t, rows, n_in, n_out))
        wv = values(pp, 1, w, n_in)
        close(dx, dy.double() @ wv, sum_bound(dy.double(), wv, n_out), t)


@pytest.mark.parametrize("t", TYPES)
def test_backward_weight(pp, t):
    import torch
    g = torch.Generator(device="cuda").manual_seed(33)
    for rows, n_in, n_out in WEIGHT:
        print("[case] backward_weight", t, rows, n_in, n_out, flush=True)
        dy = torch.randn(rows, n_out, generator=g, device="cuda").to(torch_type(t))
        kept = pp.empty_packed(0, rows, n_in)
        pp.pp_pack(0, torch.randn(rows, n_in, generator=g, device="cuda"), kept)
        dw_in = torch.randn(n_out, n_in, generator=g, device="cuda")
        dw, db = torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
        pp.pp_linear_backward_weight(dy, kept, dw_in, dw, db, workspace(pp, 2, t, rows, n_in, n_out))
        d, xv = dy.double().t().contiguous(), values(pp, 0, kept, n_in)
        want = d @ xv + dw_in.double()
        close(dw, want, sum_bound(d, xv, rows) + 2.0 ** -22 * (want.abs() + dw_in.double().abs()), "f32")
        close(db, d.sum(1), d.abs().sum(1) * ((rows + 8) * 2.0 ** -23), "f32")


@pytest.mark.parametrize("t", TYPES)
def test_exact_sums(pp, t):
    """Small whole numbers: every product and sum is exact, whatever the order and the tile."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(34)

    def whole(rows, cols, most):
        return torch.randint(-most, most + 1, (rows, cols), generator=g, device="cuda").float()
    for rows, n_in, n_out in FORWARD + INPUT + WEIGHT:
        print("[case] exact", t, rows, n_in, n_out, flush=True)
        x, w = whole(rows, n_in, 4), whole(n_out, n_in, 4)
        x[:, ::32] = 4.0
        w[:, ::32] = 4.0
        dy = whole(rows, n_out, 2).to(torch_type(t))
        wp, xp = pp.empty_packed(1, n_out, n_in), pp.empty_packed(0, rows, n_in)
        pp.pp_pack(1, w, wp)
        y = torch.empty(rows, n_out, device="cuda")
        pp.pp_linear_forward(x, wp, None, y, xp, workspace(pp, 0, "f32", rows, n_in, n_out))
        assert torch.equal(y.double(), x.double() @ w.double().t().contiguous())
        dx = torch.empty(rows, n_in, dtype=dy.dtype, device="cuda")
        pp.pp_linear_backward_input(dy, wp, dx, workspace(pp, 1, t, rows, n_in, n_out))
        assert torch.equal(dx, (dy.double() @ w.double()).to(dy.dtype))
        dw, db = torch.empty(n_out, n_in, device="cuda"), torch.empty(n_out, device="cuda")
        pp.pp_linear_backward_weight(dy, xp, None, dw, db, workspace(pp, 2, t, rows, n_in, n_out))
        d = dy.double().t().contiguous()
        assert torch.equal(dw.double(), d @ x.double()) and torch.equal(db.double(), d.sum(1))


def test_gradients_against_differences(pp):
    """The loss sum(dy * y) moves with a weight of a row by what dw says and with an input by what dx says: y is
    linear in both where their packed values are exact."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(35)
    rows, n_in, n_out = 70, 256, 200
    x = torch.randint(-4, 5, (rows, n_in), generator=g, device="cuda").float()
    x[:, ::32] = 4.0
    wv = torch.randint(-2, 3, (n_out, n_in), generator=g, device="cuda").float()
    wv[:, ::32] = 4.0
    dy = torch.randint(-3, 4, (rows, n_out), generator=g, device="cuda").float()

    def loss(x_, w_):
        w, y = pp.empty_packed(1, n_out, n_in), torch.empty(rows, n_out, device="cuda")
        pp.pp_pack(1, w_, w)
        pp.pp_linear_forward(x_, w, None, y, None, workspace(pp, 0, "f32", rows, n_in, n_out))
        return float((y.double() * dy.double()).sum())
    w, kept = pp.empty_packed(1, n_out, n_in), pp.empty_packed(0, rows, n_in)
    pp.pp_pack(1, wv, w)
    pp.pp_pack(0, x, kept)
    dx, dw = torch.empty(rows, n_in, device="cuda"), torch.empty(n_out, n_in, device="cuda")
    pp.pp_linear_backward_input(dy, w, dx, workspace(pp, 1, "f32", rows, n_in, n_out))
    pp.pp_linear_backward_weight(dy, kept, None, dw, None, workspace(pp, 2, "f32", rows, n_in, n_out))
    at = loss(x, wv)
    for i, j in [(0, 1), (199, 255), (64, 33), (131, 200)]:
        moved = wv.clone()
        moved[i, j] = 3.0 if moved[i, j] != 3.0 else 2.0
        assert loss(x, moved) - at == float(dw[i, j]) * float(moved[i, j] - wv[i, j])
    for i, j in [(0, 1), (69, 255), (33, 129), (64, 31)]:
        moved = x.clone()
        moved[i, j] = 3.0 if moved[i, j] != 3.0 else 2.0
        assert loss(moved, wv) - at == float(dx[i, j]) * float(moved[i, j] - x[i, j])


def test_sums_of_rows_far_apart(pp):
    """Rows so far apart that their offsets pass 32 bits, in every operand."""
    import torch
    ld, rows, n = 1 << 22, 600, 96     # 600 rows of 8 MiB: 4.9 GB
    g = torch.Generator(device="cuda").manual_seed(36)
    room = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda").view(rows, ld)
    x = room[:, 128:128 + n]
    x.copy_(torch.randint(-4, 5, (rows, n), generator=g, device="cuda"))
    x[:, ::32] = 4.0
    wv = torch.randint(-4, 5, (n, n), generator=g, device="cuda").float()
    wv[:, ::32] = 4.0
    w, kept = pp.empty_packed(1, n, n), pp.empty_packed(0, rows, n)
    pp.pp_pack(1, wv, w)
    y = room[:, 4096:4096 + n]
    pp.pp_linear_forward(x, w, None, y, kept, workspace(pp, 0, "bf16", rows, n, n))
    want = (x.double() @ wv.double().t().contiguous())
    assert torch.equal(y, want.bfloat16())
    dx = room[:, 8192:8192 + n]
    pp.pp_linear_backward_input(x, w, dx, workspace(pp, 1, "bf16", rows, n, n))
    assert torch.equal(dx, (x.double() @ wv.double()).bfloat16())
    dw = torch.empty(n, n, device="cuda")
    pp.pp_linear_backward_weight(x, kept, None, dw, None, workspace(pp, 2, "bf16", rows, n, n))
    assert torch.equal(dw.double(), x.double().t().contiguous() @ x.double())
