"""Every tile of the linear layer's products, whole and divided, even and with ends, over long sums (marker gpu).

The sizes are those of layer_sizes.py.  The reference is in 64 bits on the GPU, from packed values that other tests compare with the
oracle's.  Random values show wrong places and waits; that nothing of a gradient is lost on the way shows in two ways: a single value of
the sum with all the digits of its type has to come out exactly, and the errors of random sums have to be as small on average as those
of 32-bit additions."""
import pytest

from layer_helpers import TYPES, torch_type
from layer_sizes import cases
from layer_plans import FORWARD, INPUT, WEIGHT
from test_gpu_layer_tiles import close, sum_bound, values, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pp():
    from paper_2204_10562_amd import layer
    return layer


def ids(case):
    return "-".join(str(v) for v in case).replace(" ", "")


def small_on_average(got, want, n):
    """Root mean squares.  n values of 24 bits are at most 3 n / 16 additions in 32 bits (three planes, sixteen products to an addition), each
    off by 2^-25 of a sum that is on average less than what it ends as: 2^-25 sqrt(3 n / 16) of it, less than 2^-19 for
    n <= 16384; the digits that a missing last plane of a float would take are 2^-16.5 of it, of an fp16 2^-8."""
    assert n <= 16384
    err, size = (got.double() - want).square().mean().sqrt(), want.square().mean().sqrt()
    assert err <= 2.0 ** -18 * size, (float(err), float(size))


def powers(shape, g):
    """Powers of two of either sign that either format holds exactly, where each block's largest is 4."""
    import torch
    v = 2.0 ** torch.randint(0, 3, shape, generator=g, device="cuda") * (torch.randint(0, 2, shape, generator=g, device="cuda") * 2 - 1)
    v[:, ::32] = 4.0
    return v


def digits(n, t, g):
    """n values with all the digits of their type, the last one set."""
    import torch
    bits, reach = {"bf16": (8, 20), "f16": (11, 5), "f32": (24, 20)}[t]
    m = torch.randint(0, 1 << (bits - 2), (n,), generator=g, device="cuda").double() * 2 + 1 + (1 << (bits - 1))
    v = m * 2.0 ** (torch.randint(-reach, reach + 1, (n,), generator=g, device="cuda") - bits + 1).double()
    return (v * (torch.randint(0, 2, (n,), generator=g, device="cuda") * 2 - 1)).to(torch_type(t))


def places(n, sums, g):
    """For each of n results places of the sum, in turns that together reach every run of 64 of it, its ends among them."""
    import torch
    runs = -(-sums // 64)
    for turn in range(-(-runs // n)):
        at = (torch.arange(n, device="cuda") + turn * n) % runs * 64 + torch.randint(0, 64, (n,), generator=g, device="cuda")
        at[0], at[-1] = 0, sums - 1
        yield at.clamp(max=sums - 1)


@pytest.mark.parametrize("case", cases(FORWARD), ids=ids)
@pytest.mark.parametrize("t", TYPES)
def test_forward(pp, t, case):
    import torch
    rows, n_in, n_out = case[-1]
    print("[case] forward", t, case, flush=True)
    g = torch.Generator(device="cuda").manual_seed(101)
    x = torch.randn(rows, n_in, generator=g, device="cuda").to(torch_type(t))
    w, x4 = pp.empty_packed(1, n_out, n_in), pp.empty_packed(1, rows, n_in)
    pp.pp_pack(1, torch.randn(n_out, n_in, generator=g, device="cuda"), w)
    pp.pp_pack(1, x, x4)
    b = torch.randn(n_out, generator=g, device="cuda")
    room = torch.full((rows, n_out + 3), 77.0, dtype=x.dtype, device="cuda")
    kept, again = pp.empty_packed(0, rows, n_in), pp.empty_packed(0, rows, n_in)
    pp.pp_linear_forward(x, w, b, room[:, :n_out], kept, workspace(pp, 0, t, rows, n_in, n_out))
    xv, wv = values(pp, 1, x4, n_in), values(pp, 1, w, n_in).t().contiguous()
    want = xv @ wv + b.double()
    close(room[:, :n_out], want, sum_bound(xv, wv, n_in) + 2.0 ** -22 * want.abs(), t)
    if t == "f32":
        small_on_average(room[:, :n_out], want, n_in)
    assert (room[:, n_out:] == 77).all()
    pp.pp_pack(0, x, again)
    assert torch.equal(kept[0], again[0]) and torch.equal(kept[1], again[1])


@pytest.mark.parametrize("case", cases(INPUT), ids=ids)
def test_backward_input(pp, case):
    import torch
    t, (rows, n_in, n_out) = case[1], case[-1]
    print("[case] backward_input", case, flush=True)
    g = torch.Generator(device="cuda").manual_seed(102)
    w, ws = pp.empty_packed(1, n_out, n_in), workspace(pp, 1, t, rows, n_in, n_out)
    room = torch.full((rows, n_in + 3), 77.0, dtype=torch_type(t), device="cuda")
    dx = room[:, :n_in]
    dy = torch.randn(rows, n_out, generator=g, device="cuda").to(torch_type(t))
    pp.pp_pack(1, torch.randn(n_out, n_in, generator=g, device="cuda"), w)
    pp.pp_linear_backward_input(dy, w, dx, ws)
    wv = values(pp, 1, w, n_in)
    want = dy.double() @ wv
    close(dx, want, sum_bound(dy.double(), wv, n_out), t)
    if t == "f32":
        small_on_average(dx, want, n_out)
    del want, wv
    wv = powers((n_out, n_in), g)
    pp.pp_pack(1, wv, w)
    for at in places(rows, n_out, g):
        v = digits(rows, t, g)
        dy.zero_()
        dy[torch.arange(rows, device="cuda"), at] = v
        pp.pp_linear_backward_input(dy, w, dx, ws)
        assert torch.equal(dx.double(), v.double()[:, None] * wv[at].double())
    assert (room[:, n_in:] == 77).all()


@pytest.mark.parametrize("case", cases(WEIGHT), ids=ids)
def test_backward_weight(pp, case):
    import torch
    t, (rows, n_in, n_out) = case[1], case[-1]
    print("[case] backward_weight", case, flush=True)
    g = torch.Generator(device="cuda").manual_seed(103)
    kept, ws = pp.empty_packed(0, rows, n_in), workspace(pp, 2, t, rows, n_in, n_out)
    room, db = torch.full((n_out, n_in + 3), 77.0, device="cuda"), torch.empty(n_out, device="cuda")
    dw = room[:, :n_in]
    dy = torch.randn(rows, n_out, generator=g, device="cuda").to(torch_type(t))
    pp.pp_pack(0, torch.randn(rows, n_in, generator=g, device="cuda"), kept)
    d, xv = dy.double().t().contiguous(), values(pp, 0, kept, n_in)
    want, bound = d @ xv, sum_bound(d, xv, rows)
    sums, near = d.sum(1), d.abs().sum(1) * ((rows + 8) * 2.0 ** -23)
    for add in (None, torch.randn(n_out, n_in + 3, generator=g, device="cuda")[:, :n_in], dw):      # dw added to nothing, another matrix, itself
        total = want if add is None else want + add.double()
        pp.pp_linear_backward_weight(dy, kept, add, dw, db, ws)
        close(dw, total, bound + 2.0 ** -22 * (total.abs() + (total - want).abs()), "f32")
        close(db, sums, near.clone(), "f32")
        if add is None:
            small_on_average(dw, want, rows)
    del want, bound, total, xv, d
    x = powers((rows, n_in), g)
    pp.pp_pack(0, x, kept)
    for at in places(n_out, rows, g):
        v = digits(n_out, t, g)
        dy.zero_()
        dy[at, torch.arange(n_out, device="cuda")] = v
        pp.pp_linear_backward_weight(dy, kept, None, dw, db, ws)
        assert torch.equal(dw.double(), v.double()[:, None] * x[at].double())
        assert torch.equal(db.double(), v.double())
    assert (room[:, n_in:] == 77).all()
