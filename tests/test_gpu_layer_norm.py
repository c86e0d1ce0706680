"""Norms against the formulas in 64 bits (marker gpu).

Bounds, with u = 2^-24 (half a step of float32): a row's sum of squares has at most 64 additions in a thread for every 65536 columns, 6 in a wave and 16
over waves, all of one sign, and 1 / sqrt takes half of its error and 2 u of its own; x + res, the two products and the
gain add 4 u.  So y is right to (64 + 22) / 2 + 8 < 64 u of itself up to 65536 columns and 32 u for every further 65536.
"""
import itertools

import numpy as np
import pytest

from layer_helpers import Guarded, assert_within, half_step, on_gpu, packed_guarded
from oracle import layers as ol, rows as o

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [(1, 1), (3, 33), (5, 512), (1030, 513), (1025, 1030), (7, 2048), (1024, 2048), (40, 2050), (4, 4100), (3, 8200), (2, 16384), (3, 20001), (2, 32768), (2, 40000), (2, 65600)]


def data(rows, cols, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal(cols) * 0.7)
    return rng, x


def vector(v):
    import torch
    t = torch.from_numpy(np.asarray(v)).float().cuda()
    return t, t.double().cpu().numpy()


def check_packed(got, want, bound):
    """Codes and scales of values that are within `bound` of `want`: the scale is that of a largest value within its bound, and the values are
    within half a step (a whole one where the code is held at 127)."""
    codes, scales = got
    rows, cols = want.shape
    unit = np.ldexp(1.0, scales.reshape(rows, -1).astype(int) - 133)
    top = np.abs(ol.blocks(want)).max(2)
    slack = ol.blocks(np.broadcast_to(bound, want.shape)).max(2)
    tiny = top + slack < 2.0 ** -126
    assert (tiny | ((64 * unit <= top + slack) & (top - slack < 128 * unit))).all()
    v = ol.unpack("int8", codes, scales, cols)
    step = np.repeat(unit, 32, 1)[:, :cols]
    held = np.abs(codes.reshape(rows, -1)[:, :cols].astype(int)) == 127
    assert (np.abs(v - want) <= np.where(held, 1.0, 0.5) * step * (1 + 1e-6) + bound + 1e-45).all()
    return v


def unity(cols):
    return (64 + 32 * (cols // 65536)) * U


@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_forward(t, rows, cols):
    import torch
    from paper_2204_10562_amd import layer as pp
    rng, x = data(rows, cols, rows + cols)
    r = rng.standard_normal((rows, cols)) * 2
    gain, gv = vector(1 + rng.standard_normal(cols) * 0.2)
    for k, (with_res, with_gain, kept, pad, off) in enumerate([(True, True, True, 0, 0), (True, False, False, 3, 1), (False, True, True, 8, 0), (False, False, False, 0, 5)]):
        mx, xv = on_gpu(x, t, pad, off)
        mr, rv = on_gpu(r, t, pad, 0) if with_res else (None, None)
        y, total = Guarded(rows, cols, t, pad, off), Guarded(rows, cols, t, 0, off)
        y8, look_y = packed_guarded(0, rows, cols)
        s8, look_s = packed_guarded(0, rows, cols)
        inv = torch.full((rows,), 7.0, device="cuda")
        pp.pp_norm_forward(mx, mr, gain if with_gain else None, 1e-5, total.m if with_res else None, None if k == 2 else y.m, y8 if kept else None,
                           s8 if kept else None, inv)
        s, iv, want = o.norm_forward(xv, rv, gv if with_gain else None, 1e-5)
        bound = unity(cols) * np.abs(want)
        assert_within(inv.double().cpu().numpy(), iv, unity(cols) * iv, "f32")
        if k != 2:
            assert_within(y.values(), want, bound, t)
        if with_res:
            assert_within(total.values(), s, U * np.abs(s), t)
        if kept:
            check_packed(look_y(), want, bound)
            check_packed(look_s(), s, U * np.abs(s))


@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_backward(t, rows, cols):
    """The bound of dx: the mean has as many additions as the sum of squares and two more roundings to a term; then five roundings.  dgain: a row is
    an addition, and the parts 16 more."""
    import torch
    from paper_2204_10562_amd import layer as pp
    rng, s = data(rows, cols, rows * 3 + cols)
    d, extra = rng.standard_normal((rows, cols)) * 0.1, rng.standard_normal((rows, cols)) * 0.1
    gain, gv = vector(1 + rng.standard_normal(cols) * 0.2)
    dg0, dg0v = vector(rng.standard_normal(cols))
    ws = torch.full((pp.pp_norm_workspace_bytes(getattr(torch, {"bf16": "bfloat16", "f16": "float16", "f32": "float32"}[t]), rows, cols),), 255,
                    dtype=torch.uint8, device="cuda")
    for packed, with_gain, with_total, with_dg, pad, off in [(True, True, True, True, 0, 0), (False, False, False, True, 3, 1), (False, True, True, False, 8, 0)]:
        ms, sv = on_gpu(s, t, pad, off)
        inv, iv = vector(1 / np.sqrt((sv * sv).mean(1) + 1e-5))
        if packed:
            total = pp.empty_packed(0, rows, cols)
            pp.pp_pack(0, ms, total)
            sv = ol.unpack("int8", total[0].cpu().numpy(), total[1].cpu().numpy(), cols)
        else:
            total = ms
        md, dv = on_gpu(d, t, pad, 0)
        mt, tv = on_gpu(extra, t, 0, off) if with_total else (None, None)
        dx = Guarded(rows, cols, t, pad, off)
        dg = torch.full((cols + 8,), 7.0, device="cuda")
        pp.pp_norm_backward(md, total, inv, gain if with_gain else None, mt, dx.m, dg0 if with_dg else None, dg[:cols] if with_dg else None, ws)
        g = gv if with_gain else None
        want, wg = o.norm_backward(dv, sv, iv, g, tv, dg0v)
        z, gd = np.abs(sv * iv[:, None]), np.abs(dv if g is None else dv * g)
        bound = iv[:, None] * (6 * U * gd + z * (unity(cols) + 6 * U) * (gd * z).mean(1, keepdims=True)) + 2 * U * np.abs(want)
        assert_within(dx.values(), want, bound, t)
        if with_dg:
            assert_within(dg[:cols].double().cpu().numpy(), wg, (rows + 20) * U * ((np.abs(dv) * z).sum(0) + np.abs(dg0v)), "f32")
        assert (dg[cols:] == 7).all()


@pytest.mark.parametrize("rows, cols", [(5, 300), (1100, 40), (3, 20001), (2, 40000), (2, 65600)])
def test_in_place(rows, cols):
    """total may be res or x, dx may be dy or dtotal, dgain may be dgain_in: the same results."""
    import torch
    from paper_2204_10562_amd import layer as pp
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *n: torch.randn(*n, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, r, dy, dt, y, dx = (new(rows, cols) for _ in range(6))
    gain, dg0 = torch.randn(cols, generator=g, device="cuda"), torch.randn(cols, generator=g, device="cuda")
    total, inv, dg = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty_like(gain)
    ws = torch.empty(pp.pp_norm_workspace_bytes(x.dtype, rows, cols), dtype=torch.uint8, device="cuda")
    pp.pp_norm_forward(x, r, gain, 1e-6, total, y, None, None, inv)
    for at in (x, r):
        a, b, y2 = x.clone(), r.clone(), torch.empty_like(y)
        pp.pp_norm_forward(a, b, gain, 1e-6, a if at is x else b, y2)
        assert torch.equal(a if at is x else b, total) and torch.equal(y2, y)
    pp.pp_norm_backward(dy, total, inv, gain, dt, dx, dg0, dg, ws)
    for k in range(2):
        a, b, dg2 = dy.clone(), dt.clone(), dg0.clone()
        pp.pp_norm_backward(a, total, inv, gain, b, (a, b)[k], dg2, dg2, ws)
        assert torch.equal((a, b)[k], dx) and torch.equal(dg2, dg)


@pytest.mark.parametrize("cols", [70, 5000, 70000])
def test_rows_that_are_no_numbers(cols):
    """A NaN or an infinity spoils its row and no other; a row of zeros gives zeros; eps counts where a row is small."""
    import torch
    from paper_2204_10562_amd import layer as pp
    x = torch.randn(5, cols, generator=torch.Generator().manual_seed(3)).cuda()
    x[0, cols // 2], x[1, 3], x[2], x[3] = float("nan"), float("inf"), 0.0, x[3] * 1e-20
    y, y8, inv = torch.empty_like(x), pp.empty_packed(0, 5, cols), torch.empty(5, device="cuda")
    pp.pp_norm_forward(x, None, None, 1e-4, None, y, y8, None, inv)
    back = torch.empty_like(x)
    pp.pp_unpack(0, y8, back)
    assert torch.isnan(y[0]).all() and torch.isnan(y[1, 3]) and (y[1, torch.arange(cols) != 3] == 0).all()
    assert torch.isnan(back[0]).all() and (y[2] == 0).all() and (back[2] == 0).all()
    want = o.norm_forward(x[3:].double().cpu().numpy(), None, None, 1e-4)[2]
    assert_within(y[3:].double().cpu().numpy(), want, 2 * unity(cols) * np.abs(want), "f32")


def test_no_rows():
    import torch
    from paper_2204_10562_amd import layer as pp
    x, g = torch.empty(0, 70, device="cuda"), torch.arange(70.0, device="cuda")
    pp.pp_norm_forward(x, None, g, 1e-5, None, x, None, None, x[:, 0].contiguous())
    ws, dg = torch.empty(pp.pp_norm_workspace_bytes(x.dtype, 0, 70), dtype=torch.uint8, device="cuda"), torch.full((70,), 5.0, device="cuda")
    pp.pp_norm_backward(x, x, x[:, 0].contiguous(), g, None, x, g, dg, ws)
    assert torch.equal(dg, g)
    pp.pp_norm_backward(x, x, x[:, 0].contiguous(), g, None, x, None, dg, ws)
    assert (dg == 0).all()


def test_many_rows():
    """More rows than workgroups of a launch, of few columns."""
    import torch
    from paper_2204_10562_amd import layer as pp
    rows, cols = (1 << 22) + 5, 2
    x = torch.randn(rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    y, inv = torch.empty_like(x), torch.empty(rows, device="cuda")
    pp.pp_norm_forward(x, None, None, 1e-3, None, y, None, None, inv)
    want = x.double() * ((x.double() ** 2).mean(1, keepdim=True) + 1e-3).rsqrt()
    assert ((y - want).abs() <= 64 * U * want.abs() + 1e-40).all()
    dx, dg = torch.empty_like(x), torch.empty(cols, device="cuda")
    ws = torch.empty(pp.pp_norm_workspace_bytes(x.dtype, rows, cols), dtype=torch.uint8, device="cuda")
    pp.pp_norm_backward(y, x, inv, None, None, dx, None, dg, ws)
    z, dy = x.double() * inv.double()[:, None], y.double()
    exact = inv.double()[:, None] * (dy - z * (dy * z).mean(1, keepdim=True))
    assert ((dx - exact).abs() <= inv[:, None] * 80 * U * (dy.abs() + z.abs() * (dy * z).abs().mean(1, keepdim=True))).all()
    terms = dy * z
    assert ((dg - terms.sum(0)).abs() <= (rows // 1024 + 160) * U * terms.abs().sum(0)).all()
