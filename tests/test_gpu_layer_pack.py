"""Packing and activation functions on the GPU against the 64-bit oracle (marker gpu)."""
import numpy as np
import pytest

from oracle import layers as ol
from layer_helpers import Guarded, TYPES, assert_within, on_gpu, packed_guarded, torch_type

pytestmark = pytest.mark.gpu
FMT = {"int8": 0, "fp4": 1}
SIZES = [(1, 1), (1, 31), (3, 32), (2, 33), (1, 127), (5, 128), (4, 129), (17, 200), (64, 515), (1, 4096), (300, 24), (1030, 130), (9, 2056)]


@pytest.fixture(scope="module")
def pp():
    from paper_2204_10562_amd import layer
    return layer


def draw(rng, rows, cols):
    v = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((1, cols)))
    v[rng.random((rows, cols)) < 0.02] = 0
    if rows > 1:
        v[1] = 0                       # a row of zeros
    return v


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
@pytest.mark.parametrize("t", TYPES)
def test_pack_and_unpack_are_the_oracles_bits(pp, fmt, t):
    rng = np.random.default_rng(11)
    for rows, cols in SIZES:
        for pad, off in [(0, 0), (3, 1), (8, 8)]:
            print("[case]", fmt, t, rows, cols, pad, off, flush=True)
            m, x = on_gpu(draw(rng, rows, cols), t, pad, off)
            pair, check = packed_guarded(FMT[fmt], rows, cols)
            pp.pp_pack(FMT[fmt], m, pair)
            codes, scales = check()
            c0, s0 = ol.pack(fmt, x)
            np.testing.assert_array_equal(scales, s0)
            np.testing.assert_array_equal(codes, c0)
            out = Guarded(rows, cols, t, pad, off)
            pp.pp_unpack(FMT[fmt], pair, out.m)
            want = ol.unpack(fmt, c0, s0, cols)
            assert_within(out.values(), want, 0.0, t)
            if t != "f16":             # 16 bits with 8 of exponent hold every packed value
                np.testing.assert_array_equal(out.values(), want)


@pytest.mark.parametrize("fmt", ["int8", "fp4"])
@pytest.mark.parametrize("t", TYPES)
def test_pack_ends_of_the_range(pp, fmt, t):
    """Ties, subnormal numbers, the largest ones, and blocks with NaN or infinities."""
    big = {"bf16": 255 * 2.0 ** 120, "f16": 65504.0, "f32": (2 - 2.0 ** -23) * 2.0 ** 127}[t]
    low = {"bf16": -133, "f16": -24, "f32": -149}[t]
    rows = [[big, -big / 3, big / 255], [2.0 ** low, -2.0 ** low, 0.0], [2.0 ** (low + 5), 3 * 2.0 ** low, -2.0 ** low],
            [2.0 ** -14, 2.0 ** -20, 0.0], [np.nan, 1.0, 2.0], [1.0, np.inf, 2.0], [-np.inf, np.nan, 0.0], [0.0, -0.0, 0.0]]
    if t != "f16":
        rows += [[2.0 ** e, 1.5 * 2.0 ** (e - 3), -2.0 ** (e - 6)] for e in range(-130 if t == "bf16" else -145, -108)]
    x = np.zeros((len(rows) + 2, 64))
    x[:len(rows), 29:32] = rows       # the second block of every row stays finite
    x[:len(rows), 40] = 1.0
    x[-2, :32] = np.arange(32) / 8.0 * (1 if fmt == "fp4" else 0.25)    # every tie of 4 bits
    x[-2, 31] = 7.0
    x[-1, :32] = (np.arange(32) + 0.5) / 64.0                          # ties of 8 bits
    x[-1, 31] = 1.0
    m, v = on_gpu(x, t)
    pair, check = packed_guarded(FMT[fmt], *x.shape)
    pp.pp_pack(FMT[fmt], m, pair)
    codes, scales = check()
    c0, s0 = ol.pack(fmt, v)
    np.testing.assert_array_equal(scales, s0)
    np.testing.assert_array_equal(codes, c0)
    out = Guarded(*x.shape, t)
    pp.pp_unpack(FMT[fmt], pair, out.m)
    got, want = out.values(), ol.unpack(fmt, c0, s0, 64)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    fine = np.isfinite(want)
    assert_within(got[fine], want[fine], 0.0, t)


def bound_f(kind, x, f):
    """32-bit evaluation of f: x s(z) with an exponential of relative error (|z| + 4) 2^-23 in s, which moves
    s by at most that times s (1 - s), and ten roundings; gelu: the error function's few units of 1."""
    u = 2.0 ** -24
    if kind == "gelu":
        return 16 * u * np.abs(x) + 1e-44
    z = x if kind == "silu" else 2 * ol.C * (x + 0.044715 * x ** 3)
    return np.abs(f) * u * (16 + 4 * np.minimum(np.abs(z), 200)) + 1e-37


def bound_d(x):
    """f' is a sum of terms of at most 1 + |x| s (1 - s) z' < 4 in size, each with the above relative error (|z| < 100
    where s (1 - s) does not vanish), 1 - s with an error of a unit of 1."""
    u = 2.0 ** -24
    return u * 64 * (1 + np.minimum(np.abs(x), 32) ** 3 * np.exp(-np.minimum(np.abs(x), 32)) + np.minimum(np.abs(x), 32))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
def test_act_forward_and_backward(pp, kind, t, gated):
    k = {"gelu": 0, "gelu_tanh": 1, "silu": 2}[kind]
    rng = np.random.default_rng(12)
    for rows, cols in SIZES:
        for pad, off in [(0, 0), (5, 1)]:
            print("[case]", kind, t, gated, rows, cols, pad, off, flush=True)
            x, xv = on_gpu(draw(rng, rows, cols) * 3, t, pad, off)
            u, uv = on_gpu(draw(rng, rows, cols), t, pad + 1, 0) if gated else (None, None)
            dy, dv = on_gpu(draw(rng, rows, cols), t, pad, off)
            y, dx, du = Guarded(rows, cols, t, pad, off), Guarded(rows, cols, t, pad, 0), Guarded(rows, cols, t, 2, 1)
            xp, xcheck = packed_guarded(0, rows, cols)
            up, ucheck = packed_guarded(0, rows, cols) if gated else (None, None)
            pp.pp_act_forward(k, x, u, y.m, xp, up)
            got = xcheck()
            for a, b in zip(got, ol.pack("int8", xv)):
                np.testing.assert_array_equal(a, b)
            f = ol.act(kind, xv)
            b = bound_f(kind, xv, f)
            if gated:
                for p, q in zip(ucheck(), ol.pack("int8", uv)):
                    np.testing.assert_array_equal(p, q)
                b = (b + 2.0 ** -24 * np.abs(f)) * np.abs(uv)
                f = f * uv
            assert_within(y.values(), f, b, t)
            pp.pp_act_backward(k, dy, xp, up, dx.m, du.m if gated else None)
            xk = ol.kept("int8", xv)
            wx, wu = ol.act_backward(kind, dv, xv, uv)
            b = bound_d(xk) * np.abs(dv)
            if gated:
                b = b * np.abs(ol.kept("int8", uv))
                fk = ol.act(kind, xk)
                assert_within(du.values(), wu, (bound_f(kind, xk, fk) + 2.0 ** -23 * np.abs(fk)) * np.abs(dv), t)
            assert_within(dx.values(), wx, b + 2.0 ** -22 * np.abs(wx), t)


def test_act_without_checkpoints_and_in_place(pp):
    import torch
    rng = np.random.default_rng(13)
    x, xv = on_gpu(draw(rng, 33, 333), "bf16")
    y, z = Guarded(33, 333, "bf16"), Guarded(33, 333, "bf16")
    pair, _ = packed_guarded(0, 33, 333)
    pp.pp_act_forward(pp.PP_ACT_SILU, x, None, y.m)
    pp.pp_act_forward(pp.PP_ACT_SILU, x, None, z.m, pair)
    np.testing.assert_array_equal(y.values(), z.values())
    dx = Guarded(33, 333, "bf16")
    pp.pp_act_backward(pp.PP_ACT_SILU, x, pair, None, dx.m)
    pp.pp_act_backward(pp.PP_ACT_SILU, x, pair, None, x)          # dx in the place of dy
    assert torch.equal(x, dx.m)


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_act_large_and_missing_values(pp, kind):
    """Where the functions are flat, and where a kept block holds a NaN."""
    import torch
    x = torch.tensor([[0.0, -0.0, 20.0, -20.0, 90.0, -90.0, 3e4, -3e4, 1e19, -1e19, 3e38, -3e38] + [1.0] * 20 + [float("nan")] + [2.0] * 31], device="cuda")
    p = pp.empty_packed(0, 1, 64)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    pp.pp_act_forward(kind, x, None, y, p)
    v = y[0].cpu().numpy()
    assert v[0] == 0 and abs(v[2] - 20) < 1e-5 and abs(v[3]) < 1e-7 and v[4] == 90 and abs(v[5]) < 1e-37 and v[6] == np.float32(3e4) and v[7] == 0
    assert v[8] == np.float32(1e19) and v[9] == 0 and v[10] == np.float32(3e38) and v[11] == 0 and np.isnan(v[32]) and np.isfinite(np.delete(v, 32)).all()
    pp.pp_act_backward(kind, torch.ones_like(x), p, None, dx)
    d = dx[0].cpu().numpy()
    # the first block's largest value leaves the others at zero, where every f' is 1/2; f' is 1 and 0 far out
    assert (d[:8] == 0.5).all() and d[10] == 1 and d[11] == 0 and np.isnan(d[32:]).all()
    one = torch.full((1, 32), 2.5, device="cuda")
    for big in (40.0, 1e6, 1e18, 1e30):
        one[0, 0], one[0, 1] = big, -big
        q = pp.empty_packed(0, 1, 32)
        pp.pp_pack(0, one, q)
        g = torch.empty_like(one)
        pp.pp_act_backward(kind, torch.ones_like(one), q, None, g)
        assert g[0, 0] == 1 and abs(g[0, 1]) < 1e-15, (big, g[0, :2])     # silu'(-40) = -39 exp(-40)


def test_offsets_beyond_32_bits(pp):
    """A matrix of more than 2^32 bytes and 2^31 values: its first, middle and last rows."""
    import torch
    rows, cols = 70001, 32768
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(14)
    at = [0, 1, 32767, 65535, 65536, 65537, 70000]
    for r in at:
        x[r] = torch.from_numpy(rng.standard_normal(cols)).to(x)
    for fmt in ("int8", "fp4"):
        pair = pp.empty_packed(FMT[fmt], rows, cols)
        out = torch.empty_like(x)
        pp.pp_pack(FMT[fmt], x, pair)
        pp.pp_unpack(FMT[fmt], pair, out)
        for r in at:
            want = ol.kept(fmt, x[r:r + 1].double().cpu().numpy())
            np.testing.assert_array_equal(out[r:r + 1].double().cpu().numpy(), want)
        assert not out[2:32767].any() and not out[65538:70000].any()
        del out, pair


def test_no_rows(pp):
    import torch
    x = torch.empty(0, 100, device="cuda")
    p = pp.empty_packed(0, 0, 100)
    pp.pp_pack(0, x, p)
    pp.pp_unpack(0, p, x)
    pp.pp_act_forward(0, x, None, x.clone(), p)
    pp.pp_act_backward(0, x, p, None, x.clone())


def test_binding_refusals(pp):
    import torch
    x = torch.zeros(8, 64, dtype=torch.bfloat16, device="cuda")
    p = pp.empty_packed(0, 8, 64)
    for bad in (x.t(), x[:, ::2], x[0], x.to(torch.int32), x[:4]):
        with pytest.raises(ValueError):
            pp.pp_pack(0, bad, p)
    with pytest.raises(ValueError):
        pp.pp_pack(1, x, p)                                   # the other format's codes
    with pytest.raises(ValueError):
        pp.pp_act_forward(0, x, None, x.float(), p)
    with pytest.raises(pp.PPError):
        pp.pp_act_forward(3, x, None, x.clone(), p)
    with pytest.raises(pp.PPError):
        pp.pp_act_forward(0, x, None, x.clone(), p, p)         # a gate's checkpoint without a gate
    with pytest.raises(pp.PPError):
        pp.pp_act_backward(0, x, p, p, x.clone())              # no room for the gate's gradient


def test_side_stream_behind_pending_work(pp):
    import torch
    s = torch.cuda.Stream()
    x = torch.zeros(512, 1024, dtype=torch.bfloat16, device="cuda")
    p, out = pp.empty_packed(0, 512, 1024), torch.empty(512, 1024, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            x.add_(1.0)
        pp.pp_pack(0, x, p)
        pp.pp_unpack(0, p, out)
    s.synchronize()
    assert (out == 20).all()
