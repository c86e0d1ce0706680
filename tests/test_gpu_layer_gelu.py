"""gelu where little of it is left: relative to what it is, down to the ends of the types (marker gpu)."""
import numpy as np
import pytest

from oracle import layers as ol
from layer_helpers import TYPES, assert_within, on_gpu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pp():
    from paper_2204_10562_amd import layer
    return layer


def relative(x):
    """What 32 bits lose of exp(-x^2 / 2): three roundings in an exponent of x^2 / 2 (two units each for the constant's), so
    2 x^2 units of 2^-24 at most; of the functions around it, their fit and their products 40."""
    return U * (40 + 2 * x * x)


LOW = 1e-38     # 32 bits hold no normal numbers below


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("t", TYPES)
def test_tail_forward(pp, t, gated):
    import torch
    x, xv = on_gpu(np.concatenate([np.linspace(-13.5, -2, 4000), np.linspace(-2, 9, 2000), -np.logspace(-9, 0, 400)]).reshape(1, -1), t)
    u, uv = on_gpu(np.full(xv.shape, 1024.0), t)
    y = torch.empty_like(x)
    pp.pp_act_forward(pp.PP_ACT_GELU, x, u if gated else None, y)
    f = ol.act("gelu", xv)
    b = np.abs(f) * relative(xv) + LOW
    if gated:
        f, b = f * uv, (b + U * np.abs(f)) * uv
    assert_within(y.double().cpu().numpy(), f, b, t)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_tail_backward(pp, t):
    """A block holds one value, of seven bits, so the kept one is x."""
    import torch
    values = np.concatenate([-np.arange(8, 65) / 8, -np.arange(64, 109) / 8, np.arange(0, 72) / 8])
    values = values[np.array([v == 0 or (np.abs(v) * 2.0 ** (6 - np.floor(np.log2(np.abs(v) or 1)))) % 1 == 0 for v in values])]
    x, xv = on_gpu(np.repeat(values, 32).reshape(1, -1), t)
    one = torch.ones_like(x)
    xk, uk = (pp.empty_packed(pp.PP_PACK_INT8, 1, x.shape[1]) for _ in range(2))
    pp.pp_pack(pp.PP_PACK_INT8, x, xk)
    pp.pp_pack(pp.PP_PACK_INT8, one, uk)
    np.testing.assert_array_equal(ol.kept("int8", xv), xv)
    dx, du, alone = (torch.empty_like(x) for _ in range(3))
    pp.pp_act_backward(pp.PP_ACT_GELU, one, xk, uk, dx, du)
    pp.pp_act_backward(pp.PP_ACT_GELU, one, xk, None, alone)
    f, d = ol.act("gelu", xv), ol.act_slope("gelu", xv)
    phi = np.exp(-xv * xv / 2) / np.sqrt(2 * np.pi)
    size = np.abs(d - xv * phi) + np.abs(xv) * phi       # of the two terms, whose difference f' is on the negative side
    for got, want, b in ((du, f, np.abs(f) * relative(xv) + LOW), (dx, d, size * relative(xv) + LOW), (alone, d, size * relative(xv) + LOW)):
        assert_within(got.double().cpu().numpy(), want, b, t)


def test_ends(pp):
    """Exactly zero, a half and the argument where they have to be; what is missing stays so."""
    import torch
    x = torch.tensor([[0.0, -0.0, 15.0, 1e30, float("inf"), -15.0, -1e30, float("nan")] * 4], device="cuda")
    y = torch.empty_like(x)
    pp.pp_act_forward(pp.PP_ACT_GELU, x, None, y)
    v = y[0, :8].cpu().numpy()
    assert v[0] == 0 and v[1] == 0 and v[2] == 15 and v[3] == np.float32(1e30) and v[4] == np.inf and v[5] == 0 and v[6] == 0 and np.isnan(v[7])
