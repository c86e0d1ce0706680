"""How far the activation functions in float32 are from 64 bits on average (marker gpu)."""
import numpy as np
import pytest

from oracle import layers as ol
from layer_helpers import on_gpu

pytestmark = pytest.mark.gpu
KINDS = {"gelu": 0, "gelu_tanh": 1, "silu": 2}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", list(KINDS))
def test_errors_on_average(kind, gated):
    """Root mean squares over values of all sizes.  A result is rounded a few times by half a unit of the last place at most, a
    quarter on average, on the way: y and du less than one unit of 2^-24 together.  f' adds to sigmoid or Phi a term
    of up to its size that has been rounded as often: one and a half for dx."""
    from paper_2204_10562_amd import layer as pp
    import torch
    rng = np.random.default_rng(17)
    rows, cols = 300, 1024

    def values():
        return on_gpu(rng.standard_normal((rows, cols)) * np.exp(0.7 * rng.standard_normal((1, cols))), "f32")
    (x, xv), (u, uv), (dy, dv) = values(), values(), values()
    y, dx, du = (torch.empty_like(x) for _ in range(3))
    xk, uk = (pp.empty_packed(pp.PP_PACK_INT8, rows, cols) for _ in range(2))
    pp.pp_act_forward(KINDS[kind], x, u if gated else None, y, xk, uk if gated else None)
    pp.pp_act_backward(KINDS[kind], dy, xk, uk if gated else None, dx, du if gated else None)
    wx, wu = ol.act_backward(kind, dv, xv, uv if gated else None)
    for name, got, want, units in (("y", y, ol.act_forward(kind, xv, uv if gated else None), 1.0), ("dx", dx, wx, 1.5), ("du", du, wu, 1.0)):
        if want is not None:
            err = np.sqrt(np.square(got.double().cpu().numpy() - want).mean() / np.square(want).mean())
            print(kind, gated, name, err * 2 ** 24)
            assert err <= units * 2.0 ** -24, (name, err * 2 ** 24)
