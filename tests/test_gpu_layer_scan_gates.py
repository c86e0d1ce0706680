"""The gated recurrence where a gate's exponential, or its reciprocal, leaves the normal floats (marker gpu).

exp(-gate) is finite down to a gate of -88.72, but 1 / (1 + exp(-gate)) is no normal number from -87.34 on.  Bounds: those of the
recurrence's other tests, (8 + 2 |gate|) u of the smaller side of a gate and 2^-126 of either.
"""
import numpy as np
import pytest

from layer_helpers import Guarded, assert_within, on_gpu, torch_type
from oracle import rows as o
from test_gpu_layer_scan import U, floats, run, workspace

pytestmark = pytest.mark.gpu
ENDS = [86.0, 86.5, 87.0, 87.25, 87.33, 87.34, 87.4, 87.5, 88.0, 88.5, 88.7, 88.72, 88.73, 89.0, 103.0, 104.0]


@pytest.mark.parametrize("rows", [7, 70, 300])
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_forward_and_backward(t, rows):
    """Every such gate throughout a channel, and among ordinary ones; in one tile and in several."""
    gates = np.array([-g for g in ENDS] + ENDS)
    rng = np.random.default_rng(rows)
    cols = 2 * len(gates)
    gate = rng.standard_normal((rows, cols)) * 2
    gate[:, :len(gates)] = gates
    gate[rows // 3, len(gates):] = gates
    gate[-1, len(gates):] = gates[::-1]
    draw = lambda *s: rng.standard_normal(s)  # noqa: E731
    starts = [0, rows // 2, rows]
    run(t, starts, gate, draw(rows, cols), draw(2, cols), draw(rows, cols), draw(2, cols))


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_step(t):
    """Gates from -110 to 110 and at the ends, one token a row."""
    import torch
    from paper_2204_10562_amd import layer as pp
    rng = np.random.default_rng(5)
    row = np.concatenate([np.linspace(-110, 110, 4001), ENDS, [-g for g in ENDS]])
    rows, cols = 3, len(row)
    mg, gate = on_gpu(np.stack([row, row[::-1], rng.permutation(row)]), t)
    mv, v = on_gpu(rng.standard_normal((rows, cols)) + 3, t)
    state, old = floats(rng.standard_normal((rows, cols)))
    h = Guarded(rows, cols, t)
    pp.pp_scan_step(mg, mv, None, state, h.m)
    a, u = o.sigmoid(gate), o.sigmoid(-gate)
    want = a * old + u * v
    bound = U * (4 * np.maximum(np.abs(old), np.abs(v)) + np.minimum(a, u) * np.abs(v - old) * (8 + 2 * np.abs(gate)))
    assert_within(h.values(), want, bound, t)
    assert_within(state.double().cpu().numpy(), want, bound, "f32")


@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_gates_that_are_no_numbers(t):
    """An infinite gate leaves the state or the value, exactly (a value of 0 too); one that is NaN leaves NaN, in its channel alone."""
    import torch
    from paper_2204_10562_amd import layer as pp
    inf, rows = np.inf, 40
    gate = np.tile(np.array([[inf, -inf, -inf, 0.0, np.nan, 0.5]]), (rows, 1))
    gate[:5, 4], gate[6:, 4] = 0.0, 0.0
    v = np.random.default_rng(6).standard_normal((rows, 6))
    v[:, 2] = 0.0
    mg, mv = on_gpu(gate, t)[0], on_gpu(v, t)[0]
    h0 = torch.full((1, 6), 3.0, device="cuda")
    h, last = torch.empty_like(mv), torch.empty_like(h0)
    pp.pp_scan_forward(mg, mv, None, h0, h, last, None, workspace(0, t, rows, 6))
    state, steps = h0.clone(), torch.empty_like(mv)
    for r in range(rows):
        pp.pp_scan_step(mg[r:r + 1], mv[r:r + 1], None, state, steps[r:r + 1])
    for got, end in ((h, last), (steps, state)):
        assert (got[:, 0] == 3).all() and torch.equal(got[:, 1], mv[:, 1]) and (got[:, 2] == 0).all()
        assert torch.isfinite(got[:5]).all() and torch.isnan(got[5:, 4]).all() and torch.isfinite(got[:, [0, 1, 2, 3, 5]]).all()
        assert end[0, 0] == 3 and end[0, 2] == 0 and torch.isnan(end[0, 4])
    assert h.dtype == torch_type(t)
