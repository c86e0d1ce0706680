"""The example's block of packed layers, step by step against the 64-bit oracle, and its plan (marker gpu)."""
import os
import sys

import numpy as np
import pytest

from oracle import layers as ol
from conftest import ROOT

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -23


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import packed_stage
        return packed_stage
    finally:
        sys.path.pop(0)


def kept_values(pair, cols):
    return ol.unpack("int8", pair[0].cpu().numpy(), pair[1].cpu().numpy(), cols)


def f64(t):
    return t.double().cpu().numpy()


def near(got, want, scale, n):
    """n additions in 32 bits and what the function before them lost, of terms that add up to `scale` in size."""
    assert (np.abs(f64(got) - want) <= (n + 64) * EPS * scale + 1e-30).all()


@pytest.mark.parametrize("rows, width, hidden", [(1, 96, 160), (77, 200, 264), (300, 256, 520)])
def test_block_and_update(example, rows, width, hidden):
    import torch
    block = example.PackedBlock(width, hidden, rows, torch.float32, seed=rows)
    g = torch.Generator(device="cuda").manual_seed(rows + 1)
    total = [np.zeros((l.weight.shape)) for l in block.layers]
    for _ in range(2):     # two microbatches' gradients add up
        arrived = example.send(torch.randn(rows, width, generator=g, device="cuda"))
        x = example.receive(arrived, rows, width, torch.float32)
        np.testing.assert_array_equal(f64(x), kept_values(arrived, width))
        y, kept = block.forward(x)
        dy = torch.randn(rows, width, generator=g, device="cuda")
        dx = block.backward(dy, kept)
        W = [ol.unpack("fp4", l.packed[0].cpu().numpy(), l.packed[1].cpu().numpy(), l.weight.shape[1]) for l in block.layers]
        # forward, up to what the rounding of h to 8 bits adds
        x4 = ol.kept("fp4", f64(x))
        a, u = x4 @ W[0].T, x4 @ W[1].T
        ka, ku, kh = (kept_values(kept[n], hidden) for n in ("gate", "up", "h"))
        blocks = lambda v: np.abs(ol.blocks(v)).max(-1, keepdims=True)  # noqa: E731
        for k, v in ((ka, a), (ku, u), (kh, ol.act_forward("silu", a, u))):
            assert (np.abs(ol.blocks(k) - ol.blocks(v)) <= blocks(v) * (2.0 ** -6 + 1e-4)).all()
        # h in 4 bits is at most an eighth of its block's largest value away from h (a sixth, where that is beyond 6)
        h = ol.act_forward("silu", a, u)
        lost = np.broadcast_to(blocks(h) * 0.26, ol.blocks(h).shape).reshape(rows, -1)[:, :hidden]
        assert (np.abs(f64(y) - h @ W[2].T) <= lost @ np.abs(W[2]).T + 1e-4).all()
        # backward, from what was kept
        d = f64(dy)
        dh = d @ W[2]
        da, du = ol.act_backward("silu", dh, ka, ku)
        size = np.abs(d) @ np.abs(W[2])
        sa, su = (np.abs(v) for v in ol.act_backward("silu", size, ka, ku))
        near(dx, da @ W[0] + du @ W[1], sa @ np.abs(W[0]) + su @ np.abs(W[1]), width + 2 * hidden)
        for at, (dv, size, xv) in enumerate(((da, sa, kept_values(kept["x"], width)), (du, su, kept_values(kept["x"], width)), (d, np.abs(d), kh))):
            total[at] += dv.T @ xv
            layer = block.layers[at]
            bound = size.T @ np.abs(xv)
            assert (np.abs(f64(layer.grad) - total[at]) <= 4 * (rows + width + 64) * EPS * (bound + np.abs(total[at])) + 1e-30).all()
    before = [l.weight.clone() for l in block.layers]
    grads = [l.grad.clone() for l in block.layers]
    block.update(0.5)
    for l, w, gr in zip(block.layers, before, grads):
        assert torch.equal(l.weight, w.add(gr, alpha=-0.5)) and not l.grad.any()
        c, s = ol.pack("fp4", f64(l.weight))
        np.testing.assert_array_equal(l.packed[0].cpu().numpy(), c)
        np.testing.assert_array_equal(l.packed[1].cpu().numpy(), s)


def test_plan_is_the_oracles(example):
    """The measured times and bytes through the planner, against the oracle's plan of them."""
    import torch
    from oracle import ppo
    from dataclasses import replace
    from paper_2204_10562_amd.problem import GpuProblem
    forward, backward, sent, returned = example.measure(256, 512, 64, torch.bfloat16)
    assert forward > 0 and backward > 0
    assert sent == 64 * 256 + 64 * 8 and returned == 64 * 256 * 2
    w, winners = example.plan(forward, backward, sent, returned, 24)
    assert len(winners) == len(w.Ms) and all(q["T"] > 0 for q in winners)
    w = replace(w, orderings=np.ascontiguousarray(w.explicit_orderings()[:500]), N=500)
    rc, PF, PB, XF, XB = ppo.prefix_costs(w.fwd, w.bwd, w.actf, w.actb, w.bw)
    g = GpuProblem(w)
    assert rc == 0 and g.prefix() == 0
    status, got, _, _ = g.best_multi(w.Ms)
    assert status == 0
    for q, M in enumerate(w.Ms):
        rc, want, _, _ = ppo.best_plan(w.L, w.D, w.S, w.N, M, PF, PB, XF, XB, w.orderings)
        assert rc == 0 and got[q] == want


def test_command(example, capsys):
    example.main(["--rows", "64", "--width", "256", "--hidden", "512", "--layers", "16", "--type", "f16"])
    out = capsys.readouterr().out.splitlines()
    assert len(out) == 5 and out[0].startswith("block 256 -> 512") and all(l.startswith("M = ") for l in out[1:])
