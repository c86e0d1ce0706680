"""A scan of as many rows as a matrix may have: more tiles than one launch has workgroups (marker gpu).

A gate of 0 has a = 1/2, so every result is held to its neighbours: 2 h_t = h_(t-1) + v_t, 2 dv_t = dh_t + dv_(t+1), and 2 dgate_t =
(h_(t-1) - v_t) dv_t.  Each result is off by a rounding to bf16 (2^-8 of itself) and what 32 bits leave (2^-20 of the values, which are below 8),
so by twice that where two stand together.
"""
import pytest

pytestmark = pytest.mark.gpu
ROWS, STEP = 1 << 30, 1 << 26
HALF, LEFT = 2.0 ** -8, 8 * 2.0 ** -20


def test_as_many_rows_as_there_may_be():
    import torch
    from paper_2204_10562_amd import layer as pp
    print("[case] scan", ROWS, flush=True)
    t = torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(1)
    gate, v, dh = (torch.zeros(ROWS, 1, dtype=t, device="cuda") for _ in range(3))
    for at in range(0, ROWS, STEP):
        for x in (v, dh):
            x[at:at + STEP, 0] = torch.randn(STEP, generator=g, device="cuda").clamp_(-4, 4).to(t)
    h, dgate, dv = (torch.full((ROWS, 1), float("nan"), dtype=t, device="cuda") for _ in range(3))
    h0, dh_last, last, dh0 = (torch.full((1, 1), x, device="cuda") for x in (2.0, 3.0, 7.0, 7.0))
    kept = torch.full((pp.pp_scan_kept_rows(t, ROWS, 1), 1), float("nan"), device="cuda")
    ws = torch.empty(max(pp.pp_scan_workspace_bytes(c, t, ROWS, 1) for c in (0, 1)), dtype=torch.uint8, device="cuda")
    print("[case] forward", flush=True)
    pp.pp_scan_forward(gate, v, None, h0, h, last, kept, ws)
    torch.cuda.synchronize()
    print("[case] backward", flush=True)
    pp.pp_scan_backward(dh, gate, v, None, h0, kept, dh_last, dgate, dv, dh0, ws)
    torch.cuda.synchronize()
    print("[case] look", flush=True)
    near = lambda got, want, bound: bool(((got - want).abs() <= bound + LEFT).all())  # noqa: E731
    for at in range(0, ROWS, STEP):
        end = at + STEP
        v1, d1, h1, dv1, dg1 = (x[at:end, 0].float() for x in (v, dh, h, dv, dgate))
        before = torch.cat([h[at - 1, :1].float() if at else h0[0], h1[:-1]])
        behind = torch.cat([dv1[1:], dv[end, :1].float() if end < ROWS else dh_last[0]])    # (a g of the token behind)
        assert near(2 * h1, before + v1, HALF * (2 * h1.abs() + before.abs())), at
        assert near(2 * dv1, d1 + behind, HALF * (2 * dv1.abs() + behind.abs())), at
        assert near(2 * dg1, (before - v1) * dv1, HALF * (2 * dg1.abs() + before.abs() * dv1.abs() + (before - v1).abs() * dv1.abs() * (1 + HALF))), at
    assert near(last[0], h[-1].float(), HALF * h[-1].float().abs()) and near(dh0[0], dv[0].float(), HALF * dv[0].float().abs())
    del gate, v, dh, h, dgate, dv, kept, ws
    torch.cuda.empty_cache()


def test_more_single_tokens_than_threads():
    """With a gate of 0 h is (state + v) / 2, rounded once; slots from the last to the first."""
    import torch
    from paper_2204_10562_amd import layer as pp
    rows = (1 << 28) + 5
    print("[case] step", rows, flush=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    gate, v, state = torch.zeros(rows, 1, device="cuda"), torch.randn(rows, 1, generator=g, device="cuda"), torch.randn(rows, 1, generator=g, device="cuda")
    slots, h = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda"), torch.empty_like(v)
    want = (state.flip(0) + v) / 2
    pp.pp_scan_step(gate, v, slots, state, h)
    assert torch.equal(h, want) and torch.equal(state.flip(0), want)
    del gate, v, state, slots, h, want
    torch.cuda.empty_cache()
