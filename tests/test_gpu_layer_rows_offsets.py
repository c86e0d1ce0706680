"""Norms, scans and single tokens of rows whose offsets pass 2^32 bytes and 2^31 values: the same bits as of rows that lie close (marker gpu)."""
import pytest

pytestmark = pytest.mark.gpu
COLS, FAR = 1000, 1 << 30


def test_rows_far_apart():
    import torch
    from paper_2204_10562_amd import layer as pp
    t, rows = torch.bfloat16, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    room = torch.zeros((1 << 31) + 12 * COLS, dtype=t, device="cuda")
    far = [room.as_strided((rows, COLS), (FAR, 1), k * (COLS + 8)) for k in range(8)]
    near = [torch.randn(rows, COLS, generator=g, device="cuda").to(t) for _ in range(8)]
    inv, gain, dgain = torch.empty(rows, device="cuda"), torch.randn(COLS, generator=g, device="cuda"), torch.empty(COLS, device="cuda")
    ws = torch.empty(max(pp.pp_norm_workspace_bytes(t, rows, COLS), *(pp.pp_scan_workspace_bytes(c, t, rows, COLS) for c in (0, 1))), dtype=torch.uint8, device="cuda")
    kept, pool = torch.empty(pp.pp_scan_kept_rows(t, rows, COLS), COLS, device="cuda"), torch.randn(rows, COLS, generator=g, device="cuda")
    starts = torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda")
    for f, n in zip(far, near):
        f.copy_(n)
    results = []
    for a, b, c, d, e, u, v, w in (far, near):
        out = []
        pp.pp_norm_forward(a, b, gain, 1e-5, c, d, None, None, inv)
        out += [c.clone(), d.clone()]
        pp.pp_norm_backward(e, c, inv, gain, a, d, None, dgain, ws)
        out += [d.clone(), dgain.clone()]
        pp.pp_scan_forward(a, b, starts, None, c, None, kept, ws)
        pp.pp_scan_backward(e, a, b, starts, None, kept, None, u, v, None, ws)
        out += [c.clone(), u.clone(), v.clone()]
        state = pool.clone()
        pp.pp_scan_step(a, b, None, state, w)
        results.append(out + [w.clone(), state])
    assert all(torch.equal(p, q) for p, q in zip(*results))


def test_slots_far_apart():
    """A pool of states of more than 2^31 values."""
    import torch
    from paper_2204_10562_amd import layer as pp
    slots, rows = (1 << 21) + 300, 4
    state = torch.zeros(slots, 1024, device="cuda")
    at = torch.tensor([slots - 1, 5, 1 << 21, slots], dtype=torch.int32, device="cuda")       # (the last is padding)
    g = torch.Generator(device="cuda").manual_seed(2)
    gate, v, first = (torch.randn(rows, 1024, generator=g, device="cuda") for _ in range(3))
    state[at[:3].long()] = first[:3]
    h = torch.full((rows, 1024), 7.0, device="cuda")
    small, want = first.clone(), torch.full_like(h, 7.0)
    pp.pp_scan_step(gate, v, at, state, h)
    pp.pp_scan_step(gate, v, torch.tensor([0, 1, 2, 4], dtype=torch.int32, device="cuda"), small, want)
    assert torch.equal(h, want) and torch.equal(state[at[:3].long()], small[:3])
    state[at[:3].long()] = 0
    assert not state.any()
