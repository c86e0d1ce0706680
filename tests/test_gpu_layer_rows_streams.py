"""Norms, scans and losses on a stream of their own behind pending work, in recorded graphs, and with few units free (marker gpu)."""
import pytest

pytestmark = pytest.mark.gpu
TOP = 20


class Run:
    """All of the operators once, in buffers of fixed places."""

    def __init__(self, rows, cols, vocab, dtype, ws=None):
        import torch
        from paper_2204_10562_amd import layer as pp
        self.pp, self.rows, self.cols, self.dtype = pp, rows, cols, dtype
        new = lambda *s, t=dtype: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
        f32, i32 = torch.float32, torch.int32
        self.x, self.res, self.gate, self.v, self.dh = (new(rows, cols) for _ in range(5))
        self.total, self.y, self.dx, self.h, self.dgate, self.dv = (new(rows, cols) for _ in range(6))
        self.gain, self.dgain, self.inv = new(cols, t=f32), new(cols, t=f32), new(rows, t=f32)
        self.kept8 = pp.empty_packed(0, rows, cols)
        self.starts = torch.tensor([0, rows // 3, rows // 3, rows - 1], dtype=i32, device="cuda")
        self.h0, self.last, self.dh0 = (new(3, cols, t=f32) for _ in range(3))
        self.states = new(pp.pp_scan_kept_rows(dtype, rows, cols), cols, t=f32)
        self.pool, self.slots, self.one = new(rows + 3, cols, t=f32), torch.randperm(rows + 3, device="cuda")[:rows].to(i32), new(rows, cols)
        self.logits, self.dlogits, self.ds = new(rows, vocab), new(rows, vocab), new(rows, vocab)
        self.tokens = torch.randint(0, vocab, (rows,), device="cuda", dtype=i32)
        self.logp, self.entropy, self.norm, self.loss, self.g = new(rows, t=f32), new(rows, t=f32), new(rows, 2, t=f32), new(rows, t=f32), new(rows, t=f32)
        self.index, self.value = new(rows, TOP, t=i32), new(rows, TOP, t=f32)
        need = max([pp.pp_norm_workspace_bytes(dtype, rows, cols)] + [pp.pp_scan_workspace_bytes(c, dtype, rows, cols) for c in (0, 1)]
                   + [pp.pp_logprob_workspace_bytes(dtype, rows, vocab, TOP), pp.pp_distill_workspace_bytes(dtype, rows, vocab, TOP)])
        self.ws = new(need, t=torch.uint8) if ws is None else ws
        assert self.ws.numel() >= need

    def fill(self, seed):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (self.x, self.res, self.gate, self.v, self.dh, self.gain, self.h0, self.pool, self.g):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        for r in range(0, self.rows, 256):
            n = min(256, self.rows - r)
            self.logits[r:r + n] = torch.randn(n, self.logits.shape[1], generator=g, device="cuda") * 3

    def step(self):
        pp = self.pp
        pp.pp_norm_forward(self.x, self.res, self.gain, 1e-5, self.total, self.y, None, self.kept8, self.inv)
        pp.pp_norm_backward(self.dh, self.kept8, self.inv, self.gain, self.y, self.dx, self.gain, self.dgain, self.ws)
        pp.pp_scan_forward(self.gate, self.v, self.starts, self.h0, self.h, self.last, self.states, self.ws)
        pp.pp_scan_backward(self.dh, self.gate, self.v, self.starts, self.h0, self.states, self.h0, self.dgate, self.dv, self.dh0, self.ws)
        pp.pp_scan_step(self.gate, self.v, self.slots, self.pool, self.one)
        pp.pp_logprob_forward(self.logits, 0.9, self.tokens, self.logp, self.entropy, self.norm, self.index, self.value, self.ws)
        pp.pp_logprob_backward(self.logits, 0.9, self.tokens, self.norm, self.g, self.entropy, self.g, self.dlogits)
        pp.pp_distill_loss(1, self.logits, 0.9, self.index, self.value, self.g, self.loss, self.ds, self.ws)

    def results(self):
        return [t.clone() for t in (self.total, self.y, self.inv, self.dx, self.dgain, self.h, self.last, self.dgate, self.dv, self.dh0, self.pool, self.one,
                                    self.logp, self.entropy, self.index, self.value, self.dlogits, self.loss, self.ds)]


# the last: a distillation that is read once, by workgroups that meet, and a scan of many tiles
SIZES = [(3, 40, 50), (70, 300, 9000), (700, 1000, 5000), (1100, 520, 65000)]


def same(a, b):
    import torch
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("rows, cols, vocab", SIZES)
@pytest.mark.parametrize("t", ["bfloat16", "float32"])
def test_behind_pending_work(t, rows, cols, vocab):
    """Also the same bits from call to call."""
    import torch
    one = Run(rows, cols, vocab, getattr(torch, t))
    one.fill(51)
    one.step()
    want = one.results()
    torch.cuda.synchronize()
    busy = torch.randn(2048, 2048, device="cuda")
    side = torch.cuda.Stream()
    one.fill(52)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy * 1e-3
        one.fill(51)
        one.ws.fill_(255)
        one.step()
        got = one.results()
    side.synchronize()
    assert same(got, want)


@pytest.mark.parametrize("rows, cols, vocab", SIZES)
def test_recorded(rows, cols, vocab):
    """Two graphs that share a workspace, one behind the other, with eager calls between their replays."""
    import torch
    one = Run(rows, cols, vocab, torch.bfloat16)
    two = Run(rows, cols, vocab, torch.bfloat16, one.ws)
    graphs = []
    for r in (one, two):
        r.fill(61)
        r.step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r.step()
        graphs.append(g)
    for seed in (62, 63, 64):
        want = []
        for r, s in ((one, seed), (two, seed + 100)):
            r.fill(s)
            r.step()
            want.append(r.results())
            r.fill(s)
        one.ws.fill_(255 if seed & 1 else 0)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert same(one.results(), want[0]) and same(two.results(), want[1]), seed


def test_two_streams_at_once():
    """Scans and distillations whose workgroups wait for each other, on four streams at the same time, each with a workspace of its own."""
    import torch
    runs = [Run(1100, 520, 65000, torch.bfloat16) for _ in range(4)]
    want = []
    for k, r in enumerate(runs):
        r.fill(70 + k)
        r.step()
        want.append(r.results())
    for k, r in enumerate(runs):
        r.fill(70 + k)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        for s, r in zip(streams, runs):
            with torch.cuda.stream(s):
                r.pp.pp_scan_forward(r.gate, r.v, r.starts, r.h0, r.h, r.last, r.states, r.ws)
                r.pp.pp_scan_backward(r.dh, r.gate, r.v, r.starts, r.h0, r.states, r.h0, r.dgate, r.dv, r.dh0, r.ws)
                r.pp.pp_distill_loss(1, r.logits, 0.9, r.index, r.value, r.g, r.loss, r.ds, r.ws)
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        r_now = r.results()
        for i in (5, 6, 7, 8, 9, 17, 18):
            assert torch.equal(r_now[i], w[i])
