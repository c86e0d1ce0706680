"""The layer operators on a stream of their own behind pending work, and in a recorded graph (marker gpu)."""
import pytest

pytestmark = pytest.mark.gpu


class Layer:
    """One linear layer with its activation: buffers of fixed places, and a pass over all of them."""

    def __init__(self, rows, n_in, n_out, dtype):
        import torch
        from paper_2204_10562_amd import layer as pp
        self.pp, self.rows, self.dtype = pp, rows, dtype
        new = lambda r, c, t=dtype: torch.zeros(r, c, dtype=t, device="cuda")  # noqa: E731
        self.x, self.dy = new(rows, n_in), new(rows, n_out)
        self.y, self.a, self.da, self.dx = new(rows, n_out), new(rows, n_out), new(rows, n_out), new(rows, n_in)
        self.back = new(rows, n_in)
        self.weight, self.bias, self.dw, self.db = new(n_out, n_in, torch.float32), new(1, n_out, torch.float32)[0], new(n_out, n_in, torch.float32), new(1, n_out, torch.float32)[0]
        self.w = pp.empty_packed(1, n_out, n_in)
        self.xk, self.yk = pp.empty_packed(0, rows, n_in), pp.empty_packed(0, rows, n_out)
        self.ws = [torch.zeros(pp.pp_linear_workspace_bytes(c, dtype, rows, n_in, n_out), dtype=torch.uint8, device="cuda") for c in (0, 1, 2)]

    def fill(self, seed):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        for t in (self.x, self.dy, self.weight, self.bias):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    def step(self):
        pp = self.pp
        pp.pp_pack(pp.PP_PACK_FP4, self.weight, self.w)
        pp.pp_linear_forward(self.x, self.w, self.bias, self.y, self.xk, self.ws[0])
        pp.pp_act_forward(pp.PP_ACT_GELU, self.y, None, self.a, self.yk)
        pp.pp_act_backward(pp.PP_ACT_GELU, self.dy, self.yk, None, self.da)
        pp.pp_linear_backward_input(self.da, self.w, self.dx, self.ws[1])
        pp.pp_linear_backward_weight(self.da, self.xk, None, self.dw, self.db, self.ws[2])
        pp.pp_unpack(pp.PP_PACK_INT8, self.xk, self.back)

    def results(self):
        return [t.clone() for t in (self.y, self.a, self.da, self.dx, self.dw, self.db, self.back)]


SIZES = [(3, 200, 300), (40, 520, 600), (300, 1000, 700), (2000, 264, 130)]


@pytest.mark.parametrize("rows, n_in, n_out", SIZES)
@pytest.mark.parametrize("t", ["bfloat16", "float16", "float32"])
def test_behind_pending_work(t, rows, n_in, n_out):
    import torch
    one = Layer(rows, n_in, n_out, getattr(torch, t))
    one.fill(51)
    one.step()
    want = one.results()
    torch.cuda.synchronize()
    busy = torch.randn(2048, 2048, device="cuda")
    side = torch.cuda.Stream()
    one.fill(52)                       # other values, until the side stream puts the first ones back
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy * 1e-3
        one.fill(51)
        one.step()
        got = one.results()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows, n_in, n_out", SIZES)
def test_recorded(rows, n_in, n_out):
    import torch
    one = Layer(rows, n_in, n_out, torch.float16)
    one.fill(61)
    one.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step()
    for seed in (62, 63, 64, 65):
        one.fill(seed)
        one.step()
        want = one.results()
        for b in one.ws:
            b.fill_(255)               # what a workspace holds does not matter
        one.fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(one.results(), want)), seed
