"""A feed-forward block of packed layers, measured and planned.

A stage of a synchronous pipeline keeps the activations of every microbatch in flight until its
backward pass, and sends one to the next stage per microbatch.  Here a gated block holds what it
keeps in 8 bits, multiplies in 4, and sends its output in 8; its measured times and the bytes that
cross a cut then go to the planner in the place of the workload's drawn ones.

    python examples/packed_stage.py [--rows 2048] [--width 4096] [--hidden 16384] [--layers 128] [--type bf16]
"""
import argparse
import os
import sys
from dataclasses import replace

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2204_10562_amd import layer as pp, workloads  # noqa: E402
from paper_2204_10562_amd.problem import GpuProblem  # noqa: E402


class PackedLinear:
    """A linear layer: weight in 32 bits for the optimiser, in 4 for the products; gradients added up over microbatches."""

    def __init__(self, n_in, n_out, generator):
        self.weight = torch.randn(n_out, n_in, generator=generator, device="cuda") * n_in ** -0.5
        self.bias = torch.zeros(n_out, device="cuda")
        self.grad, self.bias_grad, self.bias_part = torch.zeros_like(self.weight), torch.zeros_like(self.bias), torch.empty_like(self.bias)
        self.packed = pp.empty_packed(pp.PP_PACK_FP4, n_out, n_in)
        pp.pp_pack(pp.PP_PACK_FP4, self.weight, self.packed)

    def workspace_bytes(self, dtype, rows):
        n_out, n_in = self.weight.shape
        return max(pp.pp_linear_workspace_bytes(call, dtype, rows, n_in, n_out)
                   for call in (pp.PP_LINEAR_FORWARD, pp.PP_LINEAR_BACKWARD_INPUT, pp.PP_LINEAR_BACKWARD_WEIGHT))

    def forward(self, x, kept, workspace):
        y = torch.empty(x.shape[0], self.weight.shape[0], dtype=x.dtype, device="cuda")
        pp.pp_linear_forward(x, self.packed, self.bias, y, kept, workspace)
        return y

    def backward(self, dy, kept, workspace):
        """dx; the weight's and the bias's gradients are added to."""
        dx = torch.empty(dy.shape[0], self.weight.shape[1], dtype=dy.dtype, device="cuda")
        pp.pp_linear_backward_input(dy, self.packed, dx, workspace)
        pp.pp_linear_backward_weight(dy, kept, self.grad, self.grad, self.bias_part, workspace)
        self.bias_grad += self.bias_part
        return dx

    def update(self, rate):
        self.weight.add_(self.grad, alpha=-rate)
        self.bias.add_(self.bias_grad, alpha=-rate)
        pp.pp_pack(pp.PP_PACK_FP4, self.weight, self.packed)
        self.grad.zero_()
        self.bias_grad.zero_()


class PackedBlock:
    """y = down(silu(gate(x)) * up(x)), for microbatches of `rows` rows or fewer.  forward gives y and what backward needs of this
    microbatch: four packed matrices."""

    def __init__(self, width, hidden, rows, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.width, self.hidden = width, hidden
        self.gate, self.up, self.down = PackedLinear(width, hidden, g), PackedLinear(width, hidden, g), PackedLinear(hidden, width, g)
        self.layers = (self.gate, self.up, self.down)
        self.workspace = torch.empty(max(l.workspace_bytes(dtype, rows) for l in self.layers), dtype=torch.uint8, device="cuda")

    def forward(self, x):
        rows = x.shape[0]
        kept = {name: pp.empty_packed(pp.PP_PACK_INT8, rows, cols)
                for name, cols in (("x", self.width), ("gate", self.hidden), ("up", self.hidden), ("h", self.hidden))}
        a, u = self.gate.forward(x, kept["x"], self.workspace), self.up.forward(x, None, self.workspace)
        h = torch.empty_like(a)
        pp.pp_act_forward(pp.PP_ACT_SILU, a, u, h, kept["gate"], kept["up"])
        return self.down.forward(h, kept["h"], self.workspace), kept

    def backward(self, dy, kept):
        dh = self.down.backward(dy, kept["h"], self.workspace)
        da, du = torch.empty_like(dh), torch.empty_like(dh)
        pp.pp_act_backward(pp.PP_ACT_SILU, dh, kept["gate"], kept["up"], da, du)
        return self.gate.backward(da, kept["x"], self.workspace) + self.up.backward(du, kept["x"], self.workspace)

    def update(self, rate):
        for l in self.layers:
            l.update(rate)

    def kept_bytes(self, rows):
        return pp.packed_bytes(pp.PP_PACK_INT8, rows, self.width) + 3 * pp.packed_bytes(pp.PP_PACK_INT8, rows, self.hidden)


def send(y):
    """What crosses a cut: y in 8 bits."""
    packed = pp.empty_packed(pp.PP_PACK_INT8, *y.shape)
    pp.pp_pack(pp.PP_PACK_INT8, y, packed)
    return packed


def receive(packed, rows, cols, dtype):
    x = torch.empty(rows, cols, dtype=dtype, device="cuda")
    pp.pp_unpack(pp.PP_PACK_INT8, packed, x)
    return x


def microseconds(call, times=10):
    """Mean time of a call on the GPU."""
    call()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(times):
        call()
    end.record()
    end.synchronize()
    return start.elapsed_time(end) * 1000 / times


def measure(width, hidden, rows, dtype):
    """(forward us, backward us, bytes that cross a cut forward, and backward) of a block, arrival and sending included."""
    block = PackedBlock(width, hidden, rows, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    arrived = send(torch.randn(rows, width, generator=g, device="cuda").to(dtype))
    dy = torch.randn(rows, width, generator=g, device="cuda").to(dtype) / rows
    kept = block.forward(receive(arrived, rows, width, dtype))[1]
    forward = microseconds(lambda: send(block.forward(receive(arrived, rows, width, dtype))[0]))
    backward = microseconds(lambda: block.backward(dy, kept))
    return forward, backward, pp.packed_bytes(pp.PP_PACK_INT8, rows, width), rows * width * dy.element_size()


def plan(forward, backward, sent, returned, layers=None):
    """The GPT-shaped workload's devices and orderings with these times and bytes for every layer: (workload, winners)."""
    w = workloads.gpt()
    n = w.L if layers is None else layers
    full = lambda v: np.full(n, max(1, int(round(v))), np.int64)  # noqa: E731
    w = replace(w, name="packed", L=n, fwd=full(forward), bwd=full(backward), actf=full(sent), actb=full(returned))
    g = GpuProblem(w)
    assert g.prefix() == 0
    status, winners, _, _ = g.best_multi(w.Ms)
    assert status == 0
    return w, winners


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--rows", type=int, default=2048, help="tokens of a microbatch")
    p.add_argument("--width", type=int, default=4096)
    p.add_argument("--hidden", type=int, default=16384)
    p.add_argument("--layers", type=int, default=128)
    p.add_argument("--type", choices=("bf16", "f16", "f32"), default="bf16")
    a = p.parse_args(argv)
    dtype = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[a.type]
    forward, backward, sent, returned = measure(a.width, a.hidden, a.rows, dtype)
    flops = 6.0 * a.rows * a.width * a.hidden
    print("block %d -> %d, %d rows, %s: forward %.0f us (%.0f TFLOP/s), backward %.0f us (%.0f TFLOP/s)"
          % (a.width, a.hidden, a.rows, a.type, forward, flops / forward / 1e6, backward, 2 * flops / backward / 1e6))
    w, packed = plan(forward, backward, sent, returned, a.layers)
    _, whole = plan(forward, backward, returned, returned, a.layers)
    for M, q, v in zip(w.Ms, packed, whole):
        print("M = %2d: iteration %.1f ms, devices %s, stages end at %s (activations sent whole: %.1f ms)"
              % (M, q["T"] / 1e3, q["order"], q["bounds"], v["T"] / 1e3))


if __name__ == "__main__":
    main()
