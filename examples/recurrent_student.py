"""A student with gated recurrences, distilled from a teacher's top alternatives, and then asked token by token.

A block norms the stream, makes gates and values of it with packed linear layers, mixes the tokens of every sequence with the
gated recurrence and adds the result to the stream.  The first stage of a pipeline would hold the embedding, the last one the
head and the loss; what a block keeps of a microbatch until its backward pass is in 8 bits (and the states of every 16th token).

    python examples/recurrent_student.py [--vocab 32768] [--width 1024] [--blocks 4] [--tokens 4096] [--sequences 8] [--top 20] [--steps 5] [--rate 100]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.packed_stage import PackedLinear  # noqa: E402
from paper_2204_10562_amd import layer as pp  # noqa: E402

EPS = 1e-5


class Norm:
    """y = s gain / sqrt(mean s^2 + eps) of s = x + res; the gain's gradient is added up over microbatches."""

    def __init__(self, width, dtype, rows):
        self.gain, self.grad = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        self.workspace = torch.empty(pp.pp_norm_workspace_bytes(dtype, rows, width), dtype=torch.uint8, device="cuda")

    def forward(self, x, res):
        """(y, s, what backward needs: y and s in 8 bits, 1 / root of every row)"""
        y, total, inv = torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape[0], device="cuda")
        y_kept, s_kept = (pp.empty_packed(pp.PP_PACK_INT8, *x.shape) for _ in range(2))
        pp.pp_norm_forward(x, res, self.gain, EPS, total, y, y_kept, s_kept, inv)
        return y, total, dict(y=y_kept, s=s_kept, inv=inv)

    def backward(self, dy, dtotal, kept):
        """The gradient of x, and of res."""
        dx = torch.empty_like(dy)
        pp.pp_norm_backward(dy, kept["s"], kept["inv"], self.gain, dtotal, dx, self.grad, self.grad, self.workspace)
        return dx

    def update(self, rate):
        self.gain.add_(self.grad, alpha=-rate)
        self.grad.zero_()


class RecurrentBlock:
    """x and the stream in, what is to be added to the stream and the stream out."""

    def __init__(self, width, dtype, rows, generator):
        self.norm = Norm(width, dtype, rows)
        self.gate, self.value, self.out = (PackedLinear(width, width, generator) for _ in range(3))
        self.gate.bias.copy_(torch.linspace(-1, 5, width, device="cuda"))      # from a few tokens' memory to a hundred's
        self.parts = (self.norm, self.gate, self.value, self.out)
        sizes = [l.workspace_bytes(dtype, rows) for l in (self.gate, self.value, self.out)]
        sizes += [pp.pp_scan_workspace_bytes(c, dtype, rows, width) for c in (pp.PP_SCAN_FORWARD, pp.PP_SCAN_BACKWARD)]
        self.workspace = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")

    def forward(self, x, stream, starts):
        rows, width = x.shape
        y, stream, kept = self.norm.forward(x, stream)
        gate, value = self.gate.forward(y, None, self.workspace), self.value.forward(y, None, self.workspace)
        h, states = torch.empty_like(x), torch.empty(pp.pp_scan_kept_rows(x.dtype, rows, width), width, device="cuda")
        pp.pp_scan_forward(gate, value, starts, None, h, None, states, self.workspace)
        kept.update(h=pp.empty_packed(pp.PP_PACK_INT8, rows, width), gate=gate, value=value, states=states)
        return self.out.forward(h, kept["h"], self.workspace), stream, kept

    def backward(self, dout, dstream, kept, starts):
        """The gradient of x, and of the stream that came in."""
        dh = self.out.backward(dout, kept["h"], self.workspace)
        dgate, dvalue = torch.empty_like(dh), torch.empty_like(dh)
        pp.pp_scan_backward(dh, kept["gate"], kept["value"], starts, None, kept["states"], None, dgate, dvalue, None, self.workspace)
        dy = self.gate.backward(dgate, kept["y"], self.workspace) + self.value.backward(dvalue, kept["y"], self.workspace)
        return self.norm.backward(dy, dstream, kept)

    def step(self, x, stream, slots, state):
        """One token of each of x.shape[0] sequences, whose states lie in these slots."""
        total, y, h = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        pp.pp_norm_forward(x, stream, self.norm.gain, EPS, total, y)
        pp.pp_scan_step(self.gate.forward(y, None, self.workspace), self.value.forward(y, None, self.workspace), slots, state, h)
        return self.out.forward(h, None, self.workspace), total


class Student:
    """For microbatches of `rows` tokens or fewer."""

    def __init__(self, vocab, width, blocks, dtype, rows, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.width, self.dtype, self.rows = vocab, width, dtype, rows
        self.embedding = torch.randn(vocab, width, generator=g, device="cuda")
        self.embedding_grad = torch.zeros_like(self.embedding)
        self.blocks = [RecurrentBlock(width, dtype, rows, g) for _ in range(blocks)]
        self.norm, self.head = Norm(width, dtype, rows), PackedLinear(width, vocab, g)
        self.workspace = torch.empty(self.head.workspace_bytes(dtype, rows), dtype=torch.uint8, device="cuda")

    def forward(self, tokens, starts):
        """(logits, what backward needs)"""
        x = self.embedding[tokens.long()].to(self.dtype)
        stream, kept = torch.zeros_like(x), []
        for b in self.blocks:
            x, stream, k = b.forward(x, stream, starts)
            kept.append(k)
        y, _, k = self.norm.forward(x, stream)
        return self.head.forward(y, None, self.workspace), kept + [k]

    def backward(self, dlogits, tokens, starts, kept):
        dx = self.norm.backward(self.head.backward(dlogits, kept[-1]["y"], self.workspace), None, kept[-1])
        for b, k in zip(reversed(self.blocks), reversed(kept[:-1])):
            dx = b.backward(dx, dx, k, starts)
        self.embedding_grad.index_add_(0, tokens.long(), dx.float())

    def alternatives(self, logits, top):
        """(columns, log probabilities) of the top alternatives of every row: what a teacher gives, and a server."""
        rows = logits.shape[0]
        index, logp = torch.empty(rows, top, dtype=torch.int32, device="cuda"), torch.empty(rows, top, device="cuda")
        ws = torch.empty(pp.pp_logprob_workspace_bytes(logits.dtype, rows, self.vocab, top), dtype=torch.uint8, device="cuda")
        pp.pp_logprob_forward(logits, 1.0, None, None, None, None, index, logp, ws)
        return index, logp

    def distill(self, tokens, starts, index, logp, weight):
        """The loss of every token, its gradients added to; logits and their gradient share their memory."""
        logits, kept = self.forward(tokens, starts)
        loss = torch.empty(logits.shape[0], device="cuda")
        ws = torch.empty(pp.pp_distill_workspace_bytes(logits.dtype, *logits.shape, index.shape[1]), dtype=torch.uint8, device="cuda")
        pp.pp_distill_loss(pp.PP_DISTILL_REST, logits, 1.0, index, logp, weight, loss, logits, ws)
        self.backward(logits, tokens, starts, kept)
        return loss

    def states(self, slots):
        return [torch.zeros(slots, self.width, device="cuda") for _ in self.blocks]

    def step(self, tokens, slots, states):
        """Logits behind one more token of each sequence."""
        x = self.embedding[tokens.long()].to(self.dtype)
        stream = torch.zeros_like(x)
        for b, s in zip(self.blocks, states):
            x, stream = b.step(x, stream, slots, s)
        y = torch.empty_like(x)
        pp.pp_norm_forward(x, stream, self.norm.gain, EPS, None, y)
        return self.head.forward(y, None, self.workspace)

    def update(self, rate):
        for part in [p for b in self.blocks for p in b.parts] + [self.norm, self.head]:
            part.update(rate)
        self.embedding.add_(self.embedding_grad, alpha=-rate)
        self.embedding_grad.zero_()


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--vocab", type=int, default=32768)
    p.add_argument("--width", type=int, default=1024)
    p.add_argument("--blocks", type=int, default=4)
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--sequences", type=int, default=8)
    p.add_argument("--top", type=int, default=20)
    p.add_argument("--steps", type=int, default=5)
    p.add_argument("--rate", type=float, default=100.0)
    p.add_argument("--type", choices=("bf16", "f32"), default="bf16")
    a = p.parse_args(argv)
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[a.type]
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(0, a.vocab, (a.tokens,), generator=g, device="cuda", dtype=torch.int32)
    starts = torch.linspace(0, a.tokens, a.sequences + 1).to(torch.int32).cuda()
    teacher, student = (Student(a.vocab, a.width, a.blocks, dtype, a.tokens, seed) for seed in (2, 3))
    index, logp = teacher.alternatives(teacher.forward(tokens, starts)[0], a.top)
    weight = torch.full((a.tokens,), 1.0 / a.tokens, device="cuda")
    for k in range(a.steps):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        loss = student.distill(tokens, starts, index, logp, weight)
        student.update(a.rate)
        end.record()
        end.synchronize()
        print("step %d: divergence %.4f, %.2f ms" % (k, loss.sum().item(), start.elapsed_time(end)))
    states, slots = student.states(a.sequences), torch.arange(a.sequences, dtype=torch.int32, device="cuda")
    ask = tokens[starts[:-1].long()]
    for k in range(4):
        best, value = student.alternatives(student.step(ask, slots, states), 3)
        print("token %d: %s" % (k, ", ".join("%d (%.2f)" % v for v in zip(best[0].tolist(), value[0].tolist()))))
        ask = best[:, 0].contiguous()


if __name__ == "__main__":
    main()
