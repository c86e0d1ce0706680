"""The example of a recurrent student: norms, scans and losses together with packed linear layers (marker gpu).

The reference is the same model in 64 bits on the CPU, made of the oracle's formulas, with rounding passed straight through as the packed
layers do.  In float32 both round the same numbers to 4 and 8 bits, but for such as lie within 2^-20 of a tie: one in 10^4 or fewer of the
10^4 values that are rounded here, each of which moves an entry of a row by a quarter at most.  With ten of them results move by
(1/4) sqrt(10 / 10^4) < 1 % of their norm, which is the bound; a wrong or a missing term moves them by all of it.
"""
import numpy as np
import pytest

from oracle import layers as ol, rows as o

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Linear:
    def __init__(self, l):
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        self.w, self.b = ol.kept("fp4", f(l.weight)), f(l.bias)

    def forward(self, x):
        return ol.kept("fp4", x) @ self.w.T + self.b

    def backward(self, dy, kept):
        self.dw, self.db = dy.T @ kept, dy.sum(0)
        return dy @ self.w


def near(got, want):
    got = got.double().cpu().numpy() if hasattr(got, "cpu") else got
    assert got.shape == want.shape and np.linalg.norm(got - want) <= 0.01 * np.linalg.norm(want)


def test_distillation_step():
    """Logits, losses and every gradient of a step."""
    import torch
    from examples.recurrent_student import Student
    vocab, width, rows, top = 300, 64, 70, 12
    student = Student(vocab, width, 2, torch.float32, rows, seed=5)
    rng = np.random.default_rng(1)
    starts = [0, 11, 50, 70]
    for part in [b.norm for b in student.blocks] + [student.norm]:
        part.gain.copy_(torch.from_numpy(1 + rng.standard_normal(width) * 0.1))
    tokens = torch.from_numpy(rng.integers(0, vocab, rows).astype(np.int32)).cuda()
    ts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    teacher = rng.standard_normal((rows, vocab)) * 2
    index = np.argsort(-teacher, 1)[:, :top].astype(np.int32)
    value = np.take_along_axis(o.log_softmax(teacher)[0], index, 1).astype(np.float32)
    weight = (rng.random(rows) + 0.5).astype(np.float32)
    logits, _ = student.forward(tokens, ts)
    loss = student.distill(tokens, ts, torch.from_numpy(index).cuda(), torch.from_numpy(value).cuda(), torch.from_numpy(weight).cuda())

    x = student.embedding.double().cpu().numpy()[tokens.cpu().numpy()]
    s, kept, layers = np.zeros_like(x), [], []
    for b in student.blocks:
        gate, val, out = Linear(b.gate), Linear(b.value), Linear(b.out)
        gain = b.norm.gain.double().cpu().numpy()
        s, inv, y = o.norm_forward(x, s, gain, EPS)
        g, v = gate.forward(y), val.forward(y)
        h = o.scan_forward(g, v, starts, None)[0]
        x = out.forward(h)
        kept.append((ol.kept("int8", s), inv, ol.kept("int8", y), g, v, ol.kept("int8", h), gain))
        layers.append((gate, val, out))
    head, gain = Linear(student.head), student.norm.gain.double().cpu().numpy()
    s, inv, y = o.norm_forward(x, s, gain, EPS)
    z = head.forward(y)
    near(logits, z)
    want, dz = o.distill("rest", z, 1.0, index, value.astype(np.float64), weight.astype(np.float64))
    near(loss, want)
    dx, dgain = o.norm_backward(head.backward(dz, ol.kept("int8", y)), ol.kept("int8", s), inv, gain, None, None)
    near(student.norm.grad, dgain)
    near(student.head.grad, head.dw)
    near(student.head.bias_grad, head.db)
    for b, (s8, inv, y8, g, v, h8, gain), (gate, val, out) in reversed(list(zip(student.blocks, kept, layers))):
        dh = out.backward(dx, h8)
        dg, dv, _, _ = o.scan_backward(dh, g, v, starts, None, None)
        dx, dgain = o.norm_backward(gate.backward(dg, y8) + val.backward(dv, y8), s8, inv, gain, dx, None)
        for got, ref in ((b.norm.grad, dgain), (b.gate.grad, gate.dw), (b.value.grad, val.dw), (b.out.grad, out.dw), (b.gate.bias_grad, gate.db)):
            near(got, ref)
    de = np.zeros((vocab, width))
    np.add.at(de, tokens.cpu().numpy(), dx)
    near(student.embedding_grad, de)


def test_token_by_token():
    """Asked token by token, with states in a pool's slots, it gives the logits that it gives for whole sequences.  (Of the last token of each: the
    bound is the one above, since both ways round x to 4 bits.)"""
    import torch
    from examples.recurrent_student import Student
    student = Student(200, 64, 2, torch.float32, 64, seed=6)
    rng = np.random.default_rng(2)
    length, n = 16, 4
    tokens = torch.from_numpy(rng.integers(0, 200, n * length).astype(np.int32)).cuda()
    starts = (torch.arange(n + 1, dtype=torch.int32) * length).cuda()
    whole, _ = student.forward(tokens, starts)
    states, slots = student.states(9), torch.tensor([7, 0, 3, 5], dtype=torch.int32, device="cuda")
    for t in range(length):
        logits = student.step(tokens.view(n, length)[:, t].contiguous(), slots, states)
        near(logits, whole.view(n, length, -1)[:, t].double().cpu().numpy())
    index, logp = student.alternatives(logits, 5)
    ref = torch.log_softmax(logits.double(), 1)
    assert torch.equal(index.long(), torch.topk(ref, 5).indices) and (logp - torch.topk(ref, 5).values).abs().max() < 1e-5


def test_command(capsys):
    from examples import recurrent_student
    recurrent_student.main(["--vocab", "1000", "--width", "128", "--blocks", "2", "--tokens", "256", "--sequences", "3", "--steps", "2"])
    said = capsys.readouterr().out
    assert "step 1" in said and "token 3" in said and "nan" not in said
