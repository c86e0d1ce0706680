"""What the binding of norms, scans and losses refuses before the library is called (no GPU needed: operands are stand-ins)."""
import pytest
import torch

from test_layer_binding import Operand, pp  # noqa: F401  (the fixture)

ROWS, COLS, TOP, SEQS = 4, 200, 5, 3


def operands():
    """Every entry point's arguments; those that are operands can be moved to another device one by one."""
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    m, v, c = (lambda: Operand((ROWS, COLS), bf)), (lambda: Operand((ROWS,), f32)), (lambda: Operand((COLS,), f32))
    k = lambda: (Operand((ROWS, 2, 128), torch.int8), Operand((ROWS, 2, 4), torch.uint8))  # noqa: E731
    ws, tok = (lambda: Operand((1 << 20,), torch.uint8)), (lambda: Operand((ROWS,), i32))
    starts, state, kept = (lambda: Operand((SEQS + 1,), i32)), (lambda: Operand((SEQS, COLS), f32)), (lambda: Operand((0, COLS), f32))
    index, value = (lambda: Operand((ROWS, TOP), i32)), (lambda: Operand((ROWS, TOP), f32))
    return {"pp_norm_forward": [m(), m(), c(), 1e-5, m(), m(), k(), k(), v()], "pp_norm_backward": [m(), k(), v(), c(), m(), m(), c(), c(), ws()],
            "pp_scan_forward": [m(), m(), starts(), state(), m(), state(), kept(), ws()],
            "pp_scan_backward": [m(), m(), m(), starts(), state(), kept(), state(), m(), m(), state(), ws()],
            "pp_scan_step": [m(), m(), tok(), Operand((9, COLS), f32), m()],
            "pp_logprob_forward": [m(), 1.0, tok(), v(), v(), Operand((ROWS, 2), f32), index(), value(), ws()],
            "pp_logprob_backward": [m(), 1.0, tok(), Operand((ROWS, 2), f32), v(), v(), v(), m()],
            "pp_distill_loss": [1, m(), 1.0, index(), value(), v(), v(), m(), ws()]}


def parts_of(args):
    return [o for a in args for o in (a if isinstance(a, tuple) else (a,)) if isinstance(o, Operand)]


def made(calls, name):
    """The calls of this entry point (the size of a kept state is asked of the library too)."""
    return [c for c in calls if c[0] == name]


@pytest.fixture(autouse=True)
def dims(monkeypatch):
    monkeypatch.setattr(Operand, "dim", lambda self: len(self.shape), raising=False)


@pytest.mark.parametrize("name", list(operands()))
def test_operands_on_another_device(pp, name):  # noqa: F811
    layer, calls = pp
    args = operands()[name]
    getattr(layer, name)(*args)
    assert len(made(calls, name)) == 1 and made(calls, name)[0][1][-1] == 16      # device 0's stream
    for device in (1, -1):
        for o in parts_of(args):
            o.device, o.is_cuda = device, device >= 0
            with pytest.raises(ValueError):
                getattr(layer, name)(*args)
            o.device, o.is_cuda = 0, True
    for o in parts_of(args):
        o.device = 1
    with pytest.raises(ValueError):
        getattr(layer, name)(*args)
    assert len(made(calls, name)) == 1


@pytest.mark.parametrize("name", list(operands()))
def test_operands_of_another_shape_or_type(pp, name):  # noqa: F811
    layer, calls = pp
    args = operands()[name]
    for o in parts_of(args):
        if o.dtype is torch.uint8 and len(o.shape) == 1:       # a workspace may be of any size
            continue
        shape, dtype, stride = o.shape, o.dtype, o._stride
        o.dtype = torch.float64
        with pytest.raises(ValueError):
            getattr(layer, name)(*args)
        o.dtype = dtype
        if o is parts_of(args)[0]:
            continue                                           # sets the sizes of the others
        if not (name == "pp_scan_step" and shape[0] == 9):     # (a pool may have any number of slots)
            o.shape = torch.Size((shape[0] + 1,) + tuple(shape[1:]))
            with pytest.raises(ValueError):
                getattr(layer, name)(*args)
        o.shape = shape
        if len(shape) == 2 and dtype is torch.bfloat16:
            o._stride = (COLS, 2)                              # rows that are not consecutive values
        elif len(shape) == 2:
            o._stride = (shape[1] + 1, 1)                      # floats with room between their rows
        else:
            continue
        if shape[0] > 0:
            with pytest.raises(ValueError):
                getattr(layer, name)(*args)
        o._stride = stride
    getattr(layer, name)(*args)
    assert len(made(calls, name)) == 1


@pytest.mark.parametrize("name", list(operands()))
def test_operands_that_require_a_gradient(pp, name):  # noqa: F811
    layer, calls = pp
    args = operands()[name]
    for o in [o for o in parts_of(args) if o.dtype.is_floating_point]:
        o.requires_grad = True
        with pytest.raises(ValueError, match="autograd"):
            getattr(layer, name)(*args)
        assert not made(calls, name)
        with torch.no_grad():
            getattr(layer, name)(*args)
        assert len(made(calls, name)) == 1
        calls.clear()
        o.requires_grad = False


def test_what_may_be_left_out(pp):  # noqa: F811
    layer, calls = pp
    o = operands()
    for name, optional in (("pp_norm_forward", (1, 2, 4, 6, 7, 8)), ("pp_norm_backward", (3, 4, 6)), ("pp_scan_forward", (3, 5, 6)),
                           ("pp_scan_backward", (4, 6, 9)), ("pp_scan_step", (2,)), ("pp_logprob_forward", (2, 3, 4, 5)),
                           ("pp_logprob_backward", (2, 4, 5, 6)), ("pp_distill_loss", (5, 7))):
        args = [None if i in optional else a for i, a in enumerate(o[name])]
        getattr(layer, name)(*args)
        assert len(made(calls, name)) == 1
    one = list(o["pp_scan_forward"])
    one[2], one[3], one[5] = None, None, None      # one sequence of all rows
    layer.pp_scan_forward(*one)
    assert made(calls, "pp_scan_forward")[-1][1][7:9] == (1, None)
    lone = list(o["pp_logprob_forward"])
    lone[6] = None
    with pytest.raises(ValueError):
        layer.pp_logprob_forward(*lone)
    bad = list(o["pp_scan_forward"])
    bad[2] = Operand((0,), torch.int32)
    with pytest.raises(ValueError):
        layer.pp_scan_forward(*bad)
