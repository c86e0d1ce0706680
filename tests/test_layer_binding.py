"""What the layer operators' binding refuses before the library is called (no GPU needed: operands are stand-ins)."""
import subprocess
import sys

import pytest
import torch

from conftest import ROOT


class Operand:
    """What the binding looks at of a tensor, without one."""

    def __init__(self, shape, dtype, device=0, stride=None):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, device
        self._stride = stride or tuple(torch.empty(shape, device="meta").stride())
        self.is_cuda, self.requires_grad = device >= 0, False

    def get_device(self):
        return self.device

    def stride(self):
        return self._stride

    def data_ptr(self):
        return 4096

    def is_contiguous(self):
        return self._stride == tuple(torch.empty(self.shape, device="meta").stride())

    def numel(self):
        return self.shape.numel()


class Library:
    """Notes the calls that get as far as the library."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def pp(monkeypatch):
    from paper_2204_10562_amd import layer
    library = Library()
    monkeypatch.setattr(layer, "lib", lambda: library)
    monkeypatch.setattr(layer, "_device", lambda: 0)
    monkeypatch.setattr(layer, "_raw_stream", lambda dev: 16 * (dev + 1))
    layer_calls = library.calls
    yield layer, layer_calls


ROWS, N_IN, N_OUT = 4, 200, 70


def operands():
    """Every entry point's arguments by name; those that are operands can be moved to another device one by one."""
    bf, f32 = torch.bfloat16, torch.float32

    def packed(fmt, rows, cols):
        g = -(-cols // 128)
        return (Operand((rows, g, 64 if fmt else 128), torch.uint8 if fmt else torch.int8), Operand((rows, g, 4), torch.uint8))
    x, y, w = (lambda: Operand((ROWS, N_IN), bf)), (lambda: Operand((ROWS, N_OUT), bf)), (lambda: packed(1, N_OUT, N_IN))
    dw, b, ws = (lambda: Operand((N_OUT, N_IN), f32)), (lambda: Operand((N_OUT,), f32)), (lambda: Operand((1 << 20,), torch.uint8))
    k = lambda: packed(0, ROWS, N_IN)  # noqa: E731
    return {"pp_pack": [0, x(), k()], "pp_unpack": [0, k(), x()], "pp_act_forward": [2, x(), x(), x(), k(), k()],
            "pp_act_backward": [2, x(), k(), k(), x(), x()], "pp_linear_forward": [x(), w(), b(), y(), k(), ws()],
            "pp_linear_backward_input": [y(), w(), x(), ws()], "pp_linear_backward_weight": [y(), k(), dw(), dw(), b(), ws()]}


@pytest.mark.parametrize("name", list(operands()))
def test_operands_on_another_device(pp, name):
    layer, calls = pp
    args = operands()[name]
    getattr(layer, name)(*args)
    assert len(calls) == 1 and calls[0][0] == name and calls[0][1][-1] == 16      # device 0's stream
    parts = [o for a in args for o in (a if isinstance(a, tuple) else (a,)) if isinstance(o, Operand)]
    for device in (1, -1):                                                      # another GPU, the host
        for o in parts:
            o.device, o.is_cuda = device, device >= 0
            with pytest.raises(ValueError):
                getattr(layer, name)(*args)
            o.device, o.is_cuda = 0, True
    for o in parts:                                                             # all on a GPU that is not the current one
        o.device = 1
    with pytest.raises(ValueError):
        getattr(layer, name)(*args)
    assert len(calls) == 1


@pytest.mark.parametrize("name", list(operands()))
def test_operands_that_require_a_gradient(pp, name):
    """Refused in grad mode, where the result would lack its history, and taken without."""
    layer, calls = pp
    args = operands()[name]
    parts = [o for o in args if isinstance(o, Operand) and o.dtype.is_floating_point]
    assert parts
    for o in parts:
        o.requires_grad = True
        if name == "pp_pack":      # whole numbers have no gradient: a parameter is packed as it is
            getattr(layer, name)(*args)
            assert len(calls) == 1
            calls.clear()
            continue
        with pytest.raises(ValueError, match="autograd"):
            getattr(layer, name)(*args)
        assert not calls
        with torch.no_grad():
            getattr(layer, name)(*args)
        assert len(calls) == 1
        calls.clear()
        o.requires_grad = False
    getattr(layer, name)(*args)
    assert len(calls) == 1


def test_row_stride_of_one_row(pp):
    """dw_in and dw have the same distance between their rows; one row has none."""
    layer, calls = pp
    kept = (Operand((ROWS, 2, 128), torch.int8), Operand((ROWS, 2, 4), torch.uint8))
    ws = Operand((1 << 20,), torch.uint8)
    for rows, right in ((1, True), (2, False)):
        dy, dw_in, dw = Operand((ROWS, rows), torch.bfloat16), Operand((rows, N_IN), torch.float32, stride=(N_IN + 8, 1)), Operand((rows, N_IN), torch.float32)
        if right:
            layer.pp_linear_backward_weight(dy, kept, dw_in, dw, None, ws)
            assert len(calls) == 1
        else:
            with pytest.raises(ValueError):
                layer.pp_linear_backward_weight(dy, kept, dw_in, dw, None, ws)


def test_torch_without_raw_streams():
    """A torch that lacks the name by which it gives a stream without its object: the public way, not a failing import."""
    code = ("import torch\nvars(torch._C).pop('_cuda_getCurrentRawStream', None)\nfrom paper_2204_10562_amd import layer\n"
            "assert layer._raw_stream is layer._public_stream")
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-2000:]


@pytest.mark.gpu
def test_both_ways_give_one_stream():
    from paper_2204_10562_amd import layer
    for s in (torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(s):
            assert layer._stream(0) == layer._public_stream(0) == s.cuda_stream
