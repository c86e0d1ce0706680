"""Python binding of the layer operators of libpp (include/pp_layer.h): argument marshalling only.

As in `binding`, every function takes torch tensors that already live on the GPU (all of a call on
the current device), checks dtype, device, shape and strides, and passes raw pointers plus the
current HIP stream to the C entry point of the same name; outputs and workspaces are the caller's.  A matrix is a tensor of two
dimensions whose rows are consecutive values (stride(1) == 1); a packed matrix is the pair
(codes, scales) that `empty_packed` makes.

Autograd does not see these calls.  In grad mode an operand that requires a gradient is refused (but for
pp_pack, whose results are whole numbers); the backward operators give the gradients, of which a torch.autograd.Function can be made.  A buffer that
autograd has saved must not be written to by a later call: its version does not change.
"""
import ctypes

import torch

from . import binding
from .binding import PP_OK, PPError  # noqa: F401

PP_TYPE_F32, PP_TYPE_F16, PP_TYPE_BF16 = 0, 1, 2
PP_PACK_INT8, PP_PACK_FP4 = 0, 1
PP_ACT_GELU, PP_ACT_GELU_TANH, PP_ACT_SILU = 0, 1, 2
PP_LINEAR_FORWARD, PP_LINEAR_BACKWARD_INPUT, PP_LINEAR_BACKWARD_WEIGHT = 0, 1, 2
PP_LAYER_MAX_ROWS, PP_LAYER_MAX_COLS, PP_LAYER_MAX_LD_DW = 1 << 30, 1 << 22, 1 << 24
BLOCK, GROUP = 32, 128

EXPORTS = ("pp_pack", "pp_unpack", "pp_act_forward", "pp_act_backward", "pp_linear_workspace_bytes",
           "pp_linear_forward", "pp_linear_backward_input", "pp_linear_backward_weight")

TYPES = {torch.float32: PP_TYPE_F32, torch.float16: PP_TYPE_F16, torch.bfloat16: PP_TYPE_BF16}
_CODES = {PP_PACK_INT8: (torch.int8, GROUP), PP_PACK_FP4: (torch.uint8, GROUP // 2)}
_lib = None


def lib():
    """The loaded C library with the layer operators' signatures."""
    global _lib
    if _lib is None:
        L = binding.lib()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
        L.pp_pack.argtypes = [i32, i32, i64, i64, vp, i64, vp, vp, vp]
        L.pp_unpack.argtypes = [i32, i32, i64, i64, vp, vp, vp, i64, vp]
        L.pp_act_forward.argtypes = [i32, i32, i64, i64] + [vp, i64] * 3 + [vp] * 5
        L.pp_act_backward.argtypes = [i32, i32, i64, i64, vp, i64] + [vp] * 4 + [vp, i64] * 2 + [vp]
        L.pp_linear_workspace_bytes.argtypes = [i32, i32, i64, i64, i64]
        L.pp_linear_forward.argtypes = [i32, i64, i64, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
        L.pp_linear_backward_input.argtypes = [i32, i64, i64, i64, vp, i64, vp, vp, vp, i64, vp, sz, vp]
        L.pp_linear_backward_weight.argtypes = [i32, i64, i64, i64, vp, i64, vp, vp, vp, vp, i64, vp, vp, sz, vp]
        for name in EXPORTS:
            getattr(L, name).restype = i32
        L.pp_linear_workspace_bytes.restype = sz
        _lib = L
    return _lib


def empty_packed(fmt, rows, cols, device="cuda"):
    """Room for a packed matrix: (codes, scales)."""
    dtype, width = _CODES[fmt]
    groups = -(-cols // GROUP)
    return (torch.empty(rows, groups, width, dtype=dtype, device=device),
            torch.empty(rows, groups, 4, dtype=torch.uint8, device=device))


def packed_bytes(fmt, rows, cols):
    """Bytes of a packed matrix, codes and scales."""
    return rows * -(-cols // GROUP) * (_CODES[fmt][1] + 4)


def _public_stream(dev):
    return torch.cuda.current_stream(dev).cuda_stream


# (torch's own name for the stream without its object, which takes 3 us to make; where a torch has no such name, its public one)
_device, _raw_stream = torch.cuda.current_device, getattr(torch._C, "_cuda_getCurrentRawStream", _public_stream)


def _stream(dev):
    """The current HIP stream of device `dev`, which has to be the current one."""
    if dev != _device():
        raise ValueError("operands must be on the current device (they are on cuda:%d)" % dev)
    return _raw_stream(dev)


def _check(rc):
    if rc != PP_OK:
        raise PPError(rc)


def _no_history(name):
    """As torch's own functions with out=: what a call writes has no history, which would be gradients that are silently missing."""
    if torch.is_grad_enabled():
        raise ValueError("%s requires a gradient, and autograd does not see what the layer operators do: call them under torch.no_grad() or "
                         "with detached tensors, and their backward operators for the gradients" % name)


def _matrix(t, dtype, rows, cols, name, dev):
    """(data pointer, row stride) of a matrix on device `dev`."""
    if t.get_device() != dev or t.dtype is not dtype or t.shape != (rows, cols):
        raise ValueError("%s must be a %s matrix of %d x %d on the GPU of the other operands" % (name, dtype, rows, cols))
    if t.requires_grad:
        _no_history(name)
    return _place(t, rows, cols, name)


def _place(t, rows, cols, name):
    """(data pointer, row stride)"""
    ld, step = t.stride()
    if step != 1 and cols > 1 or ld < cols and rows > 1:
        raise ValueError("%s must have rows of consecutive values that do not overlap" % name)
    return t.data_ptr(), ld if ld > cols else cols


def _first(t, name, differentiable=True):
    """(type code, rows, cols, data pointer, row stride, device) of the matrix that sets a call's type, sizes and device;
    differentiable: of which a gradient may be asked."""
    code, shape, dev = TYPES.get(t.dtype), t.shape, t.get_device()
    if code is None or len(shape) != 2 or dev < 0:
        raise ValueError("%s must be a matrix of float32, float16 or bfloat16 on the GPU" % name)
    if differentiable and t.requires_grad:
        _no_history(name)
    rows, cols = shape
    ptr, ld = _place(t, rows, cols, name)
    return code, rows, cols, ptr, ld, dev


def _packed(pair, fmt, rows, cols, name, dev):
    """Pointers of a packed matrix of these sizes on device `dev`; None: no such matrix."""
    if pair is None:
        return None, None
    codes, scales = pair
    dtype, width = _CODES[fmt]
    groups = (cols + GROUP - 1) // GROUP
    if (codes.get_device() != dev or codes.dtype is not dtype or codes.shape != (rows, groups, width) or not codes.is_contiguous()
            or scales.get_device() != dev or scales.dtype is not torch.uint8 or scales.shape != (rows, groups, 4) or not scales.is_contiguous()):
        raise ValueError("%s must be codes %s [%d][%d][%d] and scales uint8 [%d][%d][4], contiguous on the GPU of the other operands"
                         % (name, dtype, rows, groups, width, rows, groups))
    return codes.data_ptr(), scales.data_ptr()


def _vector(t, n, name, dev):
    if t is None:
        return None
    if t.get_device() != dev or t.dtype != torch.float32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError("%s must be %d contiguous float32 values on the GPU of the other operands" % (name, n))
    if t.requires_grad:
        _no_history(name)
    return t.data_ptr()


def _workspace(t, dev):
    if t is None:
        return None, 0
    if t.get_device() != dev or t.dtype != torch.uint8 or not t.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the GPU of the other operands")
    return t.data_ptr(), t.numel()


def pp_pack(fmt, x, packed):
    type_, rows, cols, px, ld, dev = _first(x, "x", False)    # (codes are whole numbers: nothing has a gradient through them)
    codes, scales = _packed(packed, fmt, rows, cols, "packed", dev)
    _check(lib().pp_pack(fmt, type_, rows, cols, px, ld, codes, scales, _stream(dev)))


def pp_unpack(fmt, packed, out):
    type_, rows, cols, po, ld, dev = _first(out, "out")
    codes, scales = _packed(packed, fmt, rows, cols, "packed", dev)
    _check(lib().pp_unpack(fmt, type_, rows, cols, codes, scales, po, ld, _stream(dev)))


def pp_act_forward(kind, x, u, y, x_kept=None, u_kept=None):
    """u: the gate's other factor, or None."""
    type_, rows, cols, px, ldx, dev = _first(x, "x")
    pu, ldu = (None, 0) if u is None else _matrix(u, x.dtype, rows, cols, "u", dev)
    py, ldy = _matrix(y, x.dtype, rows, cols, "y", dev)
    xc, xs = _packed(x_kept, PP_PACK_INT8, rows, cols, "x_kept", dev)
    uc, us = _packed(u_kept, PP_PACK_INT8, rows, cols, "u_kept", dev)
    _check(lib().pp_act_forward(kind, type_, rows, cols, px, ldx, pu, ldu, py, ldy, xc, xs, uc, us, _stream(dev)))


def pp_act_backward(kind, dy, x_kept, u_kept, dx, du=None):
    """u_kept and du: both for a gated layer, else None."""
    type_, rows, cols, pdy, lddy, dev = _first(dy, "dy")
    xc, xs = _packed(x_kept, PP_PACK_INT8, rows, cols, "x_kept", dev)
    uc, us = _packed(u_kept, PP_PACK_INT8, rows, cols, "u_kept", dev)
    pdx, lddx = _matrix(dx, dy.dtype, rows, cols, "dx", dev)
    pdu, lddu = (None, 0) if du is None else _matrix(du, dy.dtype, rows, cols, "du", dev)
    _check(lib().pp_act_backward(kind, type_, rows, cols, pdy, lddy, xc, xs, uc, us, pdx, lddx, pdu, lddu, _stream(dev)))


def pp_linear_workspace_bytes(call, dtype, rows, n_in, n_out):
    """dtype: of x or dy, as torch's."""
    return int(lib().pp_linear_workspace_bytes(call, TYPES.get(dtype, -1), rows, n_in, n_out))


def pp_linear_forward(x, w, bias, y, x_kept, workspace):
    """w: the packed weight (PP_PACK_FP4); x_kept: room for the packed x (PP_PACK_INT8), or None."""
    type_, rows, n_in, px, ldx, dev = _first(x, "x")
    n_out = w[0].shape[0]
    wc, wsc = _packed(w, PP_PACK_FP4, n_out, n_in, "w", dev)
    py, ldy = _matrix(y, x.dtype, rows, n_out, "y", dev)
    xc, xs = _packed(x_kept, PP_PACK_INT8, rows, n_in, "x_kept", dev)
    ws, nbytes = _workspace(workspace, dev)
    _check(lib().pp_linear_forward(type_, rows, n_in, n_out, px, ldx, wc, wsc, _vector(bias, n_out, "bias", dev), py, ldy,
                                   xc, xs, ws, nbytes, _stream(dev)))


def pp_linear_backward_input(dy, w, dx, workspace):
    type_, rows, n_out, pdy, lddy, dev = _first(dy, "dy")
    n_in = dx.shape[-1]
    wc, wsc = _packed(w, PP_PACK_FP4, n_out, n_in, "w", dev)
    pdx, lddx = _matrix(dx, dy.dtype, rows, n_in, "dx", dev)
    ws, nbytes = _workspace(workspace, dev)
    _check(lib().pp_linear_backward_input(type_, rows, n_in, n_out, pdy, lddy, wc, wsc, pdx, lddx, ws, nbytes, _stream(dev)))


def pp_linear_backward_weight(dy, x_kept, dw_in, dw, db, workspace):
    """dw_in: what is added to (None = nothing; may be dw); db: the bias's gradient, or None."""
    type_, rows, n_out, pdy, lddy, dev = _first(dy, "dy")
    n_in = dw.shape[-1]
    xc, xs = _packed(x_kept, PP_PACK_INT8, rows, n_in, "x_kept", dev)
    pdw, lddw = _matrix(dw, torch.float32, n_out, n_in, "dw", dev)
    pin = None
    if dw_in is not None:
        pin, ldin = _matrix(dw_in, torch.float32, n_out, n_in, "dw_in", dev)
        if ldin != lddw and n_out > 1:
            raise ValueError("dw_in and dw must have the same row stride")
    ws, nbytes = _workspace(workspace, dev)
    _check(lib().pp_linear_backward_weight(type_, rows, n_in, n_out, pdy, lddy, xc, xs, pin, pdw, lddw,
                                           _vector(db, n_out, "db", dev), ws, nbytes, _stream(dev)))
