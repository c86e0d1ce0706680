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
PP_SCAN_FORWARD, PP_SCAN_BACKWARD = 0, 1
PP_DISTILL_TOP, PP_DISTILL_REST = 0, 1
PP_TOP_MAX = 128
PP_LAYER_MAX_ROWS, PP_LAYER_MAX_COLS, PP_LAYER_MAX_LD_DW = 1 << 30, 1 << 22, 1 << 24
BLOCK, GROUP = 32, 128

EXPORTS = ("pp_pack", "pp_unpack", "pp_act_forward", "pp_act_backward", "pp_linear_workspace_bytes",
           "pp_linear_forward", "pp_linear_backward_input", "pp_linear_backward_weight",
           "pp_norm_forward", "pp_norm_workspace_bytes", "pp_norm_backward", "pp_scan_workspace_bytes", "pp_scan_kept_rows",
           "pp_scan_forward", "pp_scan_backward", "pp_scan_step", "pp_logprob_workspace_bytes", "pp_logprob_forward",
           "pp_logprob_backward", "pp_distill_workspace_bytes", "pp_distill_loss")

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
        f32 = ctypes.c_float
        L.pp_norm_forward.argtypes = [i32, i64, i64] + [vp, i64] * 2 + [vp, f32] + [vp, i64] * 2 + [vp] * 6
        L.pp_norm_workspace_bytes.argtypes = [i32, i64, i64]
        L.pp_norm_backward.argtypes = [i32, i64, i64] + [vp, i64] * 2 + [vp] * 4 + [vp, i64] * 2 + [vp, vp, vp, sz, vp]
        L.pp_scan_workspace_bytes.argtypes = [i32, i32, i64, i64]
        L.pp_scan_kept_rows.argtypes = [i32, i64, i64]
        L.pp_scan_forward.argtypes = [i32, i64, i64] + [vp, i64] * 2 + [i64, vp, vp, vp, i64, vp, vp, vp, sz, vp]
        L.pp_scan_backward.argtypes = [i32, i64, i64] + [vp, i64] * 3 + [i64] + [vp] * 4 + [vp, i64] * 2 + [vp, vp, sz, vp]
        L.pp_scan_step.argtypes = [i32, i64, i64] + [vp, i64] * 2 + [i64, vp, vp, vp, i64, vp]
        L.pp_logprob_workspace_bytes.argtypes = [i32, i64, i64, i32]
        L.pp_logprob_forward.argtypes = [i32, i64, i64, vp, i64, f32, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        L.pp_logprob_backward.argtypes = [i32, i64, i64, vp, i64, f32, vp, vp, vp, vp, vp, vp, i64, vp]
        L.pp_distill_workspace_bytes.argtypes = [i32, i64, i64, i32]
        L.pp_distill_loss.argtypes = [i32, i32, i64, i64, vp, i64, f32, i32, vp, vp, vp, vp, vp, i64, vp, sz, vp]
        for name in EXPORTS:
            getattr(L, name).restype = sz if name.endswith("_bytes") else i64 if name.endswith("_rows") else i32
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


def _values(t, shape, dtype, name, dev):
    """Pointer of contiguous values of this shape; None: none."""
    if t is None:
        return None
    if t.get_device() != dev or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be %s contiguous %s values on the GPU of the other operands" % (name, " x ".join(map(str, shape)), dtype))
    if t.requires_grad:
        _no_history(name)
    return t.data_ptr()


def _vector(t, n, name, dev):
    return _values(t, (n,), torch.float32, name, dev)


def _optional(t, dtype, rows, cols, name, dev):
    """(data pointer, row stride) of a matrix; None: none."""
    return (None, 0) if t is None else _matrix(t, dtype, rows, cols, name, dev)


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


def pp_norm_forward(x, res, gain, eps, total, y, y_kept=None, total_kept=None, inv=None):
    """res, gain: or None; total, y, y_kept, total_kept, inv: out, or None (y and y_kept not both)."""
    type_, rows, cols, px, ldx, dev = _first(x, "x")
    pr, ldr = _optional(res, x.dtype, rows, cols, "res", dev)
    pt, ldt = _optional(total, x.dtype, rows, cols, "total", dev)
    py, ldy = _optional(y, x.dtype, rows, cols, "y", dev)
    yc, ys = _packed(y_kept, PP_PACK_INT8, rows, cols, "y_kept", dev)
    tc, ts = _packed(total_kept, PP_PACK_INT8, rows, cols, "total_kept", dev)
    _check(lib().pp_norm_forward(type_, rows, cols, px, ldx, pr, ldr, _vector(gain, cols, "gain", dev), eps, pt, ldt, py, ldy, yc, ys, tc, ts,
                                 _vector(inv, rows, "inv", dev), _stream(dev)))


def pp_norm_workspace_bytes(dtype, rows, cols):
    """dtype: of dy, as torch's."""
    return int(lib().pp_norm_workspace_bytes(TYPES.get(dtype, -1), rows, cols))


def pp_norm_backward(dy, total, inv, gain, dtotal, dx, dgain_in, dgain, workspace):
    """total: the forward pass's sum, as a matrix or packed (PP_PACK_INT8); dtotal: the gradient that reaches it beside the norm, or
    None; dgain_in: what is added to (None = nothing; may be dgain); dgain: or None."""
    type_, rows, cols, pdy, lddy, dev = _first(dy, "dy")
    kept = isinstance(total, (tuple, list))
    pt, ldt = (None, 0) if kept else _matrix(total, dy.dtype, rows, cols, "total", dev)
    tc, ts = _packed(total if kept else None, PP_PACK_INT8, rows, cols, "total", dev)
    pdt, lddt = _optional(dtotal, dy.dtype, rows, cols, "dtotal", dev)
    pdx, lddx = _matrix(dx, dy.dtype, rows, cols, "dx", dev)
    ws, nbytes = _workspace(workspace, dev)
    _check(lib().pp_norm_backward(type_, rows, cols, pdy, lddy, pt, ldt, tc, ts, _vector(inv, rows, "inv", dev), _vector(gain, cols, "gain", dev),
                                  pdt, lddt, pdx, lddx, _vector(dgain_in, cols, "dgain_in", dev), _vector(dgain, cols, "dgain", dev), ws, nbytes,
                                  _stream(dev)))


def pp_scan_workspace_bytes(call, dtype, rows, cols):
    """dtype: of gate, as torch's."""
    return int(lib().pp_scan_workspace_bytes(call, TYPES.get(dtype, -1), rows, cols))


def pp_scan_kept_rows(dtype, rows, cols):
    """Rows of the states that pp_scan_forward keeps for pp_scan_backward; -1 if a size or the type is out of range."""
    return int(lib().pp_scan_kept_rows(TYPES.get(dtype, -1), rows, cols))


def _sequences(starts, dev):
    """(number of sequences, pointer of where they start)"""
    if starts is None:
        return 1, None
    if starts.dim() != 1 or starts.shape[0] < 1:
        raise ValueError("starts must be int32 values, one more than there are sequences")
    return starts.shape[0] - 1, _values(starts, tuple(starts.shape), torch.int32, "starts", dev)


def _kept_states(kept, type_, rows, cols, dev):
    return _values(kept, (lib().pp_scan_kept_rows(type_, rows, cols), cols), torch.float32, "kept", dev)


def pp_scan_forward(gate, v, starts, h0, h, h_last, kept, workspace):
    """starts: int32, the rows where sequences start and, last, where the last one ends; None = one sequence of all rows.  h0: float32
    [sequences][cols] or None = zero; h_last (the same shape), kept (float32 [pp_scan_kept_rows][cols]): out, or None."""
    type_, rows, cols, pg, ldg, dev = _first(gate, "gate")
    pv, ldv = _matrix(v, gate.dtype, rows, cols, "v", dev)
    seqs, ps = _sequences(starts, dev)
    ph, ldh = _matrix(h, gate.dtype, rows, cols, "h", dev)
    ws, nbytes = _workspace(workspace, dev)
    _check(lib().pp_scan_forward(type_, rows, cols, pg, ldg, pv, ldv, seqs, ps, _values(h0, (seqs, cols), torch.float32, "h0", dev), ph, ldh,
                                 _values(h_last, (seqs, cols), torch.float32, "h_last", dev), _kept_states(kept, type_, rows, cols, dev), ws, nbytes,
                                 _stream(dev)))


def pp_scan_backward(dh, gate, v, starts, h0, kept, dh_last, dgate, dv, dh0, workspace):
    """h0, kept: as in pp_scan_forward; dh_last: float32 [sequences][cols] or None = zero; dh0 (the same shape): out, or None."""
    type_, rows, cols, pdh, lddh, dev = _first(dh, "dh")
    pg, ldg = _matrix(gate, dh.dtype, rows, cols, "gate", dev)
    pv, ldv = _matrix(v, dh.dtype, rows, cols, "v", dev)
    seqs, ps = _sequences(starts, dev)
    pdg, lddg = _matrix(dgate, dh.dtype, rows, cols, "dgate", dev)
    pdv, lddv = _matrix(dv, dh.dtype, rows, cols, "dv", dev)
    ws, nbytes = _workspace(workspace, dev)
    _check(lib().pp_scan_backward(type_, rows, cols, pdh, lddh, pg, ldg, pv, ldv, seqs, ps, _values(h0, (seqs, cols), torch.float32, "h0", dev),
                                  _kept_states(kept, type_, rows, cols, dev), _values(dh_last, (seqs, cols), torch.float32, "dh_last", dev),
                                  pdg, lddg, pdv, lddv, _values(dh0, (seqs, cols), torch.float32, "dh0", dev), ws, nbytes, _stream(dev)))


def pp_scan_step(gate, v, slots, state, h):
    """slots: int32 [rows] of different slots (one outside the pool: the row is padding), or None = row r has slot r; state: float32
    [slots][cols], in and out."""
    type_, rows, cols, pg, ldg, dev = _first(gate, "gate")
    pv, ldv = _matrix(v, gate.dtype, rows, cols, "v", dev)
    ph, ldh = _matrix(h, gate.dtype, rows, cols, "h", dev)
    n_slots = state.shape[0]
    _check(lib().pp_scan_step(type_, rows, cols, pg, ldg, pv, ldv, n_slots, _values(slots, (rows,), torch.int32, "slots", dev),
                              _values(state, (n_slots, cols), torch.float32, "state", dev), ph, ldh, _stream(dev)))


def pp_logprob_workspace_bytes(dtype, rows, cols, top):
    """dtype: of the logits, as torch's."""
    return int(lib().pp_logprob_workspace_bytes(TYPES.get(dtype, -1), rows, cols, top))


def pp_logprob_forward(logits, temperature, tokens, logp, entropy, norm, top_index, top_logp, workspace):
    """tokens: int32 [rows], or None without logp; logp, entropy: float32 [rows], norm: float32 [rows][2], top_index, top_logp: int32 and
    float32 [rows][top] (both or none): out, or None."""
    type_, rows, cols, pl, ld, dev = _first(logits, "logits")
    if (top_index is None) != (top_logp is None):
        raise ValueError("top_index and top_logp are given both or not at all")
    top = 0 if top_index is None else top_index.shape[-1]
    ws, nbytes = _workspace(workspace, dev)
    _check(lib().pp_logprob_forward(type_, rows, cols, pl, ld, temperature, _values(tokens, (rows,), torch.int32, "tokens", dev),
                                    _vector(logp, rows, "logp", dev), _vector(entropy, rows, "entropy", dev),
                                    _values(norm, (rows, 2), torch.float32, "norm", dev), top,
                                    _values(top_index, (rows, top), torch.int32, "top_index", dev),
                                    _values(top_logp, (rows, top), torch.float32, "top_logp", dev), ws, nbytes, _stream(dev)))


def pp_logprob_backward(logits, temperature, tokens, norm, dlogp, entropy, dentropy, dlogits):
    """dlogp, dentropy: float32 [rows] or None = zero; entropy: as the forward pass gave it, needed with dentropy; dlogits may be logits."""
    type_, rows, cols, pl, ld, dev = _first(logits, "logits")
    pd, ldd = _matrix(dlogits, logits.dtype, rows, cols, "dlogits", dev)
    _check(lib().pp_logprob_backward(type_, rows, cols, pl, ld, temperature, _values(tokens, (rows,), torch.int32, "tokens", dev),
                                     _values(norm, (rows, 2), torch.float32, "norm", dev), _vector(dlogp, rows, "dlogp", dev),
                                     _vector(entropy, rows, "entropy", dev), _vector(dentropy, rows, "dentropy", dev), pd, ldd, _stream(dev)))


def pp_distill_workspace_bytes(dtype, rows, cols, top):
    """dtype: of the logits, as torch's."""
    return int(lib().pp_distill_workspace_bytes(TYPES.get(dtype, -1), rows, cols, top))


def pp_distill_loss(kind, logits, temperature, top_index, top_value, weight, loss, dlogits, workspace):
    """kind: PP_DISTILL_TOP or PP_DISTILL_REST; top_index, top_value: int32 and float32 [rows][top], the teacher's; weight: float32 [rows] or
    None = 1; loss: float32 [rows]; dlogits: or None; may be logits."""
    type_, rows, cols, pl, ld, dev = _first(logits, "logits")
    pd, ldd = _optional(dlogits, logits.dtype, rows, cols, "dlogits", dev)
    top = top_index.shape[-1]
    ws, nbytes = _workspace(workspace, dev)
    _check(lib().pp_distill_loss(kind, type_, rows, cols, pl, ld, temperature, top, _values(top_index, (rows, top), torch.int32, "top_index", dev),
                                 _values(top_value, (rows, top), torch.float32, "top_value", dev), _vector(weight, rows, "weight", dev),
                                 _vector(loss, rows, "loss", dev), pd, ldd, ws, nbytes, _stream(dev)))
