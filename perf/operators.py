"""The operators of a pipeline stage's layers, as a list of cases to time.

A stage keeps every microbatch's activations until its backward pass and sends one to the next
stage, so their bytes are what a plan turns on.  The operators hold them in 8 bits and the linear
layers' operands in 4, in blocks of 32 neighbours of a row that share a power of two:

  pack      a matrix into 8 bits (a checkpoint) or 4 bits (an operand), and read back
  act       an activation function, gated or not: forward with its checkpoints, and backward from them
  linear    y = q4(x) W4^T + b, with q8(x) kept for the backward pass where the caller trains
  dinput    dx = dy W4
  dweight   dW = dW0 + dy^T X8 and db, from the 8-bit checkpoint

A packed matrix of R rows and C columns has G = ceil(C / 128) groups per row: int8 [R][G][128]
(or, with 4 bits, uint8 [R][G][64], the even column in the low half) and uint8 scales [R][G][4];
what lies beyond column C is zero.  With a = max |v| of a block and e = floor(log2 a), 8 bits are
rint(64 v / 2^e) held to +-127 and the scale byte is e + 127; 4 bits are the nearest of 0 .5 1 1.5 2 3 4 6
(ties to the even code, 6 beyond) to v / 2^(e-2) and the byte e - 2 + 127, at least 0.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
BLOCK, GROUP = 32, 128
BYTES8, BYTES4 = 1 + 1 / BLOCK, 0.5 + 1 / BLOCK   # of a packed value, its share of the scale included


def listed():
    return [
        # one row of a checkpoint, written and read back: the latency of the two calls
        dict(name="pack one row", kind="pack", fmt="int8", type="bf16", rows=1, cols=4096),
        # the activation that crosses a cut of the GPT-shaped workload (16 MiB in 16 bits)
        dict(name="pack boundary", kind="pack", fmt="int8", type="bf16", rows=2048, cols=4096),
        # a layer's 32-bit weight into 4 bits after an update, no size round
        dict(name="pack weight odd", kind="pack", fmt="fp4", type="f32", rows=5003, cols=4099),
        # a ragged microbatch through an ungated layer, fp16
        dict(name="act ragged", kind="act", fn="gelu", gated=False, type="f16", rows=777, cols=4100),
        # several microbatches of a gated layer
        dict(name="act gated", kind="act", fn="silu", gated=True, type="bf16", rows=8192, cols=16384),
        # a token at a time through the wide layer
        dict(name="linear one row", kind="linear", type="bf16", rows=1, n_in=4096, n_out=16384, bias=True, keep=False),
        # a ragged microbatch, no size a multiple of a tile
        dict(name="linear ragged", kind="linear", type="f16", rows=333, n_in=4100, n_out=5000, bias=True, keep=True),
        # the wide layer over several microbatches of a stage
        dict(name="linear stage", kind="linear", type="bf16", rows=8192, n_in=4096, n_out=16384, bias=True, keep=True),
        # its input's gradient, ragged and whole
        dict(name="dinput ragged", kind="dinput", type="f16", rows=333, n_in=4100, n_out=5000),
        dict(name="dinput stage", kind="dinput", type="bf16", rows=8192, n_in=4096, n_out=16384),
        # few features and many tokens: the sum over the tokens is the long axis
        dict(name="dweight long", kind="dweight", type="bf16", rows=32771, n_in=520, n_out=1000, bias=True),
        dict(name="dweight stage", kind="dweight", type="bf16", rows=8192, n_in=4096, n_out=16384, bias=False),
    ]


def _log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    if n > 512 and rng.random() < 0.5:   # half of the larger sizes are round
        n = n // 128 * 128
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["pack", "act", "linear", "dinput", "dweight"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "pack":
        return dict(kind=kind, fmt=rng.choice(["int8", "fp4"]), type=t, rows=_log_int(rng, 1, 8192), cols=_log_int(rng, 32, 16384))
    if kind == "act":
        return dict(kind=kind, fn=rng.choice(["gelu", "gelu_tanh", "silu"]), gated=rng.random() < 0.5, type=t,
                    rows=_log_int(rng, 1, 4096), cols=_log_int(rng, 32, 16384))
    wide = dict(n_in=_log_int(rng, 64, 8192), n_out=_log_int(rng, 64, 8192))
    if kind == "linear":
        return dict(kind=kind, type=t, rows=_log_int(rng, 1, 8192), bias=rng.random() < 0.5, keep=rng.random() < 0.5, **wide)
    if kind == "dinput":
        return dict(kind=kind, type=t, rows=_log_int(rng, 1, 8192), **wide)
    return dict(kind=kind, type=t, rows=_log_int(rng, 1, 8192), bias=rng.random() < 0.5, **wide)


# ---------------------------------------------------------------- the packed form in plain steps

def _blocks(x):
    """A matrix in 32 bits as [R][G * 4][32], zeros behind its last column."""
    rows, cols = x.shape
    pad = -cols % GROUP
    x = x.float()
    if pad:
        x = torch.cat([x, x.new_zeros(rows, pad)], 1)
    return x.reshape(rows, -1, BLOCK)


def _power(e):
    """2^e in 32 bits for whole e of -149 .. 127, by its bits."""
    e = e.int()
    bits = torch.where(e >= -126, (e + 127) << 23, torch.ones_like(e) << (e + 149).clamp(0, 22))
    return bits.view(torch.float32)


def _encode(x, fmt):
    v = _blocks(x)
    field = (v.abs().amax(2).view(torch.int32) >> 23) & 255      # floor(log2 a) + 127, and 0 below the normal numbers
    if fmt == "int8":
        scale = field
        u = v * 64.0
    else:
        scale = torch.where(field == 255, field, (field - 2).clamp(min=0))
        u = v
    n = 127 - scale.clamp(max=254)
    half = n >> 1                                                # 2^127 is the largest power: multiply twice
    u = u * _power(half)[..., None] * _power(n - half)[..., None]
    if fmt == "int8":
        code = torch.round(u).clamp(-127, 127)
        code = torch.where((field == 255)[..., None], torch.zeros_like(code), code).to(torch.int8)
        return code.reshape(x.shape[0], -1, GROUP), scale.to(torch.uint8).reshape(x.shape[0], -1, 4)
    a = u.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    mag = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a * 0.5 + 4))     # 0 .5 1 1.5 2 3 4 6 -> 0 .. 7
    sign = u.view(torch.int32) < 0
    mag = torch.where((field == 255)[..., None], torch.zeros_like(mag), mag).to(torch.int32)
    code = mag + torch.where(sign & (mag > 0), 8, 0)
    code = code.reshape(x.shape[0], -1, 2)
    code = (code[..., 0] | code[..., 1] << 4).to(torch.uint8)
    return code.reshape(x.shape[0], -1, GROUP // 2), scale.to(torch.uint8).reshape(x.shape[0], -1, 4)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _decode(codes, scales, cols, fmt):
    """The values of a packed matrix in 32 bits."""
    rows = codes.shape[0]
    s = scales.reshape(rows, -1).int()
    if fmt == "int8":
        v = codes.reshape(rows, -1, BLOCK).float()
        p = _power(s.clamp(max=254) - 133)
    else:
        c = codes.reshape(rows, -1).int()
        c = torch.stack([c & 15, c >> 4], 2).reshape(rows, -1, BLOCK)
        table = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), device=codes.device)
        v = table[c]
        p = _power(s.clamp(max=254) - 127)
    p = torch.where(s == 255, torch.full_like(p, math.nan), p)
    return (v * p[..., None]).reshape(rows, -1)[:, :cols]


def _f(fn, x):
    if fn == "silu":
        return x / (1 + torch.exp(-x))
    if fn == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))


def _df(fn, x):
    if fn == "silu":
        s = 1 / (1 + torch.exp(-x))
        return s * (1 + x * (1 - s))
    if fn == "gelu":
        return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (x + 0.044715 * x * x * x))
    return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * c * (1 + 3 * 0.044715 * x * x)


# ---------------------------------------------------------------- inputs

def _acts(g, rows, cols, dtype):
    """Activations: normal, with a spread of sizes over the channels and a few large ones."""
    ch = torch.exp(torch.randn(cols, generator=g, device="cuda") * 0.7)
    return (torch.randn(rows, cols, generator=g, device="cuda") * ch).to(dtype)


def _grads(g, rows, cols, dtype):
    """Gradients: normal, with a spread of sizes over the tokens."""
    tok = torch.exp(torch.randn(rows, 1, generator=g, device="cuda")) * 2.0 ** -7
    return (torch.randn(rows, cols, generator=g, device="cuda") * tok).to(dtype)


def _packed(rows, cols, fmt):
    groups = -(-cols // GROUP)
    codes = torch.empty(rows, groups, GROUP if fmt == "int8" else GROUP // 2, dtype=torch.int8 if fmt == "int8" else torch.uint8, device="cuda")
    return codes, torch.empty(rows, groups, 4, dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, rows = TYPES[case["type"]], case["rows"]
    new = lambda *n, dtype=t: torch.empty(*n, dtype=dtype, device="cuda")  # noqa: E731
    s = dict(case=case, ws=None)
    if case["kind"] == "pack":
        x = _acts(g, rows, case["cols"], t)
        if case["fmt"] == "fp4":
            x = x * 0.02
        return dict(s, x=x, packed=_packed(rows, case["cols"], case["fmt"]), out=new(rows, case["cols"]))
    if case["kind"] == "act":
        c = case["cols"]
        s.update(x=_acts(g, rows, c, t), dy=_grads(g, rows, c, t), y=new(rows, c), dx=new(rows, c), x8=_packed(rows, c, "int8"),
                 u=None, u8=None, du=None)
        if case["gated"]:
            s.update(u=_acts(g, rows, c, t), u8=_packed(rows, c, "int8"), du=new(rows, c))
        return s
    n_in, n_out = case["n_in"], case["n_out"]
    if case["kind"] in ("linear", "dinput"):
        s["w"] = _encode(torch.randn(n_out, n_in, generator=g, device="cuda") * 0.02, "fp4")
    if case["kind"] == "linear":
        bias = torch.randn(n_out, generator=g, device="cuda") * 0.1 if case["bias"] else None
        x8 = _packed(rows, n_in, "int8") if case["keep"] else None
        return dict(s, x=_acts(g, rows, n_in, t), bias=bias, y=new(rows, n_out), x8=x8, kept=new(rows, n_in) if case["keep"] else None)
    s["dy"] = _grads(g, rows, n_out, t)
    if case["kind"] == "dinput":
        return dict(s, dx=new(rows, n_in))
    s["x8"] = _encode(_acts(g, rows, n_in, t), "int8")
    s["dw0"] = torch.randn(n_out, n_in, generator=g, device="cuda") * 0.01
    return dict(s, dw=new(n_out, n_in, dtype=torch.float32), db=new(n_out, dtype=torch.float32) if case["bias"] else None)


# ---------------------------------------------------------------- one pass

def _own(s):
    from paper_2204_10562_amd import layer as pp
    case = s["case"]
    kind = case["kind"]
    if kind == "pack":
        fmt = pp.PP_PACK_INT8 if case["fmt"] == "int8" else pp.PP_PACK_FP4
        pp.pp_pack(fmt, s["x"], s["packed"])
        pp.pp_unpack(fmt, s["packed"], s["out"])
        return s["out"]
    if kind == "act":
        fn = {"gelu": pp.PP_ACT_GELU, "gelu_tanh": pp.PP_ACT_GELU_TANH, "silu": pp.PP_ACT_SILU}[case["fn"]]
        pp.pp_act_forward(fn, s["x"], s["u"], y=s["y"], x_kept=s["x8"], u_kept=s["u8"])
        pp.pp_act_backward(fn, s["dy"], s["x8"], s["u8"], s["dx"], s["du"])
        return [s["y"], s["dx"]] + ([s["du"]] if case["gated"] else [])
    if s["ws"] is None:
        op = {"linear": pp.PP_LINEAR_FORWARD, "dinput": pp.PP_LINEAR_BACKWARD_INPUT, "dweight": pp.PP_LINEAR_BACKWARD_WEIGHT}[kind]
        n = pp.pp_linear_workspace_bytes(op, TYPES[case["type"]], case["rows"], case["n_in"], case["n_out"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    if kind == "linear":
        pp.pp_linear_forward(s["x"], s["w"], s["bias"], s["y"], s["x8"], s["ws"])
        if not case["keep"]:
            return s["y"]
        pp.pp_unpack(pp.PP_PACK_INT8, s["x8"], s["kept"])
        return [s["y"], s["kept"]]
    if kind == "dinput":
        pp.pp_linear_backward_input(s["dy"], s["w"], s["dx"], s["ws"])
        return s["dx"]
    pp.pp_linear_backward_weight(s["dy"], s["x8"], s["dw0"], s["dw"], s["db"], s["ws"])
    return [s["dw"]] + ([s["db"]] if case["bias"] else [])


def _plain(s):
    case = s["case"]
    kind, t = case["kind"], TYPES[case["type"]]
    if kind == "pack":
        return _decode(*_encode(s["x"], case["fmt"]), case["cols"], case["fmt"]).to(t)
    if kind == "act":
        x, dy, c = s["x"].float(), s["dy"].float(), case["cols"]
        xk = _decode(*_encode(x, "int8"), c, "int8")
        if not case["gated"]:
            return [_f(case["fn"], x).to(t), (dy * _df(case["fn"], xk)).to(t)]
        u = s["u"].float()
        uk = _decode(*_encode(u, "int8"), c, "int8")
        return [(_f(case["fn"], x) * u).to(t), (dy * _df(case["fn"], xk) * uk).to(t), (dy * _f(case["fn"], xk)).to(t)]
    if kind == "linear":
        n_in = case["n_in"]
        y = _decode(*_encode(s["x"], "fp4"), n_in, "fp4") @ _decode(*s["w"], n_in, "fp4").t()
        if s["bias"] is not None:
            y = y + s["bias"]
        return [y.to(t), _decode(*_encode(s["x"], "int8"), n_in, "int8").to(t)] if case["keep"] else y.to(t)
    if kind == "dinput":
        return (s["dy"].float() @ _decode(*s["w"], case["n_in"], "fp4")).to(t)
    dw = s["dw0"] + s["dy"].float().t() @ _decode(*s["x8"], case["n_in"], "int8")
    return [dw, s["dy"].float().sum(0)] if case["bias"] else [dw]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    t, r = SIZE[case["type"]], case["rows"]
    if case["kind"] == "pack":
        n = r * case["cols"]
        return {"bytes": n * (2 * t + (BYTES8 if case["fmt"] == "int8" else BYTES4)), "flops": 0}
    if case["kind"] == "act":
        n, two = r * case["cols"], 2 if case["gated"] else 1
        return {"bytes": n * (t * (2 + 2 * two) + two * BYTES8), "flops": 0}   # x (u) dy read, y dx (du) and the packs written
    n_in, n_out = case["n_in"], case["n_out"]
    flops = 2 * r * n_in * n_out
    if case["kind"] == "linear":
        keep = r * n_in * (BYTES8 + t) if case["keep"] else 0
        return {"bytes": r * (n_in + n_out) * t + n_in * n_out * BYTES4 + keep, "flops": flops}
    if case["kind"] == "dinput":
        return {"bytes": r * (n_in + n_out) * t + n_in * n_out * BYTES4, "flops": flops}
    return {"bytes": r * n_out * t + r * n_in * BYTES8 + 8 * n_in * n_out, "flops": flops}


# ---------------------------------------------------------------- the definition in 64 bits

def _rounded64(x, fmt):
    """The values that x has after packing, in 64 bits, from the definition: nearest multiples of a step."""
    r, c = x.shape
    v = torch.zeros(r, -(-c // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    v[:, :c] = x
    v = v.view(r, -1, BLOCK)
    top = v.abs().max(2, keepdim=True).values
    e = torch.frexp(top).exponent.double() - 1
    if fmt == "int8":
        unit = torch.exp2(e.clamp(min=-127) - 6)
        q = torch.round(v / unit).clamp(-127, 127) * unit
    else:
        unit = torch.exp2((e - 2).clamp(min=-127))
        w = v / unit
        k = torch.floor(torch.log2(w.abs().clamp(min=1.0))).clamp(max=2)     # the octave: steps of 1/2, 1, 2
        step = torch.exp2(k - 1)
        q = (torch.round(w / step) * step).clamp(-6, 6) * unit
    return torch.where(top > 0, q, torch.zeros_like(q)).view(r, -1)[:, :c]


def _weight64(packed, n_in):
    codes, scales = packed
    c = codes.flatten(1).long()
    nib = torch.empty(c.shape[0], 2 * c.shape[1], dtype=torch.long, device=c.device)
    nib[:, 0::2], nib[:, 1::2] = c % 16, c // 16
    mag = nib % 8
    ex, man = mag // 2, (mag % 2).double()
    v = torch.where(ex == 0, man * 0.5, (1 + man * 0.5) * torch.exp2((ex - 1).double()))
    v = torch.where(nib >= 8, -v, v)
    p = torch.exp2(scales.flatten(1).double() - 127).repeat_interleave(BLOCK, 1)
    return (v * p)[:, :n_in]


def _kept64(packed, n_in):
    codes, scales = packed
    p = torch.exp2(scales.flatten(1).double() - 133).repeat_interleave(BLOCK, 1)
    return (codes.flatten(1).double() * p)[:, :n_in]


def _both64(fn, x):
    """f(x) and f'(x)."""
    if fn == "gelu":
        cdf = torch.special.ndtr(x)
        return x * cdf, cdf + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if fn == "silu":
        z, dz = x, 1.0
    else:   # 0.5 (1 + tanh(z / 2)) = sigmoid(z)
        c = 2 * math.sqrt(2 / math.pi)
        z, dz = c * (x + 0.044715 * x ** 3), c * (1 + 3 * 0.044715 * x ** 2)
    s = torch.sigmoid(z)
    return x * s, s + x * s * torch.sigmoid(-z) * dz


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "pack":
        return _rounded64(s["x"].double(), case["fmt"])
    if kind == "act":
        x, dy = s["x"].double(), s["dy"].double()
        y = _both64(case["fn"], x)[0]
        f, d = _both64(case["fn"], _rounded64(x, "int8"))
        if not case["gated"]:
            return [y, dy * d]
        u = s["u"].double()
        return [y * u, dy * d * _rounded64(u, "int8"), dy * f]
    if kind == "linear":
        x = s["x"].double()
        y = torch.mm(_rounded64(x, "fp4"), _weight64(s["w"], case["n_in"]).t().contiguous())
        if s["bias"] is not None:
            y += s["bias"].double()
        return [y, _rounded64(x, "int8")] if case["keep"] else y
    if kind == "dinput":
        return torch.mm(s["dy"].double(), _weight64(s["w"], case["n_in"]))
    dw = torch.mm(s["dy"].double().t().contiguous(), _kept64(s["x8"], case["n_in"])) + s["dw0"].double()
    return [dw, s["dy"].double().sum(0)] if case["bias"] else [dw]
