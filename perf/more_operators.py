"""The operators around a stage's linear layers, as a list of cases to time.

A block of a stage norms the stream before each linear layer and mixes tokens; the last stage turns
logits into what is trained on and answered with.  The operators:

  norm      s = x + res, y = s g / sqrt(mean s^2 + eps): forward, with y and s kept in 8 bits where the
            caller trains, and backward
  scan      h_t = a_t h_(t-1) + (1 - a_t) v_t with a = sigmoid(gate), over sequences one behind the other:
            forward and backward; and one token a sequence with the state kept in place
  logprob   log probabilities of given tokens, the entropy and the top alternatives of every row of
            logits; and the gradient
  distill   the divergence from a teacher of whom the top entries of every row are known, and its
            gradient in the student's logits.  "top": the teacher's logits, as if there were no others;
            "rest": its log probabilities, all others as one more outcome (less than 2^-20 of them
            counts as none: so much rounded log probabilities may leave of 1)

8 bits: blocks of 32 neighbours of a row that share a power of two.  With a = max |v| of a block and
e = floor(log2 a), the values are rint(64 v / 2^e), held to +-127, in units of 2^(e - 6).  Such a value
is exact in bf16.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
BLOCK, GROUP = 32, 128
BYTES8 = 1 + 1 / BLOCK
EPS = 1e-5
LEAST_REST = 2.0 ** -20


def listed():
    return [
        # a token at a time on its way through a block: the latency of the call
        dict(name="norm one row", kind="norm", type="bf16", rows=1, cols=4096, res=True, kept=False, back=False),
        # a ragged microbatch, forward and backward, from the sum in its own type
        dict(name="norm ragged", kind="norm", type="f16", rows=777, cols=4100, res=True, kept=False, back=True),
        # several microbatches of a stage, what the backward pass needs kept in 8 bits
        dict(name="norm stage", kind="norm", type="bf16", rows=8192, cols=4096, res=True, kept=True, back=True),
        # a token of each of 64 sequences, states in a pool of slots
        dict(name="scan step", kind="step", type="bf16", rows=64, cols=4096, slots=100),
        # sequences of very different lengths one behind the other, trained with carried states
        dict(name="scan ragged", kind="scan", type="f16", rows=5003, cols=1000, seqs=23, carried=True),
        # one long sequence, trained
        dict(name="scan long", kind="scan", type="bf16", rows=65536, cols=2048, seqs=1, carried=False),
        # what a server answers with for one token: its probability and 20 alternatives
        dict(name="logprob one row", kind="logprob", type="bf16", rows=1, cols=131072, top=20, back=False, temperature=1.0),
        # a policy's tokens and entropies with their gradient, no size round, a temperature
        dict(name="logprob ragged", kind="logprob", type="f32", rows=333, cols=50001, top=5, back=True, temperature=0.7),
        # a teacher's pass over a microbatch: 64 alternatives of every token
        dict(name="logprob stage", kind="logprob", type="bf16", rows=2048, cols=131072, top=64, back=False, temperature=1.0),
        # few tokens, a small vocabulary in 32 bits
        dict(name="distill small", kind="distill", mode="top", type="f32", rows=16, cols=32768, top=8, temperature=2.0),
        # a ragged microbatch, no size round
        dict(name="distill ragged", kind="distill", mode="rest", type="f16", rows=777, cols=50001, top=20, temperature=1.0),
        # a microbatch of the last stage
        dict(name="distill stage", kind="distill", mode="rest", type="bf16", rows=2048, cols=131072, top=64, temperature=1.0),
    ]


def _log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    if n > 512 and rng.random() < 0.5:   # half of the larger sizes are round
        n = n // 128 * 128
    return n


def draw(rng):
    kind = rng.choice(["norm", "norm", "step", "scan", "scan", "logprob", "logprob", "distill", "distill"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "norm":
        rows, cols = _log_int(rng, 1, 16384), _log_int(rng, 32, 16384)
        rows = min(rows, (1 << 25) // cols)
        return dict(kind=kind, type=t, rows=rows, cols=cols, res=rng.random() < 0.7, kept=rng.random() < 0.5, back=rng.random() < 0.7)
    if kind == "step":
        rows = _log_int(rng, 1, 1024)
        return dict(kind=kind, type=t, rows=rows, cols=_log_int(rng, 32, 8192), slots=rows + rng.randrange(100))
    if kind == "scan":
        rows, cols = _log_int(rng, 1, 65536), _log_int(rng, 32, 8192)
        rows = min(rows, (1 << 25) // cols)
        return dict(kind=kind, type=t, rows=rows, cols=cols, seqs=min(rows, _log_int(rng, 1, 200)), carried=rng.random() < 0.5)
    rows, cols = _log_int(rng, 1, 4096), _log_int(rng, 100, 262144)
    rows = max(1, min(rows, (1 << 27) // cols))
    top = min(rng.choice([0, 1, 5, 8, 20, 64, 100]), cols // 8)
    temperature = rng.choice([1.0, 1.0, 0.7, 2.0])
    if kind == "logprob":
        return dict(kind=kind, type=t, rows=rows, cols=cols, top=top, back=rng.random() < 0.4, temperature=temperature)
    return dict(kind=kind, mode=rng.choice(["top", "rest"]), type=t, rows=rows, cols=cols, top=max(1, top), temperature=temperature)


# ---------------------------------------------------------------- inputs

def _acts(g, rows, cols, dtype):
    """Activations: normal, with a spread of sizes over the channels."""
    ch = torch.exp(torch.randn(cols, generator=g, device="cuda") * 0.7)
    return (torch.randn(rows, cols, generator=g, device="cuda") * ch).to(dtype)


def _grads(g, rows, cols, dtype):
    """Gradients: normal, with a spread of sizes over the tokens."""
    tok = torch.exp(torch.randn(rows, 1, generator=g, device="cuda")) * 2.0 ** -7
    return (torch.randn(rows, cols, generator=g, device="cuda") * tok).to(dtype)


def _gates(g, rows, cols, dtype):
    """Gates before the sigmoid: each channel has its own reach, from the last token or two to thousands."""
    bias = torch.rand(cols, generator=g, device="cuda") * 8 - 1
    return (torch.randn(rows, cols, generator=g, device="cuda") + bias).to(dtype)


def _logits(g, rows, cols, dtype):
    """Logits: normal, a few rows sharp; in some rows the upper part of the vocabulary is masked."""
    sharp = torch.exp(torch.randn(rows, 1, generator=g, device="cuda") * 0.4) * 2.5
    x = torch.randn(rows, cols, generator=g, device="cuda") * sharp
    masked = torch.arange(rows, device="cuda") % 8 == 3
    x[masked, cols - cols // 4:] = -math.inf
    return x.to(dtype)


def _starts(rows, seqs, seed):
    """Where the sequences start, and where the last ends: lengths of many sizes (some zero); padding behind the last."""
    if seqs == 1:
        return [0, rows]
    rng = random.Random(seed)
    used = rows - rng.randrange(rows // 16 + 1)
    share = [math.exp(rng.gauss(0, 1.5)) if rng.random() > 0.1 else 0.0 for _ in range(seqs)]
    if not sum(share):
        share[0] = 1.0
    at, starts = 0.0, [0]
    for s in share:
        at += s
        starts.append(int(used * at / sum(share) + 0.5))
    return starts


def _packed(rows, cols):
    groups = -(-cols // GROUP)
    return (torch.empty(rows, groups, GROUP, dtype=torch.int8, device="cuda"), torch.empty(rows, groups, 4, dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, rows, cols, kind = TYPES[case["type"]], case["rows"], case["cols"], case["kind"]
    new = lambda *n, dtype=t: torch.zeros(*n, dtype=dtype, device="cuda")  # noqa: E731
    f32, i32 = torch.float32, torch.int32
    s = dict(case=case, ws=None)
    if kind == "norm":
        s.update(x=_acts(g, rows, cols, t), res=_acts(g, rows, cols, t) * 2 if case["res"] else None, y=new(rows, cols),
                 gain=1 + torch.randn(cols, generator=g, device="cuda") * 0.1, total=new(rows, cols) if case["res"] else None, inv=new(rows, dtype=f32))
        if case["kept"]:
            s.update(y8=_packed(rows, cols), s8=_packed(rows, cols), y_kept=new(rows, cols, dtype=torch.bfloat16))
        if case["back"]:
            s.update(dy=_grads(g, rows, cols, t), dtotal=_grads(g, rows, cols, t) if case["res"] else None, dx=new(rows, cols),
                     dgain0=torch.randn(cols, generator=g, device="cuda") * 0.01, dgain=new(cols, dtype=f32))
        return s
    if kind == "step":
        slots = torch.randperm(case["slots"], generator=g, device="cuda")[:rows].to(i32)
        return dict(s, gate=_gates(g, rows, cols, t), v=_acts(g, rows, cols, t), slots=slots,
                    state=torch.randn(case["slots"], cols, generator=g, device="cuda"), h=new(rows, cols))
    if kind == "scan":
        starts, n = _starts(rows, case["seqs"], seed), case["seqs"]
        s.update(gate=_gates(g, rows, cols, t), v=_acts(g, rows, cols, t), dh=_grads(g, rows, cols, t), h=new(rows, cols), dgate=new(rows, cols),
                 dv=new(rows, cols), starts=torch.tensor(starts, dtype=i32, device="cuda"), h0=None, h_last=None, dh_last=None, dh0=None, kept=None)
        if case["carried"]:
            s.update(h0=torch.randn(n, cols, generator=g, device="cuda"), dh_last=torch.randn(n, cols, generator=g, device="cuda") * 2.0 ** -7,
                     h_last=new(n, cols, dtype=f32), dh0=new(n, cols, dtype=f32))
        return s
    s["logits"] = _logits(g, rows, cols, t)
    top = min(case["top"], cols)
    if kind == "logprob":
        tokens = (torch.rand(rows, generator=g, device="cuda") * (cols // 2)).to(i32)
        tokens[5::16] = -1                                                   # padding
        s.update(tokens=tokens, logp=new(rows, dtype=f32), entropy=new(rows, dtype=f32), norm=new(rows, 2, dtype=f32), top_index=None, top_logp=None)
        if top:
            s.update(top_index=new(rows, top, dtype=i32), top_logp=new(rows, top, dtype=f32))
        if case["back"]:
            s.update(dlogp=torch.randn(rows, generator=g, device="cuda"), dentropy=torch.randn(rows, generator=g, device="cuda") * 0.1, dlogits=new(rows, cols))
        return s
    teacher = s["logits"].float() * 0.9 + torch.randn(rows, cols, generator=g, device="cuda")
    value, index = torch.topk(teacher, top)
    if case["mode"] == "rest":
        value = (value - torch.logsumexp(teacher, 1, keepdim=True)).contiguous()
    index = index.to(i32)
    index[4::16, max(1, top // 2):] = -1                                     # a teacher that gave fewer
    weight = torch.full((rows,), (1024.0 if case["type"] == "f16" else 1.0) / rows, device="cuda")   # (fp16 gradients: scaled)
    weight[5::16] = 0.0                                                      # padding
    return dict(s, top_index=index, top_value=value, weight=weight, loss=new(rows, dtype=f32), dlogits=new(rows, cols))


# ---------------------------------------------------------------- the framework's calls

def _room(s, nbytes):
    """The workspace that a user's program keeps."""
    if s["ws"] is None:
        s["ws"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return s["ws"]


def _own(s):
    from paper_2204_10562_amd import layer as pp
    case = s["case"]
    kind, t, rows, cols = case["kind"], TYPES[case["type"]], case["rows"], case["cols"]
    if kind == "norm":
        y8, s8 = (s["y8"], s["s8"]) if case["kept"] else (None, None)
        pp.pp_norm_forward(s["x"], s["res"], s["gain"], EPS, s["total"], s["y"], y8, s8, s["inv"])
        out = [s["y"], s["inv"]] + ([s["total"]] if case["res"] else [])
        if case["kept"]:
            pp.pp_unpack(pp.PP_PACK_INT8, y8, s["y_kept"])
            out.append(s["y_kept"])
        if case["back"]:
            ws = _room(s, pp.pp_norm_workspace_bytes(t, rows, cols))
            total = s8 if case["kept"] else s["total"] if case["res"] else s["x"]
            pp.pp_norm_backward(s["dy"], total, s["inv"], s["gain"], s["dtotal"], s["dx"], s["dgain0"], s["dgain"], ws)
            out += [s["dx"], s["dgain"]]
        return out
    if kind == "step":
        pp.pp_scan_step(s["gate"], s["v"], s["slots"], s["state"], s["h"])
        return [s["h"], s["state"]]
    if kind == "scan":
        if s["kept"] is None:
            _room(s, max(pp.pp_scan_workspace_bytes(c, t, rows, cols) for c in (pp.PP_SCAN_FORWARD, pp.PP_SCAN_BACKWARD)))
            s["kept"] = torch.empty(pp.pp_scan_kept_rows(t, rows, cols), cols, dtype=torch.float32, device="cuda")
        pp.pp_scan_forward(s["gate"], s["v"], s["starts"], s["h0"], s["h"], s["h_last"], s["kept"], s["ws"])
        pp.pp_scan_backward(s["dh"], s["gate"], s["v"], s["starts"], s["h0"], s["kept"], s["dh_last"], s["dgate"], s["dv"], s["dh0"], s["ws"])
        return [s["h"], s["dgate"], s["dv"]] + ([s["h_last"], s["dh0"]] if case["carried"] else [])
    if kind == "logprob":
        top = min(case["top"], cols)
        ws = _room(s, pp.pp_logprob_workspace_bytes(t, rows, cols, top))
        pp.pp_logprob_forward(s["logits"], case["temperature"], s["tokens"], s["logp"], s["entropy"], s["norm"], s["top_index"], s["top_logp"], ws)
        out = [s["logp"], s["entropy"]] + ([s["top_index"], s["top_logp"]] if top else [])
        if case["back"]:
            pp.pp_logprob_backward(s["logits"], case["temperature"], s["tokens"], s["norm"], s["dlogp"], s["entropy"], s["dentropy"], s["dlogits"])
            out.append(s["dlogits"])
        return out
    mode = pp.PP_DISTILL_REST if case["mode"] == "rest" else pp.PP_DISTILL_TOP
    ws = _room(s, pp.pp_distill_workspace_bytes(t, rows, cols, s["top_index"].shape[1]))
    pp.pp_distill_loss(mode, s["logits"], case["temperature"], s["top_index"], s["top_value"], s["weight"], s["loss"], s["dlogits"], ws)
    return [s["loss"], s["dlogits"]]


# ---------------------------------------------------------------- plain forms

def _through8(x):
    """The values of a float32 matrix after packing in 8 bits."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x, (0, -cols % BLOCK)).reshape(rows, -1, BLOCK)
    field = (v.abs().amax(2, keepdim=True).view(torch.int32) >> 23) & 255      # floor(log2 a) + 127
    unit = ((field - 6).clamp(min=1) << 23).view(torch.float32)
    return (torch.round(v / unit).clamp(-127, 127) * unit).reshape(rows, -1)[:, :cols]


def _plain_norm(s, case):
    t = TYPES[case["type"]]
    total = s["x"].float() + s["res"].float() if case["res"] else s["x"].float()
    inv = 1 / torch.sqrt((total * total).mean(1) + EPS)
    y = total * inv[:, None] * s["gain"]
    out = [y.to(t), inv] + ([total.to(t)] if case["res"] else [])
    if case["kept"]:
        out.append(_through8(y).to(torch.bfloat16))
    if case["back"]:
        kept = _through8(total) if case["kept"] else total.to(t).float()
        unit = kept * inv[:, None]
        dy = s["dy"].float()
        dg = dy * s["gain"]
        dx = inv[:, None] * (dg - unit * (dg * unit).mean(1, keepdim=True))
        if case["res"]:
            dx = dx + s["dtotal"].float()
        out += [dx.to(t), s["dgain0"] + (dy * unit).sum(0)]
    return out


def _double_up(a, b):
    """b_t + a_t b_(t-1) + a_t a_(t-1) b_(t-2) + ... down the rows, in steps of 1, 2, 4, ...; a and b are used up."""
    d = 1
    while d < a.shape[0]:
        b[d:] += a[d:] * b[:-d]
        a[d:] = a[d:] * a[:-d]
        d *= 2
    return b


def _plain_scan(s, case):
    t, rows = TYPES[case["type"]], case["rows"]
    starts = s["starts"].long()
    f, v, dh = s["gate"].float(), s["v"].float(), s["dh"].float()
    a, u = 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(f))
    first, behind, some = starts[:-1], starts[1:] - 1, starts[1:] > starts[:-1]
    first, behind = first[some], behind[some]
    h0 = s["h0"] if case["carried"] else torch.zeros(len(starts) - 1, case["cols"], device="cuda")
    used = torch.arange(rows, device="cuda")[:, None] < starts[-1]
    # forward: what a sequence starts with is a part of its first token's b
    b, chain = u * v, a.clone()
    b[first] += a[first] * h0[some]
    chain[first] = 0
    h = _double_up(chain, b)
    before = torch.roll(h, 1, 0)
    before[first] = h0[some]
    # backward: g_t = dh_t + a_(t+1) g_(t+1), from the last row up
    b, chain = dh.clone(), torch.roll(a, -1, 0)
    chain[behind] = 0
    if case["carried"]:
        b[behind] += s["dh_last"][some]
    g = _double_up(chain.flip(0), b.flip(0)).flip(0)
    out = [h, a * u * (before - v) * g, u * g]
    out = [torch.where(used, x, torch.zeros_like(x)).to(t) for x in out]
    if case["carried"]:
        h_last, dh0 = h0.clone(), s["dh_last"].clone()
        h_last[some] = h[behind]
        dh0[some] = a[first] * g[first]
        out += [h_last, dh0]
    return out


def _order(x):
    """Whole numbers that are ordered as the numbers of a row and, where those are equal, by the lower index."""
    bits = (x + 0.0).view(torch.int32).long()                                 # (-0 is 0)
    bits = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    return (bits << 32) + (0xffffffff - torch.arange(x.shape[1], device=x.device))


def _plain_logprob(s, case):
    t, temperature = TYPES[case["type"]], case["temperature"]
    x, tokens = s["logits"].float(), s["tokens"].long()
    m = x.amax(1, keepdim=True)
    d = (x - m) / temperature
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    lp = d - torch.log(total)
    p = e / total
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    entropy = -plp.sum(1)
    at = tokens.clamp(min=0)[:, None]
    logp = torch.where(tokens >= 0, lp.gather(1, at)[:, 0], 0.0)
    out = [logp, entropy]
    top = min(case["top"], case["cols"])
    if top:
        key = torch.topk(_order(x), top).values
        index = 0xffffffff - (key & 0xffffffff)
        value = lp.gather(1, index)
        out += [torch.where(value > -math.inf, index, -1).int(), value]
    if case["back"]:
        dlogp = torch.where(tokens >= 0, s["dlogp"], 0.0)[:, None]
        dx = -p * dlogp - s["dentropy"][:, None] * (plp + p * entropy[:, None])
        dx.scatter_add_(1, at, dlogp)
        out.append((dx / temperature).to(t))
    return out


def _log_sum(x):
    m = x.amax(1, keepdim=True)
    return m + torch.log(torch.exp(x - m).sum(1, keepdim=True))


def _plain_distill(s, case):
    t, temperature, rest = TYPES[case["type"]], case["temperature"], case["mode"] == "rest"
    z = s["logits"].float() / temperature
    there = s["top_index"] >= 0
    at = s["top_index"].long().clamp(min=0)
    value = torch.where(there, s["top_value"], -math.inf)
    lp = z - _log_sum(z)
    if rest:
        lq = value.double()                                                   # (1 - sum loses what matters in 32 bits)
        left = 1 - torch.exp(lq).sum(1)
        left = torch.where(left < LEAST_REST, 0.0, left)
        listed = torch.zeros(z.shape, device="cuda").scatter_add_(1, at, there.float()) > 0
        others = torch.where(listed, -math.inf, lp)
        log_rest = _log_sum(others)[:, 0]
    else:
        lq = value / temperature
        lq = lq - _log_sum(lq)
    q = torch.exp(lq)
    lpk = lp.gather(1, at)
    loss = torch.where(q > 0, q * (lq - lpk), 0.0).sum(1)
    dz = torch.exp(lp)
    if rest:
        loss = loss + torch.where(left > 0, left * (torch.log(left) - log_rest), 0.0)
        dz = dz - torch.exp(others - log_rest[:, None]) * left.float()[:, None]
    dz.scatter_add_(1, at, -q.float())
    w = s["weight"]
    return [(loss * w).float(), (dz * (w / temperature)[:, None]).to(t)]


def _plain(s):
    case = s["case"]
    if case["kind"] == "norm":
        return _plain_norm(s, case)
    if case["kind"] == "step":
        at, f, v = s["slots"].long(), s["gate"].float(), s["v"].float()
        h = s["state"][at] / (1 + torch.exp(-f)) + v / (1 + torch.exp(f))
        s["state"][at] = h
        return [h.to(TYPES[case["type"]]), s["state"]]
    if case["kind"] == "scan":
        return _plain_scan(s, case)
    return _plain_logprob(s, case) if case["kind"] == "logprob" else _plain_distill(s, case)


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    t, kind, rows, cols = SIZE[case["type"]], case["kind"], case["rows"], case["cols"]
    n = rows * cols
    if kind == "norm":
        b = n * t * (4 if case["res"] else 2)                                 # x (res) read, (total) y written
        if case["kept"]:
            b += n * (2 * BYTES8 + 2)                                         # both packs written, one given back
        if case["back"]:
            b += n * (t * (3 if case["res"] else 2) + (BYTES8 if case["kept"] else t)) + 12 * cols
        return {"bytes": b + 4 * cols + 4 * rows, "flops": 0}
    if kind == "step":
        return {"bytes": n * (3 * t + 8), "flops": 0}
    if kind == "scan":                                                        # f v read, h written; dh f v read, df dv written
        return {"bytes": n * 8 * t + (16 * case["seqs"] * cols if case["carried"] else 0), "flops": 0}
    if kind == "logprob":
        return {"bytes": n * t * (3 if case["back"] else 1) + rows * (12 + 8 * min(case["top"], cols)), "flops": 0}
    return {"bytes": n * t * 2 + rows * (8 + 8 * min(case["top"], cols)), "flops": 0}


# ---------------------------------------------------------------- the definitions in 64 bits

def _kept64(x):
    """The values that x has after packing in 8 bits: nearest multiples of a block's step."""
    r, c = x.shape
    v = torch.zeros(r, -(-c // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    v[:, :c] = x
    v = v.view(r, -1, BLOCK)
    top = v.abs().max(2, keepdim=True).values
    unit = torch.exp2((torch.frexp(top).exponent.double() - 1).clamp(min=-127) - 6)
    q = torch.round(v / unit).clamp(-127, 127) * unit
    return torch.where(top > 0, q, torch.zeros_like(q)).view(r, -1)[:, :c]


def _exact_scan(s, case):
    """Token by token."""
    f, v, dh = s["gate"].double(), s["v"].double(), s["dh"].double()
    starts = s["starts"].tolist()
    keep, take = torch.sigmoid(f), torch.sigmoid(-f)
    bring = take * v
    h, df, dv = torch.zeros_like(f), torch.zeros_like(f), torch.zeros_like(f)
    lasts, firsts = [], []
    for n, (lo, hi) in enumerate(zip(starts, starts[1:])):
        state = s["h0"][n].double() if case["carried"] else torch.zeros(case["cols"], dtype=torch.float64, device="cuda")
        before = state
        for i in range(lo, hi):
            state = torch.addcmul(bring[i], keep[i], state, out=h[i])
        lasts.append(state)
        g = s["dh_last"][n].double() if case["carried"] else torch.zeros_like(state)
        for i in range(hi - 1, lo - 1, -1):
            g = torch.addcmul(dh[i], keep[i + 1], g, out=dv[i]) if i < hi - 1 else torch.add(dh[i], g, out=dv[i])
        firsts.append(keep[lo] * g if hi > lo else g)
        if hi > lo:
            df[lo] = before
            df[lo + 1:hi] = h[lo:hi - 1]
    df = (df - v) * dv * keep * take
    dv = dv * take
    return [h, df, dv] + ([torch.stack(lasts), torch.stack(firsts)] if case["carried"] else [])


def exact(case, seed):
    s = prepare(case, seed)
    kind, rows, cols = case["kind"], case["rows"], case["cols"]
    if kind == "norm":
        total = s["x"].double()
        if case["res"]:
            total = total + s["res"].double()
        inv = (total.square().sum(1) / cols + EPS).rsqrt()
        y = total * inv.view(-1, 1) * s["gain"].double()
        out = [y, inv] + ([total] if case["res"] else [])
        if case["kept"]:
            out.append(_kept64(y))
        if case["back"]:
            kept = _kept64(total) if case["kept"] else total.to(TYPES[case["type"]]).double()
            dy, gain, r = s["dy"].double(), s["gain"].double(), inv.view(-1, 1)
            dot = (dy * gain * kept).sum(1, keepdim=True)
            dx = r * dy * gain - kept * (r ** 3 * dot / cols)
            if case["res"]:
                dx = dx + s["dtotal"].double()
            out += [dx, s["dgain0"].double() + (dy * kept * r).sum(0)]
        return out
    if kind == "step":
        h = torch.lerp(s["v"].double(), s["state"].double()[s["slots"].long()], torch.sigmoid(s["gate"].double()))
        state = s["state"].double()
        state[s["slots"].long()] = h
        return [h, state]
    if kind == "scan":
        return _exact_scan(s, case)
    z = s["logits"].double() / case["temperature"]
    if kind == "logprob":
        lp = torch.log_softmax(z, 1)
        tokens = s["tokens"].long()
        have = tokens >= 0
        picked = lp[torch.arange(rows, device="cuda"), torch.where(have, tokens, 0)]
        entropy = torch.special.entr(lp.exp()).sum(1)
        out = [torch.where(have, picked, 0.0), entropy]
        if case["top"]:
            out += [None, torch.topk(lp, min(case["top"], cols)).values]
        if case["back"]:
            dlogp, dh = s["dlogp"].double() * have, s["dentropy"].double()
            p = lp.exp()
            inner = torch.where(p > 0, lp, 0.0) + entropy.view(-1, 1)
            dz = -p * (dlogp.view(-1, 1) + dh.view(-1, 1) * inner)
            dz[torch.arange(rows, device="cuda"), torch.where(have, tokens, 0)] += dlogp
            out.append(dz / case["temperature"])
        return out
    # distillation: the student's outcomes are the listed ones and, in "rest", all others as one
    index, value = s["top_index"].long(), s["top_value"].double()
    value = value.masked_fill(index < 0, -math.inf)
    q = value.exp() if case["mode"] == "rest" else torch.softmax(value / case["temperature"], 1)
    p = torch.softmax(z, 1)
    r = torch.arange(rows, device="cuda").view(-1, 1)
    dense = torch.zeros_like(p)
    dense.index_put_((r.expand_as(index), index.clamp(min=0)), q, accumulate=True)
    listed = torch.zeros(p.shape, dtype=torch.bool, device="cuda")
    row, col = torch.nonzero(index >= 0, as_tuple=True)
    listed[row, index[row, col]] = True
    loss = (torch.special.xlogy(q, q) - torch.special.xlogy(q, p[r, index.clamp(min=0)])).sum(1)
    dz = p - dense
    if case["mode"] == "rest":
        left = 1 - q.sum(1)
        left = left.masked_fill(left < LEAST_REST, 0.0)
        others = p.masked_fill(listed, 0.0)
        mass = others.sum(1)
        loss = loss + torch.special.xlogy(left, left) - torch.special.xlogy(left, mass)
        dz = dz - others * (left / mass).view(-1, 1)
    w = s["weight"].double()
    return [loss * w, dz * (w / case["temperature"]).view(-1, 1)]
