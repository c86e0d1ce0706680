"""Log probabilities, alternatives and distillation against the formulas in 64 bits (marker gpu).

Bounds, with u = 2^-24.  An exponent d = (x - m) k has 2.5 u of itself (difference, product, k's rounding) and exp2 2 u: a sum of n
exponentials is right to (n_add + 2) u of itself and 1.8 u for every unit of the mean |d| (in nats 2.5).  A thread adds at most 128 terms, a wave
6, the waves 4, the segments 32 a row of 2^20: n_add <= 170.  The logarithm of a sum has that error absolutely, and 4 u of its own.
exp2 gives 0 for what is no normal number: an exponential may also be off by TINY.  A temperature is the float that the call takes.
"""
import numpy as np
import pytest

from layer_helpers import Guarded, assert_within, on_gpu, torch_type
from oracle import rows as o

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TINY = 2.0 ** -126
warm = lambda x: float(np.float32(x))  # noqa: E731
SIZES = [(1, 1), (2, 7), (3, 100), (5, 1000), (2, 2048), (4, 2049), (3, 8193), (300, 500), (40, 30000), (2, 70000), (1, 140000), (1030, 2050), (9, 131072)]


def logits(rows, cols, t, seed, masked=True):
    """Normal rows of several spreads, some entries masked; ties come with 16 bits."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)) * 0.5) * 2
    if masked:
        x[1::3, cols // 2:] = -np.inf
    return rng, x


def work(n, t):
    import torch
    return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")


def sizes_of(z):
    """(ln p, p, sum of p |d|, |d|) of rows of z = x / temperature, d = z - max"""
    lp, _ = o.log_softmax(z)
    p = np.exp(lp)
    with np.errstate(invalid="ignore"):
        d = np.where(np.isfinite(z), np.abs(z - z.max(1, keepdims=True)), 0)
    return lp, p, (p * d).sum(1), d


def forward(mx, temperature, tokens, top, t, want_norm=True):
    import torch
    from paper_2204_10562_amd import layer as pp
    rows, cols = mx.shape
    tok = None if tokens is None else torch.from_numpy(tokens.astype(np.int32)).cuda()
    room = torch.full((rows + 4,), 7.0, device="cuda"), torch.full((rows + 4,), 7.0, device="cuda")
    norm = torch.empty(rows, 2, device="cuda") if want_norm else None
    index = torch.full((rows * top + 5,), 7, dtype=torch.int32, device="cuda")
    value = torch.full((rows * top + 5,), 7.0, device="cuda")
    pp.pp_logprob_forward(mx, temperature, tok, room[0][:rows] if tok is not None else None, room[1][:rows], norm,
                          index[:rows * top].view(rows, top) if top else None, value[:rows * top].view(rows, top) if top else None,
                          work(pp.pp_logprob_workspace_bytes(torch_type(t), rows, cols, top), t))
    assert all((r[rows:] == 7).all() for r in room) and (index[rows * top:] == 7).all() and (value[rows * top:] == 7).all()
    return (room[0][:rows].double().cpu().numpy(), room[1][:rows].double().cpu().numpy(), norm, index[:rows * top].view(rows, top).cpu().numpy(),
            value[:rows * top].view(rows, top).double().cpu().numpy(), tok)


def check_forward(xv, temperature, tokens, top, got):
    logp, entropy, _, index, value, _ = got
    want = o.logprob_forward(xv, temperature, tokens, top)
    lp, p, mean, d = sizes_of(xv / temperature)
    base = (180 + 2.5 * mean) * U
    rows, cols = xv.shape
    for r in range(rows):
        if 0 <= tokens[r] < cols and np.isfinite(want[0][r]):
            assert abs(logp[r] - want[0][r]) <= base[r] + 4 * U * (abs(want[0][r]) + d[r, tokens[r]])
        else:
            assert logp[r] == want[0][r]
    # H = ln S + sum e |d| / S: both sums' errors, the second's terms also with their |d|'s
    spread = (p * d * d).sum(1)
    assert (np.abs(entropy - want[1]) <= base + (190 * mean + 5 * spread + 4 * np.abs(want[1])) * U).all()
    np.testing.assert_array_equal(index, want[2])
    fine = index >= 0
    lim = base[:, None] + 8 * U * np.abs(np.where(fine, want[3], 0))
    assert (np.abs(np.where(fine, value, 0) - np.where(fine, want[3], 0)) <= lim).all() and (value[~fine] == -np.inf).all()


@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_logprob(t, rows, cols):
    import torch
    from paper_2204_10562_amd import layer as pp
    for top, temperature, pad, off in ((0, 1.0, 0, 0), (1, warm(0.7), 3, 1), (20, 2.0, 8, 0), (128, 1.0, 0, 5)):
        rng, x = logits(rows, cols, t, rows + cols + top)
        mx, xv = on_gpu(x, t, pad, off)
        tokens = rng.integers(0, cols, rows)
        tokens[2::5] = -1 - (rows & 1) * 5000
        got = forward(mx, temperature, tokens, top, t)
        check_forward(xv, temperature, tokens, top, got)
        # the gradient, and in place
        dl, dh = (torch.from_numpy(rng.standard_normal(rows)).float().cuda() for _ in range(2))
        dlv, dhv = dl.double().cpu().numpy(), dh.double().cpu().numpy()
        entropy = torch.from_numpy(got[1]).float().cuda()
        dx = Guarded(rows, cols, t, pad, off)
        pp.pp_logprob_backward(mx, temperature, got[5], got[2], dl, entropy, dh, dx.m)
        lp, p, mean, d = sizes_of(xv / temperature)
        want = o.logprob_backward(xv, temperature, tokens, dlv, dhv)
        hv = got[1][:, None]
        fine = np.where(p > 0, np.abs(np.where(p > 0, lp, 0)), 0)
        rel = (190 + 2.5 * mean[:, None] + 2.5 * d) * U
        spread = (p * d * d).sum(1)[:, None]
        he = (190 + 193 * mean[:, None] + 5 * spread + 4 * np.abs(hv)) * U
        dl_, dh_ = np.abs(dlv * (tokens >= 0))[:, None], np.abs(dhv)[:, None]
        bound = (p * (dl_ + dh_ * (fine + np.abs(hv))) * (rel + 8 * U) + dh_ * p * (he + rel)) / temperature + 4 * U * np.abs(want)
        bound += 4 * U * (np.arange(cols) == tokens[:, None]) * (1 + p) * dl_ / temperature
        bound += TINY * (dl_ + dh_ * (fine + np.abs(hv))) / temperature
        assert_within(dx.values(), want, bound, t)
        same = mx.clone()
        pp.pp_logprob_backward(same, temperature, got[5], got[2], dl, entropy, dh, same)
        assert torch.equal(same, dx.m)


def test_logprob_parts():
    """Each output alone, each gradient alone: as all together."""
    import torch
    from paper_2204_10562_amd import layer as pp
    rows, cols = 6, 5000
    rng, x = logits(rows, cols, "f32", 1)
    mx, _ = on_gpu(x, "f32")
    tokens = rng.integers(0, cols // 2, rows)
    logp, entropy, norm, index, value, tok = forward(mx, 1.0, tokens, 4, "f32")
    ws = work(pp.pp_logprob_workspace_bytes(torch.float32, rows, cols, 4), "f32")
    new = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
    a, b, c, i, v = new(rows), new(rows), new(rows, 2), torch.zeros(rows, 4, dtype=torch.int32, device="cuda"), new(rows, 4)
    pp.pp_logprob_forward(mx, 1.0, tok, a, None, None, None, None, ws)
    pp.pp_logprob_forward(mx, 1.0, None, None, b, None, None, None, ws)
    pp.pp_logprob_forward(mx, 1.0, None, None, None, c, None, None, ws)
    pp.pp_logprob_forward(mx, 1.0, tok, None, None, None, i, v, ws)
    assert (a.double().cpu().numpy() == logp).all() and (b.double().cpu().numpy() == entropy).all() and torch.equal(c, norm)
    assert (i.cpu().numpy() == index).all() and (v.double().cpu().numpy() == value).all()
    dl, dh = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")
    x1, x2 = torch.empty_like(mx), torch.empty_like(mx)
    zero = torch.zeros_like(dl)
    pp.pp_logprob_backward(mx, 1.0, tok, norm, dl, None, None, x1)
    pp.pp_logprob_backward(mx, 1.0, tok, norm, dl, b, zero, x2)
    assert torch.equal(x1, x2)
    pp.pp_logprob_backward(mx, 1.0, None, norm, None, b, dh, x1)
    pp.pp_logprob_backward(mx, 1.0, tok, norm, zero, b, dh, x2)
    assert torch.equal(x1, x2)


@pytest.mark.parametrize("cols", [50, 3000, 40000, 300000])
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_alternatives_in_any_order(t, cols):
    """Rows that are sorted, constant, of two values, of ties across the list's end, all but a few masked, and with both zeros."""
    rows, top = 8, 100
    x = np.zeros((rows, cols))
    ramp = np.linspace(-8, 8, cols)
    rng = np.random.default_rng(1)
    x[0], x[1], x[3] = ramp, ramp[::-1], (np.arange(cols) % 7 == 3) * 1.0
    x[2] = -1.5
    x[4, :] = -np.inf
    x[4, rng.integers(0, cols, 9)] = 2.0
    x[5] = np.where(rng.random(cols) < 0.5, -0.0, 0.0)
    x[6] = np.round(rng.standard_normal(cols))
    x[7] = np.where(np.arange(cols) >= cols - cols // 3, 5.0, -np.inf)
    mx, xv = on_gpu(x, t)
    tokens = np.argmax(xv, 1)
    check_forward(xv, 1.0, tokens, top, forward(mx, 1.0, tokens, top, t))


@pytest.mark.parametrize("cols", [40, 5000, 150000])
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_rows_at_their_ends(t, cols):
    """Masks of the type's lowest value, wholly and in part; nothing but -infinity; NaN and +infinity anywhere; values at the type's ends; tokens
    outside."""
    import torch
    from paper_2204_10562_amd import layer as pp
    low = {"bf16": -3.3895313892515355e38, "f16": -65504.0, "f32": -3.4028234663852886e38}[t]
    x = np.random.default_rng(cols).standard_normal((10, cols))
    x[0] = low
    x[1, cols // 2:] = low
    x[2] = -np.inf
    x[3, cols - 1] = np.nan
    x[4, cols // 3] = np.inf
    x[5], x[5, 1] = low, -low
    x[6, 0], x[6, 1:] = 0.0, -np.inf
    x[7], x[7, 3] = -np.inf, low
    x[8, 5], x[8, 6] = np.inf, np.nan
    mx, xv = on_gpu(x, t)
    tokens = np.array([0, 1, 2, 3, 4, 1, 0, 3, cols + 7, cols])
    got = forward(mx, 1.0, tokens, 6, t)
    want = o.logprob_forward(xv, 1.0, tokens, 6)
    for k in (0, 1, 4):
        # (whole rows of one value: ln of a sum of ones; entries next to -inf or the lowest value add nothing)
        with np.errstate(over="ignore"):
            w, g = want[(0, 1, 2, 2, 3)[k]].astype(np.float32).astype(np.float64), got[k]   # (twice the lowest float is -infinity)
        both = np.isfinite(w)
        np.testing.assert_array_equal(np.isnan(w), np.isnan(g))
        np.testing.assert_array_equal(w[~both & ~np.isnan(w)], g[~both & ~np.isnan(w)])
        fine = both & (np.abs(w) < 1e30)
        assert (np.abs(w - g)[fine] <= 400 * U * (1 + np.abs(w[fine]))).all()
        assert (np.abs(w - g)[both & ~fine] <= 400 * U * np.abs(w[both & ~fine])).all()
    np.testing.assert_array_equal(got[3], want[2])
    dl, dh = torch.ones(10, device="cuda"), torch.ones(10, device="cuda")
    dx = torch.empty_like(mx)
    pp.pp_logprob_backward(mx, 1.0, got[5], got[2], dl, torch.from_numpy(got[1]).float().cuda(), dh, dx)
    with np.errstate(invalid="ignore"):
        w = o.logprob_backward(xv, 1.0, tokens, np.ones(10), np.ones(10))
    assert_within(np.nan_to_num(dx.double().cpu().numpy(), nan=9.0), np.nan_to_num(w, nan=9.0), 400 * U * (1 + np.abs(np.nan_to_num(w)) + 12), t)


# ---------------------------------------------------------------- distillation

def teacher(rng, xv, top, kind, temperature):
    rows, cols = xv.shape
    z = np.where(np.isfinite(xv), xv, -30) * 0.9 + rng.standard_normal(xv.shape)
    index = np.argsort(-z, 1, kind="stable")[:, :top].astype(np.int32)
    value = np.take_along_axis(o.log_softmax(z / temperature)[0] if kind == "rest" else z, index, 1)
    if index.shape[1] < top:
        more = top - index.shape[1]
        index, value = np.pad(index, ((0, 0), (0, more)), constant_values=-1), np.pad(value, ((0, 0), (0, more)), constant_values=-np.inf)
    index[2::4, top // 2:] = -1
    index[3::4, 0] = cols + 5
    return index, value.astype(np.float32)


def distill(kind, mx, temperature, index, value, weight, t, grad=True, pad=0, off=0, in_place=False):
    import torch
    from paper_2204_10562_amd import layer as pp
    rows, cols = mx.shape
    top = index.shape[1]
    loss = torch.full((rows + 4,), 7.0, device="cuda")
    dx = Guarded(rows, cols, t, pad, off) if grad and not in_place else None
    pp.pp_distill_loss({"top": 0, "rest": 1}[kind], mx, temperature, torch.from_numpy(index).cuda(), torch.from_numpy(value).cuda(),
                       None if weight is None else torch.from_numpy(weight).cuda(), loss[:rows], mx if in_place else dx.m if grad else None,
                       work(pp.pp_distill_workspace_bytes(torch_type(t), rows, cols, top), t))
    assert (loss[rows:] == 7).all()
    return loss[:rows].double().cpu().numpy(), dx.values() if dx else None


def check_distill(kind, xv, temperature, index, value, weight, loss, dx, t):
    """loss: the sum of what is not listed has the error of a sum and everything else is in 64 bits, so ln p and ln p_rest are off by at most `base`;
    then one rounding.  A gradient is a difference of p and q, the first off by base p; beside the list p (p_rest - r) / p_rest in 32 bits."""
    rows, cols = xv.shape
    value = value.astype(np.float64)
    want, wx = o.distill(kind, xv, temperature, index, value, weight)
    lp, p, mean, d = sizes_of(xv / temperature)
    w = np.ones(rows) if weight is None else weight.astype(np.float64)
    beside = np.ones(xv.shape, bool)
    for r in range(rows):
        beside[r, index[r][(index[r] >= 0) & (index[r] < cols)]] = False
    pb = np.where(beside, p, 0)
    rest = pb.sum(1)
    share = np.divide(pb, rest[:, None], out=np.zeros_like(pb), where=rest[:, None] > 0)
    with np.errstate(invalid="ignore"):
        db = np.where(beside & np.isfinite(xv), np.abs(xv - np.where(beside, xv, -np.inf).max(1, keepdims=True)) / temperature, 0)
    base = (180 + 2.5 * (share * db).sum(1)) * U
    mass = 2.0 if kind == "rest" else 1.0
    np.testing.assert_array_equal(np.isfinite(want), np.isfinite(loss))
    fine = np.isfinite(want)
    assert (np.abs(loss - want)[fine] <= (np.abs(w) * mass * base + 2 * U * np.abs(want))[fine]).all()
    if dx is None:
        return
    scale = (np.abs(w) / temperature)[:, None]
    listed = scale * p * base[:, None] * 2 + 2 * U * np.abs(wx)
    tail = scale * share * rest[:, None] * base[:, None] * 2 + np.abs(wx) * ((185 + 2.5 * db) * U + base[:, None])
    assert_within(dx, wx, np.where(beside, tail, listed) + TINY * scale, t)


@pytest.mark.parametrize("kind", ["top", "rest"])
@pytest.mark.parametrize("rows, cols", [s for s in SIZES if s[1] > 1])
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_distill(t, rows, cols, kind):
    for top, temperature, pad, off in ((1, 1.0, 0, 0), (5, 2.0, 3, 1), (64, 1.0, 8, 0), (128, warm(0.7), 0, 5)):
        if top > 5 and top > cols // 4:
            continue
        rng, x = logits(rows, cols, t, rows * 5 + cols + top)
        mx, xv = on_gpu(x, t, pad, off)
        index, value = teacher(rng, xv, top, kind, temperature)
        weight = (rng.random(rows) * 64).astype(np.float32) if top != 5 else None
        if weight is not None:
            weight[1::3] = 0
        loss, dx = distill(kind, mx, temperature, index, value, weight, t, True, pad, off)
        check_distill(kind, xv, temperature, index, value, weight, loss, dx, t)
        only, _ = distill(kind, mx, temperature, index, value, weight, t, False)
        assert (only == loss).all()
        distill(kind, mx, temperature, index, value, weight, t, in_place=True)
        assert (mx.double().cpu().numpy() == dx).all()


@pytest.mark.parametrize("cols", [60, 5000, 150000])
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_distill_lists(t, cols):
    """The same column twice, columns listed without probability, empty lists, lists that leave nothing, students that are sure."""
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((8, cols))
    x[5, 7] = 40.0                      # a student that is sure of what is listed: the rest keeps its digits
    x[6, 9] = 40.0                      # and of what is not
    index = np.tile(np.arange(1, 9, dtype=np.int32), (8, 1))
    value = np.log(rng.uniform(0.02, 0.1, (8, 8))).astype(np.float32)
    index[0, 4:] = index[0, :4]
    index[1] = 3
    value[2, ::2] = -np.inf
    index[3] = -1
    value[4] = -np.inf
    index[7] = [cols, -1, 2 ** 31 - 1, -2 ** 31, 0, cols - 1, cols - 1, 0]
    mx, xv = on_gpu(x, t)
    for kind in ("top", "rest"):
        loss, dx = distill(kind, mx, 1.0, index, value, None, t)
        check_distill(kind, xv, 1.0, index, value, None, loss, dx, t)
        if kind == "top":
            assert (loss[3:5] == 0).all() and (dx[3:5] == 0).all()


@pytest.mark.parametrize("cols", [60, 5000, 150000])
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_distill_rows_at_their_ends(t, cols):
    low = {"bf16": -3.3895313892515355e38, "f16": -65504.0, "f32": -3.4028234663852886e38}[t]
    x = np.random.default_rng(cols).standard_normal((11, cols))
    x[0] = low
    x[1, cols // 2:] = low
    x[2] = -np.inf
    x[3, cols - 1] = np.nan
    x[4, cols // 3] = np.inf
    x[5, 2] = np.nan                    # a listed one
    x[6, 2:] = -np.inf                  # two that are not listed have something
    x[7, 4] = -np.inf                   # a listed one has nothing
    x[8], x[9] = np.nan, np.nan         # a row of weight 0, and one without a teacher
    x[10], x[10, 2:6] = -np.inf, 1.0    # nothing beside the list
    index = np.tile(np.array([2, 3, 4, 5], np.int32), (11, 1))
    index[9] = -1
    value = np.log(np.full((11, 4), 0.2)).astype(np.float32)
    weight = np.ones(11, np.float32)
    weight[8] = 0
    mx, xv = on_gpu(x, t)
    for kind in ("top", "rest"):
        loss, dx = distill(kind, mx, 1.0, index, value, weight, t)
        with np.errstate(all="ignore"):
            want, wx = o.distill(kind, xv, 1.0, index, value.astype(np.float64), weight)
        if kind == "rest":              # (without a list the rest is everything: the row's NaN is the loss's)
            assert np.isnan(loss[9]) and np.isnan(want[9])
        np.testing.assert_array_equal(np.isnan(loss), np.isnan(want))
        fine = np.isfinite(want)
        assert (loss[~fine & ~np.isnan(want)] == want[~fine & ~np.isnan(want)]).all()
        assert (np.abs(loss - want)[fine] <= 400 * U * (1 + np.abs(want[fine]))).all()
        np.testing.assert_array_equal(np.isnan(dx), np.isnan(wx))
        assert_within(np.nan_to_num(dx, nan=9.0), np.nan_to_num(wx, nan=9.0), 400 * U * (1 + np.abs(np.nan_to_num(wx))), t)


@pytest.mark.parametrize("t, rows, cols, pad", [("bf16", 1101, 61007, 1), ("bf16", 257, 262144, 0), ("f16", 517, 131071, 0), ("f32", 300, 120001, 3), ("f32", 5000, 7001, 0), ("f32", 120, 300001, 0), ("bf16", 170, 400001, 2)])
@pytest.mark.parametrize("kind", ["top", "rest"])
def test_distill_of_many(t, rows, cols, pad, kind):
    """So many logits that they are read once, by workgroups that meet (300001 float32 columns are too long for it): some rows against the formula,
    among them such as have nothing to learn or are no numbers, and all of them again in place."""
    import torch
    from paper_2204_10562_amd import layer as pp
    assert rows * cols * (4 if t == "f32" else 2) >= 1 << 27
    g = torch.Generator(device="cuda").manual_seed(rows)
    top = 30
    room = torch.empty(rows, cols + pad, dtype=torch_type(t), device="cuda")
    x = room[:, :cols]
    for r in range(0, rows, 64):
        n = min(64, rows - r)
        x[r:r + n] = torch.randn(n, cols, generator=g, device="cuda") * 3
    x[1::7, cols - cols // 3:] = -float("inf")
    index = torch.randint(0, cols // 2, (rows, top), generator=g, device="cuda", dtype=torch.int32)
    index[::3, :5] = torch.arange(5, dtype=torch.int32, device="cuda") * (cols // 5) + 3
    value = torch.log(torch.rand(rows, top, generator=g, device="cuda") * 0.02 + 0.005)
    weight = torch.rand(rows, generator=g, device="cuda") + 0.1
    weight[2::9] = 0
    bad, none, empty, lost = 10, 12, 16, 18          # a NaN, no list, nothing but -infinity, +infinity in a listed column
    x[bad, cols - 2], x[lost, 3] = float("nan"), float("inf")
    x[empty] = -float("inf")
    index[none], index[lost, 0] = -1, 3
    weight[[bad, none, empty, lost]] = 1.0
    loss, dx = torch.empty(rows, device="cuda"), torch.full_like(room, 77)
    ws = work(pp.pp_distill_workspace_bytes(torch_type(t), rows, cols, top), t)
    k = {"top": 0, "rest": 1}[kind]
    pp.pp_distill_loss(k, x, 1.0, index, value, weight, loss, dx[:, :cols], ws)
    assert pad == 0 or (dx[:, cols:] == 77).all()
    picked = sorted(set(range(0, 24)) | set(range(0, rows, rows // 12)) | {rows - 1})
    fine = [r for r in picked if r not in (bad, none, empty, lost)]
    host = lambda v, at: v[at].double().cpu().numpy()  # noqa: E731
    check_distill(kind, host(x, fine), 1.0, index[fine].cpu().numpy(), value[fine].cpu().numpy(), host(weight, fine).astype(np.float32), host(loss, fine),
                  host(dx[:, :cols], fine), t)
    assert torch.isnan(loss[[bad, lost]]).all() and torch.isnan(dx[[bad, lost], :cols]).all()
    assert torch.isinf(loss[empty]) and (dx[empty, :cols] == 0).all()
    if kind == "top":
        assert loss[none] == 0 and (dx[none, :cols] == 0).all()
    else:                                            # everything is the rest: no divergence (r - p_rest is a rounding)
        assert abs(loss[none]) <= 400 * U and (dx[none, :cols].float().abs() <= 400 * U).all()
    again = torch.empty_like(loss)
    pp.pp_distill_loss(k, x, 1.0, index, value, weight, again, x, ws)
    assert torch.equal(again.nan_to_num(5.0), loss.nan_to_num(5.0)) and torch.equal(x.nan_to_num(5.0), dx[:, :cols].nan_to_num(5.0))


def test_large_offsets():
    """Rows whose offsets pass 2^32 bytes, and 2^31 values."""
    import torch
    from paper_2204_10562_amd import layer as pp
    cols = 1000
    room = torch.zeros((1 << 31) + 5000, dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((3, cols), (1 << 30, 1), 8)
    x.copy_(torch.randn(3, cols, generator=torch.Generator().manual_seed(1)))
    xv = x.double().cpu().numpy()
    tokens = np.array([5, 6, 7])
    got = forward(x, 1.0, tokens, 5, "bf16")
    check_forward(xv, 1.0, tokens, 5, got)
    index, value = teacher(np.random.default_rng(1), xv, 5, "rest", 1.0)
    loss, dx = distill("rest", x, 1.0, index, value, None, "bf16")
    check_distill("rest", xv, 1.0, index, value, None, loss, dx, "bf16")
