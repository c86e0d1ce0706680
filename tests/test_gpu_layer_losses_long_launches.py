"""Losses of more rows than a launch has workgroups, of few columns (marker gpu): every loop over rows takes a second turn.

Bounds, with u = 2^-24 and |d| <= 16 the distance of a logit from its row's largest: a sum of exponentials is right to (180 + 2.5 mean |d|) u,
at most 220 u, and so is ln p, with 4 u of itself and of d: 400 u.  The mean |d| of a row of six is at most its entropy, 1.8, and the mean d^2 at
most 6 max(p ln^2 p) = 3.3: the entropy is right to (180 + 4.5 + 190 * 1.8 + 5 * 3.3 + 4 * 1.8) u < 600 u.  A gradient, for |dlogp| and
|dentropy| of 1: p (203 + 2.5 d) u + 8 u < 215 u for the first; for the second p (|ln p| + H) <= 2.2 times 203 u, 2.5 p d (|ln p| + H) <= 3 u, p times the
entropy's own 600 u and p's 200 u, and 10 u: 1260 u.  A distillation's loss has ln p and ln p_rest each off by 220 u and its gradient p and p_rest.
"""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
STEP = 1 << 20


def logits(rows, cols, seed):
    """Float32 logits of 16ths, so that some of a row are equal; some masked."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, cols, generator=g, device="cuda").clamp_(-4, 4) * 32).round_() / 16
    x[3::8, cols - 1] = -float("inf")
    return g, x


def room(nbytes):
    import torch
    return torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")


def within(got, want, bound):
    return bool(((got.double() - want).abs() <= bound + U * want.abs()).all())


def test_log_probabilities():
    import torch
    from paper_2204_10562_amd import layer as pp
    rows, cols, top = (1 << 22) + 5, 6, 3
    print("[case] logprob", rows, flush=True)
    g, x = logits(rows, cols, 1)
    tokens = torch.randint(-1, cols - 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
    dlogp, dentropy = (torch.rand(rows, generator=g, device="cuda") * 2 - 1 for _ in range(2))
    logp, entropy, norm, dx = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 2, device="cuda"), torch.empty_like(x)
    index, value = torch.empty(rows, top, dtype=torch.int32, device="cuda"), torch.empty(rows, top, device="cuda")
    pp.pp_logprob_forward(x, 1.0, tokens, logp, entropy, norm, index, value, room(pp.pp_logprob_workspace_bytes(x.dtype, rows, cols, top)))
    pp.pp_logprob_backward(x, 1.0, tokens, norm, dlogp, entropy, dentropy, dx)
    for at in range(0, rows, STEP):
        part = slice(at, at + STEP)
        lp = torch.log_softmax(x[part].double(), 1)
        p = lp.exp()
        plp = torch.where(p > 0, p * lp, 0.0)
        h = -plp.sum(1)
        tok, have = tokens[part].long().clamp(min=0)[:, None], tokens[part] >= 0
        assert within(logp[part], torch.where(have, lp.gather(1, tok)[:, 0], 0.0), 400 * U) and within(entropy[part], h, 600 * U), at
        order = torch.sort(x[part], dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(index[part].long(), order) and within(value[part], lp.gather(1, order), 400 * U), at
        dl, dh = (dlogp[part].double() * have)[:, None], dentropy[part].double()[:, None]
        want = -p * dl - dh * (plp + p * h[:, None])
        want.scatter_add_(1, tok, dl)
        assert within(dx[part], want, (215 + 1260) * U), at


@pytest.mark.parametrize("kind", ["top", "rest"])
def test_distillation(kind):
    """2^24 rows of 268 MB: as many workgroups that meet would be more than a launch has."""
    import torch
    from paper_2204_10562_amd import layer as pp
    rows, cols, top = 1 << 24, 4, 2
    print("[case] distill", kind, rows, flush=True)
    g, x = logits(rows, cols, 2)
    index = torch.randint(0, cols // 2, (rows, 1), generator=g, device="cuda", dtype=torch.int32) + torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    value = torch.log(torch.rand(rows, top, generator=g, device="cuda") * 0.4 + 0.05)
    weight = torch.rand(rows, generator=g, device="cuda")
    weight[5::16] = 0
    loss, dx = torch.empty(rows, device="cuda"), torch.empty_like(x)
    pp.pp_distill_loss({"top": 0, "rest": 1}[kind], x, 1.0, index, value, weight, loss, dx, room(pp.pp_distill_workspace_bytes(x.dtype, rows, cols, top)))
    for at in range(0, rows, STEP):
        part = slice(at, at + STEP)
        lp, w, i, lq = torch.log_softmax(x[part].double(), 1), weight[part].double(), index[part].long(), value[part].double()
        if kind == "top":
            lq = torch.log_softmax(lq, 1)
        q, dz = lq.exp(), lp.exp()
        want = (q * (lq - lp.gather(1, i))).sum(1)
        if kind == "rest":
            rest, beside = 1 - q.sum(1), torch.ones_like(dz).scatter_(1, i, 0.0)
            mass = (dz * beside).sum(1)
            want += rest * (rest.log() - mass.log())
            dz = dz - dz * beside * (rest / mass)[:, None]
        dz.scatter_add_(1, i, -q)
        fine = torch.isfinite(want) | (w == 0)
        assert within(loss[part][fine], torch.where(w > 0, want * w, 0.0)[fine], 440 * U) and torch.equal(loss[part][~fine], want[~fine].float()), at
        assert within(dx[part], torch.where(w[:, None] > 0, dz * w[:, None], 0.0), 660 * U), at
