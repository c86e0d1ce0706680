"""The oracle of norms, scans and losses: gradients against differences, and rows at the ends of their range (no GPU)."""
import numpy as np
import pytest

from oracle import rows as o


def differences(f, x, step=1e-6):
    """d f / d x of a scalar f, by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + step
        up = f()
        x[i] = old - step
        g[i] = (up - f()) / (2 * step)
        x[i] = old
    return g


# central differences of smooth functions of order 1: step^2 in the truncation, 1e-16 / step in the difference
NEAR = dict(rtol=1e-6, atol=2e-8)


@pytest.mark.parametrize("res", [False, True])
def test_norm(res):
    rng = np.random.default_rng(1)
    x, r, gain, w, w2 = (rng.standard_normal(s) for s in ((3, 7), (3, 7), 7, (3, 7), (3, 7)))
    r = r if res else None

    def f():
        s, _, y = o.norm_forward(x, r, gain, 1e-3)
        return (y * w).sum() + (s * w2).sum()
    s, inv, _ = o.norm_forward(x, r, gain, 1e-3)
    dx, dgain = o.norm_backward(w, s, inv, gain, w2, None)
    np.testing.assert_allclose(dx, differences(f, x), **NEAR)
    np.testing.assert_allclose(dgain, differences(f, gain), **NEAR)


@pytest.mark.parametrize("starts", [[0, 9], [1, 4, 4, 5, 8]])
def test_scan(starts):
    rng = np.random.default_rng(2)
    gate, v, w = (rng.standard_normal((9, 3)) * 2 for _ in range(3))
    h0, wl = (rng.standard_normal((len(starts) - 1, 3)) for _ in range(2))
    used = slice(starts[0], starts[-1])

    def f():
        h, last, _ = o.scan_forward(gate, v, starts, h0)
        return (h * w)[used].sum() + (last * wl).sum()
    dgate, dv, dh0, _ = o.scan_backward(w, gate, v, starts, h0, wl)
    np.testing.assert_allclose(dgate[used], differences(f, gate)[used], **NEAR)
    np.testing.assert_allclose(dv[used], differences(f, v)[used], **NEAR)
    np.testing.assert_allclose(dh0, differences(f, h0), **NEAR)


def test_logprob():
    rng = np.random.default_rng(3)
    x, wl, wh = rng.standard_normal((4, 9)) * 2, rng.standard_normal(4), rng.standard_normal(4)
    x[1, 3:6] = -np.inf
    tokens = np.array([2, 1, -1, 8])

    def f():
        logp, entropy, _, _ = o.logprob_forward(x, 0.7, tokens, 3)
        return (logp * wl).sum() + (entropy * wh).sum()
    fine = np.isfinite(x)
    with np.errstate(invalid="ignore"):
        want = differences(f, x)
    got = o.logprob_backward(x, 0.7, tokens, wl, wh)
    np.testing.assert_allclose(got[fine], want[fine], **NEAR)
    assert (got[~fine] == 0).all()


@pytest.mark.parametrize("kind", ["top", "rest"])
def test_distill(kind):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((4, 9)) * 2
    index = np.array([[1, 5, 0], [2, -1, 7], [3, 3, 8], [4, 9, -1]])
    value = np.log(rng.uniform(0.05, 0.3, (4, 3)))
    weight = np.array([1.0, 2.0, 0.5, 0.0])

    def f():
        return o.distill(kind, x, 1.3, index, value, weight)[0].sum()
    loss, dx = o.distill(kind, x, 1.3, index, value, weight)
    np.testing.assert_allclose(dx, differences(f, x), **NEAR)
    assert loss[3] == 0 and (loss[:2] > 0).all()


def test_distill_of_itself():
    """A teacher that is the student, all or a part of it known: no divergence, no gradient."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((2, 8)) * 3
    lp = o.log_softmax(x)[0]
    for kind, top in (("rest", 3), ("rest", 7), ("top", 8)):
        index = np.argsort(-lp, 1)[:, :top]
        loss, dx = o.distill(kind, x, 1.0, index, np.take_along_axis(lp, index, 1), None)
        assert np.abs(loss).max() < 1e-14 and np.abs(dx).max() < 1e-14


def test_rows_without_numbers():
    x = np.array([[-np.inf] * 4, [0, np.nan, 1, 2], [np.inf, 0, 0, 0], [1, 1, -np.inf, 0]])
    logp, entropy, index, value = o.logprob_forward(x, 1.0, np.array([1, 0, -1, 2]), 4)
    assert logp[0] == -np.inf and entropy[0] == 0 and (index[0] == -1).all()
    assert np.isnan(logp[1]) and logp[2] == 0 and np.isnan(entropy[1:3]).all() and np.isnan(value[1:3]).all()
    assert logp[3] == -np.inf and list(index[3]) == [0, 1, 3, -1]
    g = o.logprob_backward(x, 1.0, np.array([1, 0, -1, 2]), np.ones(4), np.ones(4))
    assert (g[0] == 0).all() and np.isnan(g[1:3]).all() and np.isfinite(g[3]).all()
