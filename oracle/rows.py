"""Norms, gated scans and the last stage's losses in 64 bits on the CPU (test infrastructure only): numpy, from the formulas.

Operands are float64 arrays.  Nothing here is shared with the library.
"""
import numpy as np


# ---------------------------------------------------------------- norm

def norm_forward(x, res, gain, eps):
    """(s, inv, y)"""
    s = x if res is None else x + res
    inv = 1 / np.sqrt((s * s).mean(1) + eps)
    y = s * inv[:, None]
    return s, inv, y if gain is None else y * gain


def norm_backward(dy, s, inv, gain, dtotal, dgain_in):
    """(dx, dgain) for the sum s as it was kept, its inv given"""
    z = s * inv[:, None]
    gdy = dy if gain is None else dy * gain
    dx = inv[:, None] * (gdy - z * (gdy * z).mean(1, keepdims=True))
    if dtotal is not None:
        dx = dx + dtotal
    return dx, (dy * z).sum(0) + (0 if dgain_in is None else dgain_in)


# ---------------------------------------------------------------- scan

def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1 / (1 + e), e / (1 + e))


def scan_forward(gate, v, starts, h0):
    """(h, h_last, before): before[t] is the state that token t finds; rows in no sequence are NaN"""
    cols = gate.shape[1]
    a, u = sigmoid(gate), sigmoid(-gate)
    h, before = np.full_like(v, np.nan), np.full_like(v, np.nan)
    last = np.zeros((len(starts) - 1, cols))
    for n in range(len(starts) - 1):
        s = np.zeros(cols) if h0 is None else h0[n].copy()
        for t in range(starts[n], starts[n + 1]):
            before[t] = s
            s = a[t] * s + u[t] * v[t]
            h[t] = s
        last[n] = s
    return h, last, before


def scan_backward(dh, gate, v, starts, h0, dh_last):
    """(dgate, dv, dh0, g); rows in no sequence are NaN"""
    cols = gate.shape[1]
    a, u = sigmoid(gate), sigmoid(-gate)
    before = scan_forward(gate, v, starts, h0)[2]
    g_all = np.full_like(v, np.nan)
    dh0 = np.zeros((len(starts) - 1, cols))
    for n in range(len(starts) - 1):
        g = np.zeros(cols) if dh_last is None else dh_last[n].copy()
        for t in range(starts[n + 1] - 1, starts[n] - 1, -1):
            g = dh[t] + g
            g_all[t] = g
            g = a[t] * g
        dh0[n] = g
    return a * u * (before - v) * g_all, u * g_all, dh0, g_all


# ---------------------------------------------------------------- losses

def log_softmax(z):
    """ln p of every entry, and the rows' states: "ok", "empty" (nothing but -infinity) or "bad" (a NaN or +infinity)"""
    state = np.where(np.isnan(z).any(1) | (z == np.inf).any(1), "bad", np.where((z == -np.inf).all(1), "empty", "ok"))
    m = np.where(state == "ok", np.where(np.isfinite(z), z, -np.inf).max(1, initial=-np.inf), 0.0)
    with np.errstate(all="ignore"):
        lp = z - m[:, None] - np.log(np.exp(z - m[:, None]).sum(1, keepdims=True))
    lp[state == "bad"] = np.nan
    lp[state == "empty"] = -np.inf
    return lp, state


def _times_log(p, lp):
    """p ln p, 0 where p is"""
    return np.where(p > 0, p * np.where(p > 0, lp, 0), np.where(np.isnan(p), np.nan, 0.0))


def logprob_forward(x, temperature, tokens, top):
    """(logp, entropy, top_index, top_logp)"""
    rows, cols = x.shape
    lp, state = log_softmax(x / temperature)
    logp = np.zeros(rows)
    for r in range(rows):
        if tokens[r] >= 0:
            logp[r] = lp[r, tokens[r]] if tokens[r] < cols else np.nan
    entropy = -_times_log(np.exp(lp), lp).sum(1) + 0.0
    index, value = np.full((rows, top), -1), np.full((rows, top), -np.inf)
    for r in range(rows):
        if state[r] == "bad":
            value[r] = np.nan
            continue
        order = np.argsort(-x[r], kind="stable")[:top]
        order = order[x[r, order] > -np.inf]
        index[r, :len(order)], value[r, :len(order)] = order, lp[r, order]
    return logp, entropy, index, value


def logprob_backward(x, temperature, tokens, dlogp, dentropy):
    rows, cols = x.shape
    lp, state = log_softmax(x / temperature)
    p = np.exp(lp)
    plp = _times_log(p, lp)
    entropy = -plp.sum(1, keepdims=True)
    dl, dh = dlogp * ((tokens >= 0) & (tokens < cols)), dentropy
    dz = -p * dl[:, None] - dh[:, None] * (plp + p * entropy)
    for r in range(rows):
        if 0 <= tokens[r] < cols:
            dz[r, tokens[r]] += dl[r]
        elif tokens[r] >= cols:
            dz[r] = np.nan
    dz[state == "empty"] = 0
    return dz / temperature


def distill(kind, x, temperature, index, value, weight):
    """(loss, dx); kind "top" or "rest\""""
    rows, cols = x.shape
    lp, state = log_softmax(x / temperature)
    loss, dx = np.zeros(rows), np.zeros(x.shape)
    for r in range(rows):
        if weight is not None and weight[r] == 0:
            continue
        w = 1.0 if weight is None else weight[r]
        there = (index[r] >= 0) & (index[r] < cols)
        at, val = index[r][there], value[r][there]
        if kind == "rest":
            lq, rest = val, 1 - np.exp(val).sum()
            rest = rest if rest >= 2.0 ** -20 else 0.0
        else:
            z = val / temperature
            if not (z > -np.inf).any():
                continue
            lq, rest = z - z.max() - np.log(np.exp(z - z.max()).sum()), 0.0
        q = np.exp(lq)
        if state[r] == "bad":
            loss[r], dx[r] = np.nan, np.nan
            continue
        if state[r] == "empty":
            loss[r] = w * np.inf if (q > 0).any() else 0.0
            continue
        some = q > 0
        total = (q[some] * (lq[some] - lp[r][at[some]])).sum()
        beside = np.ones(cols, bool)
        beside[at] = False
        mass = lp[r][beside]
        top = mass.max(initial=-np.inf)
        log_mass = top + np.log(np.exp(mass - top).sum()) if top > -np.inf else -np.inf
        g = np.exp(lp[r])
        if rest > 0:
            total = total + rest * (np.log(rest) - log_mass)
            if top > -np.inf:
                g[beside] -= rest * np.exp(mass - log_mass)
        np.subtract.at(g, at, q)
        loss[r], dx[r] = w * total, w / temperature * g
    return loss, dx
