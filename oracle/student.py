"""fp64 restatement of the student block's operators (numpy, from the formulas
in include/hcw.h): the gated feed-forward block, the residual norm and the
distillation loss, each with its gradients."""
from __future__ import annotations

import numpy as np
from scipy.special import erf

NONE, RMS, LAYER = 0, 1, 2
SILU, GELU, RELU = 0, 1, 2


# ------------------------------------------------------------------ gated feed-forward block
def act(kind, g):
    """act(g) and act'(g)."""
    if kind == SILU:
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if kind == GELU:
        phi = 0.5 * (1.0 + erf(g / np.sqrt(2.0)))
        return g * phi, phi + g * np.exp(-0.5 * g * g) / np.sqrt(2.0 * np.pi)
    return np.where(g > 0, g, 0.0), (g > 0).astype(np.float64)


def ffn_fwd(x, W1, W2, kind):
    h = W2.shape[1]
    g, u = x @ W1[:h].T, x @ W1[h:].T
    return (act(kind, g)[0] * u) @ W2.T


def ffn_bwd(x, dy, W1, W2, kind):
    """dx, dW1, dW2."""
    h = W2.shape[1]
    g, u = x @ W1[:h].T, x @ W1[h:].T
    ag, dag = act(kind, g)
    da = dy @ W2
    dgu = np.concatenate([da * u * dag, da * ag], axis=1)
    return dgu @ W1, dgu.T @ x, dy.T @ (ag * u)


# ------------------------------------------------------------------ residual norm
def hat(kind, v, eps):
    """vhat and the reciprocal deviation [T, 1]."""
    if kind == NONE:
        return v, np.ones((v.shape[0], 1))
    c = v - v.mean(axis=1, keepdims=True) if kind == LAYER else v
    rs = 1.0 / np.sqrt((c * c).mean(axis=1, keepdims=True) + eps)
    return c * rs, rs


def hat_grad(kind, vh, rs, e):
    if kind == NONE:
        return e
    t = e - vh * (e * vh).mean(axis=1, keepdims=True)
    if kind == LAYER:
        t = t - e.mean(axis=1, keepdims=True)
    return t * rs


def gate_rows(gate, rows_per_gate, T, d):
    if gate is None:
        return np.ones((T, d))
    rows = rows_per_gate or max(T, 1)
    return gate[np.arange(T) // rows]


def norm_fwd(r, f, gate, rows, alpha, post, post_w, post_b, pre, pre_w, pre_b, eps):
    T, d = (f if r is None else r).shape
    s = np.zeros((T, d)) if r is None else alpha * r
    if f is not None:
        v = hat(post, f, eps)[0]
        if post != NONE and post_w is not None:
            v = v * post_w
        if post == LAYER and post_b is not None:
            v = v + post_b
        s = s + gate_rows(gate, rows, T, d) * v
    if pre == NONE:
        return s, None
    x = hat(pre, s, eps)[0]
    if pre_w is not None:
        x = x * pre_w
    if pre == LAYER and pre_b is not None:
        x = x + pre_b
    return s, x


def norm_bwd(dr_out, dx_out, s, f, gate, rows, alpha, post, post_w, post_b, pre, pre_w, eps):
    """Dict of every gradient there is."""
    T, d = (dr_out if dx_out is None else dx_out).shape
    out = {}
    ds = np.zeros((T, d)) if dr_out is None else dr_out.copy()
    if dx_out is not None:
        sh, rs = hat(pre, s, eps)
        ds = ds + hat_grad(pre, sh, rs, dx_out if pre_w is None else dx_out * pre_w)
        out["dpre_w"] = (dx_out * sh).sum(axis=0)
        out["dpre_b"] = dx_out.sum(axis=0)
    out["dr"] = alpha * ds
    if f is not None:
        fh, rf = hat(post, f, eps)
        v = fh
        if post != NONE and post_w is not None:
            v = v * post_w
        if post == LAYER and post_b is not None:
            v = v + post_b
        dv = gate_rows(gate, rows, T, d) * ds
        out["df"] = hat_grad(post, fh, rf, dv if post == NONE or post_w is None else dv * post_w)
        out["dpost_w"] = (dv * fh).sum(axis=0)
        out["dpost_b"] = dv.sum(axis=0)
        step = rows or max(T, 1)
        out["dgate"] = np.stack([(ds * v)[i:i + step].sum(axis=0) for i in range(0, T, step)]) \
            if T else np.zeros((0 if rows else 1, d))
    return out


# ------------------------------------------------------------------ distillation
def _log_softmax(z):
    m = z.max(axis=1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore"):
        return z - m - np.log(np.exp(z - m).sum(axis=1, keepdims=True))


def distill(z, idx, teacher, target, weight, tau, kl, ce):
    """loss [T] and dz [T, V]; rows of weight 0 and rows of -inf alone are zero."""
    T, V = z.shape
    loss, dz = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        w = 1.0 if weight is None else weight[t]
        row = z[t]
        if w == 0.0 or not (row != -np.inf).any():
            continue
        if idx is not None and kl != 0.0:
            on = (idx[t] >= 0) & (idx[t] < V) & (teacher[t] > -np.inf)
            if on.any():
                lp = _log_softmax(teacher[t][on][None] / tau)[0]
                p, at = np.exp(lp), idx[t][on]
                lq = _log_softmax(row[None] / tau)[0]
                use = p > 0
                loss[t] += w * kl * tau * tau * (p[use] * (lp[use] - lq[at][use])).sum()
                g = np.exp(lq)
                np.subtract.at(g, at, p)
                dz[t] += w * kl * tau * g
        if target is not None and ce != 0.0 and 0 <= target[t] < V:
            lq = _log_softmax(row[None])[0]
            loss[t] -= w * ce * lq[target[t]]
            g = np.exp(lq)
            g[target[t]] -= 1.0
            dz[t] += w * ce * g
    return loss, dz
