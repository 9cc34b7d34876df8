"""fp64 restatement of the operators at a language model's two ends (numpy, from the formulas in
include/hcw.h): symbol lookup with its gradient, clipping by the global norm, products with 4-bit
weights, edits of logits."""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ symbols
def embed_fwd(ids, E, scale):
    x = np.zeros((len(ids), E.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < len(E):
            x[t] = scale * E[v]
    return x


def embed_bwd(ids, dx, V, scale, dE=None):
    out = np.zeros((V, dx.shape[1])) if dE is None else dE.copy()
    for t, v in enumerate(ids):
        if 0 <= v < V:
            out[v] += scale * dx[t]
    return out


# ------------------------------------------------------------------ clipping
def clip(grads, max_norm):
    """The norm, the factor and the clipped gradients."""
    with np.errstate(over="ignore", invalid="ignore"):
        big = max((np.abs(g).max() for g in grads if g.size), default=0.0)
        if np.isfinite(big) and big > 0:
            norm = big * np.sqrt(sum(((g / big) ** 2).sum() for g in grads))
        else:
            norm = big if not np.isnan(big) else np.nan
        for g in grads:
            if np.isnan(g).any():
                norm = np.nan
    c = max_norm / norm if norm > max_norm and np.isfinite(norm) else 1.0
    return norm, c, [c * g for g in grads]


# ------------------------------------------------------------------ weights of 4 bits
def quantize(W, group, round_scale):
    """Codes and scales of W [N, K]; round_scale: fp64 scales to the stored ones.  Division and
    rounding are those of fp32, as stated."""
    N, K = W.shape
    G = -(-K // group)
    codes, scales = np.zeros((N, K), np.int8), np.zeros((N, G))
    for g in range(G):
        w = W[:, g * group:(g + 1) * group].astype(np.float32)
        s = round_scale((np.abs(w).max(axis=1) / np.float32(7)).astype(np.float32)).astype(np.float32)
        scales[:, g] = s
        q = np.where(s[:, None] > 0, np.rint(w / np.where(s > 0, s, 1)[:, None]), 0)
        codes[:, g * group:(g + 1) * group] = np.clip(q, -8, 7)
    return codes, scales


def q4_weights(codes, scales, group):
    return codes * np.repeat(scales, group, axis=1)[:, :codes.shape[1]]


def q4_matmul(x, codes, scales, group, bias=None):
    y = x @ q4_weights(codes, scales, group).T
    return y if bias is None else y + bias


# ------------------------------------------------------------------ logits
def allowed(mask, V):
    """bool [B, V] of the bits of mask [B, W] int32."""
    words = mask.astype(np.int64) & 0xffffffff
    j = np.arange(V)
    return (words[:, j // 32] >> (j % 32) & 1).astype(bool)


def edit(z, history=None, lengths=None, prompt=None, rep=None, freq=None, pres=None, bias_idx=None,
         bias=None, mask=None):
    """The edited logits and, for tolerances, the sum of the magnitudes that enter each."""
    B, V = z.shape
    out, mag = z.copy(), np.abs(z)
    for b in range(B):
        seen, count = np.zeros(V, bool), np.zeros(V)
        if history is not None:
            n = history.shape[1] if lengths is None else min(max(lengths[b], 0), history.shape[1])
            p = 0 if prompt is None else prompt[b]
            for t in range(n):
                v = history[b, t]
                if 0 <= v < V:
                    seen[v] = True
                    count[v] += t >= p
        r = 1.0 if rep is None else rep[b]
        f = 0.0 if freq is None else freq[b]
        q = 0.0 if pres is None else pres[b]
        for j in np.nonzero(seen)[0]:
            v = out[b, j]
            v = v / r if v > 0 else v * r
            out[b, j] = v - f * count[j] - (q if count[j] else 0.0)
            mag[b, j] = abs(v) + abs(f) * count[j] + abs(q)
        if bias_idx is not None:
            for k, j in enumerate(bias_idx[b]):
                if 0 <= j < V:
                    out[b, j] += bias[b, k]
                    mag[b, j] += abs(bias[b, k])
    if mask is not None:
        out[~allowed(mask, V)] = -np.inf
    return out, mag
