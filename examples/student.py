"""A student block around the mixing stack, trained from a teacher's top logits, then run one
symbol at a time.

    python examples/student.py [--steps 40] [--tokens 256] [--width 256]

Replacing attention layers of a language model by mixing layers (Eq. (1)) leaves
the block around them as it was: norms before and after each sublayer, a gate on
what the sublayer adds to the residual stream, a gated feed-forward block.  And
it leaves a teacher: the model before the replacement.  One training step here is

    x   = N(E[ids])                               hcw_embed_fwd
    m   = mixing stack of x                       hcw_stack_fwd
    r,x = r + g1 N(m), N(r)                       hcw_residual_norm_fwd
    f   = W2 (silu(Wg x) * Wu x)                  hcw_gated_ffn_fwd
    r,x = r + g2 N(f), N(r)                       hcw_residual_norm_fwd
    z   = Wh x                                    hcw_gemm_bf16
    loss against the teacher's top logits and the next symbol, dz      hcw_distill_loss

and the same calls' backward passes in reverse (hcw_embed_bwd last), before the gradients
of all parameters are clipped together (hcw_clip_grads).  Weights, activations and their
gradients are bf16, norm weights, gates, the logits and the weight gradients
fp32.  The teacher is a frozen table: its top logits for the next symbol given the
current one and the one 4 positions before, which the mixing layer can see.

Run one symbol at a time the same block takes hcw_embed_fwd for the symbol, hcw_decode_step for
the mixing, the head's weights in 4 bits (hcw_q4_matmul) and, before the next symbol is drawn, the
penalties for symbols that occurred already (hcw_logits_edit).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_18145_gb300 import hcw as H  # noqa: E402

# Eq. (1) itself, no activation: bf16 storage moves a pre-activation by about 1 % of its spread,
# so about 0.8 % of a ReLU's decisions would differ from a finer computation's, and the gradients
# would compare to it within several per cent only.  H.HCW_CAUSAL | H.HCW_ACT_RELU trains as well.
FLAGS = H.HCW_CAUSAL
EPS = 1e-5


def init(V, d, h, L, seed=0, device="cuda"):
    """Parameters of the block: name -> tensor (bf16 maps, fp32 norms and gates)."""
    g = torch.Generator(device=device).manual_seed(seed)

    def w(*shape, std):
        return (std * torch.randn(*shape, generator=g, device=device)).to(torch.bfloat16)

    p = dict(E=w(V, d, std=1.0), W_self=w(L, d, d, std=d ** -0.5), W_nbr=w(L, d, d, std=d ** -0.5),
             W1=w(2 * h, d, std=d ** -0.5), W2=w(d, h, std=h ** -0.5), Wh=w(V, d, std=d ** -0.5))
    for name in ("n0", "n1", "n2", "m1", "m2"):         # pre-norms 0, 1, 2; post-norms 1, 2
        p[name] = torch.ones(d, device=device)
    for name in ("g1", "g2"):
        p[name] = torch.full((1, d), 0.5, device=device)
    return p


def join(p, i):
    """What both directions of the i-th join of branch and stream (1 or 2) take."""
    return dict(gate=p["g%d" % i], post=H.HCW_NORM_RMS, post_w=p["m%d" % i], pre=H.HCW_NORM_RMS,
                pre_w=p["n%d" % i], eps=EPS)


def links(L):
    """The layers' links: 4, 8, ... positions back."""
    return [2 + l for l in range(L)]


def step(p, ids, teacher, target, weight, temperature=2.0):
    """Loss of every position and the gradient of every parameter.  ids [B, n],
    teacher (symbols, logits) [B n, K], target and weight [B n]."""
    B, n = ids.shape
    V, d = p["E"].shape
    L = p["W_self"].shape[0]
    dims = links(L)
    ids = ids.reshape(-1).to(torch.int32)
    # forward
    r0, x0 = H.hcw_residual_norm_fwd(H.hcw_embed_fwd(ids, p["E"]), None, pre_w=p["n0"], eps=EPS)
    m, acts, masks = H.hcw_stack_fwd(x0.view(B, n, d), p["W_self"], p["W_nbr"], flags=FLAGS,
                                     dims=dims)
    m = m.view(B * n, d)
    r1, x1 = H.hcw_residual_norm_fwd(r0, m, **join(p, 1))
    f = H.hcw_gated_ffn_fwd(x1, p["W1"], p["W2"])
    r2, x2 = H.hcw_residual_norm_fwd(r1, f, **join(p, 2))
    z = H.hcw_gemm_bf16(x2, p["Wh"], tb=True)
    loss, dz = H.hcw_distill_loss(z, *teacher, target=target, weight=weight,
                                  temperature=temperature, kl_scale=0.5, ce_scale=0.5)
    # backward
    g = {}
    dz = dz.to(torch.bfloat16)
    g["Wh"] = H.hcw_gemm_bf16(dz, x2, ta=True)
    dx2 = H.hcw_gemm_bf16(dz, p["Wh"]).to(torch.bfloat16)
    b = H.hcw_residual_norm_bwd(None, dx2, r2, f, **join(p, 2))
    g["g2"], g["m2"], g["n2"] = b["dgate"], b["dpost_w"], b["dpre_w"]
    dx1, g["W1"], g["W2"] = H.hcw_gated_ffn_bwd(x1, b["df"], p["W1"], p["W2"])
    b = H.hcw_residual_norm_bwd(b["dr"], dx1, r1, m, **join(p, 1))
    g["g1"], g["m1"], g["n1"] = b["dgate"], b["dpost_w"], b["dpre_w"]
    dx0, g["W_self"], g["W_nbr"], _ = H.hcw_stack_bwd(
        x0.view(B, n, d), acts, masks, b["df"].view(B, n, d), p["W_self"], p["W_nbr"], flags=FLAGS,
        want_dbias=False, dims=dims)
    b = H.hcw_residual_norm_bwd(b["dr"], dx0.view(B * n, d), r0, None, pre_w=p["n0"], eps=EPS)
    g["n0"] = b["dpre_w"]
    g["E"] = H.hcw_embed_bwd(ids, b["dr"], V)
    return loss, g


def batch(table, V, B, n, K, gen):
    """Symbols drawn from the teacher's table, its top logits, and the next symbols."""
    ids = torch.randint(V, (B, n + 1), generator=gen, device=table.device)
    logits = torch.empty(B, n, V, device=table.device)
    for t in range(n):
        before = ids[:, t - 4] if t >= 4 else torch.zeros(B, dtype=torch.long, device=table.device)
        logits[:, t] = table[0, ids[:, t]] + table[1, before]
        ids[:, t + 1] = torch.multinomial(logits[:, t].softmax(-1), 1, generator=gen)[:, 0]
    top, at = logits.view(B * n, V).topk(K)
    return (ids[:, :n].to(torch.int32).contiguous(), (at.to(torch.int32).contiguous(), top.contiguous()),
            ids[:, 1:].reshape(-1).to(torch.int32).contiguous())


def packed_head(p, group=64):
    """The head's weights as hcw_q4_matmul reads them."""
    return H.hcw_q4_pack(*H.hcw_q4_quantize(p["Wh"], group), group)


def cache_for(p, B, n):
    """What hcw_decode_step keeps of the positions before."""
    L, d = p["W_self"].shape[:2]
    return torch.empty(H.hcw_decode_cache_bytes(L, B, n, d, links(L)), dtype=torch.uint8,
                       device=p["E"].device)


def next_logits(p, head, symbols, t, n, cache, group=64):
    """Logits [B, V] fp32 for what follows symbols [B] int32 at position t of a window of n, after
    the positions before it in their order."""
    L = p["W_self"].shape[0]
    r, x = H.hcw_residual_norm_fwd(H.hcw_embed_fwd(symbols, p["E"]), None, pre_w=p["n0"], eps=EPS)
    m = H.hcw_decode_step(x, p["W_self"], p["W_nbr"], None, t, n, cache, FLAGS, dims=links(L))
    r, x = H.hcw_residual_norm_fwd(r, m, **join(p, 1))
    f = H.hcw_gated_ffn_fwd(x, p["W1"], p["W2"])
    r, x = H.hcw_residual_norm_fwd(r, f, **join(p, 2))
    return H.hcw_q4_matmul(x, head, p["E"].shape[0], group, y_dtype=torch.float32)


def generate(p, prompt, n, repetition=1.1, frequency=0.05, gen=None):
    """prompt [B, at least 1] int32 continued to n symbols, drawn with penalties for those that a
    sequence holds already."""
    dev, (B, given) = prompt.device, prompt.shape
    head, cache = packed_head(p), cache_for(p, B, n)
    out = torch.full((B, n), -1, dtype=torch.int32, device=dev)
    out[:, :given] = prompt
    row = lambda v, dt: torch.full((B,), v, dtype=dt, device=dev)  # noqa: E731
    own, rep, freq = row(given, torch.int32), row(repetition, torch.float32), \
        row(frequency, torch.float32)
    for t in range(n - 1):
        z = next_logits(p, head, out[:, t].contiguous(), t, n, cache)
        if t + 1 < given:
            continue
        # symbols that are not there yet are -1: empty
        z = H.hcw_logits_edit(z, history=out, prompt=own, repetition=rep, frequency=freq, out=z)
        out[:, t + 1] = torch.multinomial(z.softmax(-1), 1, generator=gen)[:, 0].to(torch.int32)
    return out


def train(steps=40, B=8, n=32, V=97, d=256, h=512, L=1, K=16, lr=3e-3, seed=0, clip=1.0, say=print,
          keep=None):
    """Adam on fp32 copies of the parameters; returns the mean loss of every step.  keep: a dict that
    gets the trained parameters."""
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)
    table = 2.0 * torch.randn(2, V, V, generator=gen, device=dev)
    p = init(V, d, h, L, seed + 1)
    master = {k: v.float().clone() for k, v in p.items()}
    m1 = {k: torch.zeros_like(v) for k, v in master.items()}
    m2 = {k: torch.zeros_like(v) for k, v in master.items()}
    weight = torch.full((B * n,), 1.0 / (B * n), device=dev)
    losses = []
    for s in range(1, steps + 1):
        ids, teacher, target = batch(table, V, B, n, K, gen)
        loss, g = step(p, ids, teacher, target, weight)
        H.hcw_clip_grads(g.values(), clip)
        for k, w in master.items():
            m1[k].lerp_(g[k], 0.1)
            m2[k].lerp_(g[k] * g[k], 0.05)
            w -= lr * (m1[k] / (1 - 0.9 ** s)) / ((m2[k] / (1 - 0.95 ** s)).sqrt() + 1e-8)
            p[k].copy_(w)
        losses.append(loss.sum())
        if say and (s == 1 or s % 10 == 0):
            say("step %3d  loss %.4f" % (s, float(losses[-1])))
    if H.hcw_sync_status() != H.HCW_OK:
        raise RuntimeError("the device reported an error")
    if keep is not None:
        keep.update(p)
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--tokens", type=int, default=256, help="positions a step (windows of 32)")
    ap.add_argument("--width", type=int, default=256, help="a multiple of 64")
    a = ap.parse_args()
    params = {}
    train(a.steps, B=max(1, a.tokens // 32), d=a.width, h=2 * a.width, keep=params)
    start = torch.arange(2, dtype=torch.int32, device="cuda")[:, None]
    for line in generate(params, start, 32).tolist():
        print("symbols", *line)
