"""The operators of a student block that learns from a larger language model, as measurable cases:

  ffn      the gated feed-forward block (hcw_gated_ffn_fwd, hcw_gated_ffn_bwd)
  norm     the norms after one block and before the next, fused with the block's gate and the
           residual scale (hcw_residual_norm_fwd, hcw_residual_norm_bwd)
  distill  the loss against a teacher's top logits, with its gradient (hcw_distill_loss)

A case is a dict of plain values; its "kind" names the operator.  run() computes the plain form
in elementary torch operations, or, where `own` is true, makes the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def listed():
    return [
        # serving one sequence: a single token through the block (width 512, hidden 1024)
        dict(name="ffn_token", kind="ffn", T=1, d=512, h=1024, act="silu", train=False),
        # a prompt of ragged length through a wider block, ragged hidden width
        dict(name="ffn_prompt", kind="ffn", T=333, d=1024, h=2744, act="gelu", train=False),
        # the window-256 training batch: 64 windows, width 512, hidden 1024
        dict(name="ffn_train", kind="ffn", T=16384, d=512, h=1024, act="silu", train=True),
        # the block of a billion-parameter model, one batch: the throughput end
        dict(name="ffn_train_wide", kind="ffn", T=8192, d=2048, h=5632, act="silu", train=True),
        # serving 64 sequences, one position a call
        dict(name="norm_tokens", kind="norm", T=64, d=512, rows=0, layer=False, f32=False,
             step=False),
        # the window-256 training batch with LayerNorms
        dict(name="norm_train", kind="norm", T=16384, d=512, rows=0, layer=True, f32=False,
             step=True),
        # odd width and length, fp32, a gate for each sample of 256 positions
        dict(name="norm_odd_f32", kind="norm", T=4099, d=777, rows=256, layer=False, f32=True,
             step=True),
        # a wide model's batch
        dict(name="norm_train_wide", kind="norm", T=32768, d=4096, rows=0, layer=False, f32=False,
             step=True),
        # scoring eight positions against a teacher: the loss alone
        dict(name="distill_score", kind="distill", T=8, V=32000, K=32, tau=1.0, ce=False,
             f32=False, pad=0, grad=False),
        # the character LM's batch (201 symbols), with the hard labels
        dict(name="distill_chars", kind="distill", T=16384, V=201, K=16, tau=2.0, ce=True,
             f32=False, pad=0, grad=True),
        # a word-piece vocabulary of odd size, fp32 logits, hard labels at another temperature
        dict(name="distill_odd_f32", kind="distill", T=1000, V=32003, K=50, tau=2.0, ce=True,
             f32=True, pad=0, grad=True),
        # the largest vocabulary, padded columns masked
        dict(name="distill_large", kind="distill", T=2048, V=131072, K=64, tau=1.0, ce=True,
             f32=False, pad=72, grad=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["ffn", "norm", "distill"])
    if kind == "ffn":
        while True:
            T, train = _log(rng, 1, 16384), rng.random() < 0.6
            d, h = 8 * _log(rng, 8, 256), 8 * _log(rng, 16, 704)
            if (3 if train else 1) * T * d * h <= 3 * 8192 * 2048 * 5632:
                return dict(kind=kind, T=T, d=d, h=h, act=rng.choice(["silu", "gelu", "relu"]),
                            train=train)
    if kind == "norm":
        while True:
            T, d, f32 = _log(rng, 1, 65536), _log(rng, 64, 8192), rng.random() < 0.3
            if rng.random() < 0.6:
                d = (d + 7) // 8 * 8
            if T * d * (2 if f32 else 1) <= 32768 * 4096:
                return dict(kind=kind, T=T, d=d, rows=rng.choice([0, 0, 64, 256]),
                            layer=rng.random() < 0.5, f32=f32, step=rng.random() < 0.7)
    while True:
        T, V, f32 = _log(rng, 1, 16384), _log(rng, 128, 131072), rng.random() < 0.3
        if rng.random() < 0.5:
            V = (V + 63) // 64 * 64
        if T * V * (2 if f32 else 1) <= 2048 * 131072:
            return dict(kind=kind, T=T, V=V, K=_log(rng, 1, 64), tau=rng.choice([1.0, 1.0, 2.0, 3.5]),
                        ce=rng.random() < 0.6, f32=f32, pad=rng.choice([0, 0, V // 50]),
                        grad=rng.random() < 0.8)


# ------------------------------------------------------------------ inputs
def _rand(gen, *shape, std=1.0, dtype=F32):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=F32).mul_(std).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return {"case": case, **globals()["_prepare_" + case["kind"]](case, gen)}


def _prepare_ffn(c, gen):
    T, d, h = c["T"], c["d"], c["h"]
    s = dict(x=_rand(gen, T, d, dtype=BF16),                              # normed activations
             W1=_rand(gen, 2 * h, d, std=d ** -0.5, dtype=BF16),
             W2=_rand(gen, d, h, std=h ** -0.5, dtype=BF16),
             y=torch.empty(T, d, dtype=BF16, device=DEV))
    if c["train"]:
        s.update(dy=_rand(gen, T, d, std=0.02, dtype=BF16),
                 dx=torch.empty(T, d, dtype=BF16, device=DEV),
                 # gradients in the weights' type, as the optimiser takes them
                 dW1=torch.empty(2 * h, d, dtype=BF16, device=DEV),
                 dW2=torch.empty(d, h, dtype=BF16, device=DEV))
    return s


def _prepare_norm(c, gen):
    T, d, dt = c["T"], c["d"], F32 if c["f32"] else BF16
    G = 1 if c["rows"] == 0 else -(-T // c["rows"])
    # a residual stream with a few features far larger than the rest, as trained models have
    big = 1.0 + 20.0 * (torch.rand(d, generator=gen, device=DEV) < 0.01)
    s = dict(r=(_rand(gen, T, d, std=2.0) * big).to(dt),
             f=(_rand(gen, T, d) + 0.3).to(dt),
             gate=0.5 + 0.3 * _rand(gen, G, d),
             post_w=1.0 + 0.2 * _rand(gen, d), pre_w=1.0 + 0.2 * _rand(gen, d),
             post_b=0.1 * _rand(gen, d) if c["layer"] else None,
             pre_b=0.1 * _rand(gen, d) if c["layer"] else None,
             alpha=0.9)
    s.update(r_out=torch.empty_like(s["r"]), x_out=torch.empty_like(s["r"]))
    if c["step"]:
        # the stream as the forward pass stored it, and the gradients that come back
        s.update(s=(_rand(gen, T, d, std=2.0) * big).to(dt),
                 dr_out=_rand(gen, T, d, std=0.02, dtype=dt),
                 dx_out=_rand(gen, T, d, std=0.02, dtype=dt),
                 dr=torch.empty_like(s["r"]), df=torch.empty_like(s["r"]))
    return s


def _prepare_distill(c, gen):
    T, V, K = c["T"], c["V"], min(c["K"], c["V"] - c["pad"])
    live = V - c["pad"]
    z = _rand(gen, T, V, std=2.0)
    # the teacher's top logits, largest first, at symbols spread over the vocabulary
    first = torch.randint(live, (T, 1), generator=gen, device=DEV)
    idx = (first + torch.arange(K, device=DEV)[None, :] * max(1, live // K)) % live
    teacher = 14.0 - 0.9 * _rand(gen, T, K).abs().cumsum(1)
    # a student that has learnt part of it
    z.scatter_add_(1, idx, 0.6 * teacher)
    z = z.to(F32 if c["f32"] else BF16)
    z[:, live:] = -math.inf                       # padded columns of the head
    idx = idx.to(torch.int32)
    u = torch.rand(T, generator=gen, device=DEV)
    # a tenth of the positions is padding (no weight); a few have fewer teacher entries, or none
    weight = torch.where(u < 0.1, 0.0, 1.0 / T)
    have = torch.where(u > 0.95, torch.randint(K + 1, (T,), generator=gen, device=DEV), K)
    idx = torch.where(torch.arange(K, device=DEV)[None, :] < have[:, None], idx, -1)
    target = torch.randint(live, (T,), generator=gen, device=DEV).to(torch.int32)
    target = torch.where(u < 0.2, -1, target).to(torch.int32)
    # padding positions hold whatever was in memory
    z[u < 0.02] = math.nan
    return dict(z=z.contiguous(), idx=idx.to(torch.int32).contiguous(), teacher=teacher.contiguous(),
                target=target.contiguous() if c["ce"] else None, weight=weight.contiguous(),
                loss=torch.empty(T, dtype=F32, device=DEV),
                dz=torch.empty_like(z) if c["grad"] else None)


# ------------------------------------------------------------------ one pass
def run(state):
    name = ("_own_" if own else "_plain_") + state["case"]["kind"]
    return globals()[name](state["case"], state)


def _own_ffn(c, s):
    from paper_2609_18145_gb300 import hcw as H
    act = {"silu": H.HCW_GATE_SILU, "gelu": H.HCW_GATE_GELU, "relu": H.HCW_GATE_RELU}[c["act"]]
    if "workspace" not in s:
        need = H.hcw_gated_ffn_fwd_workspace_bytes(c["T"], c["d"], c["h"])
        if c["train"]:
            need = max(need, H.hcw_gated_ffn_bwd_workspace_bytes(c["T"], c["d"], c["h"]))
        s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    out = dict(y=H.hcw_gated_ffn_fwd(s["x"], s["W1"], s["W2"], act, y=s["y"],
                                     workspace=s["workspace"]))
    if c["train"]:
        out["dx"], out["dW1"], out["dW2"] = H.hcw_gated_ffn_bwd(
            s["x"], s["dy"], s["W1"], s["W2"], act, dx=s["dx"], dW1=s["dW1"], dW2=s["dW2"],
            workspace=s["workspace"])
    return out


def _own_norm(c, s):
    from paper_2609_18145_gb300 import hcw as H
    kind = H.HCW_NORM_LAYER if c["layer"] else H.HCW_NORM_RMS
    par = dict(gate=s["gate"], rows_per_gate=c["rows"], alpha=s["alpha"], post_w=s["post_w"],
               pre_w=s["pre_w"], post=kind, pre=kind, eps=EPS)
    r_out, x_out = H.hcw_residual_norm_fwd(s["r"], s["f"], post_b=s["post_b"], pre_b=s["pre_b"],
                                           r_out=s["r_out"], x_out=s["x_out"], **par)
    out = dict(r_out=r_out, x_out=x_out)
    if c["step"]:
        if "workspace" not in s:
            need = H.hcw_residual_norm_bwd_workspace_bytes(c["T"], c["d"], c["rows"])
            s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
        g = H.hcw_residual_norm_bwd(s["dr_out"], s["dx_out"], s["s"], s["f"], want_bias=c["layer"],
                                    dr=s["dr"], df=s["df"], workspace=s["workspace"],
                                    post_b=s["post_b"], **par)
        out.update(g)
    return out


def _own_distill(c, s):
    from paper_2609_18145_gb300 import hcw as H
    loss, dz = H.hcw_distill_loss(s["z"], s["idx"], s["teacher"], target=s["target"],
                                  weight=s["weight"], temperature=c["tau"], kl_scale=0.7,
                                  ce_scale=0.3 if c["ce"] else 0.0, loss=s["loss"], dz=s["dz"],
                                  want_grad=c["grad"])
    return dict(loss=loss, dz=dz) if c["grad"] else dict(loss=loss)


def _act(name, g):
    """act(g) and its derivative."""
    if name == "silu":
        sg = 1.0 / (1.0 + torch.exp(-g))
        return g * sg, sg * (1.0 + g * (1.0 - sg))
    if name == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    pos = (g > 0).float()
    return g * pos, pos


def _plain_ffn(c, s):
    h = c["h"]
    x, W1, W2 = s["x"].float(), s["W1"].float(), s["W2"].float()
    gu = x @ W1.t()
    g, u = gu[:, :h], gu[:, h:]
    ag, dg_ = _act(c["act"], g)
    a = ag * u
    out = dict(y=(a @ W2.t()).to(BF16))
    if c["train"]:
        dy = s["dy"].float()
        da = dy @ W2
        dgu = torch.cat([da * u * dg_, da * ag], dim=1)
        out.update(dx=(dgu @ W1).to(BF16), dW1=(dgu.t() @ x).to(BF16), dW2=(dy.t() @ a).to(BF16))
    return out


def _hat(layer, v):
    """The normed rows and the reciprocal deviations."""
    if layer:
        v = v - v.mean(dim=1, keepdim=True)
    rs = 1.0 / torch.sqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    return v * rs, rs


def _hat_grad(layer, hat, rs, dhat):
    t = dhat - hat * (dhat * hat).mean(dim=1, keepdim=True)
    if layer:
        t = t - dhat.mean(dim=1, keepdim=True)
    return t * rs


def _plain_norm(c, s):
    layer, T, dt = c["layer"], c["T"], s["r"].dtype
    rows = c["rows"] or T
    G = -(-T // rows)
    gate = s["gate"].repeat_interleave(rows, dim=0)[:T] if G > 1 else s["gate"]
    f = s["f"].float()
    fh, frs = _hat(layer, f)
    v = fh * s["post_w"]
    if layer:
        v = v + s["post_b"]
    st = s["alpha"] * s["r"].float() + gate * v
    sh, _ = _hat(layer, st)
    x = sh * s["pre_w"]
    if layer:
        x = x + s["pre_b"]
    out = dict(r_out=st.to(dt), x_out=x.to(dt))
    if c["step"]:
        dx = s["dx_out"].float()
        sh, srs = _hat(layer, s["s"].float())
        ds = s["dr_out"].float() + _hat_grad(layer, sh, srs, dx * s["pre_w"])
        dv = gate * ds
        df = _hat_grad(layer, fh, frs, dv * s["post_w"])
        dgate = ds * v
        if G > 1:
            pad = torch.zeros(G * rows - T, c["d"], device=DEV)
            dgate = torch.cat([dgate, pad]).view(G, rows, c["d"]).sum(dim=1)
        else:
            dgate = dgate.sum(dim=0, keepdim=True)
        out.update(dr=(s["alpha"] * ds).to(dt), df=df.to(dt), dgate=dgate,
                   dpost_w=(dv * fh).sum(dim=0), dpre_w=(dx * sh).sum(dim=0))
        if layer:
            out.update(dpost_b=dv.sum(dim=0), dpre_b=dx.sum(dim=0))
    return out


def _plain_distill(c, s):
    tau, V = c["tau"], c["V"]
    a, b = 0.7, 0.3 if c["ce"] else 0.0
    z, idx, w = s["z"].float(), s["idx"].long(), s["weight"][:, None]
    used = w != 0
    z = torch.where(used, z, 0.0)
    slot = idx >= 0
    at = idx.clamp(min=0)
    t = torch.where(slot, s["teacher"].float() / tau, -math.inf)
    tm = t.amax(dim=1, keepdim=True)
    e = torch.exp(t - torch.where(torch.isfinite(tm), tm, 0.0))
    te = e.sum(dim=1, keepdim=True)
    any_ = te > 0
    p = e / torch.where(any_, te, 1.0)
    m = z.amax(dim=1, keepdim=True)
    ez = torch.exp((z - m) / tau)
    sz = ez.sum(dim=1, keepdim=True)
    logq = (z.gather(1, at) - m) / tau - torch.log(sz)
    logp = torch.where(slot, t - tm - torch.log(torch.where(any_, te, 1.0)), 0.0)
    kl = torch.where(slot, p * (logp - logq), 0.0).sum(dim=1, keepdim=True)
    loss = a * tau * tau * kl
    if c["grad"]:
        dz = (a * tau) * (any_ * (ez / sz))
        dz.scatter_add_(1, at, torch.where(slot, -(a * tau) * p, 0.0))
    if c["ce"]:
        y = s["target"].long()[:, None]
        has = y >= 0
        y = y.clamp(min=0)
        e1 = torch.exp(z - m) if tau != 1.0 else ez
        s1 = e1.sum(dim=1, keepdim=True)
        loss = loss + b * torch.where(has, torch.log(s1) - (z.gather(1, y) - m), 0.0)
        if c["grad"]:
            dz += b * (has * (e1 / s1))
            dz.scatter_add_(1, y, torch.where(has, -b, 0.0))
    out = dict(loss=torch.where(used, w * loss, 0.0)[:, 0])
    if c["grad"]:
        out["dz"] = torch.where(used, w * dz, 0.0).to(s["z"].dtype)
    return out


# ------------------------------------------------------------------ 64 bits, by differentiation
def exact(case, seed):
    return globals()["_exact_" + case["kind"]](case, prepare(case, seed))


def _exact_ffn(c, s):
    x, W1, W2 = (s[k].double().requires_grad_(c["train"]) for k in ("x", "W1", "W2"))
    gate, up = (x @ W1.T).split(c["h"], dim=1)
    f = {"silu": lambda v: v * torch.sigmoid(v),
         "gelu": lambda v: 0.5 * v * torch.erfc(-v / math.sqrt(2.0)),
         "relu": torch.relu}[c["act"]]
    y = (f(gate) * up) @ W2.T
    if not c["train"]:
        return dict(y=y)
    dx, dW1, dW2 = torch.autograd.grad(y, (x, W1, W2), s["dy"].double())
    return dict(y=y.detach(), dx=dx, dW1=dW1, dW2=dW2)


def _exact_norm(c, s):
    d = c["d"]
    par = [k for k in ("post_w", "post_b", "pre_w", "pre_b") if s[k] is not None]
    q = {k: s[k].double() for k in ("r", "f", "gate", *par)}
    if c["step"]:
        q = {k: t.requires_grad_() for k, t in q.items()}

    def normed(v, at):
        if c["layer"]:
            var, mean = torch.var_mean(v, dim=1, unbiased=False, keepdim=True)
            return (v - mean) * torch.rsqrt(var + EPS) * q[at + "_w"] + q[at + "_b"]
        return v * torch.rsqrt(v.square().sum(1, keepdim=True) / d + EPS) * q[at + "_w"]

    group = torch.arange(c["T"], device=DEV) // (c["rows"] or c["T"])
    branch = q["gate"][group] * normed(q["f"], "post")
    r_out = s["alpha"] * q["r"] + branch
    out = dict(r_out=r_out.detach(), x_out=normed(r_out, "pre").detach())
    if c["step"]:
        # the backward pass starts from the stored stream
        st = s["s"].double().requires_grad_()
        names = [k for k in ("pre_w", "pre_b") if k in q]
        got = torch.autograd.grad(normed(st, "pre"), [st] + [q[k] for k in names],
                                  s["dx_out"].double())
        ds = s["dr_out"].double() + got[0]
        out.update({"d" + k: g for k, g in zip(names, got[1:])})
        names = ["r", "f", "gate"] + [k for k in ("post_w", "post_b") if k in q]
        out.update({"d" + k: g for k, g in
                    zip(names, torch.autograd.grad(r_out, [q[k] for k in names], ds))})
    return out


def _exact_distill(c, s):
    tau, a, b = c["tau"], 0.7, 0.3
    w = s["weight"].double()
    z = torch.where((w != 0)[:, None], s["z"].double(), 0.0).requires_grad_(c["grad"])
    lq = torch.log_softmax(z / tau, dim=1)
    slot = s["idx"] >= 0
    some = slot.any(dim=1)
    t = torch.where(slot, s["teacher"].double() / tau, -math.inf)
    t = torch.where(some[:, None], t, 0.0)
    lp = torch.log_softmax(t, dim=1)
    at = s["idx"].long().clamp(min=0)
    term = torch.where(slot, lp.exp() * (torch.where(slot, lp, 0.0) - lq.gather(1, at)), 0.0)
    loss = a * tau ** 2 * term.sum(dim=1)
    if c["ce"]:
        y = s["target"].long()
        ce = torch.logsumexp(z, dim=1) - z.gather(1, y.clamp(min=0)[:, None])[:, 0]
        loss = loss + b * torch.where(y >= 0, ce, 0.0)
    loss = loss * w
    if not c["grad"]:
        return dict(loss=loss)
    (dz,) = torch.autograd.grad(loss.sum(), z)
    return dict(loss=loss.detach(), dz=dz)


def work(case):
    c = case
    if c["kind"] == "ffn":
        T, d, h = c["T"], c["d"], c["h"]
        fwd = 2 * (2 * T * d + 3 * d * h)
        bwd = 2 * (3 * T * d + 6 * d * h)
        return {"bytes": fwd + (bwd if c["train"] else 0),
                "flops": (18 if c["train"] else 6) * T * d * h}
    if c["kind"] == "norm":
        T, d, e = c["T"], c["d"], 4 if c["f32"] else 2
        G = 1 if c["rows"] == 0 else -(-T // c["rows"])
        par = 4 * d * (G + (4 if c["layer"] else 2))
        return {"bytes": 4 * T * d * e + par + (6 * T * d * e + 2 * par if c["step"] else 0),
                "flops": T * d * (12 + (30 if c["step"] else 0))}
    T, V, K, e = c["T"], c["V"], c["K"], 4 if c["f32"] else 2
    return {"bytes": T * V * e * (2 if c["grad"] else 1) + T * (8 * K + 12),
            "flops": T * V * ((8 if c["grad"] else 4) + (4 if c["ce"] and c["tau"] != 1 else 0))}
