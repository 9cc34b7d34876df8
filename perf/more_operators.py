"""The operators at a language model's two ends, around the mixing stack, as measurable cases:

  embed    the lookup of symbols with a scale, and its gradient (hcw_embed_fwd, hcw_embed_bwd)
  clip     the norm over the gradients of all parameters, and clipping by it (hcw_clip_grads)
  q4       products of a few tokens with 4-bit weights and group scales (hcw_q4_matmul)
  logits   penalties for repeated symbols, biases and grammar masks (hcw_logits_edit)

A case is a dict of plain values; its "kind" names the operator.  run() computes the plain form
in elementary torch operations, or, where `own` is true, makes the library's calls.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def listed():
    return [
        # serving 64 sequences, one position a call
        dict(name="embed_tokens", kind="embed", T=64, V=32000, d=512, f32=False, grad=False),
        # the character LM's training batch: every symbol occurs about 80 times, some far more often
        dict(name="embed_chars", kind="embed", T=16384, V=201, d=512, f32=False, grad=True),
        # odd length, vocabulary and width, fp32
        dict(name="embed_odd_f32", kind="embed", T=4099, V=32003, d=777, f32=True, grad=True),
        # a wide model's batch over the largest vocabulary
        dict(name="embed_large", kind="embed", T=65536, V=131072, d=2048, f32=False, grad=True),
        # a one-layer student's parameters, fp32 gradients
        dict(name="clip_student", kind="clip", layers=1, V=97, d=256, h=512, f32=True, over=True),
        # eight layers of a billion-parameter model, bf16 gradients, fp32 ones of the norms
        dict(name="clip_large", kind="clip", layers=8, V=32000, d=2048, h=5632, f32=False, over=True),
        # serving one sequence: a token through the up products of a block (width 512, hidden 1024)
        dict(name="q4_token", kind="q4", T=1, N=2048, K=512, group=64, f32=False, bias=False),
        # five sequences at a head of odd size: fp32 logits, a bias, a ragged last group
        dict(name="q4_head_odd", kind="q4", T=5, N=32003, K=1000, group=32, f32=True, bias=True),
        # sixteen sequences at the head of a wide model: the throughput end
        dict(name="q4_large", kind="q4", T=16, N=131072, K=4096, group=128, f32=True, bias=False),
        # one character-LM sequence
        dict(name="logits_chars", kind="logits", B=1, V=201, H=256, M=0, f32=True, mask=False),
        # a batch over an odd word-piece vocabulary with a grammar each
        dict(name="logits_batch", kind="logits", B=64, V=32003, H=1024, M=40, f32=False, mask=True),
        # a large batch over the largest vocabulary, long histories
        dict(name="logits_large", kind="logits", B=256, V=131072, H=4096, M=300, f32=True, mask=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "clip", "q4", "logits"])
    if kind == "embed":
        while True:
            T, V, d = _log(rng, 1, 65536), _log(rng, 128, 131072), _log(rng, 16, 4096)
            if rng.random() < 0.6:
                d = (d + 7) // 8 * 8
            f32, grad = rng.random() < 0.3, rng.random() < 0.7
            if (V + T) * d * (2 if f32 else 1) <= (131072 + 65536) * 2048:
                return dict(kind=kind, T=T, V=V, d=d, f32=f32, grad=grad)
    if kind == "clip":
        while True:
            layers, V, d = _log(rng, 1, 48), _log(rng, 64, 131072), _log(rng, 64, 4096)
            h = (d * rng.choice([2, 2, 3]) * 7 // 8 + 7) // 8 * 8
            c = dict(kind=kind, layers=layers, V=V, d=d, h=h, f32=rng.random() < 0.5,
                     over=rng.random() < 0.8)
            if sum(_sizes(c)) * (2 if c["f32"] else 1) <= 400e6:
                return c
    if kind == "q4":
        while True:
            N, K = _log(rng, 64, 131072), 8 * _log(rng, 16, 1024)
            if N * K <= 131072 * 4096:
                return dict(kind=kind, T=_log(rng, 1, 16), N=N, K=K,
                            group=rng.choice([32, 64, 128]), f32=rng.random() < 0.4,
                            bias=rng.random() < 0.3)
    while True:
        B, V, f32 = _log(rng, 1, 256), _log(rng, 128, 131072), rng.random() < 0.5
        if B * V * (2 if f32 else 1) <= 256 * 131072 * 2:
            return dict(kind=kind, B=B, V=V, H=_log(rng, 1, 4096), f32=f32,
                        M=rng.choice([0, 0, 8, 40, 300]), mask=rng.random() < 0.6)


# ------------------------------------------------------------------ inputs
def _rand(gen, *shape, std=1.0, dtype=F32):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=F32).mul_(std).to(dtype)


def _symbols(gen, V, *shape):
    """Symbols as text has them: the r-th most frequent about 1 / r times as often as the first."""
    u = torch.rand(*shape, generator=gen, device=DEV)
    return (torch.exp(u * math.log(V + 1.0)).long() - 1).clamp_(0, V - 1).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    return {"case": case, **globals()["_prepare_" + case["kind"]](case, gen)}


def _prepare_embed(c, gen):
    T, V, d, dt = c["T"], c["V"], c["d"], F32 if c["f32"] else BF16
    ids = _symbols(gen, V, T)
    # a fiftieth of the positions is padding
    ids = torch.where(torch.rand(T, generator=gen, device=DEV) < 0.02, -1, ids).to(torch.int32)
    s = dict(ids=ids.contiguous(), E=_rand(gen, V, d, std=d ** -0.5, dtype=dt), scale=d ** 0.5,
             x=torch.empty(T, d, dtype=dt, device=DEV))
    if c["grad"]:
        s.update(dx=_rand(gen, T, d, std=0.02, dtype=dt),
                 dE=torch.empty(V, d, dtype=F32, device=DEV))
    return s


def _sizes(c):
    """Elements of the gradients: a layer's two maps, its feed-forward block and its small
    vectors, then the embedding, the head and the last norm."""
    d, h = c["d"], c["h"]
    return [d * d, d * d, 2 * h * d, d * h, d, d, d, d] * c["layers"] + [c["V"] * d, c["V"] * d, d]


def _flat(grads, dtype=None):
    """Zeroed buffers, one for each type, and a view of its size and type for every gradient in
    them; each starts at a multiple of 64 elements."""
    size, place = {}, []
    for g in grads:
        at = size.get(g.dtype, 0)
        place.append(at)
        size[g.dtype] = at + (g.numel() + 63) // 64 * 64
    flat = {t: torch.zeros(n, dtype=dtype or t, device=DEV) for t, n in size.items()}
    views = [flat[g.dtype][at:at + g.numel()] for g, at in zip(grads, place)]
    return [flat[t] for t in (BF16, F32) if t in flat], views


def _prepare_clip(c, gen):
    grads, n2 = [], 0.0
    for n in _sizes(c):
        # the small vectors' gradients are fp32 and larger than the maps'
        small = n == c["d"]
        std = 0.05 if small else 1e-3
        grads.append(_rand(gen, n, std=std, dtype=F32 if small or c["f32"] else BF16))
        n2 += n * std * std
    # the clipped gradients go to one buffer for each type, as an optimiser keeps them
    flat, out = _flat(grads)
    return dict(grads=grads, max_norm=math.sqrt(n2) * (0.3 if c["over"] else 3.0), flat=flat, out=out)


def _prepare_q4(c, gen):
    T, N, K, group = c["T"], c["N"], c["K"], c["group"]
    G = -(-K // group)
    # weights as a layer has them, quantised by their groups' largest magnitude
    w = torch.zeros(N, G * group, device=DEV)
    w[:, :K] = _rand(gen, N, K, std=K ** -0.5)
    w = w.view(N, G, group)
    scales = (w.abs().amax(dim=2) / 7.0).to(BF16)
    w /= scales.float().clamp(min=1e-30)[:, :, None]
    codes = w.round_().clamp_(-8, 7).to(torch.int8).view(N, G * group)[:, :K].contiguous()
    # activations with a few features far larger than the rest, as trained models have
    x = _rand(gen, T, K) * (1.0 + 20.0 * (torch.rand(K, generator=gen, device=DEV) < 0.01))
    return dict(x=x.to(BF16), codes=codes, scales=scales.contiguous(),
                bias=_rand(gen, N, std=0.1) if c["bias"] else None,
                y=torch.empty(T, N, dtype=F32 if c["f32"] else BF16, device=DEV))


def _prepare_logits(c, gen):
    B, V, H, M, dt = c["B"], c["V"], c["H"], c["M"], F32 if c["f32"] else BF16
    z = _rand(gen, B, V, std=3.0, dtype=dt)
    history = _symbols(gen, V, B, H)
    lengths = torch.randint(H // 2, H + 1, (B,), generator=gen, device=DEV).to(torch.int32)
    prompt = (lengths * torch.rand(B, generator=gen, device=DEV)).to(torch.int32)
    row = lambda lo, hi: lo + (hi - lo) * torch.rand(B, generator=gen, device=DEV)  # noqa: E731
    s = dict(z=z, history=history, lengths=lengths, prompt=prompt, repetition=row(1.0, 1.5),
             frequency=row(0.0, 0.5), presence=row(-0.2, 0.8), out=torch.empty_like(z),
             bias_idx=None, bias=None, mask=None)
    if M:
        # a request's own biases; some slots are empty
        first = torch.randint(V, (B, 1), generator=gen, device=DEV)
        idx = (first + torch.arange(M, device=DEV)[None, :] * max(1, V // M)) % V
        idx = torch.where(torch.rand(B, M, generator=gen, device=DEV) < 0.1, -1, idx)
        s.update(bias_idx=idx.to(torch.int32).contiguous(), bias=_rand(gen, B, M, std=4.0))
    if c["mask"]:
        # a grammar lets runs of symbols through; bits past the last symbol are anything
        W = -(-V // 32)
        word = torch.randint(-2 ** 31, 2 ** 31, (B, W), generator=gen, device=DEV)
        some = torch.rand(B, W, generator=gen, device=DEV)
        word = torch.where(some < 0.7, 0, torch.where(some < 0.85, -1, word))
        s["mask"] = word.to(torch.int32).contiguous()
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    name = ("_own_" if own else "_plain_") + state["case"]["kind"]
    return globals()[name](state["case"], state)


def _own_embed(c, s):
    from paper_2609_18145_gb300 import hcw as H
    out = dict(x=H.hcw_embed_fwd(s["ids"], s["E"], scale=s["scale"], x=s["x"]))
    if c["grad"]:
        if "workspace" not in s:
            need = H.hcw_embed_bwd_workspace_bytes(c["T"], c["V"], c["d"])
            s["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
        out["dE"] = H.hcw_embed_bwd(s["ids"], s["dx"], c["V"], scale=s["scale"], dE=s["dE"],
                                    workspace=s["workspace"])
    return out


def _own_clip(c, s):
    from paper_2609_18145_gb300 import hcw as H
    if "list" not in s:
        s["list"] = H.GradList(s["grads"], out=s["out"])
        s["workspace"] = torch.empty(H.hcw_clip_grads_workspace_bytes(len(s["grads"])),
                                     dtype=torch.uint8, device=DEV)
        s["norm"] = torch.empty(2, dtype=F32, device=DEV)
    norm = H.hcw_clip_grads(s["list"], s["max_norm"], norm=s["norm"], workspace=s["workspace"])
    return dict(flat=s["flat"], norm=norm)


def _own_q4(c, s):
    from paper_2609_18145_gb300 import hcw as H
    if "packed" not in s:
        s["packed"] = H.hcw_q4_pack(s["codes"], s["scales"], c["group"])
    return dict(y=H.hcw_q4_matmul(s["x"], s["packed"], c["N"], c["group"], bias=s["bias"],
                                  y=s["y"]))


def _own_logits(c, s):
    from paper_2609_18145_gb300 import hcw as H
    return dict(out=H.hcw_logits_edit(
        s["z"], history=s["history"], lengths=s["lengths"], prompt=s["prompt"],
        repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
        bias_idx=s["bias_idx"], bias=s["bias"], mask=s["mask"], out=s["out"]))


def _plain_embed(c, s):
    ids, dt = s["ids"].long(), s["E"].dtype
    have = (ids >= 0)[:, None]
    at = ids.clamp(min=0)
    out = dict(x=torch.where(have, s["scale"] * s["E"][at].float(), 0.0).to(dt))
    if c["grad"]:
        dE = torch.zeros(c["V"], c["d"], device=DEV)
        dE.index_add_(0, at, torch.where(have, s["scale"] * s["dx"].float(), 0.0))
        out["dE"] = dE
    return out


def _plain_clip(c, s):
    # a sum over every parameter is a long one
    n2 = torch.stack([(g.float() * g.float()).sum(dtype=F64) for g in s["grads"]]).sum()
    norm = torch.sqrt(n2)
    factor = (s["max_norm"] / norm).clamp(max=1.0)
    f = factor.float()
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * f)
    return dict(flat=s["flat"], norm=torch.stack([norm, factor]).float())


def _plain_q4(c, s):
    N, K, group = c["N"], c["K"], c["group"]
    scale = s["scales"].float().repeat_interleave(group, dim=1)[:, :K]
    y = s["x"].float() @ (s["codes"].float() * scale).t()
    if c["bias"]:
        y = y + s["bias"]
    return dict(y=y.to(s["y"].dtype))


def _plain_logits(c, s):
    B, V, H = c["B"], c["V"], c["H"]
    z = s["z"].float()
    at = torch.arange(H, device=DEV)[None, :]
    hist = s["history"].long()
    there = (at < s["lengths"][:, None]).float()
    mine = there * (at >= s["prompt"][:, None])
    seen = torch.zeros(B, V, device=DEV).scatter_add_(1, hist, there)
    count = torch.zeros(B, V, device=DEV).scatter_add_(1, hist, mine)
    r = s["repetition"][:, None]
    z = torch.where(seen > 0, torch.where(z > 0, z / r, z * r), z)
    z = z - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if c["M"]:
        idx = s["bias_idx"].long()
        z.scatter_add_(1, idx.clamp(min=0), torch.where(idx >= 0, s["bias"], 0.0))
    if c["mask"]:
        word = s["mask"].long()[:, :, None]
        bit = (word >> torch.arange(32, device=DEV)) & 1
        z = torch.where(bit.view(B, -1)[:, :V] != 0, z, -math.inf)
    return dict(out=z.to(s["z"].dtype))


# ------------------------------------------------------------------ 64 bits, from the definitions
def exact(case, seed):
    return globals()["_exact_" + case["kind"]](case, prepare(case, seed))


def _exact_embed(c, s):
    V, d = c["V"], c["d"]
    # one more row of zeros stands for padding
    table = torch.cat([s["E"].double(), torch.zeros(1, d, dtype=F64, device=DEV)])
    ids = s["ids"].long() % (V + 1)
    out = dict(x=table[ids] * s["scale"])
    if c["grad"]:
        # the rows in the order of their symbols: differences of running sums would lose digits,
        # so the sum goes through equal runs of the sorted rows, a column block at a time
        order = torch.argsort(ids, stable=True)
        lengths = torch.bincount(ids, minlength=V + 1)
        dE = torch.empty(V, d, dtype=F64, device=DEV)
        for j in range(0, d, 256):
            rows = s["dx"][order, j:j + 256].double()
            dE[:, j:j + 256] = torch.segment_reduce(rows, "sum", lengths=lengths, axis=0,
                                                    initial=0.0)[:V]
        out["dE"] = dE.mul_(s["scale"])
    return out


def _exact_clip(c, s):
    norm = math.sqrt(math.fsum(float(torch.dot(p, p)) for g in s["grads"]
                               for p in (q.double() for q in g.split(1 << 24))))
    factor = min(1.0, s["max_norm"] / norm)
    flat, out = _flat(s["grads"], F64)
    for g, o in zip(s["grads"], out):
        o.copy_(g.double() * factor)
    return dict(flat=flat, norm=torch.tensor([norm, factor], dtype=F64))


def _exact_q4(c, s):
    x, group = s["x"].double(), c["group"]
    y = torch.zeros(c["T"], c["N"], dtype=F64, device=DEV)
    for g, k in enumerate(range(0, c["K"], group)):
        part = x[:, k:k + group] @ s["codes"][:, k:k + group].double().T
        y += part * s["scales"][:, g].double()
    if s["bias"] is not None:
        y += s["bias"].double()
    return dict(y=y)


def _exact_logits(c, s):
    V, out = c["V"], []
    for b in range(c["B"]):
        n, p = int(s["lengths"][b]), int(s["prompt"][b])
        row = s["history"][b, :n].long()
        z = s["z"][b].double()
        seen = torch.unique(row)
        r = s["repetition"][b].double()
        z[seen] = torch.maximum(z[seen], z.new_zeros(())) / r + torch.clamp(z[seen], max=0.0) * r
        times = torch.bincount(row[p:], minlength=V).double()
        z -= s["frequency"][b].double() * times + s["presence"][b].double() * times.clamp(max=1.0)
        if s["bias_idx"] is not None:
            used = s["bias_idx"][b] >= 0
            z.index_add_(0, s["bias_idx"][b][used].long(), s["bias"][b][used].double())
        if s["mask"] is not None:
            j = torch.arange(V, device=DEV)
            z[(s["mask"][b][j // 32] & (1 << (j % 32)).to(torch.int32)) == 0] = -math.inf
        out.append(z)
    return dict(out=torch.stack(out))


def work(case):
    c = case
    if c["kind"] == "embed":
        T, V, d, e = c["T"], c["V"], c["d"], 4 if c["f32"] else 2
        # the rows that are looked up, each read once: as many symbols as T draws are expected to name
        r = torch.arange(1, V + 1, dtype=F64)
        p = 0.98 * torch.log1p(1.0 / r) / math.log(V + 1.0)
        rows = int(-torch.expm1(T * torch.log1p(-p)).sum())
        return {"bytes": 4 * T + (rows + T) * d * e + (T * d * e + 4 * V * d if c["grad"] else 0),
                "flops": T * d * (2 if c["grad"] else 1)}
    if c["kind"] == "clip":
        n = sum(_sizes(c))
        small = (4 * c["layers"] + 1) * c["d"]
        e = 4 if c["f32"] else 2
        return {"bytes": 2 * ((n - small) * e + small * 4), "flops": 3 * n}
    if c["kind"] == "q4":
        T, N, K = c["T"], c["N"], c["K"]
        return {"bytes": N * K // 2 + 2 * N * -(-K // c["group"]) + 2 * T * K
                + T * N * (4 if c["f32"] else 2) + (4 * N if c["bias"] else 0),
                "flops": 2 * T * N * K}
    B, V, H, e = c["B"], c["V"], c["H"], 4 if c["f32"] else 2
    return {"bytes": 2 * B * V * e + 4 * B * H + 8 * B * c["M"] + 20 * B
            + (B * -(-V // 32) * 4 if c["mask"] else 0),
            "flops": 4 * B * V}
