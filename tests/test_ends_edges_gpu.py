"""The operators at the model's two ends between other work: calls on two streams at once, inputs that
are written right before a call and overwritten right after it, outputs that the next call reads."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


def rnd(seed, *shape):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def ints(seed, hi, *shape):
    return torch.randint(-1, hi, shape, device="cuda", dtype=torch.int32,
                         generator=torch.Generator(device="cuda").manual_seed(seed))


def test_two_streams_at_once(H):
    T, V, d = 9000, 3000, 520
    ids, dx = [ints(k, V, T) for k in range(2)], [rnd(k, T, d).to(BF16) for k in range(2)]
    z, hist = [rnd(k, 70, 40001) for k in range(2)], [ints(k, 40001, 70, 600) for k in range(2)]
    freq = torch.full((70,), 0.3, device="cuda")
    codes, scales = H.hcw_q4_quantize(rnd(5, 5000, 1024), 64)
    packed, x = H.hcw_q4_pack(codes, scales, 64), [rnd(k, 3 + 9 * k, 1024).to(BF16) for k in range(2)]

    def calls(k, stream=None):
        g = [dx[k].clone(), z[k].clone()] if stream is None else grads[k]
        return (H.hcw_embed_bwd(ids[k], dx[k], V, stream=stream),
                H.hcw_logits_edit(z[k], history=hist[k], frequency=freq, stream=stream),
                H.hcw_q4_matmul(x[k], packed, 5000, 64, stream=stream),
                H.hcw_clip_grads(g, 1.0, stream=stream), *g)

    alone = [calls(k) for k in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        grads = [[dx[k].clone(), z[k].clone()] for k in range(2)]
        torch.cuda.synchronize()
        got = [calls(k, streams[k]) for k in range(2)]
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(a, b) for a, b in zip(alone[k], got[k]))


@pytest.mark.parametrize("B,V", [(3, 501), (90, 30011)])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("inplace", [False, True])
def test_logits_that_change_around_the_call(H, B, V, masked, inplace):
    """What a call reads is written by the launch before it and overwritten by the one behind it."""
    zs, hs = [rnd(k, B, V) for k in range(6)], [ints(k, V, B, 200) for k in range(6)]
    rep, freq = torch.full((B,), 1.4, device="cuda"), torch.full((B,), 0.3, device="cuda")
    bi, bv = ints(9, V, B, 12), rnd(9, B, 12)
    masks = [torch.randint(-2 ** 31, 2 ** 31, (B, -(-V // 32)), device="cuda").to(torch.int32)
             for _ in range(6)] if masked else None
    z, h = torch.empty(B, V, device="cuda"), torch.empty(B, 200, dtype=torch.int32, device="cuda")
    m = torch.empty_like(masks[0]) if masked else None
    kw = dict(repetition=rep, frequency=freq, bias_idx=bi, bias=bv)
    want = [H.hcw_logits_edit(zs[k], history=hs[k], mask=masks[k] if masked else None, **kw).clone()
            for k in range(6)]
    torch.cuda.synchronize()
    got = []
    for k in range(6):
        z.copy_(zs[k])
        h.copy_(hs[k])
        if masked:
            m.copy_(masks[k])
        out = H.hcw_logits_edit(z, history=h, mask=m, out=z if inplace else None, **kw)
        got.append(out.clone())
        h.fill_(0)
        z.fill_(float("nan"))
        if masked:
            m.fill_(0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_edits_one_after_the_other_in_place(H):
    """The next call's first launch begins while this call's last one is under way."""
    B, V = 80, 50021
    z = rnd(1, B, V)
    hist, freq = ints(2, V, B, 900), torch.full((B,), 0.125, device="cuda")
    one = z.clone()
    full = torch.full((B, -(-V // 32)), -1, dtype=torch.int32, device="cuda")
    for k in range(8):
        H.hcw_logits_edit(one, history=hist, frequency=freq, mask=full if k % 2 else None, out=one)
    torch.cuda.synchronize()
    two = z.clone()
    for k in range(8):
        two = H.hcw_logits_edit(two, history=hist, frequency=freq)
        torch.cuda.synchronize()
    assert torch.equal(one, two)


def test_a_workspace_for_call_after_call(H):
    """One workspace, other sizes from call to call, nothing between them."""
    jobs = [(5000, 700, 264), (70, 40000, 64), (3000, 200001, 40), (1, 9, 8), (20000, 3, 520)]
    data = [(ints(k, V, T), rnd(k, T, d).to(BF16)) for k, (T, V, d) in enumerate(jobs)]
    want = [H.hcw_embed_bwd(i, x, V) for (i, x), (T, V, d) in zip(data, jobs)]
    torch.cuda.synchronize()
    ws = torch.empty(max(H.hcw_embed_bwd_workspace_bytes(*j) for j in jobs), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        got = [H.hcw_embed_bwd(i, x, V, workspace=ws) for (i, x), (T, V, d) in zip(data, jobs)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_weights_packed_right_before_the_product(H):
    x = rnd(1, 7, 512).to(BF16)
    Ws = [rnd(k, 1000, 512) for k in range(4)]
    codes, scales = H.hcw_q4_quantize(Ws[0], 32)
    packed = H.hcw_q4_pack(codes, scales, 32)
    want = []
    for W in Ws:
        want.append(H.hcw_q4_matmul(x, H.hcw_q4_pack(*H.hcw_q4_quantize(W, 32), 32), 1000, 32))
        torch.cuda.synchronize()
    got = []
    for W in Ws:
        H.hcw_q4_quantize(W, 32, codes=codes, scales=scales)
        H.hcw_q4_pack(codes, scales, 32, packed=packed)
        got.append(H.hcw_q4_matmul(x, packed, 1000, 32))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_clipping_call_after_call(H):
    """The factor of one call is the next one's input."""
    g = [rnd(k, 3 + 50000 * k) for k in range(4)]
    ref = [t.double().clone() for t in g]
    q = H.GradList(g)
    norm, ws = torch.empty(2, device="cuda"), torch.empty(H.hcw_clip_grads_workspace_bytes(4),
                                                          dtype=torch.uint8, device="cuda")
    for k in range(6):
        H.hcw_clip_grads(q, 100.0 / 2 ** k, norm=norm, workspace=ws)
    torch.cuda.synchronize()
    total = float(torch.sqrt(sum((t * t).sum() for t in ref)))
    for t, r in zip(g, ref):
        assert bool(((t.double() - r * (3.125 / total)).abs() <= 6 * 20 * 2.0 ** -24 * r.abs() *
                     (3.125 / total) + 1e-44).all())
    assert np.isclose(float(norm[0]), 6.25, rtol=1e-5) and np.isclose(float(norm[1]), 0.5, rtol=1e-5)


def test_tensors_of_another_device_than_the_current_one(H, monkeypatch):
    x = torch.zeros(4, 64, device="cuda")
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    q = H.GradList([x])
    monkeypatch.setattr(H, "_current_device", lambda: 1)
    for f in (lambda: H.hcw_embed_fwd(i, x), lambda: H.hcw_embed_bwd(i, x, 9), lambda: H.GradList([x]),
              lambda: H.hcw_clip_grads(q, 1.0), lambda: H.hcw_q4_quantize(x),
              lambda: H.hcw_q4_matmul(x.to(BF16), i, 64), lambda: H.hcw_logits_edit(x)):
        with pytest.raises(ValueError, match="current device"):
            f()
