"""The entry points for symbols, clipping, 4-bit weights and logits refuse bad sizes, types,
pointers, alignment, overlaps and workspaces before anything launches, and do nothing where there is
nothing to do."""
import ctypes

import pytest

P = ctypes.c_void_p
LL = ctypes.c_longlong


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


@pytest.fixture(autouse=True)
def nothing_launches(H):
    before = H.hcw_launch_count()
    yield
    assert H.hcw_launch_count() == before


def places(n, step=1 << 28):
    """Addresses far apart (never read: every call here is refused)."""
    return [P((i + 1) * step) for i in range(n)]


def test_lookup_refusals(H):
    T, V, d = 100, 300, 24
    i, E, x = places(3)

    def call(i=i, E=E, T=T, V=V, d=d, dt=0, s=1.0, x=x):
        return H.lib().hcw_embed_fwd(i, E, T, V, d, dt, s, x, None)

    assert call(T=-1) == call(V=0) == call(d=0) == call(dt=2) == H.HCW_ERR_INVALID_ARG
    assert call(s=float("inf")) == call(s=float("nan")) == H.HCW_ERR_INVALID_ARG
    assert call(V=(1 << 23) + 1) == call(d=(1 << 20) + 1) == call(T=(1 << 28) + 1) == \
        H.HCW_ERR_UNSUPPORTED
    for k in "iEx":
        assert call(**{k: None}) == H.HCW_ERR_INVALID_ARG, k
        assert call(**{k: P(6)}) == H.HCW_ERR_ALIGNMENT, k
    assert call(E=P(8)) == call(x=P(8)) == H.HCW_ERR_ALIGNMENT
    assert call(x=E) == call(x=i) == call(x=P(E.value + V * d * 2 - 16)) == H.HCW_ERR_ALIASING
    assert call(T=0, i=None, E=None, x=None) == H.HCW_OK


def test_lookup_gradient_refusals(H):
    T, V, d = 100, 300, 24
    ws = H.hcw_embed_bwd_workspace_bytes(T, V, d)
    assert ws >= 4 * T * 4
    i, dx, dE, w = places(4)

    def call(i=i, dx=dx, T=T, V=V, d=d, dt=0, s=1.0, add=0, ot=1, dE=dE, w=w, n=ws):
        return H.lib().hcw_embed_bwd(i, dx, T, V, d, dt, s, add, ot, dE, w, n, None)

    assert call(T=-1) == call(V=0) == call(d=-4) == call(dt=3) == call(ot=2) == H.HCW_ERR_INVALID_ARG
    assert call(add=2) == call(add=-1) == call(s=float("nan")) == H.HCW_ERR_INVALID_ARG
    assert call(V=(1 << 23) + 1) == call(T=(1 << 28) + 1) == H.HCW_ERR_UNSUPPORTED
    for k, v in dict(i=i, dx=dx, dE=dE).items():
        assert call(**{k: None}) == H.HCW_ERR_INVALID_ARG, k
        assert call(**{k: P(v.value + 2)}) == H.HCW_ERR_ALIGNMENT, k
    assert call(dx=P(dx.value + 8)) == call(dE=P(dE.value + 8)) == H.HCW_ERR_ALIGNMENT
    assert call(w=P(w.value + 8)) == H.HCW_ERR_ALIGNMENT
    assert call(w=None) == call(n=ws - 1) == H.HCW_ERR_WORKSPACE
    assert call(dE=dx) == call(dE=i) == call(w=dE) == call(w=dx) == H.HCW_ERR_ALIASING
    # fp32 gradients are twice as long
    assert call(dE=P(dx.value - V * d * 2)) == H.HCW_ERR_ALIASING
    assert call(T=1 << 28, d=1 << 20, n=1 << 60, i=P(1 << 40), dx=P(1 << 50), dE=P(1 << 44),
                w=P(1 << 55)) == H.HCW_ERR_UNSUPPORTED     # more chunks than a grid holds
    assert call(T=0, add=1, i=None, dx=None, w=None, n=0) == H.HCW_OK
    assert H.hcw_embed_bwd_workspace_bytes(0, V, d) == 0
    assert H.hcw_embed_bwd_workspace_bytes(T, V, 0) == 0


def test_lookup_gradient_workspace_never_falls(H):
    for d in (1, 64, 777, 2048, 8192):
        last = 0
        for T in list(range(1, 200)) + [2 ** k + e for k in range(8, 24) for e in (-1, 0, 1)]:
            need = H.hcw_embed_bwd_workspace_bytes(T, 1000, d)
            assert need >= last, (T, d)
            last = need


def test_clipping_refusals(H):
    n, w, a, b, c, d = places(6)
    ws = H.hcw_clip_grads_workspace_bytes(2)
    assert ws > 0 and H.hcw_clip_grads_workspace_bytes(-1) == 0
    assert H.hcw_clip_grads_workspace_bytes(5000) > ws

    def call(g=(a, b), o=None, sizes=(100, 1000), dts=(0, 1), count=2, m=1.0, n=n, w=w, nb=ws):
        G = (P * 2)(*g)
        O = None if o is None else (P * 2)(*o)  # noqa: E741
        return H.lib().hcw_clip_grads(G, O, (LL * 2)(*sizes), (ctypes.c_int * 2)(*dts), count, m, n, w,
                                      nb, None)

    assert call(count=-1) == call(m=-1.0) == call(m=float("nan")) == H.HCW_ERR_INVALID_ARG
    assert call(n=None) == call(dts=(0, 2)) == call(sizes=(-1, 5)) == H.HCW_ERR_INVALID_ARG
    assert call(g=(a, None)) == call(o=(c, None)) == H.HCW_ERR_INVALID_ARG
    assert H.lib().hcw_clip_grads(None, None, None, None, 1, 1.0, n, w, ws, None) == \
        H.HCW_ERR_INVALID_ARG
    # (what an empty tensor's pointer is does not matter; the other one is refused)
    assert call(g=(P(3), P(b.value + 2)), sizes=(0, 8)) == H.HCW_ERR_ALIGNMENT
    assert call(g=(P(3), None), sizes=(0, 8)) == H.HCW_ERR_INVALID_ARG
    assert call(sizes=(1 << 45, 5)) == H.HCW_ERR_UNSUPPORTED
    assert call(g=(P(a.value + 1), b)) == call(g=(a, P(b.value + 2))) == H.HCW_ERR_ALIGNMENT
    assert call(n=P(n.value + 2)) == call(w=P(w.value + 8)) == H.HCW_ERR_ALIGNMENT
    assert call(w=None) == call(nb=ws - 1) == H.HCW_ERR_WORKSPACE
    # in place no two share memory; apart no output lies on anything
    assert call(g=(a, a)) == call(g=(P(b.value + 3992), b)) == call(n=a) == call(w=b) == \
        H.HCW_ERR_ALIASING
    assert call(o=(a, d)) == call(o=(c, c)) == call(o=(c, P(a.value + 196))) == H.HCW_ERR_ALIASING
    assert call(o=(c, d), n=d) == call(o=(c, d), w=c) == H.HCW_ERR_ALIASING


def test_packed_weight_refusals(H):
    N, K = 40, 264
    W, q, s, p = places(4)
    need = H.hcw_q4_bytes(N, K, 64)
    assert need == 3 * 3 * (1024 + 2 * 32)
    assert H.hcw_q4_bytes(N, K, 48) == H.hcw_q4_bytes(N, K + 4, 64) == H.hcw_q4_bytes(0, K, 64) == 0

    def quant(W=W, N=N, K=K, g=64, dt=0, q=q, s=s):
        return H.lib().hcw_q4_quantize(W, N, K, g, dt, q, s, None)

    def pack(q=q, s=s, N=N, K=K, g=64, p=p):
        return H.lib().hcw_q4_pack(q, s, N, K, g, p, None)

    for f in (quant, pack):
        assert f(N=0) == f(K=0) == f(g=16) == f(g=0) == H.HCW_ERR_INVALID_ARG
        assert f(K=260) == f(N=(1 << 24) + 1) == f(K=(1 << 20) + 8) == H.HCW_ERR_UNSUPPORTED
        assert f(q=None) == f(s=None) == H.HCW_ERR_INVALID_ARG
        assert f(q=P(q.value + 4)) == f(s=P(s.value + 2)) == H.HCW_ERR_ALIGNMENT
    assert quant(dt=5) == quant(W=None) == pack(p=None) == H.HCW_ERR_INVALID_ARG
    assert quant(W=P(4)) == pack(p=P(4)) == H.HCW_ERR_ALIGNMENT
    assert quant(q=W) == quant(s=W) == quant(s=q) == pack(p=q) == pack(p=s) == H.HCW_ERR_ALIASING


def test_packed_product_refusals(H):
    T, N, K = 5, 40, 264
    x, p, b, y = places(4)

    def call(x=x, p=p, b=b, T=T, N=N, K=K, g=64, dt=0, y=y):
        return H.lib().hcw_q4_matmul(x, p, b, T, N, K, g, dt, y, None)

    assert call(T=-1) == call(N=0) == call(g=100) == call(dt=2) == H.HCW_ERR_INVALID_ARG
    assert call(K=12) == call(T=(1 << 19) + 1) == H.HCW_ERR_UNSUPPORTED
    for k in "xpy":
        assert call(**{k: None}) == H.HCW_ERR_INVALID_ARG, k
    for k in "xpy":
        assert call(**{k: P(8)}) == H.HCW_ERR_ALIGNMENT, k
    assert call(b=P(6)) == H.HCW_ERR_ALIGNMENT
    assert call(y=x) == call(y=p) == call(y=b) == H.HCW_ERR_ALIASING
    assert call(y=P(x.value - T * N * 4 + 16), dt=1) == H.HCW_ERR_ALIASING
    assert call(T=0, x=None, y=None) == H.HCW_OK


def test_logits_refusals(H):
    B, V, Hn, M = 3, 100, 20, 5
    z, h, n, q, r, f, e, bi, b, m, o = places(11)

    def call(z=z, B=B, V=V, dt=0, h=h, n=n, q=q, Hn=Hn, r=r, f=f, e=e, bi=bi, b=b, M=M, m=m, o=o):
        return H.lib().hcw_logits_edit(z, B, V, dt, h, n, q, Hn, r, f, e, bi, b, M, m, o, None)

    assert call(B=-1) == call(V=0) == call(dt=2) == call(Hn=-1) == call(M=-1) == H.HCW_ERR_INVALID_ARG
    assert call(z=None) == call(o=None) == H.HCW_ERR_INVALID_ARG
    assert call(h=None) == call(Hn=0) == call(bi=None) == call(b=None) == call(M=0) == \
        H.HCW_ERR_INVALID_ARG
    assert call(h=None, Hn=0, q=None) == call(h=None, Hn=0, n=None) == H.HCW_ERR_INVALID_ARG
    assert call(M=1025) == call(V=(1 << 24) + 1) == call(B=(1 << 20) + 1) == H.HCW_ERR_UNSUPPORTED
    assert call(B=1 << 20, V=(1 << 20) + 1) == H.HCW_ERR_UNSUPPORTED
    for k, v in dict(z=z, h=h, n=n, q=q, r=r, f=f, e=e, bi=bi, b=b, m=m, o=o).items():
        assert call(**{k: P(v.value + 2)}) == H.HCW_ERR_ALIGNMENT, k
    assert call(z=P(z.value + 4)) == call(o=P(o.value + 4)) == H.HCW_ERR_ALIGNMENT
    for v in (h, n, q, r, f, e, bi, b, m):
        assert call(o=v) == H.HCW_ERR_ALIASING
    assert call(o=P(z.value + 16)) == H.HCW_ERR_ALIASING      # neither in place nor apart
    assert call(B=0, z=None, o=None) == H.HCW_OK


def test_the_binding_checks_what_it_is_given(H):
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    for f in (lambda: H.hcw_embed_fwd(i, x), lambda: H.hcw_embed_bwd(i, x, 9),
              lambda: H.GradList([x]), lambda: H.hcw_clip_grads([x], 1.0),
              lambda: H.hcw_q4_quantize(x), lambda: H.hcw_q4_pack(x, x),
              lambda: H.hcw_q4_matmul(x, x, 64), lambda: H.hcw_logits_edit(x)):
        with pytest.raises(ValueError, match="CUDA tensors"):
            f()
