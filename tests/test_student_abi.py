"""The student block's entry points refuse bad sizes, kinds, pointers, alignment, overlaps
and workspaces before anything launches, and do nothing where there is nothing to do."""
import ctypes

import pytest

P = ctypes.c_void_p


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


def places(n, step=1 << 26):
    """Addresses far apart (never read: every call here is refused)."""
    return [P((i + 1) * step) for i in range(n)]


def test_gated_ffn_forward_refusals(H):
    T, d, h = 100, 128, 264
    ws = H.hcw_gated_ffn_fwd_workspace_bytes(T, d, h)
    assert ws >= T * h * 2
    x, W1, W2, y, w = places(5)

    def call(x=x, W1=W1, W2=W2, T=T, d=d, h=h, act=0, y=y, w=w, n=ws):
        return H.lib().hcw_gated_ffn_fwd(x, W1, W2, T, d, h, act, y, w, n, None)

    assert call(T=-1) == H.HCW_ERR_INVALID_ARG
    assert call(d=0) == call(h=-8) == H.HCW_ERR_INVALID_ARG
    assert call(act=3) == call(act=-1) == H.HCW_ERR_INVALID_ARG
    assert call(d=132) == call(h=260) == call(d=(1 << 20) + 8) == H.HCW_ERR_UNSUPPORTED
    for k in ("x", "W1", "W2", "y"):
        assert call(**{k: None}) == H.HCW_ERR_INVALID_ARG, k
        assert call(**{k: P(8)}) == H.HCW_ERR_ALIGNMENT, k
    assert call(w=P(w.value + 4)) == H.HCW_ERR_ALIGNMENT
    assert call(w=None) == call(n=ws - 1) == call(n=0) == H.HCW_ERR_WORKSPACE
    assert call(y=x) == call(w=W2) == call(w=y) == H.HCW_ERR_ALIASING
    assert call(y=P(W1.value + 2 * h * d * 2 - 16)) == H.HCW_ERR_ALIASING
    assert call(T=0, x=None, y=None, w=None, n=0) == H.HCW_OK
    assert H.hcw_gated_ffn_fwd_workspace_bytes(0, d, h) == 0
    assert H.hcw_gated_ffn_fwd_workspace_bytes(T, d + 4, h) == 0


def test_gated_ffn_backward_refusals(H):
    T, d, h = 100, 128, 264
    ws = H.hcw_gated_ffn_bwd_workspace_bytes(T, d, h)
    assert ws >= 3 * T * h * 2
    x, dy, W1, W2, dx, dW1, dW2, w = places(8)

    def call(x=x, dy=dy, W1=W1, W2=W2, T=T, d=d, h=h, act=0, dt=0, dx=dx, dW1=dW1, dW2=dW2, w=w,
             n=ws):
        return H.lib().hcw_gated_ffn_bwd(x, dy, W1, W2, T, d, h, act, dt, dx, dW1, dW2, w, n, None)

    assert call(T=-2) == call(act=9) == call(dt=2) == H.HCW_ERR_INVALID_ARG
    assert call(d=12) == H.HCW_ERR_UNSUPPORTED
    for k in ("x", "dy", "W1", "W2", "dW1", "dW2"):
        assert call(**{k: None}) == H.HCW_ERR_INVALID_ARG, k
    assert call(dx=None, dW1=None, dW2=None) == H.HCW_ERR_INVALID_ARG
    assert call(dW2=P(dW2.value + 8)) == H.HCW_ERR_ALIGNMENT
    assert call(w=None) == call(n=256) == H.HCW_ERR_WORKSPACE
    assert call(dx=dy) == call(dW1=W1) == call(dW2=dW1) == call(w=dx) == H.HCW_ERR_ALIASING
    # fp32 gradients are twice as long
    assert call(dt=1, dW2=P(dW1.value + 2 * h * d * 2)) == H.HCW_ERR_ALIASING
    assert call(T=0, x=None, dy=None, dx=None, dW1=None, dW2=None) == H.HCW_OK


def test_residual_norm_refusals(H):
    T, d = 50, 96
    r, f, g, w, b, q, c, o, x = places(9)

    def call(r=r, f=f, g=g, rows=0, alpha=1.0, post=1, w=w, b=b, pre=2, q=q, c=c, eps=1e-5, T=T,
             d=d, dt=0, o=o, x=x):
        return H.lib().hcw_residual_norm_fwd(r, f, g, rows, alpha, post, w, b, pre, q, c, eps, T, d,
                                             dt, o, x, None)

    assert call(T=-1) == call(d=0) == call(dt=5) == H.HCW_ERR_INVALID_ARG
    assert call(post=3) == call(pre=-1) == call(rows=-1) == H.HCW_ERR_INVALID_ARG
    assert call(eps=-1.0) == call(eps=float("nan")) == H.HCW_ERR_INVALID_ARG
    assert call(alpha=float("inf")) == H.HCW_ERR_INVALID_ARG
    assert call(pre=0) == H.HCW_ERR_INVALID_ARG            # x_out without a norm
    assert call(r=None, f=None) == call(o=None, x=None) == H.HCW_ERR_INVALID_ARG
    assert call(d=8193) == H.HCW_ERR_UNSUPPORTED
    assert call(g=P(g.value + 4)) == call(x=P(x.value + 2)) == H.HCW_ERR_ALIGNMENT
    assert call(o=r) == call(x=f) == call(o=x) == call(x=q) == H.HCW_ERR_ALIASING
    # the gates of groups of two rows reach further than one gate
    past = P(g.value + d * 4)
    assert call(rows=2, o=past) == H.HCW_ERR_ALIASING
    assert call(T=0, r=None, f=None, o=None, x=None) == H.HCW_OK


def test_residual_norm_backward_refusals(H):
    T, d = 50, 96
    ws = H.hcw_residual_norm_bwd_workspace_bytes(T, d, 0)
    assert ws > 0 and H.hcw_residual_norm_bwd_workspace_bytes(T, 8193, 0) == 0
    dro, dxo, s, f, g, w, b, q, dr, df, dg, dw, db, dq, dc, wk = places(16)

    def call(dro=dro, dxo=dxo, s=s, f=f, g=g, rows=0, post=2, w=w, b=b, pre=2, q=q, T=T, d=d, dt=1,
             dr=dr, df=df, dg=dg, dw=dw, db=db, dq=dq, dc=dc, wk=wk, n=ws):
        return H.lib().hcw_residual_norm_bwd(dro, dxo, s, f, g, rows, 1.0, post, w, b, pre, q, 1e-5,
                                             T, d, dt, dr, df, dg, dw, db, dq, dc, wk, n, None)

    assert call(T=-1) == call(dt=2) == call(rows=-3) == H.HCW_ERR_INVALID_ARG
    assert call(post=1) == call(pre=1) == H.HCW_ERR_INVALID_ARG       # RMS has no bias
    assert call(post=0, db=None) == H.HCW_ERR_INVALID_ARG             # no norm, no weight
    assert call(dro=None, dxo=None) == H.HCW_ERR_INVALID_ARG
    assert call(s=None) == call(f=None) == H.HCW_ERR_INVALID_ARG
    assert call(dxo=None) == H.HCW_ERR_INVALID_ARG                    # dpre_w without dx_out
    assert call(dr=None, df=None, dg=None, dw=None, db=None, dq=None, dc=None) == \
        H.HCW_ERR_INVALID_ARG
    assert call(d=9000) == H.HCW_ERR_UNSUPPORTED
    assert call(dq=P(dq.value + 8)) == call(wk=P(wk.value + 8)) == H.HCW_ERR_ALIGNMENT
    assert call(dr=dro) == call(df=dr) == call(dg=w) == call(wk=s) == H.HCW_ERR_ALIASING
    assert call(wk=None) == call(n=ws - 1) == H.HCW_ERR_WORKSPACE


def test_distillation_refusals(H):
    T, V, K = 40, 300, 8
    z, i, t, y, w, loss, dz = places(7)

    def call(z=z, i=i, t=t, y=y, w=w, T=T, V=V, K=K, dt=0, tau=1.0, a=1.0, b=0.5, loss=loss, dz=dz):
        return H.lib().hcw_distill_loss(z, i, t, y, w, T, V, K, dt, tau, a, b, loss, dz, None)

    assert call(T=-1) == call(V=0) == call(K=-1) == call(dt=3) == H.HCW_ERR_INVALID_ARG
    assert call(tau=0.0) == call(tau=-1.0) == call(tau=float("nan")) == H.HCW_ERR_INVALID_ARG
    assert call(tau=float("inf")) == call(a=float("nan")) == call(b=float("inf")) == \
        H.HCW_ERR_INVALID_ARG
    assert call(z=None) == call(loss=None, dz=None) == H.HCW_ERR_INVALID_ARG
    assert call(i=None) == call(t=None) == call(K=0) == H.HCW_ERR_INVALID_ARG
    assert call(V=262145) == call(K=1025) == call(T=1 << 30, V=1, K=1) == H.HCW_ERR_UNSUPPORTED
    assert call(z=P(z.value + 2)) == call(w=P(w.value + 4)) == H.HCW_ERR_ALIGNMENT
    assert call(dz=z) == call(loss=w) == call(dz=loss) == H.HCW_ERR_ALIASING
    assert call(T=0, z=None, loss=None, dz=None) == H.HCW_OK


def test_the_binding_checks_what_it_is_given(H):
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for f in (lambda: H.hcw_gated_ffn_fwd(x, x, x), lambda: H.hcw_gated_ffn_bwd(x, x, x, x),
              lambda: H.hcw_residual_norm_fwd(x, x), lambda: H.hcw_residual_norm_bwd(x, x, x, x),
              lambda: H.hcw_distill_loss(x)):
        with pytest.raises(ValueError, match="CUDA tensors"):
            f()
    with pytest.raises(ValueError, match="r or f"):
        H.hcw_residual_norm_fwd(None, None)
    with pytest.raises(ValueError, match="dr_out or dx_out"):
        H.hcw_residual_norm_bwd(None, None, None, None)
