"""GPU parity of hcw_residual_norm_fwd / _bwd with the fp64 oracle.

Tolerances.  Both sides start from the same values.  The kernels work in fp32
with u = 2^-24 and round each output once (bf16: half a step of 8 significant bits, 2^-8 relative;
fp32: u).  A row quantity is a handful of operations on sums of d terms, added
up in chains of at most 16 + 5 + 16 (thread, shuffles, warps): 64 u of the sum
of the magnitudes that enter it (the A_* below, the formulas with every term
taken absolute) bounds the whole.  A sum over T rows adds at most T u more.
"""
import numpy as np
import pytest
import torch

from oracle import student as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
KU = 64 * U
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


def np64(t):
    return None if t is None else t.double().cpu().numpy()


class Problem:
    def __init__(self, T, d, dtype, seed, rows=0, gate=True, weights=True, offset=0.0):
        rng = np.random.default_rng(seed)

        def t(*shape, std=1.0, mean=0.0, dt=F32):
            return torch.from_numpy((mean + std * rng.normal(size=shape)).astype(np.float32)).to(dt).cuda()

        G = -(-T // rows) if rows else 1
        self.T, self.d, self.rows, self.dtype, self.eps = T, d, rows, dtype, 1e-5
        self.alpha = float(np.float32(0.83))
        self.r, self.f = t(T, d, std=2, mean=offset, dt=dtype), t(T, d, mean=0.3 + offset, dt=dtype)
        self.s = t(T, d, std=1.5, mean=offset, dt=dtype)
        self.dr_out, self.dx_out = t(T, d, std=0.1, dt=dtype), t(T, d, std=0.1, dt=dtype)
        self.gate = t(G, d, std=0.4, mean=0.6) if gate else None
        self.post_w, self.pre_w = (t(d, std=0.2, mean=1.0) if weights else None for _ in range(2))
        self.post_b, self.pre_b = (t(d, std=0.2) if weights else None for _ in range(2))

    def eps64(self):
        return float(np.float32(self.eps))


def abs_hat(kind, v, rs):
    return np.abs(v) if kind == S.NONE else rs * (np.abs(v) + np.abs(v).mean(axis=1, keepdims=True))


def abs_grad(kind, A_hat, rs, A_e):
    if kind == S.NONE:
        return A_e
    return rs * (A_e + A_e.mean(axis=1, keepdims=True) +
                 A_hat * (A_e * A_hat).mean(axis=1, keepdims=True))


def close(got, ref, A, what, rows=0):
    """|got - ref| <= the output's rounding + (64 + rows) u A."""
    out = 2.0 ** -8 if got.dtype == BF16 else U
    g = np64(got)
    assert g.shape == ref.shape, (what, g.shape, ref.shape)
    assert np.isfinite(g).all(), what
    bound = (KU + rows * U) * A
    bound = bound + out * (np.abs(ref) + bound) + 1e-38
    bad = np.abs(g - ref) > bound
    assert not bad.any(), (what, float((np.abs(g - ref) / bound).max()))


def check_fwd(H, p, post, pre, r=True, f=True, stream=None):
    R, F = p.r if r else None, p.f if f else None
    par = dict(post=post, post_w=p.post_w, post_b=p.post_b, pre=pre, pre_w=p.pre_w, pre_b=p.pre_b)
    # outputs inside larger buffers: nothing past their ends is written
    n = p.T * p.d
    pad = 8 * 16
    buf = [torch.full((n + pad,), 7.0, dtype=p.dtype, device="cuda") for _ in range(2)]
    got = H.hcw_residual_norm_fwd(R, F, p.gate, p.rows, p.alpha, eps=p.eps,
                                  r_out=buf[0][:n].view(p.T, p.d),
                                  x_out=buf[1][:n].view(p.T, p.d) if pre else None,
                                  want_x=bool(pre), stream=stream, **par)
    torch.cuda.synchronize()
    assert all(bool((b[n:] == 7.0).all()) for b in buf)
    q = {k: np64(v) if torch.is_tensor(v) else v for k, v in par.items()}
    gate = np64(p.gate)
    s, x = S.norm_fwd(np64(R), np64(F), gate, p.rows, p.alpha, post, q["post_w"], q["post_b"], pre,
                      q["pre_w"], q["pre_b"], p.eps64())
    A_s = np.zeros((p.T, p.d)) if R is None else p.alpha * np.abs(np64(R))
    if f:
        _, rf = S.hat(post, np64(F), p.eps64())
        A_v = abs_hat(post, np64(F), rf)
        if post and p.post_w is not None:
            A_v = A_v * np.abs(q["post_w"]) + (np.abs(q["post_b"]) if post == S.LAYER else 0)
        A_s = A_s + np.abs(S.gate_rows(gate, p.rows, p.T, p.d)) * A_v
    close(got[0], s, A_s, "r_out")
    if pre:
        _, rs = S.hat(pre, s, p.eps64())
        # s enters with its own error (64 u A_s), the deviation with that of all of s
        A_x = rs * (A_s + A_s.mean(axis=1, keepdims=True))
        A_x = A_x + np.abs(S.hat(pre, s, p.eps64())[0]) * (A_x * A_x).mean(axis=1, keepdims=True) ** 0.5
        if p.pre_w is not None:
            A_x = A_x * np.abs(q["pre_w"]) + (np.abs(q["pre_b"]) if pre == S.LAYER else 0)
        close(got[1], x, 2 * A_x, "x_out")


def check_bwd(H, p, post, pre, dr_out=True, dx_out=True, f=True, stream=None):
    A, B, F = p.dr_out if dr_out else None, p.dx_out if dx_out else None, p.f if f else None
    par = dict(post=post, post_w=p.post_w, post_b=p.post_b, pre=pre, pre_w=p.pre_w)
    call = lambda: H.hcw_residual_norm_bwd(  # noqa: E731
        A, B, p.s if dx_out else None, F, p.gate, p.rows, p.alpha, eps=p.eps, want_bias=True,
        stream=stream, **par)
    got, again = call(), call()
    torch.cuda.synchronize()
    for k in got:
        assert torch.equal(got[k], again[k]), k      # the same bits every time
    q = {k: np64(v) if torch.is_tensor(v) else v for k, v in par.items()}
    gate = np64(p.gate)
    ref = S.norm_bwd(np64(A), np64(B), np64(p.s), np64(F), gate, p.rows, p.alpha, post,
                     q["post_w"], q["post_b"], pre, q["pre_w"], p.eps64())
    want = {"dr"} | ({"df"} if f else set())
    T, d = p.T, p.d
    A_ds = np.zeros((T, d)) if A is None else np.abs(np64(A))
    if dx_out:
        want |= {"dpre_w"} | ({"dpre_b"} if pre == S.LAYER else set())
        _, rs = S.hat(pre, np64(p.s), p.eps64())
        A_hat = abs_hat(pre, np64(p.s), rs)
        A_e = np.abs(np64(B)) * (1 if q["pre_w"] is None else np.abs(q["pre_w"]))
        A_ds = A_ds + abs_grad(pre, A_hat, rs, A_e)
        close(got["dpre_w"], ref["dpre_w"], (np.abs(np64(B)) * A_hat).sum(axis=0), "dpre_w", T)
        if pre == S.LAYER:
            close(got["dpre_b"], ref["dpre_b"], np.abs(np64(B)).sum(axis=0), "dpre_b", T)
    close(got["dr"], ref["dr"], p.alpha * A_ds, "dr")
    if f:
        _, rf = S.hat(post, np64(F), p.eps64())
        A_f = abs_hat(post, np64(F), rf)
        A_g = np.abs(S.gate_rows(gate, p.rows, T, d))
        A_h = A_ds * A_g * (1 if post == S.NONE or q["post_w"] is None else np.abs(q["post_w"]))
        close(got["df"], ref["df"], abs_grad(post, A_f, rf, A_h), "df")
        if post:
            want |= {"dpost_w"} | ({"dpost_b"} if post == S.LAYER else set())
            close(got["dpost_w"], ref["dpost_w"], (A_ds * A_g * A_f).sum(axis=0), "dpost_w", T)
        if post == S.LAYER:
            close(got["dpost_b"], ref["dpost_b"], (A_ds * A_g).sum(axis=0), "dpost_b", T)
        if gate is not None:
            want |= {"dgate"}
            A_v = A_f * (1 if post == S.NONE or q["post_w"] is None else np.abs(q["post_w"]))
            if post == S.LAYER and q["post_b"] is not None:
                A_v = A_v + np.abs(q["post_b"])
            step = p.rows or T
            A_gate = np.stack([(A_ds * A_v)[i:i + step].sum(axis=0) for i in range(0, T, step)])
            close(got["dgate"], ref["dgate"], A_gate, "dgate", T)
    assert set(got) == want


KINDS = [(0, 1), (0, 2), (1, 1), (1, 2), (2, 1), (2, 2)]
WIDTHS = [1, 7, 64, 200, 257, 512, 777, 1000, 2048, 2056, 4096, 4097, 8184, 8192]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_every_width(H, d, dtype):
    for i, (post, pre) in enumerate(KINDS if d <= 512 else KINDS[2::3]):
        p = Problem(19, d, dtype, 100 * d + i)
        check_fwd(H, p, post, pre)
        check_bwd(H, p, post, pre)


@pytest.mark.parametrize("T,rows", [(1, 0), (1, 1), (5, 1), (37, 3), (64, 64), (65, 64), (700, 256),
                                    (1500, 0), (2500, 7)])
@pytest.mark.parametrize("d", [64, 136, 1000])
def test_lengths_and_gate_groups(H, T, rows, d):
    p = Problem(T, d, BF16, T + rows + d, rows=rows)
    check_fwd(H, p, 1, 1)
    check_bwd(H, p, 1, 1)
    check_bwd(H, p, 2, 2)


def test_parts_that_are_not_there(H):
    p = Problem(33, 264, BF16, 5)
    check_fwd(H, p, 1, 1, r=False)
    check_fwd(H, p, 1, 1, f=False)
    check_fwd(H, p, 2, 0)
    check_bwd(H, p, 1, 1, dr_out=False)
    check_bwd(H, p, 2, 2, dx_out=False)
    check_bwd(H, p, 1, 2, f=False)
    q = Problem(33, 264, F32, 6, gate=False, weights=False)
    check_fwd(H, q, 2, 2)
    check_bwd(H, q, 2, 2)
    # row gradients alone: no parameter gradients, no workspace
    got = H.hcw_residual_norm_bwd(p.dr_out, p.dx_out, p.s, p.f, p.gate, alpha=p.alpha, post=1,
                                  post_w=p.post_w, pre=1, pre_w=p.pre_w, eps=p.eps,
                                  want_params=False)
    full = H.hcw_residual_norm_bwd(p.dr_out, p.dx_out, p.s, p.f, p.gate, alpha=p.alpha, post=1,
                                   post_w=p.post_w, pre=1, pre_w=p.pre_w, eps=p.eps)
    assert set(got) == {"dr", "df"}
    assert all(torch.equal(got[k], full[k]) for k in got)


def test_layer_norm_under_a_large_offset(H):
    """Rows whose mean is a thousand times their deviation."""
    p = Problem(40, 512, F32, 9, offset=1000.0)
    check_fwd(H, p, 2, 2)
    check_bwd(H, p, 2, 2)


def test_rows_of_zeros_and_no_rows(H):
    z = torch.zeros(3, 96, dtype=BF16, device="cuda")
    r, x = H.hcw_residual_norm_fwd(z, z, post=1, pre=2)
    assert not r.any() and not x.any()
    e = torch.empty(0, 96, dtype=BF16, device="cuda")
    w = torch.ones(96, device="cuda")
    g = torch.ones(1, 96, device="cuda")
    r, x = H.hcw_residual_norm_fwd(e, e, g, post=1, post_w=w, pre=1, pre_w=w)
    assert r.shape == (0, 96) and x.shape == (0, 96)
    got = H.hcw_residual_norm_bwd(e, e, e, e, g, post=2, post_w=w, pre=2, pre_w=w, want_bias=True)
    for k in ("dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b"):
        assert not got[k].any(), k


def test_another_stream_than_the_current_one(H):
    p = Problem(300, 512, BF16, 11)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    check_fwd(H, p, 1, 1, stream=st)
    check_bwd(H, p, 1, 1, stream=st)


def test_a_nan_row_stays_in_its_row(H):
    p = Problem(12, 256, BF16, 12)
    r = p.r.clone()
    r[5, 3] = float("nan")
    a = H.hcw_residual_norm_fwd(p.r, p.f, p.gate, post=1, post_w=p.post_w, pre=1, pre_w=p.pre_w)
    b = H.hcw_residual_norm_fwd(r, p.f, p.gate, post=1, post_w=p.post_w, pre=1, pre_w=p.pre_w)
    rows = [i for i in range(12) if i != 5]
    assert torch.equal(a[0][rows], b[0][rows]) and torch.equal(a[1][rows], b[1][rows])
    assert b[1][5].isnan().all() and int(b[0][5].isnan().sum()) == 1
