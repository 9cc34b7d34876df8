"""GPU parity of hcw_gated_ffn_fwd / _bwd with the fp64 oracle.

Tolerances, element by element from the magnitudes that enter (the products with
every factor taken absolute).  r = 2^-8 is the rounding of a bf16 operand or
output (half a step of 8 significant bits), u = 2^-24 fp32's.  A product over K
terms accumulates in fp32: K u of its magnitude bounds any order, 2 K u here for
accumulators that cut off instead of rounding.
  g, u, da      2 K u of their magnitudes (K = d)
  act           1-Lipschitz up to the factor 1.13 (GELU's slope), act' up to 0.8 (GELU)
  a = act(g) u  r |a| + 1.13 (dg |u| + |g| du)
  y             sum (error of a) |W2| + 2 h u sum |a| |W2| + r |y|
and likewise for the gradients.  ReLU's derivative steps at 0: within the error of g it
may be either.
"""
import numpy as np
import pytest
import torch

from oracle import student as S

pytestmark = pytest.mark.gpu

R = 2.0 ** -8
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


def np64(t):
    return t.double().cpu().numpy()


def make(T, d, h, seed):
    rng = np.random.default_rng(seed)
    t = lambda std, *s: torch.from_numpy((std * rng.normal(size=s)).astype(np.float32)).to(BF16).cuda()  # noqa: E731
    return (t(1.0, T, d), t(0.1, T, d), t(d ** -0.5, 2 * h, d), t(h ** -0.5, d, h))


def bounds(x, dy, W1, W2, act):
    """(reference, error bound before the output's rounding) of y, dx, dW1, dW2."""
    T, d = x.shape
    h = W2.shape[1]
    ax, ady, aW1, aW2 = (np.abs(v) for v in (x, dy, W1, W2))
    g, u = x @ W1[:h].T, x @ W1[h:].T
    eg, eu = 2 * (d + 8) * U * (ax @ aW1[:h].T), 2 * (d + 8) * U * (ax @ aW1[h:].T)
    ag, dag = S.act(act, g)
    eag, edag = 1.13 * eg + 16 * U * np.abs(g), 0.8 * eg + 16 * U
    if act == S.RELU:
        edag = (np.abs(g) <= eg).astype(np.float64)
    a = ag * u
    ea = eag * np.abs(u) + (np.abs(ag) + eag) * eu
    ea = ea + R * (np.abs(a) + ea)
    y = a @ W2.T
    ey = ea @ aW2.T + 2 * (h + 8) * U * ((np.abs(a) + ea) @ aW2.T)
    da = dy @ W2
    eda = 2 * (d + 8) * U * (ady @ aW2)
    dg, du = da * u * dag, da * ag
    edu = eda * (np.abs(ag) + eag) + np.abs(da) * eag
    edg = eda * (np.abs(u) + eu) * (np.abs(dag) + edag) + np.abs(da) * (eu * (np.abs(dag) + edag) + np.abs(u) * edag)
    edu, edg = edu + (R + 8 * U) * (np.abs(du) + edu), edg + (R + 8 * U) * (np.abs(dg) + edg)
    D, eD = np.concatenate([dg, du], 1), np.concatenate([edg, edu], 1)
    M = np.abs(D) + eD
    dx, edx = D @ W1, eD @ aW1 + 2 * (2 * h + 8) * U * (M @ aW1)
    dW1, edW1 = D.T @ x, eD.T @ ax + 2 * (T + 8) * U * (M.T @ ax)
    dW2, edW2 = dy.T @ a, ady.T @ ea + 2 * (T + 8) * U * (ady.T @ (np.abs(a) + ea))
    for k, v in zip(("dx", "dW1", "dW2"), S.ffn_bwd(x, dy, W1, W2, act)):
        assert np.allclose(v, {"dx": dx, "dW1": dW1, "dW2": dW2}[k])
    return {"y": (y, ey), "dx": (dx, edx), "dW1": (dW1, edW1), "dW2": (dW2, edW2)}


def close(got, ref, err, what):
    g = np64(got)
    assert g.shape == ref.shape and np.isfinite(g).all(), what
    out = R if got.dtype == BF16 else U
    bound = err + out * (np.abs(ref) + err) + 1e-38
    ratio = np.abs(g - ref) / bound
    assert ratio.max(initial=0.0) <= 1.0, (what, float(ratio.max()))
    # and not merely inside the worst case: the errors are independent, so their norm is
    # far below the bounds' (8 bf16 roundings of every value's size)
    assert np.linalg.norm(g - ref) <= 8 * R * np.linalg.norm(ref) + 1e-30, what


def padded(shape, dtype):
    n = int(np.prod(shape))
    buf = torch.full((n + 64,), 7.0, dtype=dtype, device="cuda")
    return buf, buf[:n].view(*shape)


def check(H, T, d, h, act, seed, dw=BF16, stream=None):
    x, dy, W1, W2 = make(T, d, h, seed)
    ref = bounds(*(np64(v) for v in (x, dy, W1, W2)), act)
    torch.cuda.synchronize()
    bufs = [padded(s, t) for s, t in (((T, d), BF16), ((T, d), BF16), ((2 * h, d), dw), ((d, h), dw))]
    y = H.hcw_gated_ffn_fwd(x, W1, W2, act, y=bufs[0][1], stream=stream)
    dx, dW1, dW2 = H.hcw_gated_ffn_bwd(x, dy, W1, W2, act, dx=bufs[1][1], dW1=bufs[2][1],
                                       dW2=bufs[3][1], stream=stream)
    torch.cuda.synchronize()
    assert H.hcw_sync_status() == H.HCW_OK
    got = {"y": y, "dx": dx, "dW1": dW1, "dW2": dW2}
    for k, v in got.items():
        close(v, *ref[k], k)
    for b, v in bufs:
        assert bool((b[v.numel():] == 7.0).all())
    # again: the same bits; and each part alone
    y2 = H.hcw_gated_ffn_fwd(x, W1, W2, act, stream=stream)
    only_dx = H.hcw_gated_ffn_bwd(x, dy, W1, W2, act, want_dw=False, stream=stream)
    only_dw = H.hcw_gated_ffn_bwd(x, dy, W1, W2, act, want_dx=False, dw_dtype=dw, stream=stream)
    two = H.hcw_gated_ffn_bwd(x, dy, W1, W2, act, dw_dtype=dw, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
    assert all(torch.equal(a, b) for a, b in zip((dx, dW1, dW2), two))
    assert only_dx[1] is None and only_dw[0] is None
    close(only_dx[0], *ref["dx"], "dx alone")
    close(only_dw[1], *ref["dW1"], "dW1 alone")
    close(only_dw[2], *ref["dW2"], "dW2 alone")


SIZES = [(1, 8, 8), (1, 64, 128), (2, 512, 1024), (3, 72, 200), (7, 136, 64), (8, 256, 264),
         (15, 1024, 96), (16, 64, 1032), (17, 512, 128), (31, 96, 512), (64, 256, 256),
         (65, 200, 344), (127, 520, 136), (129, 64, 64), (200, 128, 1000), (255, 264, 128),
         (256, 256, 128), (257, 128, 136), (300, 768, 520), (513, 64, 2056), (1000, 328, 264)]


@pytest.mark.parametrize("T,d,h", SIZES)
def test_every_size(H, T, d, h):
    check(H, T, d, h, S.SILU, T + d + h)


@pytest.mark.parametrize("act", [S.GELU, S.RELU])
@pytest.mark.parametrize("T,d,h", [(5, 64, 72), (130, 192, 200), (300, 256, 384)])
def test_other_activations(H, act, T, d, h):
    check(H, T, d, h, act, T + act)


@pytest.mark.parametrize("T,d,h", [(1, 64, 64), (90, 128, 200), (700, 64, 136)])
def test_fp32_weight_gradients(H, T, d, h):
    check(H, T, d, h, S.SILU, T, dw=F32)


@pytest.mark.parametrize("T,d,h", [(4100, 512, 1024), (5000, 128, 264)])
def test_sums_over_many_tokens(H, T, d, h):
    """More units than pairs of SMs, and a split sum over the tokens."""
    check(H, T, d, h, S.SILU, T)


def test_gates_far_from_zero(H):
    """SiLU and GELU where exp and erf have saturated."""
    for act in (S.SILU, S.GELU):
        x, dy, W1, W2 = make(33, 64, 64, act)
        W1 = (W1.float() * 60).to(BF16)
        ref = bounds(*(np64(v) for v in (x, dy, W1, W2)), act)
        close(H.hcw_gated_ffn_fwd(x, W1, W2, act), *ref["y"], "y")
        for k, v in zip(("dx", "dW1", "dW2"), H.hcw_gated_ffn_bwd(x, dy, W1, W2, act)):
            close(v, *ref[k], k)


def test_no_tokens(H):
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    _, _, W1, W2 = make(1, 64, 72, 0)
    assert H.hcw_gated_ffn_fwd(x, W1, W2).shape == (0, 64)
    for dw in (BF16, F32):
        dx, dW1, dW2 = H.hcw_gated_ffn_bwd(x, x, W1, W2, dw_dtype=dw)
        assert dx.shape == (0, 64) and not dW1.any() and not dW2.any()


def test_batched_rows_and_another_stream(H):
    x, dy, W1, W2 = make(6 * 32, 128, 136, 3)
    y = H.hcw_gated_ffn_fwd(x, W1, W2)
    assert torch.equal(H.hcw_gated_ffn_fwd(x.view(6, 32, 128), W1, W2).view(-1, 128), y)
    torch.cuda.synchronize()
    check(H, 150, 128, 136, S.SILU, 4, stream=torch.cuda.Stream())


def test_a_nan_token_stays_in_its_row(H):
    for T in (4, 200):
        x, _, W1, W2 = make(T, 128, 136, T)
        a = H.hcw_gated_ffn_fwd(x, W1, W2)
        x[2, 5] = float("nan")
        b = H.hcw_gated_ffn_fwd(x, W1, W2)
        rows = [i for i in range(T) if i != 2]
        assert torch.equal(a[rows], b[rows]) and b[2].isnan().all()


@pytest.mark.parametrize("T,d,h", [(300, 768, 520), (4100, 256, 1024), (3000, 1024, 264)])
def test_the_same_bits_over_many_runs(H, T, d, h):
    """Nothing depends on how the kernels' warps and copies happen to be timed."""
    x, dy, W1, W2 = make(T, d, h, 9)
    first = None
    for _ in range(60):
        got = (H.hcw_gated_ffn_fwd(x, W1, W2),
               *H.hcw_gated_ffn_bwd(x, dy, W1, W2, dw_dtype=BF16))
        if first is None:
            first = got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("T,d,h", [(20000, 64, 264), (9000, 64, 2056), (1000, 520, 1416), (333, 128, 2744)])
def test_every_way_tiles_are_shared_out(H, T, d, h):
    """Whole tiles and cut ones, units of 256 and 128 hidden columns, an odd end."""
    check(H, T, d, h, S.SILU, h)
    check(H, T, d, h, S.GELU, h + 1, dw=F32)


@pytest.mark.parametrize("T,d,h", [(1, 512, 1024), (20, 128, 264), (333, 128, 2744), (4100, 256, 1024)])
def test_nothing_is_read_from_the_workspace_before_it_is_written(H, T, d, h):
    x, dy, W1, W2 = make(T, d, h, 11)
    got = []
    for fill in (0, 255):   # zeros, and NaN in every type
        ws = [torch.full((max(n, 1),), fill, dtype=torch.uint8, device="cuda")
              for n in (H.hcw_gated_ffn_fwd_workspace_bytes(T, d, h),
                        H.hcw_gated_ffn_bwd_workspace_bytes(T, d, h))]
        got.append((H.hcw_gated_ffn_fwd(x, W1, W2, workspace=ws[0]),
                    *H.hcw_gated_ffn_bwd(x, dy, W1, W2, dw_dtype=BF16, workspace=ws[1])))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("act", [S.SILU, S.GELU, S.RELU])
@pytest.mark.parametrize("T,d,h", [(1, 512, 1024), (3, 72, 200), (8, 1024, 2744)])
def test_few_tokens_round_the_output_alone(H, T, d, h, act):
    """Up to 8 tokens a is kept in two bf16 parts: off by 2^-16 of itself."""
    x, _, W1, W2 = make(T, d, h, T + act)
    x64, w1, w2 = np64(x), np64(W1), np64(W2)
    g, u = x64 @ w1[:h].T, x64 @ w1[h:].T
    eg, eu = (2 * (d + 8) * U * (np.abs(x64) @ np.abs(w).T) for w in (w1[:h], w1[h:]))
    ag, _ = S.act(act, g)
    eag = 1.13 * eg + 16 * U * np.abs(g)
    a = ag * u
    ea = eag * np.abs(u) + (np.abs(ag) + eag) * eu
    ea = ea + 2.0 ** -16 * (np.abs(a) + ea)
    y = a @ w2.T
    ey = ea @ np.abs(w2).T + 2 * (2 * h + 8) * U * ((np.abs(a) + ea) @ np.abs(w2).T)
    close(H.hcw_gated_ffn_fwd(x, W1, W2, act), y, ey, "y")
    big = (W1.float() * 1e15).to(BF16)   # a = 1e30 and more: an infinite sum stays one
    got = H.hcw_gated_ffn_fwd((x.float() * 1e8).to(BF16), big, W2, S.RELU)
    assert not torch.isfinite(got).all()
