"""GPU parity with the fp64 oracle where every CTA works through several rows: wide norm
backwards, whose sums over the rows and rings go round, and distillation by clusters that take
many rows in turn."""
import numpy as np
import pytest
import torch

from oracle import student as S
from test_distill_gpu import KU, U, make
from test_norm_gpu import Problem, check_bwd, check_fwd

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", [S.RMS, S.LAYER])
@pytest.mark.parametrize("d", [4097, 8184, 8192])
def test_wide_norms_of_many_rows(H, d, kind, dtype):
    p = Problem(2100, d, dtype, d + kind)
    check_fwd(H, p, kind, kind)
    check_bwd(H, p, kind, kind)
    check_bwd(H, Problem(1300, d, dtype, d, rows=70), kind, 3 - kind)


def rows_close(rows, z, idx, teacher, target, weight, tau, kl, ce, loss, dz):
    """The bounds of the distillation's other parity tests, for some rows of a larger call."""
    z64, t64 = z[rows].double().numpy(), teacher[rows].astype(np.float64)
    idx, target, w64 = idx[rows], target[rows], weight[rows].astype(np.float64)
    z64[w64 == 0.0] = 0.0
    rl, rz = S.distill(z64, idx, t64, target, w64, tau, kl, ce)
    gl, g = loss.double().cpu().numpy()[rows], dz[torch.as_tensor(rows).cuda()].double().cpu().numpy()
    out = 2.0 ** -8 if z.dtype == BF16 else U
    for t, row in enumerate(rows):
        w, on = abs(w64[t]), idx[t] >= 0
        if w == 0.0:
            assert gl[t] == 0.0 and not g[t].any(), row
            continue
        top, V, L = np.abs(z64[t]).max(), z64.shape[1], 0.0
        A = np.abs(rz[t])
        if on.any():
            np.add.at(A, idx[t][on], 2 * w * kl * tau)
            L += kl * tau * tau * (2 * top / tau + np.log(V) + 2 * np.abs(t64[t][on]).max() / tau +
                                   np.log(on.sum() + 1))
        if target[t] >= 0:
            A[target[t]] += 2 * w * ce
            L += ce * (2 * top + np.log(V))
        assert abs(gl[t] - rl[t]) <= KU * w * L + U * abs(rl[t]) + 1e-38, (row, gl[t], rl[t])
        bound = KU * A
        bound = bound + out * (np.abs(rz[t]) + bound) + 1e-37
        assert (np.abs(g[t] - rz[t]) <= bound).all(), row


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,V,K,gap,tau",
                         [(T, V, K, 0, tau) for T, V in ((6000, 9000), (1500, 33001))
                          for K in (12, 65) for tau in (1.0, 2.0, 3.5)] + [(24000, 8200, 12, 22000, 2.0)])
def test_clusters_that_take_many_rows(H, T, V, K, gap, tau, dtype):
    """More rows than clusters run at once, and rows of weight 0 between them: single ones, runs,
    and (gap) a run of more than 32 of every cluster's own rows."""
    z, idx, teacher, target, weight = make(T, V, K, dtype, T + K) if T < 10000 else wide(T, V, K, dtype)
    rng = np.random.default_rng(K)
    weight[rng.random(T) < 0.1] = 0.0
    weight[T // 3:T // 3 + 90] = 0.0
    if gap:
        weight[1000:1000 + gap] = 0.0
    target[rng.random(T) < 0.1] = -1
    idx[rng.random(T) < 0.1] = -1
    idx[::17, -2:] = idx[::17, :2]                       # symbols that two slots name
    z[torch.from_numpy(weight == 0.0)] = float("nan")
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    args = (z.cuda(), dev(idx), dev(teacher), dev(target), dev(weight), tau, 0.7, 0.3)
    loss, dz = H.hcw_distill_loss(*args)
    alone, _ = H.hcw_distill_loss(*args, want_grad=False)
    assert H.hcw_sync_status() == H.HCW_OK
    assert torch.equal(loss, alone)
    zero = dev(weight == 0.0)
    assert not loss[zero].any() and not dz[zero].any()
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(dz).all())
    # a sample of every stretch of the rows, and both ends
    some = np.unique(np.concatenate([np.arange(20), T - 1 - np.arange(20), rng.integers(T, size=120),
                                     np.flatnonzero(weight)[-100:]]))
    rows_close(some, z, idx, teacher, target, weight, tau, 0.7, 0.3, loss, dz)


def wide(T, V, K, dtype):
    """make(), drawn on the GPU, the symbols of a row spread from a first one."""
    gen = torch.Generator(device="cuda").manual_seed(T)
    z = torch.empty(T, V, device="cuda").normal_(0.0, 2.5, generator=gen).to(dtype).cpu()
    rng = np.random.default_rng(T)
    idx = ((rng.integers(V, size=(T, 1)) + np.arange(K) * (V // K)) % V).astype(np.int32)
    return (z, idx, (3 * rng.normal(size=(T, K))).astype(np.float32),
            rng.integers(V, size=T).astype(np.int32), (0.25 + rng.random(T)).astype(np.float32))
