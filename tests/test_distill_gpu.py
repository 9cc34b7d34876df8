"""GPU parity of hcw_distill_loss with the fp64 oracle.

Tolerances.  Both sides start from the same logits.  fp32 with u = 2^-24: an
exponential is off by a few u and by u for each unit of its exponent (below 64
here wherever it matters), a sum by the length of its chain (64 symbols a
thread, then 5 + 4 + 3 joins): 128 u of the magnitudes that enter covers both.
dz is rounded once (bf16: half a step of 8 significant bits, 2^-8 relative; fp32: u).
"""
import numpy as np
import pytest
import torch

from oracle import student as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
KU = 128 * U
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


def make(T, V, K, dtype, seed, std=2.5):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((std * rng.normal(size=(T, V))).astype(np.float32)).to(dtype)
    idx = np.stack([rng.permutation(V)[:K] if K <= V else rng.integers(V, size=K)
                    for _ in range(T)]).astype(np.int32).reshape(T, K)
    teacher = (3 * rng.normal(size=(T, K))).astype(np.float32)
    target = rng.integers(V, size=T).astype(np.int32)
    weight = (0.25 + rng.random(T)).astype(np.float32)
    return z, idx, teacher, target, weight


def check(H, z, idx, teacher, target, weight, tau, kl, ce, stream=None):
    T, V = z.shape
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    n, pad = T * V, 64
    buf = torch.full((n + pad,), 7.0, dtype=z.dtype, device="cuda")
    args = (z.cuda(), dev(idx), dev(teacher), dev(target), dev(weight), tau, kl, ce)
    loss, dz = H.hcw_distill_loss(*args, dz=buf[:n].view(T, V), stream=stream)
    torch.cuda.synchronize()
    assert bool((buf[n:] == 7.0).all())
    alone, none = H.hcw_distill_loss(*args, want_grad=False, stream=stream)
    torch.cuda.synchronize()
    assert none is None and torch.equal(torch.nan_to_num(alone, 9.0), torch.nan_to_num(loss, 9.0))
    z64 = z.double().numpy()
    t64 = None if teacher is None else teacher.astype(np.float64)
    w64 = None if weight is None else weight.astype(np.float64)
    with np.errstate(invalid="ignore"):
        rl, rz = S.distill(z64, idx, t64, target, w64, tau, kl, ce)
    g, gl = dz.double().cpu().numpy(), loss.double().cpu().numpy()
    out = 2.0 ** -8 if z.dtype == BF16 else U
    for t in range(T):
        w = 1.0 if w64 is None else w64[t]
        if not np.isfinite(rl[t]):
            assert np.isposinf(gl[t]) == np.isposinf(rl[t])
            continue
        # magnitudes: kl tau (q + sum p) + ce (q1 + [y]), and the loss's terms
        A = np.abs(rz[t])
        L = 0.0
        fin = z64[t][np.isfinite(z64[t])]
        top = np.abs(fin).max() if fin.size else 0.0
        if idx is not None and kl:
            on = (idx[t] >= 0) & (idx[t] < V)
            A = A.copy()
            np.add.at(A, idx[t][on], 2 * abs(w) * kl * tau)
            L += kl * tau * tau * (2 * top / tau + np.log(V) + np.abs(t64[t][on]).max(initial=0, where=np.isfinite(t64[t][on])) * 2 / tau + np.log(len(idx[t]) + 1))
        if target is not None and ce and 0 <= target[t] < V:
            A[target[t]] += 2 * abs(w) * ce
            L += ce * (2 * top + np.log(V))
        assert abs(gl[t] - rl[t]) <= KU * abs(w) * L + U * abs(rl[t]) + 1e-38, (t, gl[t], rl[t])
        bound = KU * A
        bound = bound + out * (np.abs(rz[t]) + bound) + 1e-37
        bad = np.abs(g[t] - rz[t]) > bound
        assert not bad.any(), (t, np.argmax(bad), float((np.abs(g[t] - rz[t]) / bound).max()))


SIZES = [(1, 1, 1), (3, 2, 1), (5, 37, 4), (9, 201, 16), (4, 256, 64), (3, 1000, 65), (6, 1024, 8),
         (7, 1025, 8), (5, 4097, 33), (3, 8193, 20), (2, 32003, 50), (9, 50257, 7), (1, 65535, 100),
         (2, 131072, 64), (1, 262144, 1024), (1, 262143, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,V,K", SIZES)
def test_every_size(H, T, V, K, dtype):
    z, idx, teacher, target, weight = make(T, V, K, dtype, V + K)
    check(H, z, idx, teacher, target, weight, 1.0, 0.7, 0.3)
    check(H, z, idx, teacher, target, weight, 2.0, 0.7, 0.3)
    check(H, z, idx, teacher, None, None, 3.5, 1.0, 0.0)


@pytest.mark.parametrize("V", [130, 1024, 5000])
def test_many_rows(H, V):
    z, idx, teacher, target, weight = make(321, V, 12, BF16, V)
    check(H, z, idx, teacher, target, weight, 1.5, 0.5, 0.5)


@pytest.mark.parametrize("V,K", [(100, 12), (3001, 12), (3000, 200)])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_slots_and_rows_that_are_empty(H, V, K, tau):
    z, idx, teacher, target, weight = make(14, V, K, BF16, V)
    idx[0] = -1                     # no slot, a label
    idx[1], target[1] = -1, -1      # neither
    idx[2, 1:] = -7                 # one slot
    teacher[3] = -np.inf            # slots without probability
    teacher[4, ::2] = -np.inf
    idx[5, :] = idx[5, 0]           # one symbol in every slot
    idx[6, 3] = idx[6, 0]
    target[6] = idx[6, 0]           # the label is a symbol that occurs twice
    target[7] = idx[7, 2]
    weight[8] = 0.0
    weight[9] = -0.5
    teacher[10, 0] = 3e38           # a slot that takes everything
    idx[11, ::3] = -1
    teacher[11, ::3] = np.nan       # what an empty slot holds is not read as a logit
    check(H, z, idx, teacher, target, weight, tau, 0.7, 0.3)


@pytest.mark.parametrize("V", [100, 3001])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_masked_symbols(H, V, dtype):
    z, idx, teacher, target, weight = make(10, V, 8, dtype, V)
    low = torch.finfo(dtype).min
    z[0, V // 2:] = -float("inf")
    z[1, V // 2:] = low
    z[2, :] = -float("inf")         # nothing can occur: 0 and 0
    z[3, 1:] = -float("inf")        # one symbol left
    z[4, :] = low                   # every symbol alike
    z[5, :] = float("nan")
    weight[5] = 0.0                 # a row without weight is not looked at
    z[6, :8] = -float("inf")
    for t in (0, 1):
        idx[t] = np.arange(8)
        target[t] = 3
    idx[3] = 0
    target[3] = 0
    idx[6] = 20 + np.arange(8)
    target[6] = 30
    check(H, z, idx, teacher, target, weight, 1.0, 0.7, 0.3)
    check(H, z, idx, teacher, target, weight, 2.0, 0.7, 0.3)
    # a symbol that cannot occur, named by the label or the teacher: +inf
    z[7, 5] = -float("inf")
    target[7] = 5
    z[8, 6] = -float("inf")
    idx[8, 0] = 6
    check(H, z, idx, teacher, target, weight, 1.0, 0.7, 0.3)


@pytest.mark.parametrize("V", [100, 3001, 140000])
def test_nan_and_inf_stay_in_their_row(H, V):
    z, idx, teacher, target, weight = make(4, V, 4, F32, V)
    z[1, V // 3] = float("nan")
    z[2, V - 1] = float("inf")
    a = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    loss, dz = H.hcw_distill_loss(z.cuda(), a(idx), a(teacher), a(target), a(weight), 1.0, 0.5, 0.5)
    assert loss.isnan().tolist() == [False, True, True, False]
    assert dz[1].isnan().all() and dz[2].isnan().all()
    assert dz[0].isfinite().all() and dz[3].isfinite().all()


@pytest.mark.parametrize("V", [100, 3001])
def test_symbols_past_the_vocabulary_are_reported(H, V):
    z, idx, teacher, target, weight = make(3, V, 4, BF16, V)
    assert H.hcw_sync_status() == H.HCW_OK
    idx[0, 1] = V
    check(H, z, idx, teacher, target, weight, 1.0, 0.7, 0.3)
    assert H.hcw_sync_status() == H.HCW_ERR_INVALID_ARG
    target[2] = V + 5
    idx[0, 1] = -1
    check(H, z, idx, teacher, target, weight, 1.0, 0.7, 0.3)
    assert H.hcw_sync_status() == H.HCW_ERR_INVALID_ARG
    assert H.hcw_sync_status() == H.HCW_OK


def test_parts_alone_and_no_rows(H):
    z, idx, teacher, target, weight = make(6, 500, 5, BF16, 3)
    check(H, z, None, None, target, weight, 2.0, 1.0, 0.4)      # labels alone: temperature unused
    check(H, z, idx, teacher, target, weight, 2.0, 0.0, 1.0)
    check(H, z, idx, teacher, target, None, 2.0, 1.0, 0.0)
    e = torch.empty(0, 500, dtype=BF16, device="cuda")
    loss, dz = H.hcw_distill_loss(e)
    assert loss.shape == (0,) and dz.shape == (0, 500)


@pytest.mark.parametrize("V", [200, 9000])
def test_another_stream_and_the_same_bits(H, V):
    z, idx, teacher, target, weight = make(50, V, 9, BF16, V)
    st = torch.cuda.Stream()
    check(H, z, idx, teacher, target, weight, 1.0, 0.7, 0.3, stream=st)
    a = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    args = (z.cuda(), a(idx), a(teacher), a(target), a(weight), 2.0, 0.7, 0.3)
    one, two = H.hcw_distill_loss(*args), H.hcw_distill_loss(*args)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [256, 257, 1023, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 8191, 8193])
def test_rows_of_several_warps(H, V, dtype):
    """Every number of warps a row, rows that start at odd places, named ends."""
    z, idx, teacher, target, weight = make(11, V, 40, dtype, V)
    idx[1, 0], idx[1, 1] = 0, V - 1          # the row's ends are named ...
    target[1], target[2] = V - 1, 0          # ... and labels
    idx[2, 5] = 0
    idx[3, 1] = idx[3, 39] = idx[3, 0]       # a symbol three times, far apart
    weight[4] = 0.0
    z[4, :] = float("nan")
    z[5, : V // 2] = -float("inf")
    z[6, :] = -float("inf")
    z[6, V - 1] = 1.0
    target[5] = target[6] = V - 1
    idx[5], idx[6] = -1, -1
    for tau in (1.0, 2.0, 3.5):
        check(H, z[:4], idx[:4], teacher[:4], target[:4], weight[:4], tau, 0.7, 0.3)
        check(H, z[5:], idx[5:], teacher[5:], target[5:], weight[5:], tau, 0.7, 0.3)
    a = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    loss, dz = H.hcw_distill_loss(z.cuda(), a(idx), a(teacher), a(target), a(weight), 2.0, 0.7, 0.3)
    torch.cuda.synchronize()
    assert float(loss[4]) == 0.0 and bool((dz[4] == 0).all())
    assert bool(torch.isfinite(dz[3]).all()) and bool(torch.isfinite(dz[5]).all())


@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_empty_slots_in_long_rows(H, tau):
    test_slots_and_rows_that_are_empty(H, 9001, 12, tau)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_masked_symbols_in_long_rows(H, dtype):
    test_masked_symbols(H, 9001, dtype)


def test_symbols_past_a_long_vocabulary_are_reported(H):
    test_symbols_past_the_vocabulary_are_reported(H, 9001)
