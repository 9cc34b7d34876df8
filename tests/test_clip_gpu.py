"""GPU parity of hcw_clip_grads with the fp64 oracle.

Tolerances, u = 2^-24.  A thread adds up to 64 squares in four chains of 16 multiply-adds and three
additions, a warp its threads in 5 more: every term is positive, so the sum is off by at most 24 u
relative, its root by half of that, by another half for the sum's rounding to fp32 before it and u for
its own: 13.5 u.  The factor is a quotient with that root: 14.5 u.  Below
2^-126 fp32's half step is 2^-150 whatever the value: norm and factor, which are returned in fp32, are
off by that there.  An output is one product (u) rounded once (half a step).
"""
import math

import numpy as np
import pytest
import torch

from oracle import ends as E

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: U}


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


def make(sizes, dtypes, seed=0, std=1.0, at=0):
    """Gradients that start `at` elements behind a 256-byte boundary, with guards around them."""
    g = torch.Generator().manual_seed(seed)
    bufs, grads = [], []
    for n, dt in zip(sizes, dtypes):
        b = torch.full((n + at + 64,), 7.0, dtype=dt)
        b[at:at + n] = (std * torch.randn(n, generator=g)).to(dt)
        b = b.cuda()
        bufs.append(b)
        grads.append(b[at:at + n])
    return bufs, grads


def check(H, sizes, dtypes, limit, seed=0, std=1.0, at=0, apart=None, stream=None):
    bufs, grads = make(sizes, dtypes, seed, std, at)
    before = [g.clone() for g in grads]
    limit = float(np.float32(min(limit, 1e300)) if limit < 3e38 else np.inf)   # as it arrives
    n64, c64, ref = E.clip([g.double().cpu().numpy() for g in grads], limit)
    outs = grads
    obufs = bufs
    if apart is not None:
        obufs, outs = make(sizes, dtypes, seed + 1, 1.0, apart)
    need = H.hcw_clip_grads_workspace_bytes(len(sizes))
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    norm = H.hcw_clip_grads(H.GradList(grads, None if apart is None else outs), limit,
                            workspace=ws[:need], stream=stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xFF).all())
    n, c = norm.double().cpu().tolist()
    assert abs(n - n64) <= 14 * U * n64 + 2.0 ** -150 and \
        abs(c - c64) <= 15 * U * c64 + 2.0 ** -150, (n, n64, c, c64)
    for k, (o, b, r, old, dt) in enumerate(zip(outs, obufs, ref, before, dtypes)):
        got = o.double().cpu().numpy()
        bound = 16 * U * np.abs(r)
        bound = bound + HALF[dt] * (np.abs(r) + bound) + 1e-44
        assert (np.abs(got - r) <= bound).all(), k
        if c64 == 1.0:
            assert torch.equal(o, old)
        head = at if apart is None else apart
        assert bool((b[:head] == 7.0).all()) and bool((b[head + sizes[k]:] == 7.0).all())
        if apart is not None:
            assert torch.equal(grads[k], old)
    return norm


SIZES = [[1], [7], [16384], [16385], [5, 1, 0, 33], [16384 * 3 + 5, 2, 40000], [100003, 65536, 777, 8],
         [3] * 32, [3] * 33, [1000 + i for i in range(100)]]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), s[0]))
def test_every_size(H, sizes, dtype):
    dts = [dtype] * len(sizes)
    check(H, sizes, dts, 0.5)
    check(H, sizes, dts, 1e6)
    check(H, sizes, dts, 0.5, apart=0)
    check(H, sizes, dts, 1e6, apart=0)


@pytest.mark.parametrize("at", [1, 2, 3, 5, 7])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_any_alignment(H, dtype, at):
    sizes = [1, 3, 9, 16383, 16384, 16390, 50001]
    dts = [dtype] * len(sizes)
    check(H, sizes, dts, 0.7, at=at)
    check(H, sizes, dts, 0.7, at=at, apart=at)
    check(H, sizes, dts, 0.7, at=at, apart=0)
    check(H, sizes, dts, 0.7, at=0, apart=at)


def test_types_side_by_side(H):
    sizes = [300, 70000, 5, 16384, 1]
    check(H, sizes, [BF16, F32, F32, BF16, BF16], 3.0)
    check(H, sizes, [F32, BF16, BF16, F32, F32], 3.0, apart=0)


@pytest.mark.parametrize("count", [511, 512, 513, 1500])
def test_many_tensors(H, count):
    rng = np.random.default_rng(count)
    sizes = rng.integers(0, 300, size=count).tolist()
    dts = [BF16 if b else F32 for b in rng.integers(2, size=count)]
    check(H, sizes, dts, 1.0)
    check(H, sizes, dts, 1.0, apart=0)


@pytest.mark.parametrize("std", [1e-44, 1e-38, 1e-30, 1e-21, 1e-19, 1e17, 1e19, 1e25, 1e36])
def test_squares_that_leave_the_range(H, std):
    check(H, [20000, 77], [F32, F32], 1e9 * std, std=std)   # not clipped
    n = check(H, [20000], [F32], 1e-3 if std > 1 else 1e-3 * std, std=std)
    assert bool(torch.isfinite(n[0]))
    if std > 1e-38:
        check(H, [20000, 77], [BF16, F32], 2.0 * std, std=std)


def test_small_and_large_side_by_side(H):
    g = torch.cat([torch.full((16384 * 2,), 1e-25), torch.full((3,), 1e25)]).cuda()
    norm = H.hcw_clip_grads([g], 1.0)
    assert abs(float(norm[0]) - math.sqrt(3) * 1e25) <= 14 * U * 2e25
    assert bool((g[:5] == 0).all()) or float(g[:5].max()) < 1e-44
    assert abs(float(g[-1]) - 3 ** -0.5) < 1e-6


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_leaves_the_gradients(H, bad):
    for dt in (BF16, F32):
        g = torch.randn(50000, device="cuda").to(dt)
        g[33333] = bad
        old = g.clone()
        norm = H.hcw_clip_grads([g], 1.0)
        assert not math.isfinite(float(norm[0])) and float(norm[1]) == 1.0
        assert math.isnan(float(norm[0])) == math.isnan(bad)
        assert torch.equal(torch.nan_to_num(g, 9.0), torch.nan_to_num(old, 9.0))


def test_a_norm_past_fp32_still_clips(H):
    g = torch.full((1000,), 3e38, device="cuda")
    norm = H.hcw_clip_grads([g], 1.0)
    assert math.isinf(float(norm[0]))
    assert abs(float(g[0]) - 1000 ** -0.5) < 1e-6


def test_zeros_no_tensors_and_the_norm_alone(H):
    g = torch.zeros(40000, device="cuda")
    assert H.hcw_clip_grads([g], 1.0).tolist() == [0.0, 1.0]
    assert H.hcw_clip_grads([g], 0.0).tolist() == [0.0, 1.0]
    assert H.hcw_clip_grads([], 1.0).tolist() == [0.0, 1.0]
    assert H.hcw_clip_grads([g[:0]], 1.0).tolist() == [0.0, 1.0]
    r = torch.randn(40000, device="cuda")
    old = r.clone()
    n = H.hcw_clip_grads([r], float("inf"))
    assert abs(float(n[0]) - float(old.double().norm())) <= 14 * U * float(n[0]) and float(n[1]) == 1.0
    assert torch.equal(r, old)
    out = torch.full_like(r, 7.0)
    H.hcw_clip_grads(H.GradList([r], [out]), float("inf"))
    assert torch.equal(out, old)
    H.hcw_clip_grads([r], 0.0)
    assert bool((r == 0).all())


def test_the_same_bits_another_stream_and_a_graph(H):
    sizes, dts = [300001, 16, 70000], [F32, F32, BF16]
    _, one = make(sizes, dts)
    _, two = make(sizes, dts)
    a, b = H.hcw_clip_grads(one, 1.0), H.hcw_clip_grads(two, 1.0, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    assert torch.equal(a, b) and all(torch.equal(x, y) for x, y in zip(one, two))
    _, grads = make(sizes, dts)
    start = [g.clone() for g in grads]
    q = H.GradList(grads)
    norm, ws = torch.empty(2, device="cuda"), torch.empty(
        H.hcw_clip_grads_workspace_bytes(3), dtype=torch.uint8, device="cuda")
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        H.hcw_clip_grads(q, 1.0, norm=norm, workspace=ws)
    for k in (1.0, 3.0):
        for g, s in zip(grads, start):
            g.copy_(s * k)
        graph.replay()
        torch.cuda.synchronize()
        assert abs(float(norm[0]) - k * float(a[0])) <= 2 ** -8 * k * float(a[0])
    for g, s in zip(grads, start):
        g.copy_(s)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(norm, a) and all(torch.equal(x, y) for x, y in zip(grads, one))


def test_tensors_that_share_memory_are_refused(H):
    g = torch.randn(1000, device="cuda")
    with pytest.raises(H.HcwError):
        H.hcw_clip_grads([g, g[100:300]], 1.0)
    with pytest.raises(H.HcwError):
        H.hcw_clip_grads(H.GradList([g], [g]), 1.0)
    H.hcw_clip_grads(H.GradList([g, g], [g.clone(), g.clone()]), 1.0)   # only read: allowed
    with pytest.raises(ValueError):
        H.hcw_clip_grads([g.view(10, 100).t()], 1.0)
    with pytest.raises(TypeError):
        H.hcw_clip_grads([g.half()], 1.0)
    with pytest.raises(ValueError):
        H.GradList([g], [g.view(10, 100).clone()])
