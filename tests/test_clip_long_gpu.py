"""hcw_clip_grads above some 10 M elements, where a launch's chunks are the long ones (64 elements a
thread for the norm, 32 for the product), against fp64 (tolerances: test_clip_gpu.py)."""
import math

import numpy as np
import pytest
import torch

from test_clip_gpu import BF16, F32, HALF, U, H  # noqa: F401 (H is the fixture)

pytestmark = pytest.mark.gpu

CHUNK = 512 * 64


def tensors(sizes, dtypes, seed, std, at):
    """Gradients that start `at` elements behind a boundary, with guards around them."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    bufs = []
    for n, dt in zip(sizes, dtypes):
        b = torch.full((at + n + 64,), 7.0, dtype=dt, device="cuda")
        b[at:at + n] = (std * torch.randn(n, generator=gen, device="cuda", dtype=torch.float64)).to(dt)
        bufs.append(b)
    return bufs, [b[at:at + n] for b, n in zip(bufs, sizes)]


def check(H, sizes, dtypes, part=0.25, seed=0, std=1.0, at=0, apart=None):  # noqa: F811
    """Clipped to `part` of the norm."""
    assert sum(sizes) > 608 * 16384                   # (four long chunks an SM)
    bufs, grads = tensors(sizes, dtypes, seed, std, at)
    before = [g.clone() for g in grads]
    # (std may be small: scaled, so that no square leaves fp64's range; sums of fp64 lose nothing here)
    total = std * math.sqrt(math.fsum(float(((g.double() / std) ** 2).sum()) for g in before))
    limit = float(np.float32(part * total))
    want = min(1.0, limit / total)
    outs, obufs, first = grads, bufs, at
    if apart is not None:
        first = apart
        obufs, outs = tensors(sizes, dtypes, seed + 1, 1.0, apart)
    need = H.hcw_clip_grads_workspace_bytes(len(sizes))
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    norm, factor = H.hcw_clip_grads(H.GradList(grads, None if apart is None else outs), limit,
                                    workspace=ws[:need]).double().cpu().tolist()
    assert bool((ws[need:] == 0xFF).all())
    assert abs(norm - total) <= 14 * U * total + 2.0 ** -150, (norm, total)
    assert abs(factor - want) <= 15 * U * want, (factor, want)
    for k, (o, b, old, dt) in enumerate(zip(outs, obufs, before, dtypes)):
        ref = old.double() * want
        bound = 16 * U * ref.abs()
        bound = bound + HALF[dt] * (ref.abs() + bound) + 1e-44
        assert bool(((o.double() - ref).abs() <= bound).all()), k
        assert bool((b[:first] == 7.0).all()) and bool((b[first + sizes[k]:] == 7.0).all())
        if apart is not None:
            assert torch.equal(grads[k], old)
        if want == 1.0:
            assert torch.equal(o, old)


FEW = [CHUNK * 300 + 17, 1, CHUNK, 0, 1 << 22, CHUNK - 1, 5, CHUNK // 2 + 3, 777, CHUNK + 1]
MANY = [int(n) for n in np.random.default_rng(1).integers(0, 600000, size=60)] + [1, 0, CHUNK, CHUNK + 7]
MOST = [int(n) for n in np.random.default_rng(2).integers(0, 60000, size=700)] + [11000000]


@pytest.mark.parametrize("kind", ["bf16", "f32", "mixed"])
@pytest.mark.parametrize("sizes", [[12000001], FEW, MANY, MOST], ids=lambda s: str(len(s)))
def test_long_chunks(H, sizes, kind):  # noqa: F811
    dts = [{"bf16": BF16, "f32": F32}.get(kind, (BF16, F32, F32, BF16, BF16)[i % 5])
           for i in range(len(sizes))]
    check(H, sizes, dts)
    check(H, sizes, dts, apart=0)
    check(H, sizes, dts, part=2.0)
    check(H, sizes, dts, part=2.0, apart=0)


@pytest.mark.parametrize("at,apart", [(1, None), (3, None), (1, 1), (3, 0), (0, 3), (5, 2)])
@pytest.mark.parametrize("kind", ["bf16", "f32", "mixed"])
def test_any_alignment(H, kind, at, apart):  # noqa: F811
    for sizes in (FEW, MANY):
        dts = [{"bf16": BF16, "f32": F32}.get(kind, (F32, BF16)[i % 2]) for i in range(len(sizes))]
        check(H, sizes, dts, at=at, apart=apart)


@pytest.mark.parametrize("std", [1e-30, 1e-21, 1e19, 1e25])
def test_squares_that_leave_the_range(H, std):  # noqa: F811
    check(H, FEW, [F32] * len(FEW), std=std)
    check(H, FEW, [BF16, F32] * (len(FEW) // 2), std=std, at=3, apart=1)


def test_one_that_is_not_finite_leaves_them_all(H):  # noqa: F811
    bufs, grads = tensors(FEW, [F32] * len(FEW), 3, 1.0, 1)
    grads[4][4000001] = float("nan")
    before = [g.clone() for g in grads]
    norm, factor = H.hcw_clip_grads(grads, 1.0).tolist()
    assert math.isnan(norm) and factor == 1.0
    assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in zip(grads, before))


def test_every_element_is_taken_once(H):  # noqa: F811
    """Ones: the norm's square is the number of elements, each comes out as the factor."""
    for dt in (BF16, F32):
        grads = [torch.ones(n, dtype=dt, device="cuda") for n in FEW]
        n = sum(FEW)
        norm, factor = H.hcw_clip_grads(grads, 1.0).tolist()
        assert abs(norm ** 2 - n) <= 28 * U * n
        for g in grads:
            assert bool((g == torch.tensor(factor, device="cuda").to(dt)).all())
