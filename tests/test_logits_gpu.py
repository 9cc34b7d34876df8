"""GPU parity of hcw_logits_edit with the fp64 oracle.

Tolerances, u = 2^-24.  An edited logit takes one product or quotient, two products, two subtractions
and an addition for each of its slots, each in fp32: (6 + slots) u of the magnitudes that enter.  The
output is rounded once: half a step, bf16 2^-8, fp32 u.  What is not edited keeps its bits, and what
an edit takes past fp32's largest number is infinite.
"""
import numpy as np
import pytest
import torch

from oracle import ends as E

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, F32: U}
KEYS = ("history", "lengths", "prompt", "repetition", "frequency", "presence", "bias_idx", "bias", "mask")


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


def make(B, V, Hn, M, dtype, mask=True, seed=0):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((3 * rng.normal(size=(B, V))).astype(np.float32)).to(dtype)
    a = dict(history=np.minimum((V ** rng.random((B, Hn))).astype(np.int64) - 1, V - 1).astype(np.int32),
             lengths=rng.integers(0, Hn + 1, size=B).astype(np.int32),
             prompt=rng.integers(-1, Hn + 1, size=B).astype(np.int32),
             repetition=(1 + rng.random(B)).astype(np.float32),
             frequency=rng.normal(size=B).astype(np.float32),
             presence=rng.normal(size=B).astype(np.float32))
    if Hn > 4:
        a["history"][:, 3] = -1
    if M:
        a["bias_idx"] = rng.integers(-1, V, size=(B, M)).astype(np.int32)
        a["bias"] = (2 * rng.normal(size=(B, M))).astype(np.float32)
    if mask:
        a["mask"] = rng.integers(-2 ** 31, 2 ** 31, size=(B, -(-V // 32))).astype(np.int32)
    if not Hn:
        for k in ("history", "lengths", "prompt"):
            del a[k]
    return z, a


def run(H, z, a, out=None, stream=None):
    dev = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in a.items()}
    return H.hcw_logits_edit(z, out=out, stream=stream, **dev)


def check(H, z, a, stream=None):
    B, V = z.shape
    n = B * V
    buf = torch.full((n + 64,), 7.0, dtype=z.dtype, device="cuda")
    out = run(H, z.cuda(), a, buf[:n].view(B, V), stream)
    torch.cuda.synchronize()
    assert bool((buf[n:] == 7.0).all())
    again = buf.clone()
    again[:n] = z.cuda().flatten()
    same = again[:n].view(B, V)
    run(H, same, a, same, stream)                     # in place: the same bits
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(same, 9.0, 8.0, 6.0), torch.nan_to_num(out, 9.0, 8.0, 6.0))
    assert bool((again[n:] == 7.0).all())
    f = {k: v.astype(np.float64) if v.dtype == np.float32 else v for k, v in a.items()}
    z64 = z.double().numpy()
    with np.errstate(invalid="ignore"):
        ref, mag = E.edit(z64, f.get("history"), f.get("lengths"), f.get("prompt"), f.get("repetition"),
                          f.get("frequency"), f.get("presence"), f.get("bias_idx"), f.get("bias"),
                          f.get("mask"))
        # what lies past fp32's largest number is infinite (products are fp32)
        ref = np.where(np.abs(ref) > float(np.finfo(np.float32).max), np.copysign(np.inf, ref), ref)
        slots = f["bias_idx"].shape[1] if "bias_idx" in f else 0
        got = out.double().cpu().numpy()
        fin = np.isfinite(ref)
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert np.array_equal(got[~fin & ~np.isnan(ref)], ref[~fin & ~np.isnan(ref)])
        bound = (6 + slots) * U * mag
        bound = bound + HALF[z.dtype] * (np.abs(ref) + bound) + 1e-37
        bad = fin & ~(np.abs(got - ref) <= bound)
        assert not bad.any(), np.argwhere(bad)[:4]
        kept = fin & (ref == z64)
        assert np.array_equal(got[kept], z64[kept])
    return out


SIZES = [(1, 1, 1, 0), (1, 5, 3, 2), (2, 33, 40, 7), (3, 201, 256, 0), (5, 1000, 1, 40), (2, 4099, 3000, 300),
         (1, 32003, 1024, 16), (4, 50257, 100, 1024), (1, 131072, 500, 64), (7, 1023, 70, 3), (40, 8192, 64, 5),
         (65, 32003, 90, 9)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,V,Hn,M", SIZES)
def test_every_size(H, B, V, Hn, M, dtype):
    z, a = make(B, V, Hn, M, dtype, seed=V)
    check(H, z, a)
    del a["mask"]
    check(H, z, a)


@pytest.mark.parametrize("drop", ["history", "penalties", "repetition", "frequency", "presence", "lengths",
                                  "prompt", "bias", "everything"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_parts_that_are_not_there(H, drop, dtype):
    z, a = make(3, 777, 50, 6, dtype)
    gone = {"history": ("history", "lengths", "prompt"), "bias": ("bias_idx", "bias"),
            "penalties": ("repetition", "frequency", "presence"), "everything": KEYS}.get(drop, (drop,))
    for k in gone:
        del a[k]
    check(H, z, a)
    a.pop("mask", None)
    check(H, z, a)


@pytest.mark.parametrize("V", [100, 20001])
def test_masks(H, V):
    z, a = make(6, V, 30, 4, F32)
    a["mask"][0] = 0                              # nothing can occur
    a["mask"][1] = -1
    a["mask"][2] = 0
    a["mask"][2, (V - 1) // 32] = np.int64(1 << ((V - 1) % 32)).astype(np.int32)   # the last one alone
    a["mask"][3] = 1                              # every 32nd
    z[4, 3] = float("nan")
    z[4, 9] = float("inf")
    z[4, 11] = -float("inf")
    z[5] = torch.finfo(F32).min
    out = check(H, z, a)
    assert bool((out[0] == -float("inf")).all())
    assert int(torch.isfinite(out[2]).sum()) == 1
    a["mask"][4] = 0
    assert bool((check(H, z, a)[4] == -float("inf")).all())


@pytest.mark.parametrize("V", [64, 9000])
def test_slots_that_name_one_symbol(H, V):
    z, a = make(4, V, 20, 700, F32)
    a["bias_idx"][0] = 5                          # all of them
    a["bias_idx"][1, ::2] = V - 1
    a["bias_idx"][2] = -1
    a["bias_idx"][3] = np.arange(700) % V
    a["bias"][1, 0] = -np.inf                     # a symbol that is ruled out
    del a["mask"]
    out = check(H, z, a)
    assert float(out[1, V - 1]) == -float("inf")


def test_counts_of_long_histories(H):
    z, a = make(2, 300, 70000, 0, F32, mask=False)
    a["history"][0] = 7
    a["lengths"][:] = 70000
    a["prompt"][0] = 1
    a["prompt"][1] = 70000                        # nothing of its own: no frequency, no presence
    check(H, z, a)
    a["lengths"][:] = (-3, 1 << 20)               # taken to 0 .. H
    check(H, z, a)


def test_symbols_past_the_vocabulary_are_reported(H):
    z, a = make(3, 90, 20, 4, BF16)
    check(H, z, a)
    assert H.hcw_sync_status() == H.HCW_OK
    a["lengths"][:] = 20
    a["history"][1, 2] = 90
    check(H, z, a)
    assert H.hcw_sync_status() == H.HCW_ERR_INVALID_ARG
    a["history"][1, 2] = 0
    a["bias_idx"][2, 1] = 2 ** 31 - 1
    check(H, z, a)
    assert H.hcw_sync_status() == H.HCW_ERR_INVALID_ARG
    assert H.hcw_sync_status() == H.HCW_OK


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rows_at_odd_places(H, dtype):
    for V in range(1, 40):
        z, a = make(9, V, 12, 3, dtype, seed=V)
        check(H, z, a)
    for V in (2047, 2049, 4095, 4097, 16383, 16385, 16391):
        z, a = make(3, V, 12, 3, dtype, seed=V)
        check(H, z, a)


def test_another_stream_a_graph_and_no_rows(H):
    z, a = make(5, 3001, 40, 8, BF16)
    one = check(H, z, a).clone()
    st = torch.cuda.Stream()
    assert torch.equal(one, check(H, z, a, stream=st))
    dev = {k: torch.from_numpy(v).cuda() for k, v in a.items()}
    zd, out = z.cuda(), torch.empty(5, 3001, dtype=BF16, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        H.hcw_logits_edit(zd, out=out, **dev)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, one)
    assert H.hcw_logits_edit(zd[:0]).shape == (0, 3001)


def test_shapes_are_checked(H):
    z = torch.zeros(3, 64, device="cuda")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    for kw in (dict(history=i(2, 5)), dict(history=i(15)), dict(history=i(3, 5), lengths=i(2)),
               dict(repetition=f(4)), dict(bias_idx=i(3, 2)), dict(bias=f(3, 2)),
               dict(bias_idx=i(3, 2), bias=f(3, 4)), dict(mask=i(3, 3)), dict(out=f(64, 3))):
        with pytest.raises(ValueError):
            H.hcw_logits_edit(z, **kw)
    for kw in (dict(history=i(3, 5).long()), dict(mask=f(3, 2)), dict(presence=i(3)),
               dict(bias_idx=i(3, 2), bias=i(3, 2))):
        with pytest.raises(TypeError):
            H.hcw_logits_edit(z, **kw)


LARGE = [(60, 50001, 300, 64), (200, 20003, 4000, 90), (3, 1500001, 40, 1024), (40, 131072, 4097, 5),
         (900, 8191, 60, 20), (40, 131072, 0, 30), (40, 131072, 700, 0), (30, 60001, 20000, 40)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,V,Hn,M", LARGE)
def test_large_batches(H, B, V, Hn, M, dtype):
    """Sizes at which the named symbols have a launch of their own, with and without a mask."""
    z, a = make(B, V, Hn, M, dtype, seed=V)
    if Hn > 100:
        a["history"][0] = a["history"][0, 5]                       # one symbol all along
        a["history"][1] = np.arange(Hn) * 31 % V                   # every symbol another one
        a["lengths"][:2], a["prompt"][:2] = Hn, (Hn // 2, 0)
    if M > 4:
        a["bias_idx"][0] = 5                                       # one symbol in every slot
        a["bias_idx"][1, ::2] = V - 1
        a["bias_idx"][2, 1] = a["history"][2, 0] if Hn else 0      # a symbol of the history too
    a["mask"][0] = -1
    a["mask"][1, : 9] = 0
    a["mask"][2] = 0
    check(H, z, a)
    del a["mask"]
    check(H, z, a)


def test_rows_at_odd_places_in_large_batches(H):
    for V in (16385, 16386, 16391, 33003):
        for dtype in (BF16, F32):
            z, a = make(257, V, 5, 2, dtype, seed=V)
            check(H, z, a)


def test_a_large_batch_in_a_graph(H):
    z, a = make(64, 50001, 300, 64, F32)
    one = check(H, z, a).clone()
    dev = {k: torch.from_numpy(v).cuda() for k, v in a.items()}
    zd, out, st = z.cuda(), torch.empty(64, 50001, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        # the history is written right before the call that reads it
        past = dev["history"] + 0
        H.hcw_logits_edit(zd, out=out, **dict(dev, history=past))
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, one)
