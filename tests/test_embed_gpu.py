"""GPU parity of hcw_embed_fwd and hcw_embed_bwd with the fp64 oracle.

Tolerances, u = 2^-24 and h half a step of the output's type (bf16 2^-8, fp32 u).  The lookup
multiplies once in fp32 (u) and rounds once (h).  A gradient is a sum of n rows in fp32, which any
order of adding keeps within (n - 1) u of the sum of the magnitudes, times the scale (u), plus what
was there (u), rounded once (h).
"""
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


def symbols(rng, V, T, pad=0.1):
    """A few symbols often, most of them never, some padding."""
    ids = np.minimum((V ** rng.random(T)).astype(np.int64) - 1 + (rng.random(T) < 0.2), V - 1)
    return np.where(rng.random(T) < pad, -1 - rng.integers(3, size=T), ids).astype(np.int32)


def check_fwd(H, ids, table, scale, stream=None):
    T, d = len(ids), table.shape[1]
    buf = torch.full((T * d + 64,), 7.0, dtype=table.dtype, device="cuda")
    x = H.hcw_embed_fwd(torch.from_numpy(ids).cuda(), table.cuda(), scale, x=buf[:T * d].view(T, d),
                        stream=stream)
    torch.cuda.synchronize()
    assert bool((buf[T * d:] == 7.0).all())
    ref = E.embed_fwd(ids, table.double().numpy(), np.float32(scale).astype(np.float64))
    err = np.abs(x.double().cpu().numpy() - ref)
    assert (err <= (HALF[table.dtype] + 2 * U) * np.abs(ref) + 1e-38).all()


def check_bwd(H, ids, dx, V, scale, out=F32, base=None, stream=None, poison=0.0):
    T, d = dx.shape
    n = V * d
    buf = torch.full((n + 64,), 7.0, dtype=out, device="cuda")
    dE = buf[:n].view(V, d)
    if base is not None:
        dE.copy_(base)
    need = H.hcw_embed_bwd_workspace_bytes(T, V, d)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    if poison:
        ws[:need // 4 * 4].view(torch.float32).fill_(poison)
    H.hcw_embed_bwd(torch.from_numpy(ids).cuda(), dx.cuda(), V, scale, dE=dE,
                    accumulate=base is not None, workspace=ws[:need], stream=stream)
    torch.cuda.synchronize()
    assert bool((buf[n:] == 7.0).all()) and bool((ws[need:] == 0xA5).all())
    s = float(np.float32(scale))
    x64 = dx.double().numpy()
    b64 = None if base is None else base.double().numpy()
    ref = E.embed_bwd(ids, x64, V, s, b64)
    mag = E.embed_bwd(ids, np.abs(x64), V, abs(s), None if b64 is None else np.abs(b64))
    count = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)[:, None]
    got = dE.double().cpu().numpy()
    bound = (count + 3) * U * mag
    bound = bound + HALF[out] * (np.abs(ref) + bound) + 1e-37
    named = count[:, 0] > 0
    assert (np.abs(got - ref) <= bound)[named].all(), float((np.abs(got - ref) / bound)[named].max())
    # no token: zeros, or left alone
    rest = np.zeros_like(ref) if base is None else b64
    assert np.array_equal(got[~named], rest[~named])
    return dE


SIZES = [(1, 1, 1), (1, 5, 8), (3, 2, 7), (33, 300, 64), (64, 31, 513), (257, 1000, 24), (100, 151, 2048),
         (1000, 152, 40), (1000, 153, 256), (2049, 40000, 33), (4099, 3203, 777), (5000, 17, 96),
         (700, 9001, 9), (90, 5003, 1), (1500, 4001, 63), (300, 2503, 130), (400, 200003, 7)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", SIZES)
def test_every_size(H, T, V, d, dtype):
    rng = np.random.default_rng(T + V + d)
    ids = symbols(rng, V, T)
    table = torch.from_numpy(rng.normal(size=(V, d)).astype(np.float32)).to(dtype)
    dx = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32)).to(dtype)
    check_fwd(H, ids, table, d ** 0.5)
    check_fwd(H, ids, table, 1.0)
    check_bwd(H, ids, dx, V, d ** 0.5, poison=float("nan"))
    check_bwd(H, ids, dx, V, 0.3, out=BF16)
    base = torch.from_numpy(rng.normal(size=(V, d)).astype(np.float32))
    check_bwd(H, ids, dx, V, -1.0, base=base)
    check_bwd(H, ids, dx, V, 1.0, out=BF16, base=base.to(BF16))


@pytest.mark.parametrize("T", [1, 31, 32, 33, 127, 128, 129, 1023, 1025, 4095, 4097, 20000])
def test_runs_over_chunks(H, T):
    """One symbol for every token, two, and runs that end where a chunk does."""
    rng = np.random.default_rng(T)
    d, V = 72, 500
    dx = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32)).to(BF16)
    at = np.arange(T)
    for ids in (np.full(T, 3), at % 2 * 499, at // 8 % V, at // 32 % V, at // 33 % V, at // 300 % V,
                (T - 1 - at) // 64 % V, np.full(T, -1)):
        check_bwd(H, ids.astype(np.int32), dx, V, 1.0, poison=float("nan"))


@pytest.mark.parametrize("T", [16384, 16385, 24577, 40001, 100000])
@pytest.mark.parametrize("V,d", [(1, 8), (3, 24), (201, 16), (5003, 9), (40000, 8), (99000, 4), (120000, 4)])
def test_many_tokens(H, T, V, d):
    rng = np.random.default_rng(T + V)
    ids = symbols(rng, V, T)
    ids[::11] = ids[0]
    ids[T - 100:] = V - 1
    dx = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32))
    at = torch.from_numpy(np.where(ids < 0, V, ids)).long()
    want = torch.zeros(V + 1, d, dtype=torch.float64).index_add_(0, at, dx.double())[:V]
    mag = torch.zeros(V + 1, d, dtype=torch.float64).index_add_(0, at, dx.double().abs())[:V]
    dE = torch.full((V, d), float("nan"), device="cuda")
    H.hcw_embed_bwd(torch.from_numpy(ids).cuda(), dx.cuda(), V, dE=dE)
    assert bool(((dE.double().cpu() - want).abs() <= T * U * mag).all())
    again = H.hcw_embed_bwd(torch.from_numpy(ids).cuda(), dx.cuda(), V)
    assert torch.equal(again, dE)
    assert H.hcw_sync_status() == H.HCW_OK


@pytest.mark.parametrize("V", [256 * 152 - 1, 256 * 152 + 1, 131072, 262144, 1 << 20])
def test_vocabularies_of_one_and_two_sorting_passes(H, V):
    rng = np.random.default_rng(V)
    T, d = 3000, 16
    ids = rng.integers(V, size=T).astype(np.int32)
    ids[::7] = ids[0]
    ids[1::5] = V - 1
    dx = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32))
    want = torch.zeros(V, d, dtype=torch.float64).index_add_(0, torch.from_numpy(ids).long(), dx.double())
    mag = torch.zeros(V, d, dtype=torch.float64).index_add_(0, torch.from_numpy(ids).long(),
                                                           dx.double().abs())
    got = H.hcw_embed_bwd(torch.from_numpy(ids).cuda(), dx.cuda(), V).double().cpu()
    assert bool(((got - want).abs() <= 3000 * U * mag).all())


def test_symbols_past_the_vocabulary_are_reported(H):
    rng = np.random.default_rng(5)
    V, d = 90, 24
    ids = rng.integers(V, size=50).astype(np.int32)
    table = torch.from_numpy(rng.normal(size=(V, d)).astype(np.float32))
    dx = torch.from_numpy(rng.normal(size=(50, d)).astype(np.float32))
    check_fwd(H, ids, table, 2.0)
    check_bwd(H, ids, dx, V, 2.0)
    assert H.hcw_sync_status() == H.HCW_OK
    ids[7], ids[20] = V, 2 ** 31 - 1
    check_fwd(H, ids, table, 2.0)
    assert H.hcw_sync_status() == H.HCW_ERR_INVALID_ARG
    check_bwd(H, ids, dx, V, 2.0)
    assert H.hcw_sync_status() == H.HCW_ERR_INVALID_ARG
    assert H.hcw_sync_status() == H.HCW_OK


def test_nothing_to_do(H):
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    table = torch.ones(5, 8, device="cuda")
    assert H.hcw_embed_fwd(ids, table).shape == (0, 8)
    dE = torch.full((5, 8), 3.0, device="cuda")
    H.hcw_embed_bwd(ids, table[:0], 5, dE=dE, accumulate=True)
    assert bool((dE == 3.0).all())
    H.hcw_embed_bwd(ids, table[:0], 5, dE=dE)
    assert bool((dE == 0.0).all())


def test_padding_and_nan_keep_to_their_rows(H):
    ids = torch.tensor([1, -1, 2, 1, -5], dtype=torch.int32, device="cuda")
    dx = torch.ones(5, 16, device="cuda")
    dx[1] = float("nan")       # padding's gradient is not looked at
    dx[2, 3] = float("inf")
    dE = H.hcw_embed_bwd(ids, dx, 4)
    assert dE[1].tolist() == [2.0] * 16 and bool(torch.isinf(dE[2, 3]))
    assert bool((dE[0] == 0).all()) and bool((dE[3] == 0).all()) and bool(torch.isfinite(dE[1]).all())
    table = torch.ones(4, 16, device="cuda")
    table[0] = float("nan")
    x = H.hcw_embed_fwd(ids, table)
    assert bool((x[1] == 0).all()) and bool((x[4] == 0).all()) and bool((x[0] == 1).all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_the_same_bits_another_stream_and_a_graph(H, dtype):
    rng = np.random.default_rng(9)
    T, V, d = 5000, 700, 264
    ids = symbols(rng, V, T)
    dx = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32)).to(dtype)
    one = check_bwd(H, ids, dx, V, 1.5).clone()
    st = torch.cuda.Stream()
    assert torch.equal(one, check_bwd(H, ids, dx, V, 1.5, stream=st))
    dev_ids, dev_dx = torch.from_numpy(ids).cuda(), dx.cuda()
    dE, ws = torch.empty(V, d, device="cuda"), torch.empty(
        H.hcw_embed_bwd_workspace_bytes(T, V, d), dtype=torch.uint8, device="cuda")
    with torch.cuda.stream(st):
        H.hcw_embed_bwd(dev_ids, dev_dx, V, 1.5, dE=dE, workspace=ws)   # also loads the code
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        H.hcw_embed_bwd(dev_ids, dev_dx, V, 1.5, dE=dE, workspace=ws)
    for _ in range(3):
        dE.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(one, dE)
    # other symbols in the same buffers
    other = symbols(np.random.default_rng(10), V, T)
    dev_ids.copy_(torch.from_numpy(other))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(dE, check_bwd(H, other, dx, V, 1.5))


def test_many_tokens_on_two_streams_and_in_a_graph(H):
    rng = np.random.default_rng(12)
    T, V, d = 40000, 900, 24
    ids = [torch.from_numpy(symbols(rng, V, T)).cuda() for _ in range(2)]
    dx = [torch.randn(T, d, device="cuda") for _ in range(2)]
    want = [H.hcw_embed_bwd(i, x, V) for i, x in zip(ids, dx)]
    got = [torch.full((V, d), float("nan"), device="cuda") for _ in range(2)]
    ws = [torch.empty(H.hcw_embed_bwd_workspace_bytes(T, V, d), dtype=torch.uint8, device="cuda")
          for _ in range(2)]
    st = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for k in range(2):
            H.hcw_embed_bwd(ids[k], dx[k], V, dE=got[k], workspace=ws[k], stream=st[k])
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st[0]):
        H.hcw_embed_bwd(ids[0], dx[0], V, dE=got[0], workspace=ws[0])
    ids[0].copy_(ids[1])
    dx[0].copy_(dx[1])
    for _ in range(3):
        got[0].fill_(float("nan"))
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[1])


def test_shapes_of_batches(H):
    ids = torch.randint(0, 50, (4, 7), dtype=torch.int32, device="cuda")
    table = torch.randn(50, 24, device="cuda")
    x = H.hcw_embed_fwd(ids, table)
    assert x.shape == (4, 7, 24) and torch.equal(x, table[ids.long()])
    dE = H.hcw_embed_bwd(ids, x, 50)
    assert dE.shape == (50, 24)
    with pytest.raises(ValueError):
        H.hcw_embed_bwd(ids, x[:, :6].contiguous(), 50)
    with pytest.raises(ValueError):
        H.hcw_embed_bwd(ids, x, 50, accumulate=True)
    with pytest.raises(ValueError):
        H.hcw_embed_fwd(ids, table, x=torch.empty(7, 4, 24, device="cuda"))
    with pytest.raises(TypeError):
        H.hcw_embed_fwd(ids.long(), table)
    with pytest.raises(ValueError):
        H.hcw_embed_fwd(ids, table.t())


@pytest.mark.parametrize("at", [1, 2, 3])
def test_ids_that_start_anywhere(H, at):
    rng = np.random.default_rng(at)
    for T in (1, 5, 3000):
        ids = torch.from_numpy(symbols(rng, 500, T + at)).cuda()
        table, dx = torch.randn(500, 40, device="cuda"), torch.randn(T, 40, device="cuda")
        apart = ids[at:].clone()
        assert torch.equal(H.hcw_embed_fwd(ids[at:], table), H.hcw_embed_fwd(apart, table))
        assert torch.equal(H.hcw_embed_bwd(ids[at:], dx, 500), H.hcw_embed_bwd(apart, dx, 500))
