"""The lookup's gradient of many tokens, bit by bit: gradients that are whole numbers up to 8, so that
every sum in fp32 is exact while it stays below 2^24 (8 x 400000 < 2^22) and equals the sum in whole
numbers whatever the order.  A row that is lost or added twice shows wherever it lies.  A bf16 output
is that sum rounded once."""
import numpy as np
import pytest
import torch

from test_embed_gpu import BF16, F32, H, symbols  # noqa: F401 (H is the fixture)

pytestmark = pytest.mark.gpu


def whole(seed, *shape, dtype=F32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-8, 9, shape, generator=gen, device="cuda").to(dtype)


def sums(ids, dx, V):
    at = torch.where((ids < 0) | (ids >= V), V, ids).long()
    out = torch.zeros(V + 1, dx.shape[1], dtype=torch.float64, device="cuda")
    return out.index_add_(0, at, dx.double())[:V]


def check(H, ids, dx, V):  # noqa: F811
    """Written and accumulated, fp32 and bf16, with a workspace of exactly its bytes."""
    T, d = dx.shape
    ids = torch.from_numpy(np.ascontiguousarray(ids, dtype=np.int32)).cuda()
    want = sums(ids, dx, V)
    need = H.hcw_embed_bwd_workspace_bytes(T, V, d)
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    for out in (F32, BF16):
        ws[:need] = 0xFF                              # NaN, and symbols that are none
        buf = torch.full((V * d + 64,), float("nan"), dtype=out, device="cuda")
        dE = buf[:V * d].view(V, d)
        H.hcw_embed_bwd(ids, dx, V, 0.5, dE=dE, workspace=ws[:need])
        assert torch.equal(dE, (0.5 * want).float().to(out))
        assert bool(buf[V * d:].isnan().all()) and bool((ws[need:] == 0xFF).all())
    base = whole(V, V, d)
    dE = base.clone()
    H.hcw_embed_bwd(ids, dx, V, -2.0, dE=dE, accumulate=True, workspace=ws[:need])
    assert torch.equal(dE.double(), base.double() - 2.0 * want)
    assert bool((ws[need:] == 0xFF).all())
    assert H.hcw_sync_status() == H.HCW_OK


@pytest.mark.parametrize("T", [16384, 16385, 40001, 100000, 160001])
@pytest.mark.parametrize("V,d,dtype", [(1, 8, F32), (3, 24, F32), (201, 600, BF16), (500, 777, BF16),
                                       (5003, 133, F32), (40000, 40, BF16), (99000, 8, F32),
                                       (120000, 4, F32), (200003, 72, BF16), (262144, 9, F32),
                                       (1 << 20, 16, BF16)])
def test_many_tokens(H, T, V, d, dtype):  # noqa: F811
    rng = np.random.default_rng(T + V)
    ids = symbols(rng, V, T)
    ids[::11] = ids[0]
    ids[T - 100:] = V - 1
    check(H, ids, whole(T, T, d, dtype=dtype), V)


@pytest.mark.parametrize("T", [63, 64, 65, 4097, 20000, 77825, 160001])
@pytest.mark.parametrize("V,d,dtype", [(500, 72, BF16), (500, 261, F32), (40000, 40, BF16), (200003, 8, F32)])
def test_long_runs(H, T, V, d, dtype):  # noqa: F811
    """One symbol for every token, two, one beside many, and runs that end where a chunk does or not."""
    dx, at = whole(T, T, d, dtype=dtype), np.arange(T)
    for ids in (np.full(T, 3), np.full(T, V - 1), at % 2 * 499, np.where(at % 3, 7, at % V),
                at // 64 % V, at // 256 % V, at // 300 % V, (T - 1 - at) // 2000 % V, np.full(T, -1)):
        check(H, ids, dx, V)


@pytest.mark.parametrize("d,dtype", [(2048, BF16), (2048, F32), (8200, BF16), (1000, F32)])
def test_workspaces_where_the_chunks_grow(H, d, dtype):  # noqa: F811
    """Batches around the sizes from which a chunk has twice the tokens."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count // 2 * 2
    elems = 8 if dtype == BF16 else 4
    tiles = -(-d // (32 * elems))
    for log2 in (6, 7):
        first = -(-(8 * sms << log2) // tiles)
        for T in (first - 1, first, first + 1):
            ids = symbols(np.random.default_rng(T), 300, T)
            check(H, ids, whole(T, T, d, dtype=dtype), 300)
