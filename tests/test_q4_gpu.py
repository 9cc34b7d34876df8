"""GPU parity of hcw_q4_quantize, hcw_q4_pack and hcw_q4_matmul with the fp64 oracle.

Tolerances, u = 2^-24.  A product of a bf16 number and a code is exact in fp32.  An MMA adds 16 of
them to the sum so far; it may cut instead of rounding, so 4 u of the magnitudes that enter it for
each.  A group takes group / 16 of them, its scaled sum joins the others (one rounding of the
product and the sum each, K / group in all), eight warps' parts and the bias follow.  The output is
rounded once: half a step, bf16 2^-8, fp32 u.
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


def make(T, N, K, group, seed=0):
    rng = np.random.default_rng(seed)
    codes = rng.integers(-8, 8, size=(N, K)).astype(np.int8)
    scales = torch.from_numpy((0.5 + rng.random((N, -(-K // group)))).astype(np.float32) / 8).to(BF16)
    x = torch.from_numpy(rng.normal(size=(T, K)).astype(np.float32)).to(BF16)
    bias = torch.from_numpy(rng.normal(size=N).astype(np.float32))
    return torch.from_numpy(codes), scales, x, bias


def check(H, codes, scales, x, bias, group, dtype, stream=None):
    (T, K), N = x.shape, codes.shape[0]
    need = H.hcw_q4_bytes(N, K, group)
    pbuf = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    packed = H.hcw_q4_pack(codes.cuda(), scales.cuda(), group, packed=pbuf[:need])
    torch.cuda.synchronize()
    assert bool((pbuf[need:] == 0xA5).all())
    buf = torch.full((T * N + 64,), 7.0, dtype=dtype, device="cuda")
    y = H.hcw_q4_matmul(x.cuda(), packed, N, group, bias=None if bias is None else bias.cuda(),
                        y=buf[:T * N].view(T, N), stream=stream)
    torch.cuda.synchronize()
    assert bool((buf[T * N:] == 7.0).all())
    c64, s64, x64 = codes.numpy().astype(np.float64), scales.double().numpy(), x.double().numpy()
    b64 = None if bias is None else bias.double().numpy()
    ref = E.q4_matmul(x64, c64, s64, group, b64)
    mag = E.q4_matmul(np.abs(x64), np.abs(c64), np.abs(s64), group, None if bias is None else np.abs(b64))
    G = -(-K // group)
    bound = (4 * (group // 16) + 2 * G + 8 + 2) * U * mag
    bound = bound + HALF[dtype] * (np.abs(ref) + bound) + 1e-37
    err = np.abs(y.double().cpu().numpy() - ref)
    assert (err <= bound).all(), float((err / bound).max())
    return y


SIZES = [(1, 1, 8), (1, 16, 64), (1, 17, 72), (3, 33, 200), (8, 64, 256), (9, 40, 1000), (16, 100, 2048),
         (1, 2048, 512), (5, 3203, 1000), (16, 48, 8192), (17, 50, 136), (40, 31, 640), (2, 5000, 4096),
         (1, 40000, 64), (9, 30000, 320), (3, 40, 5000), (16, 33, 9000), (10, 6000, 4232), (2, 20, 33800),
         (12, 40, 66000)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T,N,K", SIZES)
def test_every_size(H, T, N, K, group):
    codes, scales, x, bias = make(T, N, K, group, T + N + K)
    check(H, codes, scales, x, None, group, BF16)
    check(H, codes, scales, x, bias, group, F32)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N,K", [(1, 8), (7, 40), (64, 256), (33, 1000)])
def test_quantised_codes_and_scales(H, N, K, group, dtype):
    g = torch.Generator().manual_seed(N + K)
    W = torch.randn(N, K, generator=g).to(dtype)
    if K >= 256:
        W[0, :group] = 0                      # a group of zeros
        W[1, 5] = 1e30                        # one that is nothing but its largest
        W[2, :group] = 1e-40                  # below what a scale holds
    codes, scales = H.hcw_q4_quantize(W.cuda(), group)
    ref, rs = E.quantize(W.float().numpy(), group,
                         lambda s: torch.from_numpy(s).to(BF16).float().numpy())
    assert np.array_equal(scales.double().cpu().numpy(), rs)
    assert np.array_equal(codes.cpu().numpy(), ref)


@pytest.mark.parametrize("N,K", [(200, 1024), (40000, 264), (3000, 4104)])
def test_a_token_does_not_depend_on_the_others(H, N, K):
    codes, scales, x, bias = make(16, N, K, 64)
    packed = H.hcw_q4_pack(codes.cuda(), scales.cuda(), 64)
    x = x.cuda()
    all_ = H.hcw_q4_matmul(x, packed, N, 64, y_dtype=F32)
    for T in (1, 3, 8, 9):
        assert torch.equal(H.hcw_q4_matmul(x[:T].contiguous(), packed, N, 64, y_dtype=F32), all_[:T])
    more = H.hcw_q4_matmul(torch.cat([x, x, x]), packed, N, 64, y_dtype=F32)
    assert torch.equal(more, torch.cat([all_, all_, all_]))


def test_nan_and_infinity_keep_to_their_token(H):
    codes, scales, x, bias = make(9, 70, 264, 32)
    x[2, 5] = float("nan")
    x[8, 7] = float("inf")
    codes[:, 7] = 3
    packed = H.hcw_q4_pack(codes.cuda(), scales.cuda(), 32)
    y = H.hcw_q4_matmul(x.cuda(), packed, 70, 32)
    assert bool(y[2].isnan().all()) and bool((y[8] == float("inf")).all())
    assert bool(y[[0, 1, 3, 4, 5, 6, 7]].isfinite().all())


def test_what_lies_behind_the_last_token_and_feature_is_not_read(H):
    T, N, K = 3, 40, 200
    codes, scales, x, bias = make(T, N, K, 64)
    buf = torch.full((20 * K,), float("nan"), dtype=BF16, device="cuda")
    buf[:T * K] = x.cuda().flatten()
    packed = H.hcw_q4_pack(codes.cuda(), scales.cuda(), 64)
    y = H.hcw_q4_matmul(buf[:T * K].view(T, K), packed, N, 64)
    assert bool(y.isfinite().all())


def test_another_stream_a_graph_and_no_tokens(H):
    codes, scales, x, bias = make(5, 300, 512, 128)
    one = check(H, codes, scales, x, bias, 128, F32).clone()
    st = torch.cuda.Stream()
    assert torch.equal(one, check(H, codes, scales, x, bias, 128, F32, stream=st))
    packed, b = H.hcw_q4_pack(codes.cuda(), scales.cuda(), 128), bias.cuda()
    dx, y = x.cuda(), torch.empty(5, 300, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        H.hcw_q4_matmul(dx, packed, 300, 128, bias=b, y=y)
    y.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, one)
    assert H.hcw_q4_matmul(dx[:0], packed, 300, 128).shape == (0, 300)


def test_shapes_are_checked(H):
    codes, scales, x, bias = make(4, 64, 256, 64)
    packed = H.hcw_q4_pack(codes.cuda(), scales.cuda(), 64)
    x = x.cuda()
    assert H.hcw_q4_matmul(x.view(2, 2, 256), packed, 64, 64).shape == (2, 2, 64)
    for bad in (lambda: H.hcw_q4_matmul(x, packed, 64, 32), lambda: H.hcw_q4_matmul(x, packed, 80, 64),
                lambda: H.hcw_q4_matmul(x[:, :128].contiguous(), packed, 64, 64),
                lambda: H.hcw_q4_matmul(x, packed, 64, 64, bias=torch.zeros(63, device="cuda")),
                lambda: H.hcw_q4_matmul(x, packed, 64, 64, y=torch.empty(64, 4, device="cuda")),
                lambda: H.hcw_q4_pack(codes.cuda(), scales.cuda(), 32),
                lambda: H.hcw_q4_pack(codes.cuda(), scales.cuda(), 64, packed=packed[:-16])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: H.hcw_q4_matmul(x.float(), packed, 64, 64),
                lambda: H.hcw_q4_pack(codes.cuda().float(), scales.cuda(), 64)):
        with pytest.raises(TypeError):
            bad()


@pytest.mark.parametrize("T", [1, 9])
@pytest.mark.parametrize("N,K", [(16, 264), (40, 520), (24, 1096), (3, 1920)])
def test_fewer_pieces_than_warps_at_the_end_of_an_allocation(H, N, K, T):
    """Rows of 3 to 15 pieces, which fewer warps take than share them: what is read ends with the weights."""
    group = 64
    codes, scales, x, bias = make(T, N, K, group, seed=5)
    need = H.hcw_q4_bytes(N, K, group)
    room = torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    packed = H.hcw_q4_pack(codes.cuda(), scales.cuda(), group, packed=room[-need:])
    y = H.hcw_q4_matmul(x.cuda(), packed, N, group, bias=bias.cuda(), y_dtype=F32)
    want = check(H, codes, scales, x, bias, group, F32)
    assert torch.equal(y, want)
