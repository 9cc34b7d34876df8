"""hcw_q4_matmul where a CTA's warps go through several rounds of row tiles: heads of more rows than
the SMs hold at once, with random codes and scales, against fp64.

Tolerance: as in test_q4_gpu.py, in terms of the magnitudes that enter: 4 u for each of a group's MMAs, 2 u
a group for its scaled sum, 8 warps' parts and the bias, and half a step of the output."""
import pytest
import torch

from test_q4_gpu import BF16, F32, HALF, U, H  # noqa: F401 (H is the fixture)

pytestmark = pytest.mark.gpu


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count // 2 * 2


def make(T, N, K, group, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(-8, 8, (N, K), generator=gen, device="cuda", dtype=torch.int8)
    scales = ((0.5 + torch.rand(N, -(-K // group), generator=gen, device="cuda")) / 8).to(BF16)
    x = torch.randn(T, K, generator=gen, device="cuda").to(BF16)
    return codes, scales, x, torch.randn(N, generator=gen, device="cuda")


def check(H, T, N, K, group, dtype):  # noqa: F811
    codes, scales, x, bias = make(T, N, K, group, T + N + K + group)
    need = H.hcw_q4_bytes(N, K, group)
    # (what lies behind the weights would be seen in a sum)
    room = torch.full((need + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
    packed = H.hcw_q4_pack(codes, scales, group, packed=room[:need])
    assert bool((room[need:] == 0x7f).all())
    buf = torch.full((T * N + 64,), 7.0, dtype=dtype, device="cuda")
    y = H.hcw_q4_matmul(x, packed, N, group, bias=bias, y=buf[:T * N].view(T, N))
    assert bool((buf[T * N:] == 7.0).all())
    G = -(-K // group)
    x64 = x.double()
    for r in range(0, N, 1 << 15):
        rows = slice(r, min(N, r + (1 << 15)))
        w = codes[rows].double() * scales[rows].double().repeat_interleave(group, dim=1)[:, :K]
        ref = x64 @ w.T + bias[rows].double()
        mag = x64.abs() @ w.abs().T + bias[rows].double().abs()
        bound = (4 * (group // 16) + 2 * G + 8 + 2) * U * mag
        bound = bound + HALF[dtype] * (ref.abs() + bound) + 1e-37
        err = (y[:, rows].double() - ref).abs()
        assert bool((err <= bound).all()), (r, float((err / bound).max()))
    assert H.hcw_sync_status() == H.HCW_OK


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 3, 8, 9, 16])
@pytest.mark.parametrize("K", [136, 1096, 4232])
def test_several_rounds_of_row_tiles(H, T, K, group):  # noqa: F811
    # two rounds of two row tiles for each of 14 warps, then an odd number of tiles, the last one ragged
    check(H, T, 16 * 2 * 14 * sms() + 16 + 5, K, group, F32 if K != 1096 else BF16)


@pytest.mark.parametrize("T", [2, 16])
@pytest.mark.parametrize("tiles", [2, 3, 13, 14, 27, 28, 41, 57, 70])
def test_row_tiles_around_the_rules(H, T, tiles):  # noqa: F811
    """A team a tile, as many as an SM holds, pairs in one round, in one and a bit, in several."""
    for more in (-1, 0, 1):
        check(H, T, 16 * (tiles * sms() + more) - 3, 264, 64, F32)


@pytest.mark.parametrize("T", [17, 33, 40])
def test_more_tokens_than_a_pass_takes(H, T):  # noqa: F811
    check(H, T, 16 * 2 * 14 * sms() + 16 + 5, 264, 64, F32)
    check(H, T, 16 * 15 * sms() + 1, 4232, 128, BF16)


@pytest.mark.parametrize("N,K", [(34048, 1096), (34064, 1096), (70021, 4232)])
def test_a_token_does_not_depend_on_the_others(H, N, K):  # noqa: F811
    codes, scales, x, _ = make(16, N, K, 64, 3)
    packed = H.hcw_q4_pack(codes, scales, 64)
    all_ = H.hcw_q4_matmul(x, packed, N, 64, y_dtype=F32)
    for T in (1, 8, 9):
        assert torch.equal(H.hcw_q4_matmul(x[:T].contiguous(), packed, N, 64, y_dtype=F32), all_[:T])
    assert torch.equal(H.hcw_q4_matmul(torch.cat([x, x[:3]]), packed, N, 64, y_dtype=F32),
                       torch.cat([all_, all_[:3]]))
