"""Tensors of more than 2^31 elements at the model's two ends: what lies behind that offset is
computed as what lies before it (tolerances: test_embed_gpu.py, test_clip_gpu.py, test_q4_gpu.py and
test_logits_gpu.py)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


@pytest.fixture(autouse=True)
def memory():
    if torch.cuda.get_device_properties(0).total_memory < 60e9:
        pytest.skip("needs 60 GB")
    yield
    torch.cuda.empty_cache()


def test_a_table_past_2_31(H):
    V, d = (1 << 20) + 7, 2056                     # 2.16e9 elements
    E = torch.zeros(V, d, dtype=BF16, device="cuda")
    ids = torch.tensor([V - 1, 5, V - 1, -1, V - 2, 0, (1 << 31) // d + 1], dtype=torch.int32, device="cuda")
    rows = torch.randn(7, d, device="cuda").to(BF16)
    for i, v in enumerate(ids.tolist()):
        if v >= 0:
            E[v] = rows[i]
    rows[0] = rows[2]
    x = H.hcw_embed_fwd(ids, E)
    rows[3] = 0
    assert torch.equal(x, rows)
    E.fill_(7.0)
    H.hcw_embed_bwd(ids, x, V, dE=E)
    want = x.float()
    assert torch.equal(E[V - 1], (want[0] + want[2]).to(BF16)) and torch.equal(E[V - 2], x[4])
    assert torch.equal(E[5], x[1]) and torch.equal(E[0], x[5]) and torch.equal(E[(1 << 31) // d + 1], x[6])
    assert int(E.view(-1).view(torch.int16).count_nonzero()) == \
        sum(int(E[v].count_nonzero()) for v in set(ids.tolist()) if v >= 0)


def test_tokens_past_2_31(H):
    T, V, d = (1 << 21) + 3, 9, 1024               # 2.15e9 elements
    dx = torch.zeros(T, d, dtype=BF16, device="cuda")
    ids = torch.full((T,), 4, dtype=torch.int32, device="cuda")
    ids[-2:] = 7
    dx[-3:] = torch.randn(3, d, device="cuda").to(BF16)
    dx[0] = 1.0
    dE = H.hcw_embed_bwd(ids, dx, V)
    assert torch.equal(dE[7], dx[-1].float() + dx[-2].float())
    assert torch.equal(dE[4], 1.0 + dx[-3].float())
    x = H.hcw_embed_fwd(ids, dE.to(BF16), x=dx)
    assert torch.equal(x[-1], dE[7].to(BF16)) and torch.equal(x[-3], dE[4].to(BF16))


def test_gradients_past_2_31(H):
    n = (1 << 31) + 4099
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[-4098] = 3.0
    g[-1] = 4.0
    norm = H.hcw_clip_grads([g], 1.0)
    assert abs(float(norm[0]) - 5.0) < 1e-5
    assert abs(float(g[-1]) - 0.8) < 2 ** -8 and abs(float(g[-4098]) - 0.6) < 2 ** -8


def test_logits_past_2_31(H):
    B, V = 8200, 262144                            # 2.15e9 elements
    z = torch.ones(B, V, dtype=BF16, device="cuda")
    hist = torch.full((B, 3), -1, dtype=torch.int32, device="cuda")
    hist[-1] = torch.tensor([V - 1, 3, V - 1], dtype=torch.int32)
    pres, freq = torch.full((B,), 0.5, device="cuda"), torch.full((B,), 0.25, device="cuda")
    for out in (None, z):
        out = H.hcw_logits_edit(z, history=hist, presence=pres, frequency=freq, out=out)
        assert float(out[-1, V - 1]) == 0.0 and float(out[-1, 3]) == 0.25
        assert bool((out[:-1] == 1).all()) and int((out[-1] != 1).sum()) == 2


def test_weights_past_2_31(H):
    N, K = (1 << 19) + 8, 8192                     # 4.3e9 weights
    codes = torch.zeros(N, K, dtype=torch.int8, device="cuda")
    codes[-1] = 7
    codes[-1, ::2] = -8
    codes[(1 << 31) // K] = 1
    scales = torch.ones(N, K // 128, dtype=BF16, device="cuda")
    packed = H.hcw_q4_pack(codes, scales, 128)
    del codes
    x = torch.randn(3, K, device="cuda").to(BF16)
    y = H.hcw_q4_matmul(x, packed, N, 128, y_dtype=F32)
    x64 = x.double()
    want = 7 * x64[:, 1::2].sum(1) - 8 * x64[:, ::2].sum(1)
    mag = 8 * x64.abs().sum(1)
    assert bool(((y[:, -1].double() - want).abs() <= 200 * U * mag).all())
    assert bool(((y[:, (1 << 31) // K].double() - x64.sum(1)).abs() <= 200 * U * mag).all())
    assert int((y != 0).sum()) == 6
