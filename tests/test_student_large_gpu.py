"""Tensors of more than 2^31 elements: the operators' rows past that offset.

Rows stand for themselves in the norms and the distillation: the last rows of a large call
are, bit for bit, those of a call on these rows alone.  The feed-forward block's products may
be cut differently there; they are held to the fp64 form within its tests' bounds, and with dy
zero up to the last rows the weight gradients are those rows' alone.
"""
import pytest
import torch

from oracle import student as S
from test_ffn_gpu import bounds, close, np64

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB on the device")
    return hcw


def rand(*shape, std=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(sum(shape))
    return torch.empty(*shape, dtype=BF16, device="cuda").normal_(0.0, std, generator=gen)


def test_distillation(H):
    T, V, K, last = 16500, 131073, 9, 24      # an odd V: rows start at odd places
    z = rand(T, V)
    idx = torch.randint(V, (T, K), device="cuda", dtype=torch.int32)
    te = torch.randn(T, K, device="cuda")
    y = torch.randint(V, (T,), device="cuda", dtype=torch.int32)
    assert z.numel() > 2 ** 31
    loss, dz = H.hcw_distill_loss(z, idx, te, y, temperature=2.0, kl_scale=0.7, ce_scale=0.3)
    part = [t[-last:].clone() for t in (z, idx, te, y)]
    rl, rz = H.hcw_distill_loss(*part, temperature=2.0, kl_scale=0.7, ce_scale=0.3)
    assert H.hcw_sync_status() == H.HCW_OK
    assert torch.isfinite(rl).all()
    # another number of CTAs may share a row: sums in another order
    assert ((loss[-last:] - rl).abs() <= 1e-5 * rl.abs()).all()
    assert ((dz[-last:].float() - rz.float()).abs() <= 2.0 ** -7 * rz.float().abs() + 1e-7).all()


def test_distillation_of_short_rows(H):
    T, V, last = 1100000, 2001, 40
    z = rand(T, V)
    y = torch.randint(V, (T,), device="cuda", dtype=torch.int32)
    loss, dz = H.hcw_distill_loss(z, target=y, kl_scale=0.0, ce_scale=1.0)
    rl, rz = H.hcw_distill_loss(z[-last:].clone(), target=y[-last:].clone(), kl_scale=0.0, ce_scale=1.0)
    assert H.hcw_sync_status() == H.HCW_OK
    assert torch.equal(loss[-last:], rl) and torch.equal(dz[-last:], rz)


@pytest.mark.parametrize("T,d,kind", [(530000, 4096, 1), (2800000, 777, 2)])
def test_norms(H, T, d, kind):
    last = 40
    r, f = rand(T, d), rand(T, d)
    w = torch.rand(d, device="cuda") + 0.5
    b = torch.rand(d, device="cuda") if kind == H.HCW_NORM_LAYER else None
    par = dict(post=kind, post_w=w, pre=kind, pre_w=w, alpha=0.9)
    s, x = H.hcw_residual_norm_fwd(r, f, post_b=b, pre_b=b, **par)
    cut = lambda t: t[T - last:].clone()  # noqa: E731
    s1, x1 = H.hcw_residual_norm_fwd(cut(r), cut(f), post_b=b, pre_b=b, **par)
    assert torch.equal(s[-last:], s1) and torch.equal(x[-last:], x1)
    g = H.hcw_residual_norm_bwd(r, x, s, f, post_b=b, want_params=False, **par)
    g1 = H.hcw_residual_norm_bwd(cut(r), cut(x), s1, cut(f), post_b=b, want_params=False, **par)
    assert H.hcw_sync_status() == H.HCW_OK
    assert torch.equal(g["dr"][-last:], g1["dr"]) and torch.equal(g["df"][-last:], g1["df"])


def test_feed_forward_block(H):
    T, d, h, last = 54000, 64, 40008, 64
    x, W1, W2 = rand(T, d), rand(2 * h, d, std=d ** -0.5), rand(d, h, std=h ** -0.5)
    dy = torch.zeros(T, d, dtype=BF16, device="cuda")
    dy[-last:] = rand(last, d, std=0.1)
    assert T * h > 2 ** 31
    y = H.hcw_gated_ffn_fwd(x, W1, W2)
    dx, dW1, dW2 = H.hcw_gated_ffn_bwd(x, dy, W1, W2, dw_dtype=torch.float32)
    assert H.hcw_sync_status() == H.HCW_OK
    ref = bounds(*(np64(v) for v in (x[-last:], dy[-last:], W1, W2)), S.SILU)
    close(y[-last:], *ref["y"], "y")
    close(dx[-last:], *ref["dx"], "dx")
    close(dW1, *ref["dW1"], "dW1")
    close(dW2, *ref["dW2"], "dW2")
    assert not dx[:-last].any()
