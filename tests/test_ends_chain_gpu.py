"""Edits of logits that the launch right before them wrote, one call after the other without a pause:
the same bits as with a pause after every call."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


@pytest.mark.parametrize("B,V,Hn", [(64, 32003, 700), (40, 131072, 4100), (90, 8191, 60), (3, 501, 20)])
@pytest.mark.parametrize("masked", [False, True])
def test_logits_of_the_launch_before(H, B, V, Hn, masked):
    K, group = 256, 64
    gen = torch.Generator(device="cuda").manual_seed(V)
    packed = H.hcw_q4_pack(*H.hcw_q4_quantize(torch.randn(V, K, generator=gen, device="cuda"), group), group)
    xs = torch.randn(6, B, K, generator=gen, device="cuda").to(torch.bfloat16)
    hist = torch.randint(-1, V, (6, B, Hn), generator=gen, device="cuda", dtype=torch.int32)
    freq, rep = torch.full((B,), 0.25, device="cuda"), torch.full((B,), 1.5, device="cuda")
    bi = torch.randint(-1, V, (B, 9), generator=gen, device="cuda", dtype=torch.int32)
    bv = torch.randn(B, 9, generator=gen, device="cuda")
    mask = torch.randint(-2 ** 31, 2 ** 31, (B, -(-V // 32)), generator=gen,
                         device="cuda").to(torch.int32) if masked else None
    z, h = torch.empty(B, V, device="cuda"), torch.empty(B, Hn, dtype=torch.int32, device="cuda")

    def calls(pause):
        got = []
        for k in range(6):
            h.copy_(hist[k])
            H.hcw_q4_matmul(xs[k], packed, V, group, y=z)
            pause()
            H.hcw_logits_edit(z, history=h, frequency=freq, repetition=rep, bias_idx=bi, bias=bv,
                              mask=mask, out=z)
            pause()
            # the edited logits again, apart
            got += [z.clone(), H.hcw_logits_edit(z, history=h, frequency=freq, bias_idx=bi, bias=bv,
                                                 mask=mask)]
            pause()
        torch.cuda.synchronize()
        return got

    want, got = calls(torch.cuda.synchronize), calls(lambda: None)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
