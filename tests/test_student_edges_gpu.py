"""Calls of the student block's operators at their edges: parts that are not there, values that
are not finite, extreme sizes, other streams than the current one."""
import numpy as np
import pytest
import torch

from oracle import student as S
from test_distill_gpu import check as distill_check, make as distill_problem
from test_ffn_gpu import make as ffn_problem
from test_norm_gpu import Problem, check_fwd

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


@pytest.mark.parametrize("post,pre", [(0, 1), (0, 2), (1, 2), (2, 1), (2, 2), (2, 0)])
def test_without_a_branch_its_gate_and_norm_are_not_read(H, post, pre):
    p = Problem(33, 264, BF16, 7)
    check_fwd(H, p, post, pre, f=False)
    p.gate[0, 5], p.post_w[7], p.post_b[9] = float("nan"), float("inf"), float("nan")
    check_fwd(H, p, post, pre, f=False)


@pytest.mark.parametrize("T,d,rows", [(200000, 64, 0), (40000, 512, 256), (8000, 2048, 0),
                                      (4000, 8192, 100)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", [S.RMS, S.LAYER])
def test_a_norm_that_gives_up_ends_and_says_so(H, T, d, rows, dtype, kind):
    p = Problem(T, d, dtype, d, rows=rows)
    par = dict(gate=p.gate, rows_per_gate=rows, alpha=p.alpha, post=kind, post_w=p.post_w,
               post_b=p.post_b, pre=kind, pre_w=p.pre_w)
    calls = (lambda: H.hcw_residual_norm_fwd(p.r, p.f, pre_b=p.pre_b, **par),
             lambda: tuple(H.hcw_residual_norm_bwd(p.dr_out, p.dx_out, p.s, p.f,
                                                   want_bias=kind == S.LAYER, **par).values()))
    for call in calls:
        whole = call()
        assert H.hcw_sync_status() == H.HCW_OK
        for fetches in (1, 3, 5):
            H.hcw_selftest_norm_starve(fetches)
            try:
                call()
            finally:
                assert H.hcw_selftest_norm_starve(0) == fetches
            assert H.hcw_sync_status() == H.HCW_ERR_TIMEOUT
        again = call()
        assert H.hcw_sync_status() == H.HCW_OK
        assert all(torch.equal(a, b) for a, b in zip(whole, again))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 31, 33, 201, 256, 257, 1000, 1024])
def test_rows_with_a_label_and_no_teacher(H, V, dtype):
    z, idx, teacher, target, weight = distill_problem(700, V, 3, dtype, V)
    distill_check(H, z, None, None, target, weight, 1.0, 1.0, 0.4)
    idx[:] = -1
    distill_check(H, z, idx, teacher, target, weight, 2.0, 0.7, 0.3)


@pytest.mark.parametrize("V,K", [(5000, 32), (5000, 7), (9001, 32)])
def test_slots_that_name_the_same_symbols(H, V, K):
    """Every symbol by two slots or more, in rows of a cluster."""
    z, idx, teacher, target, weight = distill_problem(400, V, K, BF16, V + K)
    idx[:, K // 2:] = idx[:, : K - K // 2]
    idx[::3, 1:] = idx[::3, :1]
    distill_check(H, z, idx, teacher, target, weight, 1.0, 0.7, 0.3)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("V,K", [(100, 12), (1000, 40), (3001, 12), (5000, 50), (3000, 200), (33001, 64)])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.5])
def test_the_teachers_logits_count_by_their_differences(H, V, K, tau, dtype):
    """Logits in quarters, and the same ones 2^20 higher and lower: exact in fp32, and so are
    their differences, from which everything follows.  The same bits."""
    z, idx, teacher, target, weight = distill_problem(9, V, K, dtype, V)
    teacher = np.round(teacher * 4) / 4
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    got = [H.hcw_distill_loss(z.cuda(), dev(idx), dev((teacher + c).astype(np.float32)), dev(target),
                              dev(weight), tau, 0.7, 0.3) for c in (0.0, 2.0 ** 20, -2.0 ** 20)]
    assert bool(torch.isfinite(got[0][0]).all())
    for loss, dz in got[1:]:
        assert torch.equal(loss, got[0][0]) and torch.equal(dz, got[0][1])
    distill_check(H, z, idx, teacher.astype(np.float32), target, weight, tau, 0.7, 0.3)


@pytest.mark.parametrize("act", [S.SILU, S.GELU, S.RELU])
@pytest.mark.parametrize("T", [4, 20, 200])
def test_a_nan_in_a_gate_row_is_not_hidden(H, T, act):
    """NaN in one gate: in every output that this hidden column enters, and in no other."""
    d, h, at = 128, 136, 3
    x, dy, W1, W2 = ffn_problem(T, d, h, T)
    W1[at, 5] = float("nan")
    assert H.hcw_gated_ffn_fwd(x, W1, W2, act).isnan().all()
    dx, dW1, dW2 = H.hcw_gated_ffn_bwd(x, dy, W1, W2, act)
    assert dx.isnan().all() and dW2[:, at].isnan().all()
    assert dW1[at].isnan().all() and dW1[h + at].isnan().all()
    keep = [i for i in range(h) if i != at]
    assert dW2[:, keep].isfinite().all()
    assert dW1[keep].isfinite().all() and dW1[[h + i for i in keep]].isfinite().all()
    # a token's: in its own row alone
    x, dy, W1, W2 = ffn_problem(T, d, h, T)
    x[2, 5] = float("nan")
    y = H.hcw_gated_ffn_fwd(x, W1, W2, act)
    dx = H.hcw_gated_ffn_bwd(x, dy, W1, W2, act, want_dw=False)[0]
    rows = [i for i in range(T) if i != 2]
    for t in (y, dx):
        assert t[2].isnan().all() and t[rows].isfinite().all()


def test_memory_of_a_call_on_another_stream_is_its_own(H):
    """While the side stream is busy the current one goes on: it gets none of the memory of the
    calls that wait there, and gives them none that it still works on."""
    x, dy, W1, W2 = ffn_problem(700, 128, 264, 1)
    p = Problem(700, 128, BF16, 2, rows=64)
    par = dict(gate=p.gate, rows_per_gate=64, post=S.RMS, post_w=p.post_w, pre=S.RMS, pre_w=p.pre_w)
    z = distill_problem(700, 500, 3, BF16, 3)
    zs = [torch.as_tensor(t).cuda() for t in z]

    def calls(stream=None):
        y = H.hcw_gated_ffn_fwd(x, W1, W2, stream=stream)
        dx, dW1, dW2 = H.hcw_gated_ffn_bwd(x, dy, W1, W2, stream=stream)
        r, v = H.hcw_residual_norm_fwd(p.r, p.f, stream=stream, **par)
        g = H.hcw_residual_norm_bwd(p.dr_out, p.dx_out, p.s, p.f, stream=stream, **par)
        loss, dz = H.hcw_distill_loss(*zs, stream=stream)
        return (y, dx, dW1, dW2, r, v, *g.values(), loss, dz)

    want = calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        # blocks of many sizes that the current stream has in use, and then lets go of
        sizes = [1 << k for k in range(9, 23)] + [t.numel() * t.element_size() for t in want]
        torch.cuda._sleep(2_000_000)
        for t in [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]:
            t.fill_(255)
        del t
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = calls(side)
        dropped = calls(side)
        del dropped
        mine = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes
                for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        assert all(bool((t == 255).all()) for t in mine)
        del got, mine


def test_rows_in_another_order_are_refused(H):
    """As many elements are not enough."""
    t = lambda *s, dtype=BF16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    par = dict(rows_per_gate=2, post=S.RMS, pre=S.RMS)
    r, f, gate = t(6, 8), t(6, 8), t(3, 8, dtype=F32)
    H.hcw_residual_norm_fwd(r.view(2, 3, 8), f, gate, **par)
    H.hcw_residual_norm_bwd(r.view(2, 3, 8), f, r, f, gate, **par)
    for bad in (dict(f=t(8, 6)), dict(gate=t(8, 3, dtype=F32)), dict(r_out=t(4, 12))):
        with pytest.raises(ValueError):
            H.hcw_residual_norm_fwd(**{"r": r, "f": f, "gate": gate, **par, **bad})
    for bad in (dict(s=t(8, 6)), dict(gate=t(8, 3, dtype=F32)), dict(df=t(12, 4))):
        with pytest.raises(ValueError):
            H.hcw_residual_norm_bwd(**{"dr_out": r, "dx_out": r, "s": r, "f": f, "gate": gate, **par,
                                       **bad})
    W1, W2 = t(32, 8), t(8, 16)
    for bad in (t(8, 6), t(3, 16)):
        with pytest.raises(ValueError):
            H.hcw_gated_ffn_fwd(r, W1, W2, y=bad)
        with pytest.raises(ValueError):
            H.hcw_gated_ffn_bwd(r, bad, W1, W2)
    z = t(2, 3, 40)
    ok = dict(idx=t(2, 3, 4, dtype=torch.int32), teacher=t(2, 3, 4, dtype=F32),
              target=t(6, dtype=torch.int32), weight=t(2, 3, dtype=F32))
    H.hcw_distill_loss(z, **ok)
    for bad in (dict(target=t(3, 2, dtype=torch.int32)), dict(weight=t(3, 2, dtype=F32)),
                dict(idx=t(3, 2, 4, dtype=torch.int32), teacher=t(3, 2, 4, dtype=F32)),
                dict(dz=t(3, 2, 40)), dict(loss=t(3, 2, dtype=F32))):
        with pytest.raises(ValueError):
            H.hcw_distill_loss(z, **{**ok, **bad})
    assert H.hcw_sync_status() == H.HCW_OK


@pytest.mark.parametrize("rows", [0, 1 << 30])
def test_norms_of_as_many_rows_as_an_int_counts(H, rows):
    T, last = 2 ** 31 - 1, 700
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB on the device")
    new = lambda: torch.empty(T, 1, dtype=BF16, device="cuda").normal_()  # noqa: E731
    cut = lambda t: t[T - last:].clone()  # noqa: E731
    r, f = new(), new()
    gate = torch.rand(-(-T // rows) if rows else 1, 1, device="cuda")
    one = dict(alpha=0.9, post=S.RMS, pre=S.RMS)
    par = dict(gate=gate, rows_per_gate=rows, **one)
    s, x = H.hcw_residual_norm_fwd(r, f, **par)
    s1, x1 = H.hcw_residual_norm_fwd(cut(r), cut(f), gate=gate[-1:].clone(), **one)
    assert torch.equal(cut(s), s1) and torch.equal(cut(x), x1)
    got = H.hcw_residual_norm_bwd(r, x, s, f, **par)
    part = H.hcw_residual_norm_bwd(cut(r), x1, s1, cut(f), gate=gate[-1:].clone(), **one)
    assert torch.equal(cut(got["dr"]), part["dr"]) and torch.equal(cut(got["df"]), part["df"])
    # the sums: dpre_w = sum x shat over blocks of rows in fp64, within 2^16 fp32 roundings (a
    # thread adds up its CTA's rows one after the other, 2^31 / 152 / 64 of them and more)
    want = size = 0.0
    for i in range(0, T, 1 << 27):
        b = slice(i, min(i + (1 << 27), T))
        sd = s[b].double()
        t = x[b].double() * sd * torch.rsqrt(sd * sd + 1e-5)
        want, size = want + float(t.sum()), size + float(t.abs().sum())
        del sd, t
    assert abs(float(got["dpre_w"]) - want) <= 2.0 ** -24 * (2 ** 31 / 152 / 64) * size
    assert H.hcw_sync_status() == H.HCW_OK


def test_a_feed_forward_block_of_as_many_rows_as_an_int_counts(H):
    T, d, h, last = 2 ** 31 - 1, 8, 8, 999
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 215e9:
        pytest.skip("needs 215 GB on the device")
    _, _, W1, W2 = ffn_problem(1, d, h, 5)
    x = torch.empty(T, d, dtype=BF16, device="cuda").normal_()
    end = x[T - last:].clone()
    y = H.hcw_gated_ffn_fwd(x, W1, W2)
    assert torch.equal(y[T - last:], H.hcw_gated_ffn_fwd(end, W1, W2))
    del y
    dx, none, _ = H.hcw_gated_ffn_bwd(x, x, W1, W2, want_dw=False)
    assert none is None
    assert torch.equal(dx[T - last:], H.hcw_gated_ffn_bwd(end, end, W1, W2, want_dw=False)[0])
    assert H.hcw_sync_status() == H.HCW_OK
    del dx, x
    torch.cuda.empty_cache()


def test_the_example_learns_with_the_stacks_usual_activation(monkeypatch):
    """The step's gradients are held to fp64 without a ReLU (whose decisions near 0 differ); with it
    the same calls have to bring the loss down clearly."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "student.py")
    spec = importlib.util.spec_from_file_location("student_relu", path)
    student = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(student)
    monkeypatch.setattr(student, "FLAGS", student.H.HCW_CAUSAL | student.H.HCW_ACT_RELU)
    losses = student.train(steps=60, say=None)
    assert all(v == v for v in losses) and sum(losses[-5:]) / 5 < 0.8 * losses[0]


@pytest.mark.parametrize("post", [S.NONE, S.RMS, S.LAYER])
def test_an_infinite_gate_gives_infinities(H, post):
    """gate v alone: no bias that is not there times the gate."""
    p = Problem(9, 264, F32, 3)
    p.gate[0, 5] = float("inf")
    s, _ = H.hcw_residual_norm_fwd(p.r, p.f, p.gate, alpha=0.5, post=post, post_w=p.post_w,
                                   pre=S.LAYER)
    assert s[:, 5].isinf().all() and not s.isnan().any()
