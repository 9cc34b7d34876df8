"""The fp64 oracle of the student block's operators: its gradients against
central differences of its own forward, and closed forms."""
import numpy as np
import pytest

from oracle import student as S

STEP = 1e-5
# central differences in fp64: truncation ~ STEP^2 f''' ~ 1e-10, rounding ~ 1e-16 |f| / STEP
# ~ 1e-11 |f| with sums |f| below 1e3 here
TOL = 1e-6


def differences(fn, v):
    g = np.zeros_like(v)
    for i in np.ndindex(v.shape):
        keep = v[i]
        v[i] = keep + STEP
        hi = fn()
        v[i] = keep - STEP
        lo = fn()
        v[i] = keep
        g[i] = (hi - lo) / (2 * STEP)
    return g


@pytest.mark.parametrize("kind", [S.SILU, S.GELU, S.RELU])
def test_ffn_gradients_are_the_differences(kind):
    rng = np.random.default_rng(1)
    x, W1, W2 = rng.normal(size=(5, 4)), rng.normal(size=(12, 4)), rng.normal(size=(4, 6))
    dy = rng.normal(size=(5, 4))
    f = lambda: float((S.ffn_fwd(x, W1, W2, kind) * dy).sum())  # noqa: E731
    for got, v in zip(S.ffn_bwd(x, dy, W1, W2, kind), (x, W1, W2)):
        assert np.abs(got - differences(f, v)).max() < TOL


@pytest.mark.parametrize("post", [S.NONE, S.RMS, S.LAYER])
@pytest.mark.parametrize("pre", [S.RMS, S.LAYER])
@pytest.mark.parametrize("rows", [0, 2])
def test_norm_gradients_are_the_differences(post, pre, rows):
    rng = np.random.default_rng(2)
    T, d = 5, 6
    r, f = rng.normal(size=(T, d)), rng.normal(size=(T, d))
    gate = rng.normal(size=(3 if rows else 1, d))
    pw, pb, qw, qb = (rng.normal(size=d) for _ in range(4))
    a, b = rng.normal(size=(T, d)), rng.normal(size=(T, d))

    def fwd():
        s, x = S.norm_fwd(r, f, gate, rows, 0.7, post, pw, pb, pre, qw, qb, 1e-3)
        return float((s * a).sum() + (x * b).sum())

    s, _ = S.norm_fwd(r, f, gate, rows, 0.7, post, pw, pb, pre, qw, qb, 1e-3)
    got = S.norm_bwd(a, b, s, f, gate, rows, 0.7, post, pw, pb, pre, qw, 1e-3)
    want = {"dr": r, "df": f, "dgate": gate, "dpre_w": qw}
    if post != S.NONE:
        want["dpost_w"] = pw
    if post == S.LAYER:
        want["dpost_b"] = pb
    if pre == S.LAYER:
        want["dpre_b"] = qb
    for k, v in want.items():
        assert np.abs(got[k] - differences(fwd, v)).max() < TOL, k


@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distillation_gradient_is_the_differences(tau):
    rng = np.random.default_rng(3)
    T, V, K = 6, 9, 4
    z = rng.normal(size=(T, V))
    idx = np.stack([rng.permutation(V)[:K] for _ in range(T)])
    idx[1, 2:] = -1             # empty slots
    idx[2] = -1                 # no slot
    idx[3, 1] = idx[3, 0]       # a symbol twice
    teacher = rng.normal(size=(T, K)) * 3
    teacher[4, 1] = -np.inf
    target = np.array([1, 2, 3, int(idx[3, 0]), -1, 0])
    weight = np.array([1.0, 0.5, 2.0, 1.0, 1.0, 0.0])
    args = (idx, teacher, target, weight, tau, 0.7, 0.3)
    _, dz = S.distill(z, *args)
    assert np.abs(dz - differences(lambda: float(S.distill(z, *args)[0].sum()), z)).max() < TOL


def test_distillation_of_the_teachers_own_distribution_is_zero():
    rng = np.random.default_rng(4)
    z = rng.normal(size=(3, 8))
    idx = np.tile(np.arange(8), (3, 1))
    loss, dz = S.distill(z, idx, z + 2.0, None, None, 1.7, 1.0, 0.0)
    assert np.abs(loss).max() < 1e-14 and np.abs(dz).max() < 1e-14


def test_norm_of_a_constant_row():
    v = np.full((1, 4), 3.0)
    assert np.abs(S.hat(S.LAYER, v, 1e-5)[0]).max() == 0.0
    assert np.abs(S.hat(S.RMS, v, 0.0)[0] - 1.0).max() < 1e-15
