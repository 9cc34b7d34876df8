"""The fp64 forms of the operators at the model's two ends: gradients against differences, the
clipped norm against its limit, quantised weights against the originals, edits worked out by hand."""
import numpy as np
import pytest

from oracle import ends as E


def test_lookup_gradient_against_differences():
    rng = np.random.default_rng(0)
    T, V, d, scale = 12, 7, 3, 1.7
    ids = rng.integers(-2, V + 2, size=T)
    table, w = rng.normal(size=(V, d)), rng.normal(size=(T, d))
    dE = E.embed_bwd(ids, w, V, scale)
    for v in range(V):
        for j in range(d):
            up, down = table.copy(), table.copy()
            up[v, j] += 1e-5
            down[v, j] -= 1e-5
            num = ((E.embed_fwd(ids, up, scale) - E.embed_fwd(ids, down, scale)) * w).sum() / 2e-5
            assert abs(num - dE[v, j]) < 1e-8
    assert np.array_equal(E.embed_bwd(ids, w, V, scale, dE), 2 * dE) or \
        np.allclose(E.embed_bwd(ids, w, V, scale, dE), 2 * dE, rtol=1e-14)


def test_clipped_gradients_have_the_limit_as_norm():
    rng = np.random.default_rng(1)
    grads = [rng.normal(size=n) for n in (1, 5, 0, 100)]
    n, c, out = E.clip(grads, 2.0)
    assert abs(n - np.linalg.norm(np.concatenate(grads))) < 1e-12 * n
    assert abs(np.linalg.norm(np.concatenate(out)) - 2.0) < 1e-12
    n, c, out = E.clip(grads, 1e3)
    assert c == 1.0 and all(np.array_equal(a, b) for a, b in zip(out, grads))
    assert E.clip([np.array([1.0, np.inf])], 1.0)[:2] == (np.inf, 1.0)
    assert np.isnan(E.clip([np.array([1.0, np.nan])], 1.0)[0])
    assert abs(E.clip([np.array([3e200, 4e200])], 1.0)[0] / 5e200 - 1) < 1e-15
    assert E.clip([], 1.0)[:2] == (0.0, 1.0)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantised_weights_lie_within_half_a_step(group):
    rng = np.random.default_rng(2)
    W = rng.normal(size=(5, 200)).astype(np.float32)
    codes, scales = E.quantize(W, group, lambda s: s)
    back = E.q4_weights(codes, scales, group)
    assert codes.min() >= -8 and codes.max() <= 7
    assert (np.abs(back - W) <= 0.5001 * np.repeat(scales, group, axis=1)[:, :200]).all()
    assert (np.abs(codes).max(axis=1) == 7).all()
    assert not E.quantize(np.zeros((1, 40), np.float32), group, lambda s: s)[0].any()


def test_edits_by_hand():
    z = np.array([[2.0, -1.0, 0.5, 3.0]])
    out, _ = E.edit(z, history=np.array([[0, 1, 1, 2, -1, 9]]), prompt=[1], rep=[2.0], freq=[0.25],
                    pres=[0.5], bias_idx=np.array([[3, 3, -1]]), bias=np.array([[1.0, 0.5, 7.0]]),
                    mask=np.array([[0b1011]], np.int32))
    assert np.array_equal(out, [[1.0, -2.0 - 0.5 - 0.5, -np.inf, 4.5]])
    assert np.array_equal(E.edit(z)[0], z)
