"""The 64-bit reference of the operators around the scan: hand-written values, and its gradients against central
differences."""
import numpy as np
import pytest

import sequence_reference as ref


def _differences(f, v, dirs, h=1e-6):
    """Directional derivatives of the scalar f at v by central differences."""
    return np.array([(f(v + h * d) - f(v - h * d)) / (2 * h) for d in dirs])


def test_gated_by_hand():
    # one channel, rate softplus(decay) = log 4 at decay = log(4 - 1), rate 1; open and half open gates
    decay, big = np.array([np.log(3.0)]), 60.0
    x = np.array([[[1.0, 2.0]]])
    y, h, _ = ref.gated_fwd(x, np.array([[[big, 0.0]]]), np.array([[[big, 0.0]]]), decay, rate=1.0)
    a0, a1 = 0.25, 0.5
    h0 = np.sqrt(1 - a0 ** 2) * 1.0
    h1 = a1 * h0 + np.sqrt(1 - a1 ** 2) * 0.5 * 2.0
    assert np.allclose(y, [[[h0, h1]]]) and np.allclose(h, h1)
    y, h, _ = ref.gated_fwd(x, np.array([[[big, 0.0]]]), np.array([[[big, 0.0]]]), decay, rate=1.0,
                            starts=np.array([[0, 1]]), h0=np.array([[5.0]]))
    assert np.allclose(y, [[[a0 * 5 + h0, np.sqrt(1 - a1 ** 2)]]])


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_gated_gradients_by_differences(reverse, packed):
    rng = np.random.default_rng(3)
    B, D, L = 2, 3, 7
    v = dict(x=rng.standard_normal((B, D, L)), ga=rng.standard_normal((B, D, L)), gx=rng.standard_normal((B, D, L)),
             decay=rng.standard_normal(D) - 2, h0=rng.standard_normal((B, D)))
    starts = (rng.random((B, L)) < 0.3).astype(np.uint8) if packed else None
    w, wT = rng.standard_normal((B, D, L)), rng.standard_normal((B, D))

    def loss(**k):
        y, h, _ = ref.gated_fwd(**{**v, **k}, starts=starts, reverse=reverse)
        return (y * w).sum() + (h * wT).sum()

    g = ref.gated_bwd(v["x"], v["ga"], v["gx"], v["decay"], w, starts=starts, reverse=reverse, h0=v["h0"], dhT=wT)
    for name, key in (("x", "dx"), ("ga", "dgate_a"), ("gx", "dgate_x"), ("decay", "ddecay"), ("h0", "dh0")):
        dirs = rng.standard_normal((5,) + v[name].shape)
        want = _differences(lambda t: loss(**{name: t}), v[name], dirs)
        got = np.array([(g[key] * d).sum() for d in dirs])
        assert np.allclose(got, want, rtol=1e-6, atol=1e-7), name


@pytest.mark.parametrize("residual", [False, True])
def test_norm_gradients_by_differences(residual):
    rng = np.random.default_rng(4)
    x, r = rng.standard_normal((4, 9)), rng.standard_normal((4, 9)) if residual else None
    weight, bias, w, ws = rng.standard_normal(9), rng.standard_normal(9), rng.standard_normal((4, 9)), rng.standard_normal((4, 9))

    def loss(x=x, weight=weight, bias=bias):
        y, s, _, _ = ref.norm_fwd(x, weight, bias, r)
        return (y * w).sum() + ((s * ws).sum() if residual else 0)

    g = ref.norm_bwd(x if r is None else x + r, weight, w, ws if residual else None)
    for name, val, key in (("x", x, "ds"), ("weight", weight, "dweight"), ("bias", bias, "dbias")):
        dirs = rng.standard_normal((5,) + val.shape)
        want = _differences(lambda t: loss(**{name: t}), val, dirs)
        assert np.allclose([(g[key] * d).sum() for d in dirs], want, rtol=1e-6, atol=1e-7), name


def test_embedding_by_hand():
    weight = np.arange(6.0).reshape(3, 2)
    ids = np.array([[2, -1], [0, 3], [2, 2]])
    out = ref.embed_fwd(ids, weight, 2.0)
    assert np.array_equal(out, [[[8, 10], [0, 0]], [[0, 2], [0, 0]], [[8, 10], [8, 10]]])
    g = ref.embed_bwd(ids, np.ones((3, 2, 2)), 3, 0.5)
    assert np.array_equal(g, [[0.5, 0.5], [0, 0], [1.5, 1.5]])
