"""The 64-bit definition of norms around a block: its gradients against differences, and what it says at its ends."""
import numpy as np
import pytest

from oracle import decoder as od


def _inputs(rng, T, H, post, gate):
    d = dict(y=rng.standard_normal((T, H)), h=rng.standard_normal((T, H)), pre_weight=rng.uniform(0.5, 1.5, H), pre_bias=rng.standard_normal(H))
    if post:
        d.update(post_weight=rng.uniform(0.5, 1.5, H), post_bias=rng.standard_normal(H))
    if gate:
        d["gate"] = rng.standard_normal(H if gate == "row" else (T, H))
    return d


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", [None, "row", "token"])
def test_gradients_against_differences(layer, post, gate):
    rng = np.random.default_rng(3)
    d = _inputs(rng, 3, 7, post, gate)
    gx, gh = rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    rest = dict(eps=1e-3, layer=layer, post=post, y_scale=0.7, h_scale=1.3)

    def f():
        h, x = od.block_norm(**d, **rest)
        return (h * gh).sum() + (x * gx).sum()

    got = od.block_norm_bwd(gx=gx, gh=gh, **d, **rest)
    for name, a in d.items():
        want, step = np.empty_like(a), 1e-5
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + step
            up = f()
            a[i] = keep - step
            want[i] = (up - f()) / (2 * step)
            a[i] = keep
        np.testing.assert_allclose(got[name], want, rtol=1e-6, atol=1e-7)


def test_what_is_absent():
    rng = np.random.default_rng(4)
    d = _inputs(rng, 2, 5, False, None)
    h, x = od.block_norm(None, d["h"], 0.0, h_scale=2.0)
    np.testing.assert_allclose(h, 2 * d["h"])
    np.testing.assert_allclose((x * x).mean(-1), 1.0)                     # RMS norm without weight
    h, x = od.block_norm(d["y"], None, 0.0, layer=True)
    np.testing.assert_allclose(h, d["y"])
    np.testing.assert_allclose([x.mean(-1), x.var(-1)], [[0, 0], [1, 1]], atol=1e-12)
