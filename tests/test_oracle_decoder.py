"""The 64-bit definitions of what stands between the linear layers, against properties and differences (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import decoder as od


def _angles(rng, tokens, rot):
    a = rng.uniform(-20, 20, (tokens, rot // 2))
    return np.cos(a), np.sin(a)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot,norm", [(16, 16, True), (24, 8, True), (16, 0, True), (16, 8, False)])
def test_gradient_of_norm_and_rotation_against_differences(D, rot, norm, interleaved):
    rng = np.random.default_rng(D + rot)
    x, w, g = rng.standard_normal((3, 2, D)), rng.uniform(0.5, 1.5, D), rng.standard_normal((3, 2, D))
    cos, sin = _angles(rng, 3, rot)

    def f(x, w):
        return (od.qk_norm_rope(x, w, 1e-3, cos, sin, interleaved, norm) * g).sum()

    dx, dw = od.qk_norm_rope_bwd(x, w, 1e-3, cos, sin, g, interleaved, norm)
    step = 1e-5                                   # central differences: error ~ step^2 f''' + 1e-16 f / step
    for i in np.ndindex(*x.shape):
        d = np.zeros_like(x)
        d[i] = step
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * step) - dx[i]) < 1e-7
    if norm:
        for i in range(D):
            d = np.zeros(D)
            d[i] = step
            assert abs((f(x, w + d) - f(x, w - d)) / (2 * step) - dw[i]) < 1e-7


def test_rotation_keeps_lengths_and_relative_angles():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 1, 8))
    base = rng.uniform(0, 1, 4)
    dots = []
    for p in (0, 5):                              # positions (p + 3, p): only their distance counts
        a = np.stack([(p + 3) * base, p * base])
        y = od.rotate(x, np.cos(a), np.sin(a), False)
        assert np.allclose((y * y).sum(-1), (x * x).sum(-1))
        dots.append(y[0, 0] @ y[1, 0])
    assert abs(dots[0] - dots[1]) < 1e-12


def test_codes_are_the_8_bit_floating_type():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(od.e4m3_values(), want, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20001), 2.0 ** np.linspace(-14, 8, 5001), [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10]])
    want = torch.from_numpy(x).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(od.e4m3_encode(x.astype(np.float32)), want)


@pytest.mark.parametrize("D", [64, 96, 256])
def test_places_in_a_block_are_each_taken_once(D):
    for values in (False, True):
        assert np.array_equal(np.sort(od.places(D, values).ravel()), np.arange(32 * D))


def test_tokens_written_one_by_one_stand_where_a_whole_write_puts_them():
    rng = np.random.default_rng(3)
    n, heads, D = 45, 2, 64
    new = rng.standard_normal((n, heads, D)).astype(np.float32) * (1 + np.arange(n))[:, None, None]     # growing: exponents move
    table, got = np.array([[2, 0]]), []
    for values in (False, True):
        for steps in ([n], [1] * n, [20, 20, 5]):
            codes, exps = np.full((3, heads, 1, 32 * D), 9, dtype=np.uint8), np.zeros((3, heads, 1), dtype=np.uint8)
            at = 0
            for m in steps:
                at += m
                od.cache_write(codes, exps, values, table, np.array([at]), np.array([0, m]), new[at - m:at])
            got.append((codes, exps, od.cache_dense(codes, exps, values, table, np.array([n]), 0)[0]))
        whole = got[-3]
        for codes, exps, x in got[-2:]:
            assert np.array_equal(exps, whole[1])
            # moved codes are rounded once more only where they became subnormal: by half of 2^-9 at the last exponent
            step = 2.0 ** (exps[table[0][np.arange(n) // 32], :, 0].astype(int) - 127 - 9)
            assert np.all(np.abs(x - whole[2]) <= step[..., None])
            assert np.all(np.abs(x - new) <= np.maximum(np.abs(new) / 16, step[..., None]))


def test_attention_of_equal_keys_is_a_mean_and_masks_leave_rows_empty():
    q, k, v = np.ones((3, 2, 4)), np.ones((5, 1, 4)), np.arange(20.0).reshape(5, 1, 4)
    there = np.ones(5, dtype=bool)
    out, lse, _ = od.attention(q, k, v, there, 5, 0.5, True, 0)
    assert np.allclose(out[0, 0], v[:3, 0].mean(0)) and np.allclose(out[2, 1], v[:, 0].mean(0)) and np.allclose(lse[2], 2 + np.log(5))
    out, lse, _ = od.attention(np.ones((7, 2, 4)), k, v, there, 5, 0.5, True, 0)          # more queries than tokens
    assert np.all(out[:2] == 0) and np.all(lse[:2] == -np.inf)
    out, _, _ = od.attention(q, k, v, there, 5, 0.5, True, 1)
    assert np.allclose(out[:, 0], v[2:, 0])


def test_gradient_of_log_probabilities_against_differences():
    rng = np.random.default_rng(5)
    x, t = rng.standard_normal((4, 9)) * 2, np.array([0, 8, -1, 3])
    x[3, 5] = -np.inf
    g, h = rng.standard_normal(4), rng.standard_normal(4)

    def f(x):
        lp = od.log_probs(x, 0.7)
        return sum(g[r] * lp[r, t[r]] for r in range(4) if t[r] >= 0) + (h * od.entropy(lp)).sum()

    d = od.log_probs_grad(x, t, g, h, 0.7)
    for i in np.ndindex(*x.shape):
        if np.isinf(x[i]):
            assert d[i] == 0
            continue
        e = np.zeros_like(x)
        e[i] = 1e-5
        assert abs((f(x + e) - f(x - e)) / 2e-5 - d[i]) < 1e-7


def test_alternatives_prefer_lower_indices_and_nan():
    x = np.array([[1.0, 3.0, 3.0, -np.inf, 0.0], [-np.inf, np.nan, 7.0, -np.inf, np.inf]])
    assert od.alternatives(x, 4).tolist() == [[1, 2, 0, 4], [1, 4, 2, 0]]
