"""Head gradients row by row: gradients of very different sizes beside each other."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2406_02913_amd import szo
from test_gpu_head import HALF, TYPES, U, _np, _off, _room, forward

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _spread(R, V, K, kind, places, seed=0):
    """Gradients from 2^13 down over `places` powers of two, in no order; targets that are unlikely, and logits of a few units, so that every entry of d counts."""
    rng = np.random.default_rng(seed + R + V + places)
    x, w = (torch.from_numpy(a).to(TYPES[kind]).to(DEV) for a in (rng.standard_normal((R, K)) * 0.25, rng.standard_normal((V, K)) * 0.25))
    t = torch.from_numpy(rng.integers(0, V, R).astype(np.int32)).to(DEV)
    g = 2.0 ** (13 - places * rng.permutation(R) / max(R - 1, 1)) * rng.choice([-1, 1], R) * (0.6 + 0.4 * rng.random(R))
    return x, w, t, torch.from_numpy(g).float().to(DEV)


def _gradients(x, w, t, g, want=(True, True), scale=1.0):
    _, stats = forward(x, w, t, scale)
    d = szo.make_head_desc(x, w, t, stats=stats, scale=scale)
    gx, gw = (torch.full_like(a, 7.0) if on else None for a, on in zip((x, w), want))
    szo.szo_head_logprobs_bwd(d, g, gx, gw, _room(szo.szo_head_bwd_workspace_bytes(d)))
    return gx, gw


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("R,V,K,places", [(40, 6000, 64, 24), (7, 40000, 64, 20), (300, 3000, 128, 24), (25, 3000, 64, 0), (40, 6000, 64, 8)])
def test_each_row_has_the_bits_of_its_own_gradient(R, V, K, places, kind):
    x, w, t, g = _spread(R, V, K, kind, places)
    gx, gw = _gradients(x, w, t, g)
    xn, wn, tn, gn = _np(x), _np(w), t.cpu().numpy(), _np(g)
    off, half = _off(xn, wn, 1.0), HALF[kind]
    dn = od.log_probs_grad(xn @ wn.T, tn, gn, np.zeros(R), 1.0)
    p = np.where(np.arange(V)[None, :] == tn[:, None], gn[:, None] - dn, dn)
    # d: its rounding, logit and sum, and in fp16 2^-25 of what the row's largest entry is lifted to, 2^13 or more
    floor = 0 if kind == "bf16" else 2.0 ** -38 * np.abs(gn)[:, None]
    d_err = half * np.abs(dn) + (1 + half) * np.abs(p) * (4 * off + 2.0 ** -17) + floor
    # states beside it in fp16: up to 2^15, times what the row's gradient is smaller by, off by 2^-25: relative to the largest state of the batch at most 2^-39 times that
    least = 0 if kind == "bf16" else 2.0 ** -25
    x_err = 0 if kind == "bf16" else 2 * np.abs(xn).max() * 2.0 ** -39 * 2 * np.abs(gn).max() / np.abs(gn)[:, None] * np.ones_like(xn)
    for got, want, err, size, n in ((gx, dn @ wn, d_err @ np.abs(wn), np.abs(dn) @ np.abs(wn), V),
                                    (gw, dn.T @ xn, d_err.T @ np.abs(xn) + ((1 + half) * np.abs(dn).T @ x_err if kind == "f16" else 0), np.abs(dn).T @ np.abs(xn), R)):
        bad = np.abs(_np(got) - want) - (half * np.abs(want) + least + (1 + half) * (err + (n / 8 + 40) * U * size))
        assert np.all(bad <= 0), (bad.max(), np.argwhere(bad > 0)[:4])
    # and in the mean: rows of x_grad are off by no more than the roundings of d and of the result in the mean of squares, wherever the result is not subnormal
    rows = np.abs(gn) * np.abs(wn).mean() > 2.0 ** -10
    relative = np.linalg.norm(_np(gx) - dn @ wn, axis=1) / np.linalg.norm(dn @ wn, axis=1)
    assert rows.any() and np.all(relative[rows] <= half * 1.2 + 4 * off), (relative.max(), half)


@pytest.mark.parametrize("R", [40, 300])
def test_x_grad_is_the_same_alone(R):
    x, w, t, g = _spread(R, 3000, 128, "f16", 24)
    t[::7] = -1
    both, alone = _gradients(x, w, t, g), _gradients(x, w, t, g, (True, False))
    assert torch.equal(both[0], alone[0])
    assert torch.equal(both[1], _gradients(x, w, t, g, (False, True))[1])


@pytest.mark.parametrize("largest", [2.0 ** 120, 2.0 ** 127, 2.0 ** -20, 2.0 ** -120, 2.0 ** -149, 0.0])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_gradients_of_any_size(kind, largest):
    """Where the result is beyond the type it is infinite or 0, and one row's size does nothing to the others."""
    R, V, K = 20, 700, 64
    x, w, t, g = _spread(R, V, K, kind, 4)
    g /= 2.0 ** 13
    want = _gradients(x, w, t, g, (True, False))[0]
    g[3] = largest
    gx, gw = _gradients(x, w, t, g)
    rest = [i for i in range(R) if i != 3]
    # Another factor of all rows moves roundings: each call's d and result are off by half a step, and in fp16 by 2^-25 where the result is subnormal
    dn = np.abs(od.log_probs_grad(_np(x) @ _np(w).T, t.cpu().numpy(), _np(g), np.zeros(R), 1.0))[rest]
    off = 2 * (HALF[kind] + 4 * _off(_np(x), _np(w), 1.0) + 2.0 ** -17) * 1.01
    assert np.all(np.abs(_np(gx) - _np(want))[rest] <= off * (dn @ np.abs(_np(w)) + np.abs(_np(want))[rest]) + 2.0 ** -24)
    assert torch.isfinite(gx[rest]).all() and not torch.isnan(gw).any()
    if largest == 0:
        assert (gx[3] == 0).all()
    if kind == "bf16" and largest <= 1:
        dn = od.log_probs_grad(_np(x) @ _np(w).T, t.cpu().numpy(), _np(g), np.zeros(R), 1.0)
        assert np.all(np.abs(_np(gx) - dn @ _np(w))[3] <= 2.0 ** -6 * np.linalg.norm((dn @ _np(w))[3]) + 2.0 ** -133)


@pytest.mark.parametrize("g", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_a_gradient_that_is_not_finite_stays_in_its_row(kind, g):
    x, w, t, by = _spread(20, 700, 64, kind, 4)
    by /= 2.0 ** 13
    by[3] = g
    gx, _ = _gradients(x, w, t, by)
    rest = [i for i in range(20) if i != 3]
    assert torch.isfinite(gx[rest]).all() and not torch.isfinite(gx[3]).any()
