"""Rows that are split over workgroups, of every kind of logits: parts without a finite one, NaN and infinities in one part, equal logits in several."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2406_02913_amd import szo
from test_gpu_token_logprobs import DEV, STORE, U, check_forward, logits

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def rows(V, kind, R=14):
    """A row of each kind, and a target in it."""
    x, t = logits(R, V, kind, seed=V)
    low, part = torch.finfo(x.dtype).min, V // 8
    x[0, part:] = -INF                            # one part alone has finite ones
    x[1, :V - part] = -INF
    x[2, :] = -INF
    x[2, [5, 3 * part + 7, V - 1]] = torch.tensor([1.0, 1.0, 2.0], dtype=x.dtype)        # three, fewer than are asked for
    x[3, :] = -INF
    x[4, :] = low
    x[5, 2 * part:] = low
    x[6, 6 * part + 1] = NAN
    x[7, V - 1] = INF
    x[8, 0], x[8, 3 * part], x[8, V - 1] = NAN, INF, -INF
    x[9, :] = 0.5                                 # equal everywhere: the lowest indices
    x[10, :] = (torch.arange(V) % 5).to(x.dtype)  # many equal ones in every part
    x[11, ::part] = 60.0                          # equal largest ones, one in each part
    x[12, :] = NAN
    x[13, :] = torch.linspace(-200, 200, V).to(x.dtype)                                   # the best in the last part
    t[2], t[11], t[1] = 3 * part + 7, 2 * part, V - 1
    return x, t


@pytest.mark.parametrize("kind,V", [("f32", 131072), ("f32", 131075), ("f32", 32768), ("bf16", 131077), ("f16", 131072)])
@pytest.mark.parametrize("top", [1, 20, 32])
def test_rows_in_parts(kind, V, top):
    x, t = rows(V, kind)
    d = szo.make_logprobs_desc(x.to(DEV), top_index=torch.empty(len(x), top, dtype=torch.int32, device=DEV))
    assert szo.szo_logprobs_workspace_bytes(d) > 16                # in parts
    got, _, _ = check_forward(x, t, top, scale=0.8)
    assert np.array_equal(got["top_index"][9], np.arange(top)) and (got["top_index"] >= 0).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_the_same_rows_whole_and_in_parts(kind):
    """600 copies of the rows are too many to be split: statistics agree to their rounding, alternatives are the same."""
    x, t = rows(131072, kind)
    out = []
    for copies in (1, 43):
        dev = x.to(DEV).repeat(copies, 1)
        index = torch.full((len(dev), 9), -1, dtype=torch.int32, device=DEV)
        logp, entropy = torch.empty(len(dev), device=DEV), torch.empty(len(dev), device=DEV)
        d = szo.make_logprobs_desc(dev, torch.as_tensor(np.tile(t, copies), dtype=torch.int32, device=DEV), logp, entropy, top_index=index)
        need = szo.szo_logprobs_workspace_bytes(d)
        assert (need > 16) == (copies == 1)
        szo.szo_token_logprobs(d, torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV))
        out.append([a[-len(x):].cpu().numpy() for a in (index, logp, entropy)])
    assert np.array_equal(out[0][0], out[1][0])
    for a, b in zip(out[0][1:], out[1][1:]):
        assert np.array_equal(np.isfinite(a), np.isfinite(b)) and np.array_equal(np.isnan(a), np.isnan(b))
        fine = np.isfinite(a)
        # sums of 131072 terms in chains of at most V / 256, terms of up to 200 in size for the entropy
        assert np.all(np.abs(a[fine] - b[fine]) <= 2 * (131072 / 256 + 112) * U * (1 + np.abs(a[fine])) + 8 * U * 400)


@pytest.mark.parametrize("kind,V", [("f32", 131075), ("bf16", 131072)])
def test_gradient_from_statistics_of_parts(kind, V):
    x, t = rows(V, kind)
    R = len(x)
    dev = x.to(DEV)
    stats, entropy, logp = torch.empty(R, 2, device=DEV), torch.empty(R, device=DEV), torch.empty(R, device=DEV)
    d = szo.make_logprobs_desc(dev, torch.as_tensor(t, dtype=torch.int32, device=DEV), logp, entropy, stats)
    szo.szo_token_logprobs(d, torch.full((szo.szo_logprobs_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV))
    g = torch.linspace(-1, 1, R, device=DEV)
    grad = torch.empty_like(dev)
    szo.szo_token_logprobs_bwd(d, g, None, grad)
    raw, gn = x.float().numpy(), g.cpu().numpy().astype(np.float64)
    want, lp = od.log_probs_grad(raw, t, gn, np.zeros(R)), od.log_probs(raw)
    nan = np.isnan(lp).any(-1)
    have = grad.float().cpu().numpy()
    assert np.isnan(have[nan]).all() and (have[3] == 0).all()
    rel, floor = STORE[kind]
    p = np.exp(lp[~nan])
    # p to (V / 512 + 160) roundings, as of a whole row
    off = (V / 512 + 160) * U * np.abs(gn[~nan])[:, None] * (p + (want[~nan] != 0))
    assert np.all(np.abs(have[~nan] - want[~nan]) <= rel * np.abs(want[~nan]) + floor + 2 * off)
