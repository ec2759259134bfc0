"""Log probabilities of given tokens, entropy, alternatives and their gradient against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2406_02913_amd import szo

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
STORE = {"f32": (2.0 ** -24, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}
U = 2.0 ** -24


def forward(x, targets, top, scale=1.0, pad=0, loss=False):
    """x: tensor on the CPU, of its type -> outputs as numpy, the descriptor"""
    R, V = x.shape
    dev = torch.full((R, V + pad), float("nan"), dtype=x.dtype, device=DEV)[:, pad // 2:pad // 2 + V]
    dev.copy_(x)
    out = dict(logp=torch.full((R,), 7.0, device=DEV), entropy=torch.full((R,), 7.0, device=DEV), stats=torch.full((R, 2), 7.0, device=DEV))
    if top:
        out.update(top_logp=torch.full((R, top), 7.0, device=DEV), top_index=torch.full((R, top), -7, dtype=torch.int32, device=DEV))
    acc = torch.full((1,), 0.5, dtype=torch.float64, device=DEV) if loss else None
    d = szo.make_logprobs_desc(dev, torch.as_tensor(targets, dtype=torch.int32, device=DEV), scale=scale, loss_acc=acc, loss_scale=0.25, **out)
    room = torch.full((szo.szo_logprobs_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV)
    szo.szo_token_logprobs(d, room)
    got = {n: t.cpu().numpy() for n, t in out.items()}
    if loss:
        got["loss"] = acc.item()
    return got, d, out


def check_forward(x, targets, top, scale=1.0, pad=0):
    got, d, out = forward(x, targets, top, scale, pad, loss=True)
    raw = x.float().numpy()
    lp = od.log_probs(raw, scale)
    R, V = raw.shape
    ok = np.isfinite(lp).any(-1)
    # u = scale (x - max): two roundings; each exponential 2 more and |u| U; the sum over V in chains of V / 512 and 9 levels; a logarithm
    with np.errstate(invalid="ignore"):
        spread = scale * np.nan_to_num(np.abs(raw - raw.max(-1, keepdims=True)), posinf=0)
    common = (V / 512 + 32 + 4 * 20) * U
    target_ok = [0 <= t < V for t in targets]
    for r in range(R):
        want = lp[r, targets[r]] if target_ok[r] else 0.0
        have = got["logp"][r]
        if np.isfinite(want):
            assert abs(have - want) <= common + 4 * U * (spread[r, targets[r]] + abs(want)) if target_ok[r] else have == 0
        else:
            assert np.array_equal(have, np.float32(want), equal_nan=True)
    h = od.entropy(lp)
    nothing = np.isneginf(lp).all(-1)
    assert np.array_equal(np.isnan(h[~nothing]), np.isnan(got["entropy"][~nothing])) and (got["entropy"][nothing] == 0).all()
    fine = ok & np.isfinite(h)
    # entropy = log S - sum u p: terms of |u| p, whose sum is at most the entropy plus log S
    assert np.all(np.abs(got["entropy"][fine] - h[fine]) <= 2 * common * (1 + h[fine] + np.log(V)))
    if top:
        index = od.alternatives(raw, top)
        assert np.array_equal(got["top_index"], index)
        want = np.take_along_axis(lp, index, 1)
        have = got["top_logp"]
        a, b = np.isfinite(want), np.isfinite(have)
        assert np.array_equal(a, b) and np.array_equal(np.isnan(want), np.isnan(have))
        assert np.all(np.abs(have[a] - want[a]) <= common + 4 * U * (np.take_along_axis(spread, index, 1)[a] + np.abs(want[a])))
    kept = [r for r in range(R) if target_ok[r]]
    want = 0.5 - 0.25 * got["logp"][kept].astype(np.float64).sum()
    assert np.array_equal(got["loss"], want, equal_nan=True) or abs(got["loss"] - want) <= 1e-12 * (1 + np.abs(got["logp"][kept].astype(np.float64)).sum())
    return got, d, out


def logits(R, V, kind, seed=0, peak=6.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, V)) * 2
    t = rng.integers(0, V, R)
    x[np.arange(R), t] += peak * rng.random(R)
    return torch.from_numpy(x).to(TYPES[kind]), t


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,V,top,pad", [(1, 1, 1, 0), (2, 2, 2, 1), (3, 7, 5, 3), (5, 33, 32, 0), (4, 100, 1, 5), (9, 1000, 20, 8), (3, 2047, 3, 1), (2, 2049, 32, 0),
                                         (1, 32000, 5, 0), (17, 50257, 20, 0), (3, 131072, 8, 7), (300, 513, 0, 0)])
def test_forward(R, V, top, pad, kind):
    x, t = logits(R, V, kind, seed=V)
    check_forward(x, t, top, scale=1.0 if V % 2 else 0.8, pad=pad)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_equal_logits_take_the_lower_index(kind):
    x = torch.zeros(4, 5000, dtype=TYPES[kind])
    x[1] = torch.arange(5000) % 7
    x[2, 2500:] = 1
    x[3, :] = -0.0
    x[3, 4000] = 0.0
    check_forward(x, [0, 4999, 3, 9], 32)


def test_masked_rows():
    """Masks by -inf and by the type's lowest value; rows that keep one token, a few, or none; targets that are masked."""
    x, _ = logits(8, 4096, "f32", 3)
    inf = float("inf")
    x[0, :] = -inf
    x[1, 1:] = -inf
    x[2, :4095] = -inf
    x[3, 3:] = -inf
    x[4, 2000:] = torch.finfo(torch.float32).min
    x[5, :] = torch.finfo(torch.float32).min
    x[6, ::2] = -inf
    check_forward(x, [5, 0, 17, 2, 4000, 7, 2, 1], 20)
    y = x.to(torch.bfloat16)
    y[4, 2000:] = torch.finfo(torch.bfloat16).min
    y[5, :] = torch.finfo(torch.bfloat16).min
    check_forward(y, [5, 0, 17, 2, 4000, 7, 2, 1], 20)


def test_nan_and_infinite_logits_stay_in_their_row():
    x, t = logits(5, 3001, "f32", 4)
    x[1, 77] = float("nan")
    x[2, 3000] = float("inf")
    x[3, 5], x[3, 2999] = float("nan"), float("-inf")
    got, _, _ = check_forward(x, t, 6)
    assert np.isnan(got["logp"][1:4]).all() and np.isfinite(got["logp"][[0, 4]]).all() and got["top_index"][1, 0] == 77


def test_sorted_rows_and_far_apart_logits():
    """Descending rows put the largest logits side by side; logits of thousands; one token with all the weight."""
    x = torch.stack([torch.arange(9000, 0, -1).float(), torch.arange(9000).float(), torch.linspace(-6e4, 6e4, 9000), torch.zeros(9000)])
    x[3, 8999] = 1000
    check_forward(x, [0, 8999, 8999, 1], 32)


def test_ignored_targets_and_missing_outputs():
    x, _ = logits(6, 300, "bf16", 6)
    got, d, _ = check_forward(x, [-1, -100, 300, 299, 0, 2 ** 31 - 1], 3)
    assert (got["logp"][[0, 1, 2, 5]] == 0).all()
    logp = torch.empty(6, device=DEV)
    d = szo.make_logprobs_desc(x.to(DEV), torch.tensor([1, 2, 3, 4, 5, 6], dtype=torch.int32, device=DEV), logp)
    szo.szo_token_logprobs(d, torch.empty(szo.szo_logprobs_workspace_bytes(d), dtype=torch.uint8, device=DEV))
    want = od.log_probs(x.float().numpy())[np.arange(6), np.arange(1, 7)]
    assert np.abs(logp.cpu().numpy() - want).max() < 1e-5
    index = torch.empty(6, 2, dtype=torch.int32, device=DEV)
    d = szo.make_logprobs_desc(x.to(DEV), top_index=index)
    szo.szo_token_logprobs(d, torch.empty(szo.szo_logprobs_workspace_bytes(d), dtype=torch.uint8, device=DEV))
    assert np.array_equal(index.cpu().numpy(), od.alternatives(x.float().numpy(), 2))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("R,V,pad", [(1, 1, 0), (3, 5, 2), (7, 1003, 1), (4, 9000, 0), (2, 50257, 0)])
def test_gradient(R, V, pad, kind):
    x, t = logits(R, V, kind, seed=V + 1)
    if R > 2:
        t[1] = -100
        x[2, 1:] = -float("inf")
    if R > 3:
        x[3, :] = -float("inf")
    _, d, out = forward(x, t, 0, 0.9, pad)
    rng = np.random.default_rng(2)
    g, h = (rng.standard_normal(R).astype(np.float32) for _ in range(2))
    for use_g, use_h in ((True, True), (True, False), (False, True)):
        grad = torch.full((R, V + 3), 7.0, dtype=x.dtype, device=DEV)[:, 1:V + 1]
        szo.szo_token_logprobs_bwd(d, torch.from_numpy(g).to(DEV) if use_g else None, torch.from_numpy(h).to(DEV) if use_h else None, grad)
        want = od.log_probs_grad(x.float().numpy(), t, g if use_g else 0 * g, h if use_h else 0 * h, 0.9)
        rel, floor = STORE[kind]
        # p to (V / 512 + 110) U relative as in the forward; log p + H to as much of 1 + its size
        lp = od.log_probs(x.float().numpy(), 0.9)
        with np.errstate(invalid="ignore"):
            p = np.nan_to_num(np.exp(lp))
            size = np.abs(np.nan_to_num(lp, neginf=0)) + od.entropy(lp)[:, None] + np.log(V + 1)
        off = (V / 512 + 160) * U * (np.abs(g)[:, None] * (p + (want != 0)) + np.abs(h)[:, None] * p * (1 + np.nan_to_num(size)))
        assert np.all(np.abs(grad.float().cpu().numpy() - want) <= rel * np.abs(want) + floor + 2 * off)


def test_gradient_in_place_of_the_logits():
    x, t = logits(5, 777, "f32", 9)
    _, d, out = forward(x, t, 0)
    g = torch.ones(5, device=DEV)
    a = torch.empty(5, 777, device=DEV)
    szo.szo_token_logprobs_bwd(d, g, None, a)
    szo.szo_token_logprobs_bwd(d, g, None, d.keep[0])
    assert torch.equal(a, d.keep[0])


def test_rows_behind_32_bits_and_equal_runs():
    R, V = 9000, 131072                          # 4.7 GB of fp32
    x = torch.randn(R, V, device=DEV)
    t = torch.randint(V, (R,), dtype=torch.int32, device=DEV)
    logp, top = torch.empty(R, device=DEV), torch.empty(R, 2, dtype=torch.int32, device=DEV)
    d = szo.make_logprobs_desc(x, t, logp, top_index=top)
    room = torch.empty(szo.szo_logprobs_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    szo.szo_token_logprobs(d, room)
    first = logp.clone(), top.clone()
    szo.szo_token_logprobs(d, room)
    assert torch.equal(first[0], logp) and torch.equal(first[1], top)
    for r in (0, 8191, 8192, 8999):
        row = x[r].double()
        want = (row[t[r]] - torch.logsumexp(row, 0)).item()
        assert abs(logp[r].item() - want) < 1e-5 and torch.equal(top[r].long(), torch.topk(row, 2).indices)
