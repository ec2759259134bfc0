"""Log probabilities straight from final states and a head, and their gradients, against the 64-bit definition on the same 16-bit values."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2406_02913_amd import szo

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
U = 2.0 ** -24

# rows, vocabulary, width, type, layout
CASES = [(1, 1, 64, "bf16", "plain"), (1, 257, 64, "f16", "plain"), (3, 1000, 128, "bf16", "strided"), (17, 300, 192, "f16", "plain"), (16, 2048, 512, "bf16", "plain"),
         (33, 5000, 64, "bf16", "strided"), (64, 513, 64, "bf16", "plain"), (65, 700, 128, "f16", "strided"), (100, 256, 320, "bf16", "plain"), (128, 1300, 256, "bf16", "plain"),
         (129, 1025, 64, "bf16", "plain"), (300, 777, 192, "f16", "plain"), (257, 2049, 128, "bf16", "strided"), (512, 511, 576, "bf16", "plain"), (40, 20000, 1024, "f16", "plain")]


def _laid(x, layout):
    if layout == "plain":
        return x.contiguous()
    room = torch.full((x.shape[0], x.shape[1] + 24), float("nan"), dtype=x.dtype, device=x.device)       # nothing between rows counts
    room[:, 8:8 + x.shape[1]] = x
    return room[:, 8:8 + x.shape[1]]


def _setup(R, V, K, kind, layout="plain", seed=0):
    rng = np.random.default_rng(seed + R + V + K)
    w = rng.standard_normal((V, K)) * 2 / np.sqrt(K)
    targets = rng.integers(0, V, R).astype(np.int32)
    x = rng.standard_normal((R, K)) + 2 * rng.random((R, 1)) * w[targets]
    if R > 4:
        targets[[1, 3]] = [-1, V]                              # ignored
    x, w = (_laid(torch.from_numpy(a).to(TYPES[kind]).to(DEV), layout) for a in (x, w))
    return x, w, torch.from_numpy(targets).to(DEV), rng


def _np(t):
    return t.double().cpu().numpy()


def _room(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)                   # NaN bytes: nothing is read that was not written


def _off(x, w, scale):
    """What a scaled logit may be off by: K products in fp32, 32 of them an instruction with a rounding at least for every eight, then the difference to the largest."""
    K = x.shape[1]
    reach = np.abs(scale) * (np.abs(x) @ np.abs(w).T).max(initial=0)
    return ((K / 8 + 8) * U + 2 * U) * reach


def forward(x, w, t, scale=1.0, check=True, loss=None):
    R = len(x)
    logp, stats = torch.full((R,), 7.0, device=DEV), torch.full((R, 2), 7.0, device=DEV)
    d = szo.make_head_desc(x, w, t, logp, stats, scale, loss_acc=loss, loss_scale=0.25)
    szo.szo_head_logprobs(d, _room(szo.szo_head_workspace_bytes(d)))
    return logp, stats


@pytest.mark.parametrize("scale", [1.0, 0.7])
@pytest.mark.parametrize("case", CASES)
def test_forward(case, scale):
    R, V, K, kind, layout = case
    x, w, t, _ = _setup(*case)
    loss = torch.full((1,), 3.0, dtype=torch.float64, device=DEV)
    logp, stats = forward(x, w, t, scale, loss=loss)
    xn, wn, tn = _np(x), _np(w), t.cpu().numpy()
    off = _off(xn, wn, scale)
    logits = xn @ wn.T
    lp = od.log_probs(logits, scale)
    there = (tn >= 0) & (tn < V)
    want = np.where(there, lp[np.arange(R), np.clip(tn, 0, V - 1)], 0.0)
    # exponentials of 2^-21, sums of up to 64 terms after each other and a logarithm of 2^-22
    assert np.all(np.abs(_np(logp) - want) <= np.where(there, 3 * off + 2.0 ** -18 + 2.0 ** -22 * np.abs(want), 0))
    assert np.all(np.abs(_np(stats)[:, 0] - logits.max(1)) <= off / scale + U * np.abs(logits.max(1)))
    total = np.exp(scale * (logits - logits.max(1, keepdims=True))).sum(1)
    assert np.all(np.abs(_np(stats)[:, 1] - total) <= total * (2 * off + 2.0 ** -18))
    assert abs(loss.item() - 3.0 + 0.25 * _np(logp).sum()) <= 1e-9 * R


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    R, V, K, kind, layout = case
    x, w, t, rng = _setup(*case)
    scale = 0.8
    _, stats = forward(x, w, t, scale)
    g = torch.from_numpy(rng.standard_normal(R) / 1000).float().to(DEV)              # small: fp16 would lose them as they are
    gx, gw = _laid(torch.full_like(x, 7.0), layout), _laid(torch.full_like(w, 7.0), layout)
    d = szo.make_head_desc(x, w, t, stats=stats, scale=scale)
    szo.szo_head_logprobs_bwd(d, g, gx, gw, _room(szo.szo_head_bwd_workspace_bytes(d)))
    xn, wn, tn, gn = _np(x), _np(w), t.cpu().numpy(), _np(g)
    off = _off(xn, wn, scale)
    dn = od.log_probs_grad(xn @ wn.T, tn, gn, np.zeros(R), scale)
    there = ((tn >= 0) & (tn < V))[:, None]
    hit = (np.arange(V)[None, :] == tn[:, None]) & there
    p = np.abs(np.where(hit, scale * gn[:, None] - dn, dn))                          # the size of what is subtracted at the target
    # p is off by its logit and by its sum; d is rounded to the type once more, in fp16 to 2^-25 of what the largest gradient is lifted to, 2^13 or more
    half = HALF[kind]
    floor = 0 if kind == "bf16" else 2.0 ** -25 * 2.0 ** -13 * np.abs(scale * gn).max()
    d_err = half * np.abs(dn) + (1 + half) * p * (4 * off + 2.0 ** -17) + floor * there
    least = 0 if kind == "bf16" else 2.0 ** -25                                      # where the output is subnormal
    for got, want, err, size, n in ((gx, dn @ wn, d_err @ np.abs(wn), np.abs(dn) @ np.abs(wn), V), (gw, dn.T @ xn, d_err.T @ np.abs(xn), np.abs(dn).T @ np.abs(xn), R)):
        bad = np.abs(_np(got) - want) - (half * np.abs(want) + least + (1 + half) * (err + (n / 8 + 40) * U * size))
        assert np.all(bad <= 0), (bad.max(), np.argwhere(bad > 0)[:4])
    assert (gx[~torch.from_numpy(there[:, 0]).to(DEV)] == 0).all()


@pytest.mark.parametrize("g", [1.0042, 1.0, 1.97, 0.502, 3.1e-5])
def test_a_gradient_that_all_rows_share_is_rounded_well(g):
    """Targets that are unlikely: d is nearly the gradient in every row, and its rounding the whole row's error."""
    R, V, K = 64, 3000, 256
    rng = np.random.default_rng(7)
    x, w = (torch.from_numpy(a).bfloat16().to(DEV) for a in (rng.standard_normal((R, K)) * 0.1, rng.standard_normal((V, K)) * 0.1))
    t = torch.from_numpy(rng.permutation(V)[:R].astype(np.int32)).to(DEV)
    _, stats = forward(x, w, t)
    d = szo.make_head_desc(x, w, t, stats=stats)
    by_x, by_w = torch.empty_like(x), torch.empty_like(w)
    szo.szo_head_logprobs_bwd(d, torch.full((R,), g, device=DEV), by_x, by_w, _room(szo.szo_head_bwd_workspace_bytes(d)))
    p = np.exp(od.log_probs(_np(x) @ _np(w).T))
    assert p.max() < 2.0 ** -6
    d = -g * p
    d[np.arange(R), t.cpu().numpy()] += g
    # d lies between 1.95 and 1.99 times a power of two: off by 2^-8 / 1.95 of it at most; the result's own rounding is 2^-8 / sqrt(3) in the mean of squares, at most
    bound = 2.0 ** -8 * np.sqrt(1 / 1.95 ** 2 + 1 / 3)
    for got, want in ((by_x, d @ _np(w)), (by_w, d.T @ _np(x))):
        assert np.linalg.norm(_np(got) - want) <= bound * np.linalg.norm(want), np.linalg.norm(_np(got) - want) / np.linalg.norm(want)


def test_one_gradient_alone_and_no_targets():
    x, w, t, rng = _setup(70, 600, 128, "bf16")
    _, stats = forward(x, w, t)
    g = torch.randn(70, device=DEV)
    d = szo.make_head_desc(x, w, t, stats=stats)
    room = _room(szo.szo_head_bwd_workspace_bytes(d))
    both, alone = [torch.empty_like(x), torch.empty_like(w)], [torch.empty_like(x), torch.empty_like(w)]
    szo.szo_head_logprobs_bwd(d, g, *both, room)
    szo.szo_head_logprobs_bwd(d, g, alone[0], None, room)
    szo.szo_head_logprobs_bwd(d, g, None, alone[1], room)
    assert torch.equal(both[0], alone[0]) and torch.equal(both[1], alone[1])
    szo.szo_head_logprobs_bwd(szo.make_head_desc(x, w, None, stats=stats), g, *both, room)
    assert (both[0] == 0).all() and (both[1] == 0).all()
    logp, _ = forward(x, w, None)
    assert (logp == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_gradients_in_place(kind):
    x, w, t, _ = _setup(200, 1500, 192, kind)
    _, stats = forward(x, w, t)
    g = torch.randn(200, device=DEV)
    d = szo.make_head_desc(x, w, t, stats=stats)
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    szo.szo_head_logprobs_bwd(d, g, gx, gw, _room(szo.szo_head_bwd_workspace_bytes(d)))
    szo.szo_head_logprobs_bwd(d, g, x, w, _room(szo.szo_head_bwd_workspace_bytes(d)))
    assert torch.equal(x, gx) and torch.equal(w, gw)


@pytest.mark.parametrize("rows", [20, 300])
def test_rows_without_a_target_may_hold_anything(rows):
    x, w, t, _ = _setup(rows, 900, 128, "bf16")
    x[1], x[3, 5] = float("nan"), float("inf")
    logp, stats = forward(x, w, t)
    assert (logp[[1, 3]] == 0).all() and torch.isfinite(logp).all()
    g = torch.ones(rows, device=DEV)
    g[1] = float("nan")
    d = szo.make_head_desc(x, w, t, stats=stats)
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    szo.szo_head_logprobs_bwd(d, g, gx, gw, _room(szo.szo_head_bwd_workspace_bytes(d)))
    assert (gx[[1, 3]] == 0).all() and torch.isfinite(gx).all() and torch.isfinite(gw).all()


@pytest.mark.parametrize("rows", [20, 300])
def test_nan_and_infinities_stay_in_their_rows(rows):
    x, w, t, _ = _setup(rows, 900, 128, "bf16")
    x[5], x[7, 0], x[8, 0], w[:, 0] = float("nan"), float("inf"), float("-inf"), 1.0
    logp, stats = forward(x, w, t)
    assert torch.isnan(logp[[5, 7]]).all()                                             # every logit +inf
    assert torch.isneginf(logp[8]) and stats[8, 1] == 0                                # a row of -inf alone
    rest = [i for i in range(rows) if i not in (5, 7, 8)]
    assert torch.isfinite(logp[rest]).all()
    d = szo.make_head_desc(x, w, t, stats=stats)
    gx = torch.empty_like(x)
    szo.szo_head_logprobs_bwd(d, torch.ones(rows, device=DEV), gx, None, _room(szo.szo_head_bwd_workspace_bytes(d)))
    assert torch.isfinite(gx[rest]).all() and torch.isnan(gx[[5, 7]]).any() and (gx[8] == 0).all()


def test_huge_logits_and_scales():
    x, w, t, _ = _setup(40, 300, 64, "bf16")
    x *= 1e4
    logp, stats = forward(x, w, t, 3.0)
    want = od.log_probs(_np(x) @ _np(w).T, 3.0)[np.arange(40), np.clip(t.cpu().numpy(), 0, 299)]
    ok = ((t >= 0) & (t < 300)).cpu().numpy()
    assert np.all(np.abs(_np(logp) - want)[ok] <= 3 * _off(_np(x), _np(w), 3.0) + 2.0 ** -18 + 2.0 ** -22 * np.abs(want[ok]))
    logp, _ = forward(x, w, t, 2.3e38)
    assert not torch.isnan(logp[t == torch.from_numpy((_np(x) @ _np(w).T).argmax(1)).to(DEV)]).any()


def test_pieces_of_the_vocabulary_and_parts_of_sums():
    """More of d than is held at a time: 4200 rows of 40000, three products by pieces, with sums of x_grad added up over them."""
    torch.manual_seed(3)
    R, V, K = 4200, 40000, 64
    x, w = torch.randn(R, K, device=DEV).bfloat16(), (torch.randn(V, K, device=DEV) / 8).bfloat16()
    t = torch.randint(V, (R,), device=DEV, dtype=torch.int32)
    logp, stats = forward(x, w, t)
    g = torch.randn(R, device=DEV) / R
    d = szo.make_head_desc(x, w, t, stats=stats)
    need = szo.szo_head_bwd_workspace_bytes(d)
    assert need < 2 * R * V
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    szo.szo_head_logprobs_bwd(d, g, gx, gw, _room(need))
    logits = x.double() @ w.double().t()
    lp = logits - torch.logsumexp(logits, -1, keepdim=True)
    hit = lp.gather(1, t.long()[:, None])[:, 0]
    off = (K / 8 + 10) * U * (x.double().abs().amax(0) * w.double().abs().amax(0)).sum().item()
    assert ((logp - hit).abs() <= 3 * off + 2.0 ** -18 + 2.0 ** -22 * hit.abs()).all()
    dn = -lp.exp_()
    dn[torch.arange(R, device=DEV), t.long()] += 1
    dn *= g.double()[:, None]
    # each d is rounded to 8 bits and off by its logit: a sum is off by at most that share of the sum of sizes
    share = 2.0 ** -8 + 4 * off + 2.0 ** -17
    for got, want, size, n in ((gx, dn @ w.double(), dn.abs() @ w.double().abs(), V), (gw, dn.t() @ x.double(), dn.abs().t() @ x.double().abs(), R)):
        assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * (share + (n / 8 + 40) * U) * size).all()


def test_empty_batches():
    w = torch.randn(50, 64, device=DEV).bfloat16()
    x, t = torch.empty(0, 64, device=DEV).bfloat16(), torch.empty(0, dtype=torch.int32, device=DEV)
    forward(x, w, t)
    gw = torch.full_like(w, 3.0)
    d = szo.make_head_desc(x, w, t)
    szo.szo_head_logprobs_bwd(d, torch.empty(0, device=DEV), torch.empty_like(x), gw, _room(16))
    assert (gw == 0).all()


def test_captured_and_replayed_beside_eager_calls_on_another_stream():
    x, w, t, _ = _setup(300, 5000, 256, "bf16")
    g = torch.randn(300, device=DEV)

    def call():
        out = [torch.empty(300, device=DEV), torch.empty(300, 2, device=DEV), torch.empty_like(x), torch.empty_like(w), torch.zeros(1, dtype=torch.float64, device=DEV)]
        d = szo.make_head_desc(x, w, t, out[0], out[1], loss_acc=out[4])
        rooms = _room(szo.szo_head_workspace_bytes(d)), _room(szo.szo_head_bwd_workspace_bytes(d))
        return out, lambda: (out[4].zero_(), szo.szo_head_logprobs(d, rooms[0]), szo.szo_head_logprobs_bwd(d, g, out[2], out[3], rooms[1]))

    want, run = call()
    run()
    torch.cuda.synchronize()
    got, again = call()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again()
    graph, (held, captured) = torch.cuda.CUDAGraph(), call()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        captured()
    for _ in range(4):
        for o in held:
            o.fill_(9.0)
        graph.replay()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
