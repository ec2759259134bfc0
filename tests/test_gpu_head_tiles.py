"""Every tile that sizes choose for log probabilities through the head and for their gradients, in both types, against the 64-bit definition."""
import pytest
import torch

from paper_2406_02913_amd import szo
from test_gpu_head import HALF, TYPES, U, _room

pytestmark = pytest.mark.gpu
DEV = "cuda"

# rows, vocabulary, width (a single step of 64, and more steps than LDS holds) -> what the plan says: forward tile; pieces, tile of d; tile of x_grad, parts; tile of weight_grad
WAYS = [(130, 11987, 64, (128, 128, 1, 128, 128, 128, 64, 23, 128)), (133, 16481, 64, (128, 192, 1, 128, 192, 128, 64, 32, 128)),
        (205, 16481, 128, (128, 256, 1, 128, 256, 128, 64, 32, 128)), (300, 16481, 64, (128, 320, 1, 128, 320, 128, 64, 32, 128)),
        (701, 11987, 64, (128, 384, 1, 128, 384, 128, 64, 23, 128)), (1291, 10877, 64, (128, 448, 1, 128, 448, 128, 64, 12, 128)),
        (130, 32987, 64, (256, 256, 1, 256, 256, 128, 64, 64, 128)), (601, 101, 4096, (128, 64, 1, 128, 64, 128, 128, 1, 128)),
        (2001, 99, 4096, (128, 64, 1, 128, 64, 128, 256, 1, 128)), (4100, 100, 2048, (128, 64, 1, 128, 64, 128, 320, 1, 128)),
        (4100, 100, 1024, (128, 64, 1, 128, 64, 128, 192, 1, 128)), (1288, 1003, 6592, (128, 64, 1, 128, 64, 128, 384, 1, 128)),
        (1538, 997, 6592, (128, 64, 1, 128, 64, 256, 256, 1, 128)), (388, 7999, 6464, (128, 128, 1, 128, 128, 128, 448, 5, 256)),
        (385, 7999, 4160, (128, 128, 1, 128, 128, 256, 256, 7, 256)), (391, 7999, 1600, (128, 128, 1, 128, 128, 128, 192, 6, 128)),
        (130, 11987, 448, (128, 128, 1, 128, 128, 128, 64, 21, 128)), (133, 16481, 320, (128, 192, 1, 128, 192, 128, 64, 28, 128)),
        (205, 16481, 576, (128, 256, 1, 128, 256, 128, 64, 12, 128)), (300, 16481, 448, (128, 320, 1, 128, 320, 128, 64, 12, 128)),
        (701, 11987, 512, (128, 384, 1, 128, 384, 128, 128, 10, 128)), (1291, 10877, 448, (128, 448, 1, 128, 448, 128, 192, 9, 128)),
        (131, 33001, 320, (256, 256, 1, 256, 256, 128, 64, 28, 128)),
        (100, 65599, 320, (128, 128, 1, 128, 128, 128, 128, 85, 256)), (3100, 50001, 576, (256, 256, 2, 256, 256, 128, 320, 5, 128))]


def test_the_ways_are_all_tiles_that_there_are():
    forward, grad, by_x, by_w = ({w[3][a:b] for w in WAYS} for a, b in ((0, 2), (3, 5), (5, 7), (8, 9)))
    tiles = {(128, n) for n in range(128, 449, 64)} | {(256, 256)}
    assert forward >= tiles and grad >= tiles and by_x >= tiles and by_w == {(128,), (256,)}


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("R,V,K,want", WAYS)
def test_every_way_that_sizes_choose(R, V, K, want, kind):
    gen = torch.Generator(device=DEV).manual_seed(R + V + K)
    scale = 0.9
    x = torch.randn(R, K, device=DEV, generator=gen).to(TYPES[kind])
    w = (torch.randn(V, K, device=DEV, generator=gen) * (2 / K ** 0.5)).to(TYPES[kind])
    t = torch.randint(V, (R,), device=DEV, generator=gen, dtype=torch.int32)
    t[::9] = -1
    g = torch.randn(R, device=DEV, generator=gen)
    logp, stats = torch.full((R,), 7.0, device=DEV), torch.full((R, 2), 7.0, device=DEV)
    d = szo.make_head_desc(x, w, t, logp, stats, scale)
    assert szo.szo_head_plan(d) == want
    szo.szo_head_logprobs(d, _room(szo.szo_head_workspace_bytes(d)))
    gx, gw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    szo.szo_head_logprobs_bwd(d, g, gx, gw, _room(szo.szo_head_bwd_workspace_bytes(d)))

    x64, w64, there = x.double(), w.double(), (t >= 0)[:, None]
    z = x64 @ w64.t()
    top = z.amax(1)
    lse = torch.logsumexp(scale * z, 1)
    want_logp = torch.where(there[:, 0], scale * z.gather(1, t.long().clamp(min=0)[:, None])[:, 0] - lse, 0.0)
    # a scaled logit: K products in fp32, 32 of them an instruction with a rounding at least for every eight, then the difference to the largest
    off = ((K / 8 + 8) * U + 2 * U) * scale * (x64.abs() @ w64.abs().t()).max().item()
    assert ((logp - want_logp).abs() <= torch.where(there[:, 0], 3 * off + 2.0 ** -18 + 2.0 ** -22 * want_logp.abs(), 0.0)).all()
    assert ((stats[:, 0] - top).abs() <= off / scale + U * top.abs()).all()
    total = torch.exp(lse - scale * top)
    assert ((stats[:, 1] - total).abs() <= total * (2 * off + 2.0 ** -18)).all()

    by = scale * g.double()[:, None] * there
    p = torch.exp(scale * z - lse[:, None]).mul_(by)
    dn = -p
    dn[torch.arange(R, device=DEV), t.long().clamp(min=0)] += by[:, 0]
    half, least = HALF[kind], 0 if kind == "bf16" else 2.0 ** -25
    # d: its rounding, logit and sum, and in fp16 2^-25 of what a row's gradient is lifted to; there the states that stand beside it are off by 2^-25 of 2^15 times what the row's gradient is smaller by
    floor = 0 if kind == "bf16" else 2.0 ** -38 * by.abs()
    err = half * dn.abs() + (1 + half) * p.abs() * (4 * off + 2.0 ** -17) + floor
    size = dn.abs()
    beside = 0
    if kind == "f16":
        shift = 2 * by.abs().max() / torch.where(by.abs() > 0, by.abs(), float("inf"))
        beside = (1 + half) * ((size * shift).sum(0) * 2 * x64.abs().max() * 2.0 ** -39)[:, None]
    for got, exact, e, s, n in ((gx, dn @ w64, err @ w64.abs(), size @ w64.abs(), V), (gw, dn.t() @ x64, err.t() @ x64.abs() + beside, size.t() @ x64.abs(), R)):
        bad = (got.double() - exact).abs() - (half * exact.abs() + least + (1 + half) * (e + (n / 8 + 40) * U * s))
        assert (bad <= 0).all(), (bad.max(), (bad > 0).nonzero()[:4])
    assert (gx[::9] == 0).all()
