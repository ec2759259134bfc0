"""Every way in which rows and cache go to waves, with ragged batches, masks, missing pages, NaN and odd strides, against the 64-bit definition.

The ways are chosen by sizes, among them hints (max_q, max_len, rows of q that no sequence has), so small sequences run through the ways of large batches; that a case
takes the way it is written for is asked of the library."""
import math

import numpy as np
import pytest
import torch

from attn_reference import attention
from oracle import decoder as od
from paper_2406_02913_amd import szo
from test_gpu_attn_cached import DEV, STORE, TYPES
from test_gpu_kv_cache import Both

pytestmark = pytest.mark.gpu


def filled(lengths, heads, D, missing=()):
    def change(x):
        x[1, 20, 0, 3] = np.nan                                  # one feature of one value
        x[0, min(45, x.shape[1] - 1), heads - 1, 7] = np.nan     # a key

    b = Both(lengths, heads, D, 64, seed=D)
    b.write(lengths, lengths, "f32", change)
    for s, page in missing:
        b.table[s, page] = -1 if s % 2 else 10 ** 6
    return b


def check(b, lengths, new, group, kind, way, rows=None, max_q=None, max_len=None, causal=True, window=0, layout="plain", lse_too=True):
    D, heads = b.D, b.heads * group
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(start[-1])
    rows = T if rows is None else rows
    q = torch.from_numpy(b.rng.standard_normal((T, heads, D))).to(TYPES[kind])
    if layout == "odd":                           # addresses and strides that are no multiples of a vector
        dev = torch.full((rows, heads, D + 3), float("nan"), dtype=q.dtype, device=DEV)[..., 1:D + 1]
        out = torch.full((rows, heads, D + 1), 7.0, dtype=q.dtype, device=DEV)[..., :D]
    else:
        dev = torch.full((rows, heads, D), float("nan"), dtype=q.dtype, device=DEV)
        out = torch.full((rows, heads, D), 7.0, dtype=q.dtype, device=DEV)
    dev[:T] = q.to(DEV)
    lse = torch.full((rows, heads), 7.0, device=DEV) if lse_too else None
    b.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    scale = 1 / math.sqrt(D)
    d = szo.make_attn_desc(b.cache(), dev, out, torch.from_numpy(start).to(DEV), max(new) if max_q is None else max_q, max(lengths) if max_len is None else max_len, scale,
                           causal, window, lse)
    plan = szo.szo_attn_plan(d)
    assert plan == way, (way, plan)
    room = torch.full((szo.szo_attn_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV)        # NaN bytes: nothing is read that was not written
    szo.szo_attn_cached(d, room)
    got = out.float().cpu().numpy().astype(np.float64)
    got_lse = None if lse is None else lse.cpu().numpy().astype(np.float64)
    assert (got[T:] == 7).all() and (got_lse is None or (got_lse[T:] == 7).all())                      # rows that no sequence has
    rel, floor = STORE[kind]
    for s, n in enumerate(lengths):
        if not new[s]:
            continue
        k, there = od.cache_dense(b.codes[0], b.exps[0], False, b.table, lengths, s)
        v, _ = od.cache_dense(b.codes[1], b.exps[1], True, b.table, lengths, s)
        x = q[start[s]:start[s + 1]].double().numpy()
        want, want_lse, size = attention(x, k, v, there, n, scale, causal, window)
        y = got[start[s]:start[s + 1]]
        # scores: D products in fp32 (16 per instruction, one rounding each at most), scaled and shifted: |s| and the sum of sizes bound them
        reach = scale * max((np.abs(np.nan_to_num(k)).max(initial=0) * np.abs(x)).sum(-1).max(initial=0), 1)
        off = (D / 8 + 8) * 2.0 ** -24 * reach * 1.5 + 2.0 ** -21
        # weights in fp16: 2^-11 relative; tiny ones 2^-25 of the largest
        weights, tiny = 2.0 ** -11 + 2 * off, n * 2.0 ** -25 * np.abs(np.nan_to_num(v)).max(initial=0) * 2
        fine = np.isfinite(want)
        assert np.array_equal(fine, np.isfinite(y)), (s, np.argwhere(fine != np.isfinite(y))[:5])
        err = np.abs(np.where(fine, y - want, 0))
        assert np.all(err <= np.where(fine, rel * np.abs(want) + floor + weights * size + tiny, 0)), (s, err.max())
        if lse is not None:
            z = got_lse[start[s]:start[s + 1]]
            empty, ok = np.isneginf(want_lse), np.isfinite(want_lse)
            assert np.array_equal(empty, np.isneginf(z)) and np.array_equal(np.isnan(want_lse), np.isnan(z)) and (y[empty] == 0).all()
            assert np.all(np.abs(z[ok] - want_lse[ok]) <= 2 * off + 2.0 ** -22 * np.abs(want_lse[ok]))


MASKS = [(True, 0), (False, 0), (True, 70)]
SIDE_BY_SIDE = (4, 1, 1, 0)
KINDS = ("bf16", "f16")


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_side_by_side_by_the_number_of_tiles(D):
    """2048 tiles and more."""
    lengths, new = [300, 33, 190, 1, 0, 64], [170, 33, 45, 1, 0, 40]
    b = filled(lengths, 8, D, missing=[(0, 2), (2, 0)])
    for kind in KINDS:
        for causal, window in MASKS:
            check(b, lengths, new, 4, kind, SIDE_BY_SIDE, rows=8192, max_q=8192, causal=causal, window=window, max_len=8192)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_side_by_side_where_there_is_no_cache_to_share(D):
    """1024 tiles and more with eight blocks at most; odd strides, no log sums."""
    lengths, new = [200, 100, 256, 31], [200, 37, 130, 31]
    b = filled(lengths, 8, D, missing=[(1, 0)])
    for kind in KINDS:
        for causal, window in MASKS:
            check(b, lengths, new, 4, kind, SIDE_BY_SIDE, rows=4200, max_q=4200, causal=causal, window=window, layout="odd", lse_too=causal)


def test_side_by_side_with_rows_of_many_heads_a_key_head():
    """Tiles that hold parts of a token's heads: 7 and 40 of them, of one key head."""
    for group, heads in ((7, 2), (40, 1)):
        lengths, new = [150, 70], [90, 70]
        check(filled(lengths, heads, 64), lengths, new, group, "bf16", SIDE_BY_SIDE, rows=65536, max_q=65536, max_len=1000)


def test_side_by_side_at_its_own_size():
    """Nothing but the sizes of the call itself: one prompt of 2100 tokens, 8 key heads."""
    lengths = [2100]
    check(filled(lengths, 8, 64), lengths, lengths, 4, "bf16", SIDE_BY_SIDE)


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("group,new", [(4, 1), (1, 9), (8, 2)])
def test_eight_waves_and_parts(D, group, new):
    lengths = [1, 40, 1300, 33, 64, 65, 200, 129, 31, 32, 500, 7, 96, 290, 5, 128]
    b = filled(lengths, 8, D, missing=[(2, 3), (6, 0)])
    for kind in KINDS:
        for causal, window, parts in ((True, 0, 2), (False, 0, 2), (True, 1100, 1)):
            check(b, lengths, [min(new, n) for n in lengths], group, kind, (1, 8, parts, 0), causal=causal, window=window, max_len=2100)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("sequences,max_len,parts", [(24, 1 << 17, 5), (9, 1 << 18, 14), (64, 1 << 16, 2), (140, 1 << 15, 1)])
def test_codes_that_pass_the_caches_by(D, sequences, max_len, parts):
    r = np.random.default_rng(sequences)
    lengths = [int(x) for x in r.integers(1, 60, sequences)]
    new = [min(n, int(x)) for n, x in zip(lengths, r.integers(0, 4, sequences))]
    lengths[3], new[3] = 400, 3
    b = filled(lengths, 8, D, missing=[(3, 1)])
    for kind in KINDS:
        for causal in (True, False):
            check(b, lengths, new, 2, kind, (1, 4, parts, 1), causal=causal, max_len=max_len)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("group,new,ways", [(1, 1, [(8, 0), (20, 0), (32, 0), (64, 1)]), (3, 1, [(8, 0), (20, 0), (32, 0), (64, 1)]), (5, 3, [(8, 0), (20, 0), (32, 0), (64, 1)]),
                                            (8, 4, [(1, 0), (5, 0), (12, 0), (64, 1)]), (4, 30, [(1, 0), (5, 0), (12, 0), (51, 0)])])
def test_parts_of_few_and_of_many_rows(D, group, new, ways):
    """Both ways of joining parts, odd numbers of rows a part, more parts than there are blocks."""
    lengths, news = [900, 33, 1], [new, min(new, 33), 1]
    b = filled(lengths, 1, D, missing=[(0, 5)])
    for kind in KINDS:
        for max_len, (parts, once) in zip((900, 2500, 6000, 1 << 20), ways):
            check(b, lengths, news, group, kind, (1, 4, parts, once), max_len=max_len)
