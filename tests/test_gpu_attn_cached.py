"""Attention over the 8-bit cache against the 64-bit definition on the same codes."""
import math

import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2406_02913_amd import szo
from test_gpu_kv_cache import Both

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
STORE = {"bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}


def check(b, lengths, new, group, kind, causal=True, window=0, scale=None, max_len=None, q=None, layout="plain", lse_too=True):
    D, heads = b.D, b.heads * group
    scale = 1 / math.sqrt(D) if scale is None else scale
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(start[-1])
    if q is None:
        q = b.rng.standard_normal((T, heads, D))
    q = torch.from_numpy(q).to(TYPES[kind])
    if layout == "odd":
        dev = torch.zeros(T, heads, D + 3, dtype=q.dtype, device=DEV)[..., 1:D + 1]
        out = torch.full((T, heads, D + 1), 7.0, dtype=q.dtype, device=DEV)[..., :D]
    else:                                        # a head's rows far apart, as in one buffer of all projections
        dev = torch.zeros(T, heads + 2, D, dtype=q.dtype, device=DEV)[:, 1:-1]
        out = torch.full((T, heads, D), 7.0, dtype=q.dtype, device=DEV)
    dev.copy_(q)
    lse = torch.full((T, heads), 7.0, device=DEV) if lse_too else None
    b.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    d = szo.make_attn_desc(b.cache(), dev, out, torch.from_numpy(start).to(DEV), max(new), max(lengths) if max_len is None else max_len, scale, causal, window, lse)
    room = torch.full((szo.szo_attn_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV)        # NaN bytes: nothing is read that was not written
    szo.szo_attn_cached(d, room)
    got, got_lse = out.float().cpu().numpy().astype(np.float64), None if lse is None else lse.cpu().numpy().astype(np.float64)
    rel, floor = STORE[kind]
    for s, n in enumerate(lengths):
        if not new[s]:
            continue
        k, there = od.cache_dense(b.codes[0], b.exps[0], False, b.table, lengths, s)
        v, _ = od.cache_dense(b.codes[1], b.exps[1], True, b.table, lengths, s)
        x = q[start[s]:start[s + 1]].double().numpy()
        want, want_lse, size = od.attention(x, k, v, there, n, scale, causal, window)
        y, z = got[start[s]:start[s + 1]], None if got_lse is None else got_lse[start[s]:start[s + 1]]
        # scores: D products in fp32 (16 per instruction, one rounding each at most), scaled and shifted: |s| and the sum of sizes bound them
        reach = np.abs(scale) * max((np.abs(np.nan_to_num(k)).max(initial=0) * np.abs(x)).sum(-1).max(initial=0), 1)
        off = (D / 8 + 8) * 2.0 ** -24 * reach * 1.5 + 2.0 ** -21
        # weights in fp16: 2^-11 relative; tiny ones 2^-25 of the largest
        weights = 2.0 ** -11 + 2 * off
        tiny = n * 2.0 ** -25 * np.abs(np.nan_to_num(v)).max(initial=0) * 2
        fine = np.isfinite(want)
        assert np.array_equal(fine, np.isfinite(y)), (s, np.argwhere(fine != np.isfinite(y))[:5])
        err = np.abs(np.where(fine, y - want, 0))
        assert np.all(err <= np.where(fine, rel * np.abs(want) + floor + weights * size + tiny, 0)), (s, err.max())
        if z is not None:
            empty = np.isneginf(want_lse)
            assert np.array_equal(empty, np.isneginf(z)) and (y[empty] == 0).all()
            ok = np.isfinite(want_lse)
            assert np.all(np.abs(z[ok] - want_lse[ok]) <= 2 * off + 2.0 ** -22 * np.abs(want_lse[ok]))
    return got


def filled(lengths, heads, D, page, seed=0, change=None):
    b = Both(lengths, heads, D, page, seed)
    b.write(lengths, lengths, "f32", change)
    return b


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,group,page", [(64, 2, 1, 32), (96, 1, 3, 64), (128, 2, 4, 64), (128, 1, 7, 96), (256, 1, 2, 32)])
def test_one_token_behind_lengths_of_all_kinds(D, heads, group, page, kind):
    lengths = [1, 2, 31, 32, 33, 64, 65, 200, 513]
    check(filled(lengths, heads, D, page), lengths, [1] * 9, group, kind)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,group", [(64, 1, 4), (96, 2, 1), (128, 1, 4), (256, 1, 5)])
def test_few_queries_ragged(D, heads, group, kind):
    lengths, new = [5, 40, 129, 300, 77], [5, 3, 11, 1, 0]
    check(filled(lengths, heads, D, 64), lengths, new, group, kind)


@pytest.mark.parametrize("D,heads,group", [(64, 2, 2), (96, 1, 1), (128, 2, 3), (256, 1, 1)])
def test_prompts(D, heads, group):
    lengths = [150, 1, 33, 200]
    b = filled(lengths, heads, D, 64)
    check(b, lengths, lengths, group, "bf16")
    check(b, lengths, [97, 1, 20, 65], group, "f16")


@pytest.mark.parametrize("new", [[1, 1], [40, 9], [70, 100]])
@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 33), (True, 64), (True, 1000), (False, 20)])
def test_masks(new, causal, window):
    lengths = [130, 100]
    check(filled(lengths, 1, 64, 32), lengths, new, 2, "bf16", causal, window)


def test_queries_before_the_first_token_see_nothing():
    b = filled([20, 40], 1, 128, 32)
    b.lengths.zero_()
    for new in ([30, 45], [150, 40]):
        check(b, [20, 40], new, 2, "bf16")
    check(b, [0, 40], [3, 2], 2, "bf16")                        # an empty sequence
    check(b, [0, 0], [1, 1], 2, "bf16", causal=False)


def test_what_lies_behind_the_length_has_no_influence():
    """NaN codes behind the length, in the same block and in the next one; the cache's random bytes hold such codes as well."""
    b = filled([70], 1, 64, 64)
    off = od.places(64, True)
    page, sub = b.table[0, 70 // 64], 70 % 64 // 32
    for codes, values in ((b.codes[0], False), (b.codes[1], True)):
        codes[page, 0, sub][od.places(64, values)[6:]] = 0x7F
    assert off.shape == (32, 64)
    for i in range(2):
        b.dev[i].copy_(torch.from_numpy(b.codes[i]))
    for new in ([1], [9], [70]):
        assert np.isfinite(check(b, [70], new, 2, "bf16")).all()
    assert np.isfinite(check(b, [70], [9], 2, "bf16", causal=False)).all()


def test_nan_keys_and_values_reach_only_rows_that_see_them():
    def change(x):
        x[1, 50, 0, 3] = np.nan                                  # one feature of one value
        x[0, 60, 0, 7] = np.inf                                  # a key: everything that sees it

    b = filled([90], 1, 64, 32, change=change)
    got = check(b, [90], [90], 1, "bf16")
    assert np.isfinite(got[:50]).all() and np.isnan(got[50:60, 0, 3]).all() and np.isfinite(got[50:60, 0, :3]).all() and np.isnan(got[60:]).all()
    got = check(b, [90], [90], 1, "bf16", window=8)
    assert np.isfinite(got[68:]).all() and np.isnan(got[57, 0, 3]) and np.isfinite(got[58, 0, 3])


def test_strong_scores_and_uneven_blocks():
    """Scores of hundreds; blocks of values 2^12 apart; a row's weight on one token only."""
    def change(x):
        x[0] *= 8
        x[1, 32:64] *= 4096
        x[1, 64:96] *= 2.0 ** -12
        x[1, 96:128] = 0

    b = filled([200], 2, 128, 64, change=change)
    check(b, [200], [1], 2, "bf16", scale=1.0)
    check(b, [200], [120], 2, "f16", scale=1.0)
    check(b, [200], [200], 1, "bf16", scale=-0.3)


def test_uniform_weights_with_zero_scale():
    check(filled([500], 1, 128, 64), [500], [2], 4, "bf16", scale=0.0)


def test_pages_outside_the_cache_are_not_attended_to():
    b = filled([200, 60], 1, 64, 32)
    b.table[0, 2], b.table[0, 0], b.table[1, :] = -5, 10 ** 8, -1
    for new in ([1, 1], [60, 30]):
        check(b, [200, 60], new, 2, "bf16")


def test_length_hint_that_is_wrong_still_gives_the_right_result():
    b = filled([3000], 1, 128, 64)
    for hint in (0, 1, 3000, 100000):
        check(b, [3000], [1], 4, "bf16", max_len=hint)
        check(b, [3000], [20], 4, "bf16", max_len=hint)


def test_odd_addresses_and_strides_and_no_lse():
    b = filled([100, 37], 2, 64, 64)
    check(b, [100, 37], [1, 1], 2, "bf16", layout="odd")
    check(b, [100, 37], [50, 37], 2, "f16", layout="odd", lse_too=False)


def test_many_heads_and_sequences():
    lengths = [int(x) for x in np.random.default_rng(1).integers(1, 120, 40)]
    check(filled(lengths, 4, 64, 32), lengths, [1] * 40, 8, "bf16")


def test_runs_are_equal_and_streams_and_graphs_work():
    b = filled([700, 300], 2, 128, 64)
    q = torch.randn(2, 8, 128, device=DEV).bfloat16()
    out = torch.empty_like(q)
    d = szo.make_attn_desc(b.cache(), q, out, torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV), 1, 700, 0.09)
    room = torch.empty(szo.szo_attn_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    szo.szo_attn_cached(d, room)
    want = out.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out.zero_()
        szo.szo_attn_cached(d, room)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        szo.szo_attn_cached(d, room)
    for _ in range(3):
        q.copy_(torch.randn_like(q.float()))
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        szo.szo_attn_cached(d, room)
        torch.cuda.synchronize()
        assert torch.equal(out, replayed)


def test_a_long_cache_behind_32_bits():
    """Codes behind 4 GiB; 40000 tokens."""
    heads, D, n = 8, 128, 40000
    per = -(-n // 64)
    k, v, ke, ve = szo.new_kv_cache(70000, 64, heads, D)
    table = torch.arange(70000 - per, 70000, dtype=torch.int32, device=DEV)[None]
    lengths = torch.tensor([n], dtype=torch.int32, device=DEV)
    cache = szo.make_kv_cache(k, v, ke, ve, table, lengths)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x = torch.randn(n, heads, D, device=DEV, generator=gen)
    start = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    szo.szo_kv_cache_write(cache, szo.make_kv_tokens(x, x, start, n))
    kv = torch.empty(n, heads, D, device=DEV), torch.empty(n, heads, D, device=DEV)
    szo.szo_kv_cache_read(cache, szo.make_kv_tokens(*kv, start, n))
    q = torch.randn(1, 2 * heads, D, device=DEV, generator=gen).bfloat16()
    out = torch.empty_like(q)
    d = szo.make_attn_desc(cache, q, out, torch.tensor([0, 1], dtype=torch.int32, device=DEV), 1, n, 0.5)
    szo.szo_attn_cached(d, torch.empty(szo.szo_attn_workspace_bytes(d), dtype=torch.uint8, device=DEV))
    for h in range(2 * heads):
        s = 0.5 * (kv[0][:, h // 2].double().cpu() @ q[0, h].double().cpu())
        w = torch.softmax(s, 0)
        vals = kv[1][:, h // 2].double().cpu()
        want, size = w @ vals, w @ vals.abs()
        # fp16 weights and scores of up to |s| = 40: as in check()
        off = (D / 8 + 8) * 2.0 ** -24 * 0.5 * float((q[0, h].abs().float().cpu().sum() * kv[0].abs().max().cpu())) * 1.5
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * off) * size + 2 * n * 2.0 ** -25 * float(vals.abs().max())
        assert ((out[0, h].double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("drop", [6.0, 12.0, 16.0])
def test_many_small_weights_beside_a_large_one(drop):
    """40000 tokens with weights of e^-drop beside one of 1: what they add up to keeps the precision of a single weight."""
    n, D = 40000, 64
    per = -(-n // 64)
    k, v, ke, ve = szo.new_kv_cache(per, 64, 1, D)
    lengths = torch.tensor([n], dtype=torch.int32, device=DEV)
    cache = szo.make_kv_cache(k, v, ke, ve, torch.arange(per, dtype=torch.int32, device=DEV)[None], lengths)
    start = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    keys, values = torch.zeros(n, 1, D, device=DEV), torch.ones(n, 1, D, device=DEV)
    keys[777, 0, 0], values[777] = 16.0, 0.0
    szo.szo_kv_cache_write(cache, szo.make_kv_tokens(keys, values, start, n))
    q = torch.zeros(1, 1, D, device=DEV, dtype=torch.float16)
    q[0, 0, 0] = 1.0
    out, lse = torch.empty_like(q), torch.empty(1, 1, device=DEV)
    d = szo.make_attn_desc(cache, q, out, torch.tensor([0, 1], dtype=torch.int32, device=DEV), 1, n, drop / 16, lse=lse)
    szo.szo_attn_cached(d, torch.empty(szo.szo_attn_workspace_bytes(d), dtype=torch.uint8, device=DEV))
    rest = (n - 1) * math.exp(-drop)
    # a weight to 2^-11, the output to 2^-11, the sums of 40000 equal terms in chains of some hundreds in fp32
    assert (out.double() - rest / (1 + rest)).abs().max().item() <= (2.0 ** -10 + 2.0 ** -14) * rest / (1 + rest)
    assert abs(lse.item() - (drop + math.log1p(rest))) < 1e-5


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,window", [(64, 0), (96, 700), (128, 0), (128, 40)])
def test_eight_waves_share_a_tile(D, window, kind):
    """Some hundred tiles with a long cache among them: as many workgroups as the chip has CUs, or half."""
    def change(x):
        x[1, 900, 0, 3] = np.nan
        x[0, 1030, 1, 5] = np.nan

    lengths = [1070, 1, 0, 33, 64, 257, 290, 1024, 8, 95]
    b = filled(lengths, 8, D, 64, change=change)
    check(b, lengths, [1] * 10, 4, kind, window=window)
    check(b, lengths, [20, 1, 0, 9, 3, 17, 1, 1, 8, 2], 4, kind, window=window)
    check(b, lengths, [60, 1, 0, 9, 3, 17, 1, 1, 8, 2], 2, kind, causal=False, window=window)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,group,new", [(64, 1, 1), (96, 3, 5), (128, 4, 1), (128, 2, 8), (128, 5, 13), (256, 4, 1), (256, 1, 40)])
def test_many_parts(D, group, new, kind):
    """A long sequence beside short ones: most parts of those hold nothing."""
    lengths = [1601, 5, 130]
    b = filled(lengths, 1, D, 32)
    check(b, lengths, [new, 1, new], group, kind)
    check(b, lengths, [new, 1, new], group, kind, window=100)
    check(b, lengths, [new, 1, new], group, kind, max_len=40000)          # more parts than blocks


def test_hints_of_any_size_choose_among_right_ways():
    lengths = [300, 40, 1, 700]
    b = filled(lengths, 2, 128, 64)
    for hint in (1, 300, 800, 1600, 5000, 33000, 1 << 20, 1 << 30):
        for new in ([1, 1, 1, 1], [5, 2, 1, 9], [100, 40, 1, 90]):
            check(b, lengths, new, 4, "bf16", max_len=hint)
