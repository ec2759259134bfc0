"""Attention over the cache at the ends of its ranges: exponents of values far apart, scores of any size, windows of any size."""
import math

import numpy as np
import pytest
import torch

from paper_2406_02913_amd import szo
from test_gpu_attn_cached import DEV, STORE, TYPES, check, filled

pytestmark = pytest.mark.gpu


def attend(k, v, q, scale, new, causal=True, kind="bf16", max_len=None, page=64):
    """One sequence: k, v fp32 [length, heads, D], the queries q [new, heads * group, D] -> out, lse and what the cache holds, as numpy."""
    n, heads, D = k.shape
    pages = -(-n // page)
    mem = szo.new_kv_cache(pages, page, heads, D)
    lengths = torch.tensor([n], dtype=torch.int32, device=DEV)
    cache = szo.make_kv_cache(*mem, torch.arange(pages, dtype=torch.int32, device=DEV)[None], lengths)
    start = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    szo.szo_kv_cache_write(cache, szo.make_kv_tokens(k.to(DEV), v.to(DEV), start, n))
    held = torch.empty(2, n, heads, D, device=DEV)
    szo.szo_kv_cache_read(cache, szo.make_kv_tokens(held[0], held[1], start, n))
    q = q.to(TYPES[kind]).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    d = szo.make_attn_desc(cache, q, out, torch.tensor([0, new], dtype=torch.int32, device=DEV), new, n if max_len is None else max_len, scale, causal, lse=lse)
    szo.szo_attn_cached(d, torch.full((szo.szo_attn_workspace_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV))
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), held.double().cpu().numpy(), q.double().cpu().numpy()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n,new,max_len", [(33, 1, None), (64, 3, None), (300, 1, None), (300, 40, None), (3000, 1, None), (3000, 20, None), (2500, 1200, None)])
@pytest.mark.parametrize("value,at", [(1e36, 32), (3e38, 0), (1e36, -1), (2.0 ** 90, 35)])
def test_blocks_of_zeros_beside_a_huge_value_count_in_the_sum(value, at, n, new, max_len, D):
    """Equal scores: the output is the huge value over the number of tokens, whatever the exponents of the other blocks are."""
    k, v = torch.zeros(n, 1, D), torch.zeros(n, 1, D)
    at = min(at, n - 1) % n
    v[at] = value
    out, lse, held, _ = attend(k, v, torch.ones(new, 2, D), 1.0, new, max_len=max_len)
    sees = np.arange(n - new + 1, n + 1)
    want = np.where(sees > at, held[1, at, 0, 0] / sees, 0.0)[:, None, None]
    # a weight to fp16 and the output to bf16; the sum of n equal terms in fp32, in chains of at most n / 16 steps with as many roundings
    assert np.all(np.abs(out - want) <= (2.0 ** -8 + 2.0 ** -11 + (n / 16 + 16) * 2.0 ** -24) * want)
    assert np.all(np.abs(lse - np.log(sees)[:, None]) <= (n / 16 + 16) * 2.0 ** -24 + 2.0 ** -22 * np.log(sees)[:, None] + 2.0 ** -21)


def test_exponents_that_fall_and_rise_from_block_to_block():
    """Values from 2^-40 to 2^120 by turns, scores that do not go with them, against the definition: sums of a part's waves and of parts as well."""
    def change(x):
        power = np.random.default_rng(5).integers(-40, 119, x.shape[1] // 32 + 1)
        x[1] = np.clip(x[1], -2, 2) * (2.0 ** power.astype(float))[np.arange(x.shape[1]) // 32][:, None, None]

    for lengths, new in (([700], [1]), ([700], [50]), ([2000, 90], [2, 1]), ([300], [300])):
        b = filled(lengths, 1, 64, 64, seed=sum(lengths), change=change)
        check(b, lengths, new, 2, "bf16")


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("kind,power", [("bf16", 10), ("bf16", 20), ("bf16", 24), ("bf16", 30), ("bf16", 60), ("bf16", 100), ("bf16", 119), ("f16", 24), ("f16", 100)])
@pytest.mark.parametrize("n,new", [(40, 1), (500, 7), (2000, 1), (300, 300)])
def test_scores_of_any_size_that_fp32_holds(n, new, kind, power, sign):
    """Scores j * 2^power, j of 1 to 15, with either sign: the weights stand on the largest that a query sees, and are shared by its equals."""
    rng = np.random.default_rng(n + power)
    j = rng.integers(1, 16, n)
    j[0] = 8
    high = 0 if kind == "bf16" else power - 14
    k, v = torch.zeros(n, 1, 64), torch.from_numpy(rng.integers(-8, 9, (n, 1, 64)).astype(np.float32))       # held exactly
    v *= 2.0 ** (3 * (torch.arange(n) // 32 % 3))[:, None, None]          # equal scores in blocks of different exponents
    k[:, 0, 5] = torch.from_numpy(j * 2.0 ** high).float()
    q = torch.zeros(new, 2, 64)
    q[:, :, 5] = sign * 2.0 ** (power - high)
    out, lse, held, _ = attend(k, v, q, 1.0, new, kind=kind)
    assert np.array_equal(held[1], v.double().numpy()) and np.array_equal(held[0], k.double().numpy())
    for i in range(new):
        see = n - new + i + 1
        s = sign * j[:see] * 2.0 ** power
        w = np.exp(s - s.max())
        want = (w / w.sum()) @ v[:see, 0].double().numpy()
        size = (w / w.sum()) @ np.abs(v[:see, 0].double().numpy())
        rel, floor = STORE[kind]
        # neighbouring scores lie 2^10 apart and more: equal ones have equal weights, each to 2^-11, all others 0
        assert np.all(np.abs(out[i] - want) <= rel * np.abs(want) + floor + (2.0 ** -11 + 2.0 ** -16) * size), (i, s.max())
        # one rounding of the largest score's product by log2(e), of log2(e) itself, and of the way back
        assert np.all(np.abs(lse[i] - (s.max() + math.log(w.sum()))) <= 2.0 ** -21 * abs(s.max()) + 2.0 ** -20)


@pytest.mark.parametrize("scale", [1e4, szo.MOST_SCALE, -szo.MOST_SCALE])
@pytest.mark.parametrize("n,new", [(40, 1), (300, 40)])
def test_scores_of_zero_beside_keys_as_large_as_they_get(n, new, scale):
    """Queries of zeros, and such that see only a zero feature of their keys: equal weights, though scale times the keys' exponent passes fp32."""
    k, v = torch.full((n, 1, 64), 3e38), torch.from_numpy(np.random.default_rng(n).integers(-8, 9, (n, 1, 64)).astype(np.float32))
    k[:, 0, 9] = 0
    q = torch.zeros(new, 2, 64)
    q[:, 1, 9] = 5.0
    out, lse, held, _ = attend(k, v, q, scale, new)
    for i in range(new):
        see = n - new + i + 1
        want, size = held[1][:see, 0].mean(0), np.abs(held[1][:see, 0]).mean(0)
        # equal weights, rounded to bf16; sums of n equal terms
        assert np.all(np.abs(out[i] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -18) * size)
        assert np.all(np.abs(lse[i] - math.log(see)) <= 2.0 ** -19)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 64, 2 ** 30])
@pytest.mark.parametrize("causal", [True, False])
def test_windows_wider_than_any_sequence_hide_nothing(window, causal):
    lengths = [40, 75, 130, 20]
    b = filled(lengths, 2, 64, 64)
    for new in ([1, 1, 1, 1], [40, 9, 130, 20], [40, 33, 50, 1]):
        q = b.rng.standard_normal((sum(new), 4, 64))
        wide = check(b, lengths, new, 2, "bf16", causal, window, q=q)
        assert np.array_equal(wide, check(b, lengths, new, 2, "bf16", causal, 0, q=q))


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 20, 5])
def test_windows_with_more_new_tokens_than_the_length(window):
    b = filled([20, 64], 1, 64, 32)
    check(b, [20, 64], [30, 100], 2, "bf16", True, window)
    check(b, [20, 64], [30, 100], 2, "bf16", False, window)
