"""The reference of whole heads against the definition, query by query (no GPU)."""
import numpy as np
import pytest

from attn_reference import attention
from oracle import decoder as od


@pytest.mark.parametrize("n,length", [(1, 1), (3, 7), (9, 9), (12, 8), (4, 0)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 3), (False, 2)])
def test_whole_heads_and_query_by_query(n, length, causal, window):
    rng = np.random.default_rng(n + length)
    q, k, v = rng.standard_normal((n, 4, 8)), rng.standard_normal((length, 2, 8)), rng.standard_normal((length, 2, 8))
    there = rng.random(length) < 0.8
    if length > 5:
        v[5, 1, 3], k[6, 0, 2] = np.nan, np.nan
    got, want = attention(q, k, v, there, length, 0.3, causal, window), od.attention(q, k, v, there, length, 0.3, causal, window)
    for a, b, name in zip(got[:2], want[:2], ("out", "lse")):
        assert np.array_equal(np.isnan(a), np.isnan(b)), name
        fine = np.isfinite(b)
        assert np.allclose(a[fine], b[fine], rtol=1e-12, atol=1e-12) and np.array_equal(a[~fine & ~np.isnan(b)], b[~fine & ~np.isnan(b)]), name
