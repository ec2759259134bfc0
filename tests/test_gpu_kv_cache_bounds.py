"""What the cache's calls do where token_start and the tensors of tokens do not agree: rows that the tensors do not have are neither read nor written."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2406_02913_amd import szo
from test_gpu_kv_cache import TYPES, Both

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("D,heads", [(64, 2), (128, 1)])
@pytest.mark.parametrize("start,lengths", [([0, 20, 45], [20, 25]), ([-5, 20, 30], [20, 33]), ([0, 50, 60], [90, 40]), ([0, 2 ** 31 - 1, 2 ** 31 - 1], [30, 7]),
                                           ([-2 ** 31, -7, 12], [5, 40]), ([20, 5, 30], [50, 50]), ([25, 2 ** 31 - 1, -2 ** 31], [64, 64])])
def test_rows_beyond_the_tensors_are_left_out(start, lengths, D, heads, kind):
    """30 rows in the middle of a larger buffer whose other rows stay as they are; the calls go by what lies in [0, 30)."""
    tokens, dtype = 30, TYPES[kind]
    b = Both([100, 100], heads, D, 64)
    wide = torch.full((2, tokens + 200, heads, D), float("nan"), dtype=dtype, device=DEV)
    x = torch.from_numpy(b.rng.standard_normal((2, tokens, heads, D))).to(dtype)
    wide[:, 100:100 + tokens] = x.to(DEV)
    new = wide[:, 100:100 + tokens]
    b.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    on = torch.tensor(start, dtype=torch.int32, device=DEV)
    szo.szo_kv_cache_write(b.cache(), szo.make_kv_tokens(new[0], new[1], on, 200))
    rows = [(max(a, 0), max(min(z, tokens), 0)) for a, z in zip(start, start[1:])]
    for s, (lo, hi) in enumerate(rows):
        if lo < hi:
            for i in range(2):
                od.cache_write(b.codes[i], b.exps[i], bool(i), b.table[s:s + 1], lengths[s:s + 1], [lo, hi], x[i].float().numpy())
    b.same()
    wide.fill_(7)
    szo.szo_kv_cache_read(b.cache(), szo.make_kv_tokens(new[0], new[1], on, 200))
    want = torch.full((2, tokens, heads, D), 7.0, dtype=dtype)
    for s, (lo, hi) in enumerate(rows):
        for i in range(2):
            dense, _ = od.cache_dense(b.codes[i], b.exps[i], bool(i), b.table, lengths, s)
            for row in range(lo, hi):
                at = lengths[s] - (hi - row)
                if at >= 0:
                    want[i, row] = torch.from_numpy(dense[at]).to(dtype)
    got = wide.cpu()
    assert (got[:, :100] == 7).all() and (got[:, 100 + tokens:] == 7).all()
    assert np.array_equal(got[:, 100:100 + tokens].float().numpy(), want.float().numpy())
