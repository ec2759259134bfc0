"""Alternatives of rows with NaN in them, wherever they stand: NaN comes before everything, the lower index first."""
import numpy as np
import pytest
import torch

from test_gpu_token_logprobs import TYPES, check_forward, logits

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,top", [(1, 1), (5, 5), (32, 32), (300, 8), (5000, 20)])
def test_nan_at_the_first_index(V, top, kind):
    x, t = logits(4, V, kind, seed=V)
    x[0, 0] = NAN                                 # alone
    x[1, :] = NAN                                 # a row of them
    x[2, ::2] = NAN
    x[3, 0], x[3, V - 1] = NAN, INF if V > 1 else NAN
    got, _, _ = check_forward(x, t, top)
    assert (got["top_index"][:, 0] == 0).all() and (got["top_index"] >= 0).all()
    assert np.array_equal(got["top_index"][1], np.arange(top))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_nan_at_the_first_index_of_a_row_in_parts(kind):
    x, t = logits(3, 131072, kind, seed=1)
    x[0, 0] = NAN
    x[1, 0], x[1, 70000] = NAN, NAN
    x[2, :] = NAN
    got, _, _ = check_forward(x, t, 6)
    assert got["top_index"][1, :2].tolist() == [0, 70000] and got["top_index"][2].tolist() == list(range(6))
    assert TYPES[kind] == x.dtype
