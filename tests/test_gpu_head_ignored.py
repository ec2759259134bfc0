"""Rows of a head that have no target: gradient 0 whatever the weight holds."""
import pytest
import torch

from paper_2406_02913_amd import szo
from test_gpu_head import _room, _setup, forward

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(20, 900), (300, 900), (20, 9000), (300, 40000)])
def test_rows_without_a_target_have_gradient_0_beside_a_weight_that_is_not_finite(rows, vocab, kind):
    x, w, t, _ = _setup(rows, vocab, 128, kind)
    w[5, 7], w[11, 9], w[12, 9] = float("nan"), float("inf"), float("-inf")
    t[::3] = -1
    t[1] = vocab
    _, stats = forward(x, w, t)
    d = szo.make_head_desc(x, w, t, stats=stats)
    gx = torch.full_like(x, 7.0)
    szo.szo_head_logprobs_bwd(d, torch.randn(rows, device=DEV), gx, None, _room(szo.szo_head_bwd_workspace_bytes(d)))
    none = [i for i in range(rows) if i % 3 == 0 or i == 1]
    assert (gx[none] == 0).all() and torch.isnan(gx[2]).any()
