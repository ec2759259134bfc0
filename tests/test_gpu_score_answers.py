"""The example that runs a decoder's operators together: what it scores at once is what it scores token by token."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import score_answers                                                    # noqa: E402

from oracle import decoder as od                                        # noqa: E402

pytestmark = pytest.mark.gpu


def test_answers_at_once_and_token_by_token():
    r = score_answers.main(["--layers", "2", "--prompts", "3"])
    model, new, had = r["model"], r["new"], r["had"]
    parts, targets = r["fed"].split(new), r["targets"].split(new)
    at_once = r["logp"].split(new)
    # the same tokens one at a time, sequences that are done feeding a token that nobody looks at
    steps = []
    for t in range(max(new)):
        token = torch.stack([p[min(t, len(p) - 1)] for p in parts])
        target = torch.stack([x[t] if t < len(x) else torch.full_like(x[0], -1) for x in targets])
        s = model.hidden_states(token, [1] * len(new), [h + t for h in had])
        steps.append(model.log_probs(s, target)[0])
    for i, n in enumerate(new):
        one = torch.stack([steps[t][i] for t in range(n)])
        # Not the same numbers: an answer's tokens in one block share an exponent that grows with the block when they come one by one, and activations are
        # rounded to bf16 (2^-8) at five places of two blocks; log probabilities of 2000 tokens are about -8
        assert (one - at_once[i]).abs().max().item() < 0.25, (i, one, at_once[i])
    assert abs(r["loss"][0].item() + r["logp"].double().mean().item()) < 0.1
    assert torch.isfinite(r["g"]).all() and r["decoded"].shape == (6, 4)


def test_log_probs_of_the_head_are_those_of_its_logits():
    model = score_answers.Decoder(layers=1, sequences=2)
    s = torch.randn(5, 512, device="cuda")
    t = torch.tensor([1, 5, 1999, -1, 7], dtype=torch.int32, device="cuda")
    logp, entropy, index, loss = model.log_probs(s, t, top=4)
    x = model.head(s).cpu().numpy()
    lp = od.log_probs(x)
    want = np.where(t.cpu().numpy() >= 0, lp[np.arange(5), t.cpu().numpy()], 0)
    assert np.abs(logp.cpu().numpy() - want).max() < 1e-5
    assert np.array_equal(index.cpu().numpy(), od.alternatives(x, 4))
    assert abs(loss.item() + want.sum() / 5) < 1e-5
