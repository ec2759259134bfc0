"""Norms around blocks, attention behind shared prefixes and the head's log probabilities as a user runs them together: forward, gradients, in a graph, on a stream."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import score_answers                                                    # noqa: E402

from paper_2406_02913_amd import szo                                    # noqa: E402

pytestmark = pytest.mark.gpu
BF = 2.0 ** -8                                                          # a rounding to bf16, relative


def room(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def inputs(T, H, V, seed):
    g = torch.Generator().manual_seed(seed)
    def rand(*shape):
        return torch.randn(*shape, generator=g, dtype=torch.float64)
    y, h = rand(T, H).bfloat16(), rand(T, H).bfloat16()
    post, pre, gate = (1 + 0.1 * rand(H)).float(), (1 + 0.1 * rand(H)).float(), (0.5 + 0.1 * rand(H)).float()
    w = (rand(V, H) * H ** -0.5).bfloat16()
    t = torch.randint(V, (T,), generator=g, dtype=torch.int32)
    t[::5] = -1
    return y, h, post, pre, gate, w, t


class Run:
    """The last block's output, final norm, head and loss, and the way back to the block."""

    def __init__(self, T, H, V, seed):
        y, h, post, pre, gate, w, t = (x.cuda() for x in inputs(T, H, V, seed))
        self.x, self.h_out = torch.empty_like(y), torch.empty_like(h)
        self.logp, self.stats = torch.empty(T, device="cuda"), torch.empty(T, 2, device="cuda")
        self.loss = torch.zeros(1, dtype=torch.float64, device="cuda")
        self.by_logp = torch.full((T,), -1.0, device="cuda")
        self.by_x, self.by_w = torch.empty_like(self.x), torch.empty_like(w)
        self.by_y, self.by_h = torch.empty_like(y), torch.empty_like(h)
        self.by_gate, self.by_post, self.by_pre = (torch.empty(H, device="cuda") for _ in range(3))
        self.norm = szo.make_block_desc(y, h, self.h_out, self.x, post_weight=post, gate=gate, pre_weight=pre)
        self.head = szo.make_head_desc(self.x, w, t, self.logp, self.stats, loss_acc=self.loss)
        self.grads = szo.make_block_grads(self.norm, self.by_x, None, self.by_y, self.by_h, self.by_gate, self.by_post, None, self.by_pre)
        self.rooms = (room(szo.szo_head_workspace_bytes(self.head)), room(szo.szo_head_bwd_workspace_bytes(self.head)), room(szo.szo_block_workspace_bytes(self.norm)))

    def __call__(self, stream=None):
        s = stream
        szo.szo_block_norm(self.norm, stream=s)
        szo.szo_head_logprobs(self.head, self.rooms[0], stream=s)
        szo.szo_head_logprobs_bwd(self.head, self.by_logp, self.by_x, self.by_w, self.rooms[1], stream=s)
        szo.szo_block_norm_bwd(self.norm, self.grads, self.rooms[2], stream=s)

    def outputs(self):
        return [self.x, self.h_out, self.logp, self.by_x, self.by_w, self.by_y, self.by_h, self.by_gate, self.by_post, self.by_pre]


def gradients(T, H, V, seed):
    y, h, post, pre, gate, w, t = inputs(T, H, V, seed)
    leaves = [v.double().requires_grad_() for v in (y, h, gate, post, pre, w)]
    y, h, gate, post, pre, w = leaves
    def rms(v, f):
        return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-6) * f
    x = rms(h + gate * rms(y, post), pre)
    keep = t >= 0
    logp = torch.where(keep, (x @ w.T).log_softmax(-1).gather(1, t.clamp(min=0).long()[:, None])[:, 0], 0.0)
    (-logp.sum()).backward()
    return logp.detach(), [v.grad for v in leaves]


def relative(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


SIZES = [(1, 64, 50, 1), (7, 192, 1000, 2), (40, 512, 777, 3), (300, 1024, 5000, 4)]


@pytest.mark.parametrize("T,H,V,seed", SIZES)
def test_loss_and_gradients_through_head_and_norms(T, H, V, seed):
    r = Run(T, H, V, seed)
    r()
    logp, (by_y, by_h, by_gate, by_post, by_pre, by_w) = gradients(T, H, V, seed)
    # x is rounded to bf16: H terms of size |x w| BF with signs at random make a logit's error BF |x| |w| / sqrt(3) or so, |w| = 1 at |x| = 1 here: five times that is as far as it comes
    assert (r.logp.cpu().double() - logp).abs().max().item() < 5 * BF * 1.3
    if T == 1:                                                           # the one target is ignored: no gradients at all
        assert r.loss.item() == 0 and all((v == 0).all() for v in (r.by_w, r.by_y, r.by_h, r.by_gate, r.by_post, r.by_pre))
        return
    assert abs(r.loss.item() + logp.sum().item()) < 5 * BF * 1.3 * T ** 0.5 * 2
    # relative to the whole gradient: x, the gradient by logits and by x are rounded to bf16 on the way, and the result, each by BF at most; a changed logit moves p by as much again
    for name, got, want in (("w", r.by_w, by_w), ("y", r.by_y, by_y), ("h", r.by_h, by_h), ("gate", r.by_gate, by_gate), ("post", r.by_post, by_post), ("pre", r.by_pre, by_pre)):
        assert relative(got, want) < 5 * BF, (name, relative(got, want))


def test_captured_beside_an_eager_run_of_the_same():
    r = Run(40, 512, 777, 3)
    r()
    torch.cuda.synchronize()
    want = [v.clone() for v in r.outputs()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r()
    for k in range(4):
        for v in r.outputs():
            v.zero_()
        r.loss.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(r.outputs(), want)), k
        loss = r.loss.item()
        assert abs(loss + want[2].double().sum().item()) < 1e-4 * abs(loss), k
        Run(7, 192, 1000, 2)()


def test_runs_on_several_streams_at_once():
    runs = [Run(*size) for size in SIZES[1:]]
    for r in runs:
        r()
    torch.cuda.synchronize()
    want = [[v.clone() for v in r.outputs()] for r in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    for r in runs:
        for v in r.outputs():
            v.zero_()
    torch.cuda.synchronize()
    for k in range(3):
        for r, s in zip(runs, streams):
            r(stream=s)
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        assert all(torch.equal(a, b) for a, b in zip(r.outputs(), w))


def test_candidates_behind_shared_pages_are_those_behind_their_own():
    """A decoder's states behind prompts on shared pages and on pages of each sequence."""
    def states(together):
        model = score_answers.Decoder(layers=2, sequences=4, most=128)
        g = torch.Generator().manual_seed(5)
        prompts = [torch.randint(model.vocab, (n,), generator=g) for n in (70, 33)]
        had, answers = [70, 70, 33, 33], torch.randint(model.vocab, (10,), generator=g).cuda()
        if together:
            model.hidden_states(torch.cat(prompts).cuda(), [70, 0, 33, 0], [0] * 4)
            shared = model.share([70, 33], 2)
            assert shared == [64, 32]
            model.hidden_states(torch.cat([p[s:] for p, s in zip(prompts, shared)]).cuda(), [0, 6, 0, 1], [70, 64, 33, 32])
        else:
            model.hidden_states(torch.cat([prompts[0], prompts[0], prompts[1], prompts[1]]).cuda(), had, [0] * 4)
        return model.hidden_states(answers, [3, 1, 2, 4], had).float()
    a, b = states(True), states(False)
    # the second candidate's last tokens of a prompt go through blocks of fewer tokens, whose exponent is theirs, and sums have another order: roundings to bf16 and 8 bits on the way
    assert relative(a, b.double().cpu()) < 0.05


def test_example_shares_the_pages_of_a_prompt():
    r = score_answers.main(["--layers", "1", "--prompts", "3"])
    model = r["model"]
    filled = [h // model.page for h in r["had"]]
    assert max(filled) > 0
    for i in range(0, 6, 2):
        a, b = model.table[i].tolist(), model.table[i + 1].tolist()
        assert a[:filled[i]] == b[:filled[i]] and not set(a[filled[i]:]) & set(b[filled[i]:])
