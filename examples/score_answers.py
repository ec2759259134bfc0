"""Scores candidate answers, decodes and fine-tunes with a small decoder of sparse int4 linears.

A decoder block's linears are the library's sensitive-sparse int4 layers; between them stand its norms of queries and keys with the rotation,
its 8-bit key/value cache and the attention over it, and behind the head its log probabilities.  Prompts go into the cache once; every candidate
answer is scored behind its prompt by the log probabilities of its tokens, as classification by a language model does; then a few tokens are
decoded greedily, and a zeroth-order step moves the head's sensitive weights by the answers' likelihood.

    python examples/score_answers.py [--layers 2] [--prompts 3]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2406_02913_amd import szo                                    # noqa: E402
from paper_2406_02913_amd.stack import build_linear                     # noqa: E402

DEV = "cuda"


def rms(x):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)


class Linear:
    """A sparse int4 layer for any number of tokens: bf16 in, fp32 out."""

    def __init__(self, seed, N, K, base):
        self.lin = build_linear(seed, 1, N, K, 64, density=1e-3, nnz_base=base, sigma=K ** -0.5)
        self.next_base = base + (self.lin.nnz + 3) // 4 * 4

    def desc(self, x, y):
        w = self.lin
        return szo.make_desc(x.shape[0], w.N, w.K, w.group, w.nnz, w.nnz_base, x, w.qweight, w.scales, w.tile_ptr, w.sp_idx, w.sp_val, y=y)

    def __call__(self, x, sign=0, step=0, eps=0.0):
        x = x.to(torch.bfloat16)
        y = torch.empty(x.shape[0], self.lin.N, device=DEV)
        szo.szo_linear_fwd(self.desc(x, y), 7, step, sign, eps)
        return y


class Decoder:
    def __init__(self, layers=2, hidden=512, q_heads=8, kv_heads=2, head_dim=64, vocab=2000, sequences=6, most=256, page=64):
        self.q_heads, self.kv_heads, self.head_dim, self.vocab = q_heads, kv_heads, head_dim, vocab
        gen = torch.Generator(device=DEV)
        gen.manual_seed(1)
        self.embedding = torch.randn(vocab, hidden, device=DEV, generator=gen)
        base, self.blocks = 0, []
        for layer in range(layers):
            block = {}
            for i, (name, n, k) in enumerate((("q", q_heads * head_dim, hidden), ("k", kv_heads * head_dim, hidden), ("v", kv_heads * head_dim, hidden),
                                              ("o", hidden, q_heads * head_dim))):
                block[name] = Linear(10 * layer + i, n, k, base)
                base = block[name].next_base
            block["q_norm"], block["k_norm"] = (1 + 0.1 * torch.randn(head_dim, device=DEV, generator=gen) for _ in range(2))
            block["memory"] = szo.new_kv_cache(sequences * most // page, page, kv_heads, head_dim)
            self.blocks.append(block)
        self.head = Linear(999, vocab, hidden, base)
        angle = torch.arange(most, device=DEV)[:, None] * 10000.0 ** (-torch.arange(0, head_dim, 2, device=DEV) / head_dim)
        self.cos, self.sin = angle.cos().contiguous(), angle.sin().contiguous()
        # every sequence has its own pages here; a server would hand them out as sequences grow
        self.table = torch.arange(sequences * most // page, dtype=torch.int32, device=DEV).view(sequences, -1)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=DEV)

    def hidden_states(self, tokens, new, had):
        """Appends tokens (i64 [sum(new)], sequence after sequence) behind `had` cached ones of each sequence; their final states."""
        start = torch.tensor([0] + list(new), device=DEV).cumsum(0).to(torch.int32)
        self.lengths.copy_(torch.tensor([h + n for h, n in zip(had, new)], dtype=torch.int32))
        positions = torch.cat([torch.arange(h, h + n, dtype=torch.int32) for h, n in zip(had, new)]).to(DEV)
        T, D, longest = len(tokens), self.head_dim, max(h + n for h, n in zip(had, new))
        x = self.embedding[tokens]
        for block in self.blocks:
            h = rms(x)
            q, k, v = (block[n](h).view(T, -1, D) for n in "qkv")
            q_out, k_out = torch.empty_like(q, dtype=torch.bfloat16), torch.empty_like(k, dtype=torch.bfloat16)
            szo.szo_qk_norm_rope(szo.make_qk_desc(q, k, positions, self.cos, self.sin, q_out, k_out, q_weight=block["q_norm"], k_weight=block["k_norm"]))
            cache = szo.make_kv_cache(*block["memory"], self.table, self.lengths)
            szo.szo_kv_cache_write(cache, szo.make_kv_tokens(k_out, v.to(torch.bfloat16), start, max(new)))
            out = torch.empty_like(q_out)
            attn = szo.make_attn_desc(cache, q_out, out, start, max(new), longest, D ** -0.5)
            szo.szo_attn_cached(attn, torch.empty(szo.szo_attn_workspace_bytes(attn), dtype=torch.uint8, device=DEV))
            x = x + block["o"](out.view(T, -1))
        return rms(x)

    def log_probs(self, states, targets, top=0, **perturbed):
        """Log probabilities of targets, their entropy, and the best `top` tokens."""
        logits, R = self.head(states, **perturbed), len(states)
        logp, entropy = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
        index = torch.empty(R, top, dtype=torch.int32, device=DEV) if top else None
        loss = torch.zeros(1, dtype=torch.float64, device=DEV)
        d = szo.make_logprobs_desc(logits, targets, logp, entropy, top_index=index, loss_acc=loss, loss_scale=1.0 / max(1, R))
        szo.szo_token_logprobs(d, torch.empty(szo.szo_logprobs_workspace_bytes(d), dtype=torch.uint8, device=DEV))
        return logp, entropy, index, loss


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--prompts", type=int, default=3)
    args = ap.parse_args(argv)
    n = args.prompts
    model = Decoder(layers=args.layers, sequences=2 * n)
    gen = torch.Generator().manual_seed(3)
    # two candidates for every prompt: sequences 2 i and 2 i + 1 hold prompt i
    prompts = [torch.randint(model.vocab, (int(torch.randint(5, 90, (1,), generator=gen)),), generator=gen) for _ in range(n) for _ in range(2)]
    for i in range(n):
        prompts[2 * i + 1] = prompts[2 * i]
    answers = [torch.randint(model.vocab, (int(torch.randint(1, 9, (1,), generator=gen)),), generator=gen) for _ in range(2 * n)]

    # the prompts without their last token go into the cache; that token and the answer are what is scored
    had = [len(p) - 1 for p in prompts]
    model.hidden_states(torch.cat([p[:-1] for p in prompts]).to(DEV), had, [0] * len(had))
    new = [len(a) for a in answers]
    fed = torch.cat([torch.cat([p[-1:], a[:-1]]) for p, a in zip(prompts, answers)]).to(DEV)
    targets = torch.cat(answers).to(torch.int32).to(DEV)
    states = model.hidden_states(fed, new, had)
    logp, entropy, _, _ = model.log_probs(states, targets)
    scores = [s.mean().item() for s in logp.split(new)]
    for i in range(n):
        better = max((0, 1), key=lambda c: scores[2 * i + c])
        print(f"prompt of {len(prompts[2 * i])} tokens: candidates {scores[2 * i]:.3f} {scores[2 * i + 1]:.3f} -> {better}")

    # greedy decoding behind the prompts: one token of every sequence at a time
    token, decoded = torch.stack([p[-1] for p in prompts]).to(DEV), []
    ones = [1] * len(had)
    for t in range(4):
        s = model.hidden_states(token, ones, [h + t for h in had])
        _, _, best, _ = model.log_probs(s, torch.full((len(had),), -1, dtype=torch.int32, device=DEV), top=3)
        token = best[:, 0].long()
        decoded.append(token)
    print("decoded:", torch.stack(decoded, 1).tolist())

    # a zeroth-order step of the head by the answers' negative log likelihood
    eps, lr, before = 1e-3, 1e-3, model.head.lin.sp_val.clone()
    loss = [model.log_probs(states, targets, sign=sign, step=0, eps=eps)[3] for sign in (1, -1)]
    g = torch.zeros(1, dtype=torch.float64, device=DEV)
    szo.szo_spsa_g(loss[0], loss[1], eps, g)
    w = model.head.lin
    szo.szo_sparse_update(w.sp_val, None, w.nnz, w.nnz_base, 7, 0, g, lr)
    print(f"zeroth-order step: loss {loss[0].item():.6f} {loss[1].item():.6f}, g {g.item():.4f}, "
          f"{(w.sp_val != before).sum().item()} of {w.nnz} sensitive weights moved")
    return dict(scores=scores, logp=logp, entropy=entropy, decoded=torch.stack(decoded, 1), fed=fed, new=new, had=had, targets=targets, model=model, loss=loss, g=g)


if __name__ == "__main__":
    main()
