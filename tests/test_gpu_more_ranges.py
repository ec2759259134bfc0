"""Offsets beyond 32 bits: rows, pages and strides far apart give what they give side by side."""
import pytest
import torch

from paper_2406_02913_amd import szo

pytestmark = pytest.mark.gpu
DEV = "cuda"


def room(n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("rows,vocab", [(448, 60), (70, 500)])
def test_head_with_rows_as_far_apart_as_they_may_be(rows, vocab):
    far, K = 1 << 22, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(rows, K, device=DEV, generator=g).bfloat16()
    w = torch.randn(vocab, K, device=DEV, generator=g).bfloat16()
    t = torch.randint(vocab, (rows,), device=DEV, generator=g, dtype=torch.int32)
    by = torch.randn(rows, device=DEV, generator=g)

    def apart(v):
        wide = torch.empty((len(v) - 1) * far + K, dtype=v.dtype, device=DEV).as_strided((len(v), K), (far, 1))
        wide.copy_(v)
        return wide

    def run(x, w):
        logp, stats = torch.empty(rows, device=DEV), torch.empty(rows, 2, device=DEV)
        d = szo.make_head_desc(x, w, t, logp, stats)
        szo.szo_head_logprobs(d, room(szo.szo_head_workspace_bytes(d)))
        szo.szo_head_logprobs_bwd(d, by, x, w, room(szo.szo_head_bwd_workspace_bytes(d)))       # in place
        return logp, stats, x, w

    want, got = run(x.clone(), w.clone()), run(apart(x), apart(w))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_block_norm_with_tokens_far_apart():
    H, far = 520, (1 << 31) + 8
    buffer = torch.empty(far + 8 * 1024, dtype=torch.bfloat16, device=DEV)
    at = [buffer[1024 * i:].as_strided((2, H), (far, 1)) for i in range(6)]
    g = torch.Generator(device=DEV).manual_seed(2)
    values = [torch.randn(2, H, device=DEV, generator=g).bfloat16() for _ in range(4)]
    w = torch.randn(H, device=DEV, generator=g)

    def run(y, h, gx, gh, h_out, x_out):
        for to, v in zip((y, h, gx, gh), values):
            to.copy_(v)
        szo.szo_block_norm(szo.make_block_desc(y, h, h_out, x_out, norm=szo.NORM_LAYER, post_weight=w, pre_weight=w))
        d = szo.make_block_desc(y, h, norm=szo.NORM_LAYER, post_weight=w, pre_weight=w)
        sums = [torch.empty(H, device=DEV) for _ in range(2)]
        outs = [h_out.clone(), x_out.clone()]
        szo.szo_block_norm_bwd(d, szo.make_block_grads(d, gx, gh, y, h, post_weight_grad=sums[0], pre_weight_grad=sums[1]), room(szo.szo_block_workspace_bytes(d)))
        return outs + sums + [y, h]

    got = run(*at)
    want = run(*(torch.empty(2, H, dtype=torch.bfloat16, device=DEV) for _ in range(6)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_shared_attention_over_pages_beyond_4_gib():
    heads, D, page, group, B, shared = 2, 128, 64, 4, 12, 192
    lengths = [shared + 3 + 17 * i for i in range(B)]
    per = -(-max(lengths) // page)
    few, many = B * per, (1 << 32) // (page * heads * D) + B * per + 5
    g = torch.Generator().manual_seed(3)
    near = torch.randperm(few, generator=g).view(B, per).to(torch.int32)
    near[:, :shared // page] = near[0, :shared // page]
    table = {few: near, many: near + (many - few)}
    k, v = (torch.randn(sum(lengths), heads, D, generator=g).bfloat16().to(DEV) for _ in range(2))
    q = torch.randn(B, heads * group, D, generator=g).bfloat16().to(DEV)
    start = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).to(DEV)
    for s in range(1, B):                                                # what lies on the same pages is the same
        a, n = int(start[s]), shared
        k[a:a + n], v[a:a + n] = k[:n], v[:n]
    groups = szo.make_attn_groups(ints([0, B]), ints([shared]), B, shared)

    def run(pages):
        memory = szo.new_kv_cache(pages, page, heads, D)
        cache = szo.make_kv_cache(*memory, table[pages].to(DEV), ints(lengths))
        szo.szo_kv_cache_write(cache, szo.make_kv_tokens(k, v, start, max(lengths)))
        out = torch.empty_like(q)
        d = szo.make_attn_desc(cache, q, out, ints(list(range(B + 1))), 1, 1 << 17, D ** -0.5)
        assert szo.szo_attn_shared_plan(d, groups)[0] == 1
        szo.szo_attn_shared(d, groups, room(szo.szo_attn_shared_workspace_bytes(d, groups)))
        return out

    got, want = run(many), run(few)
    assert torch.isfinite(want.float()).all() and torch.equal(got, want)
