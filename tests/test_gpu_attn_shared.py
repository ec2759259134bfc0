"""Attention of sequences that share prefixes, against the 64-bit definition on the same codes: what the call says must be what each sequence by itself gives."""
import numpy as np
import pytest
import torch

from paper_2406_02913_amd import szo
import test_gpu_attn_cached as one

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Shared:
    """A cache whose groups' sequences name the same pages for their first shared[g] tokens."""

    def __init__(self, lengths, starts, shared, heads, D, page, seed=0, change=None):
        self.b, self.starts, self.shared = one.filled(lengths, heads, D, page, seed, change), starts, shared
        for g, n in enumerate(shared):
            first, pages = starts[g], n // page
            for s in range(first, starts[g + 1]):
                self.b.table[s, :pages] = self.b.table[first, :pages]

    def check(self, monkeypatch, lengths, new, group, kind, max_sequences=None, max_shared=None, max_len=1 << 17, plan=None, **kw):
        """max_len: a hint; one as large as this makes small batches go together, in many parts."""
        def call(d, room):
            if plan is not None:
                plan.append(szo.szo_attn_shared_plan(d, groups))
            szo.szo_attn_shared(d, groups, room)

        groups = szo.make_attn_groups(ints(self.starts), ints(self.shared), max_sequences or max(b - a for a, b in zip(self.starts, self.starts[1:])),
                                      max(self.shared) if max_shared is None else max_shared)
        with monkeypatch.context() as m:
            m.setattr(szo, "szo_attn_workspace_bytes", lambda d: szo.szo_attn_shared_workspace_bytes(d, groups))
            m.setattr(szo, "szo_attn_cached", call)
            return one.check(self.b, lengths, new, group, kind, max_len=max_len, **kw)


# lengths, groups of sequences, shared tokens
SIZES = [([97, 130, 65, 64], [0, 4], [64]), ([70, 300, 290, 40, 33, 200, 199, 198], [0, 1, 3, 5, 8], [64, 256, 32, 192]), ([513], [0, 1], [512]),
         ([1030, 1024, 1100], [0, 3], [1024])]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,group", [(64, 2, 1), (96, 1, 3), (128, 2, 4), (128, 1, 7), (256, 1, 2)])
@pytest.mark.parametrize("lengths,starts,shared", SIZES)
def test_one_token_each(monkeypatch, lengths, starts, shared, D, heads, group, kind):
    Shared(lengths, starts, shared, heads, D, 32).check(monkeypatch, lengths, [1] * len(lengths), group, kind)


@pytest.mark.parametrize("D,heads,group,kind", [(64, 1, 4, "bf16"), (128, 2, 4, "f16"), (96, 2, 1, "bf16"), (256, 1, 5, "bf16")])
def test_answers_of_several_tokens(monkeypatch, D, heads, group, kind):
    lengths, starts, shared = [97, 130, 70, 64, 400, 420], [0, 4, 6], [64, 384]
    s = Shared(lengths, starts, shared, heads, D, 64)
    s.check(monkeypatch, lengths, [33, 60, 0, 1, 16, 30], group, kind, layout="odd")
    s.check(monkeypatch, lengths, [1, 2, 3, 4, 5, 6], group, kind, lse_too=False)


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 20), (True, 33), (True, 64), (True, 150), (True, 1000), (False, 40)])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 9, 30], [90, 70, 66]])
def test_masks_that_end_inside_the_prefix(monkeypatch, causal, window, new):
    """The last of these begin before the prefix ends: their first queries see a part of it."""
    lengths = [130, 100, 131]
    Shared(lengths, [0, 3], [96], 1, 64, 32).check(monkeypatch, lengths, new, 2, "bf16", causal=causal, window=window)


def test_prefixes_that_are_no_whole_blocks_or_longer_than_a_sequence(monkeypatch):
    lengths = [130, 100, 131, 20]
    s = Shared(lengths, [0, 3, 4], [96, 0], 1, 64, 32)
    for shared in ([95, 0], [97, 0], [64, 31], [33, 500], [-5, 7], [96, -2147483648]):
        s.shared = shared
        s.check(monkeypatch, lengths, [1, 4, 2, 20], 2, "bf16", max_shared=128)
    # shorter than what the group shares: its own length holds
    s = Shared([130, 131, 64], [0, 3], [96], 1, 64, 32)
    s.b.lengths.zero_()
    s.check(monkeypatch, [130, 131, 50], [1, 1, 2], 2, "bf16")
    s.check(monkeypatch, [130, 131, 0], [1, 1, 2], 2, "bf16")


def test_sequences_of_no_group_and_groups_without_any(monkeypatch):
    lengths = [130, 100, 131, 77, 40]
    s = Shared(lengths, [1, 3], [96], 1, 128, 32)
    s.check(monkeypatch, lengths, [1, 3, 2, 5, 1], 4, "bf16")
    s = Shared(lengths, [0, 0, 2, 2, 5, 5], [64, 96, 32, 32, 0], 1, 128, 32)
    s.check(monkeypatch, lengths, [1, 3, 2, 5, 1], 4, "bf16")
    s.check(monkeypatch, lengths, [0, 0, 0, 0, 1], 4, "bf16")


def test_hints_that_are_too_small(monkeypatch):
    """Rows without a place beside the others go by themselves; a prefix counts up to what the hint says."""
    lengths = [130, 100, 131, 98, 120]
    s = Shared(lengths, [0, 5], [96], 2, 64, 32)
    for most in (1, 2, 4):
        s.check(monkeypatch, lengths, [1, 4, 1, 3, 4], 4, "bf16", max_sequences=most)
    for most in (0, 31, 32, 70):
        s.check(monkeypatch, lengths, [1, 4, 1, 3, 4], 4, "bf16", max_shared=most)


def test_more_groups_and_sequences_than_a_wave_has_lanes(monkeypatch):
    rng = np.random.default_rng(2)
    lengths = [32 + int(n) for n in rng.integers(1, 40, 150)]
    starts = [0] + sorted(rng.choice(np.arange(1, 150), 79, replace=False).tolist()) + [150]
    Shared(lengths, starts, [32] * 80, 1, 64, 32).check(monkeypatch, lengths, [1] * 150, 3, "bf16")
    Shared(lengths, [0, 150], [32], 1, 64, 32).check(monkeypatch, lengths, [1 if i % 3 else 0 for i in range(150)], 1, "bf16")


# head_dim, key heads, group, sequences, new tokens of each, hint of lengths -> what the plan says
WAYS = [(64, 8, 2, 70, 60, 200, (1, 4, 1, 1)), (64, 8, 2, 80, 60, 1 << 17, (1, 1, 4, 1)),                 # tiles side by side
        (128, 8, 4, 70, 60, 200, (1, 4, 1, 1)), (256, 8, 2, 70, 61, 200, (1, 4, 1, 1)),
        (128, 8, 4, 40, 10, 1 << 17, (1, 1, 4, 1)),                  # four waves a tile, whole
        (128, 4, 4, 64, 1, 1 << 17, (1, 1, 8, 8)),                   # eight, in parts
        (96, 16, 2, 256, 1, 2000, (1, 1, 8, 1)), (64, 8, 4, 256, 1, 3000, (1, 1, 8, 1)),            # eight, whole
        (64, 8, 1, 64, 1, 200, (1, 1, 4, 24)), (256, 2, 2, 64, 1, 600, (1, 1, 4, 32)), (96, 2, 3, 40, 1, 2400, (1, 1, 8, 42)),
        (64, 1, 2, 5, 1, 200, (0, 0, 0, 0))]                          # each by itself


@pytest.mark.parametrize("D,heads,group,sequences,new,hint,want", WAYS)
def test_every_way_that_sizes_choose(monkeypatch, D, heads, group, sequences, new, hint, want):
    """With groups that end inside tiles and lengths on both sides of a block's end."""
    third = sequences // 3
    lengths = [64 + new + i * 7 % 40 for i in range(third)] + [32 + new + i * 5 % 37 for i in range(third, sequences)]
    many = [max(1, new - i % 4) for i in range(sequences)]
    plan = []
    Shared(lengths, [0, third, sequences], [64, 32], heads, D, 32).check(monkeypatch, lengths, many, group, "bf16", max_len=hint, plan=plan)
    assert plan == [want]


def test_pages_that_are_not_there_and_nan(monkeypatch):
    lengths = [130, 100, 131]

    def change(x):
        x[1, 50, 0, 3] = np.nan                                  # a value of the first sequence's prefix: everybody's
        x[0, 130 + 98, 0, 7] = np.inf                            # a key of the second one's own

    s = Shared(lengths, [0, 3], [96], 1, 64, 32, change=change)
    got = s.check(monkeypatch, lengths, [3, 3, 3], 1, "bf16")
    assert np.isnan(got[:, 0, 3]).all() and np.isfinite(got[[0, 1, 2, 6, 7, 8], 0, :3]).all()
    s = Shared(lengths, [0, 3], [96], 1, 64, 32)
    s.b.table[:, 1] = -1                                         # nothing is there for anybody
    s.b.table[2, 4] = 1 << 30
    s.check(monkeypatch, lengths, [3, 1, 3], 2, "bf16")


def _plain(seed=5, B=6, D=128, heads=2, group=4, pre=256):
    torch.manual_seed(seed)
    lengths = [pre + 5 + 13 * i for i in range(B)]
    s = Shared(lengths, [0, B], [pre], heads, D, 32, seed)
    s.b.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    q = torch.randn(B, heads * group, D, device=DEV).bfloat16()
    groups = szo.make_attn_groups(ints([0, B]), ints([pre]), B, pre)

    def call():
        out, lse = torch.full_like(q, 3.0), torch.full(q.shape[:2], 3.0, device=DEV)
        d = szo.make_attn_desc(s.b.cache(), q, out, ints(list(range(B + 1))), 1, 1 << 17, D ** -0.5, lse=lse)
        room = torch.empty(szo.szo_attn_shared_workspace_bytes(d, groups), dtype=torch.uint8, device=DEV)
        return (out, lse), lambda: szo.szo_attn_shared(d, groups, room)

    return s, q, groups, lengths, call


def test_a_group_whose_first_sequence_is_done(monkeypatch):
    """It has no new tokens, and its pages are somebody else's or nobody's by now."""
    lengths = [300, 290, 310, 275, 260, 333]
    s = Shared(lengths, [0, 3, 6], [256, 224], 2, 128, 32)
    s.b.table[0], s.b.table[3] = -1, np.roll(s.b.table[4], 3)
    s.check(monkeypatch, [0] + lengths[1:3] + [64] + lengths[4:], [0, 1, 2, 0, 3, 1], 4, "bf16")


def test_queries_left_out_and_rows_behind_the_last_sequence_stay_as_they_are():
    s, q, groups, lengths, _ = _plain()
    q = torch.randn(20, 8, 128, device=DEV).bfloat16()
    out = torch.full_like(q, 3.0)
    start = [0, 3, 4, 9, 10, 11, 12]
    d = szo.make_attn_desc(s.b.cache(), q, out, ints(start), 2, 1 << 17, 128 ** -0.5)            # two queries of a sequence at most
    szo.szo_attn_shared(d, groups, torch.empty(szo.szo_attn_shared_workspace_bytes(d, groups), dtype=torch.uint8, device=DEV))
    left = [2, 6, 7, 8] + list(range(12, 20))
    assert (out[left] == 3).all()
    want = torch.full_like(q, 3.0)
    d = szo.make_attn_desc(s.b.cache(), q, want, ints(start), 2, max(lengths), 128 ** -0.5)
    szo.szo_attn_cached(d, torch.empty(szo.szo_attn_workspace_bytes(d), dtype=torch.uint8, device=DEV))
    assert torch.allclose(out.float(), want.float(), rtol=2.0 ** -7, atol=2.0 ** -7)             # two roundings, weights of 11 bits


def test_captured_and_replayed_with_sequences_that_grow():
    s, q, groups, lengths, call = _plain()
    (out, lse), run = call()
    graph = torch.cuda.CUDAGraph()
    run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run()
    for step in range(4):
        s.b.lengths.copy_(torch.tensor([n - step for n in lengths], dtype=torch.int32))
        out.fill_(9.0)
        graph.replay()
        (want, want_lse), eager = call()
        eager()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_two_calls_at_once_on_two_streams():
    _, _, _, _, call = _plain()
    (want, _), run = call()
    run()
    torch.cuda.synchronize()
    calls = [(torch.cuda.Stream(), call()) for _ in range(2)]
    for _ in range(5):
        for stream, (_, go) in calls:
            with torch.cuda.stream(stream):
                go()
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for _, ((out, _), _) in calls)
