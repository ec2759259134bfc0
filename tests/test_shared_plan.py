"""Which batches go over a shared prefix together, and how their tiles are counted: on the host, no kernel is launched."""
import ctypes as C

import pytest

from paper_2406_02913_amd import szo

P = 0x10000                                    # never dereferenced


def plan(groups, sequences, prefix, own, new=1, window=0, heads=8, group=4, D=128, most=None, tokens=None):
    """Groups of equally many sequences; at most `own` tokens of a sequence's own."""
    cache = szo.KvCache(pages=1000, page_tokens=32, kv_heads=heads, head_dim=D, sequences=sequences, max_pages=1000, k=P, v=P, k_exp=P, v_exp=P, page_table=P, lengths=P)
    d = szo.AttnDesc(cache=cache, q_heads=heads * group, type=szo.BF16, causal=1, window=window, scale=1.0, max_q=new, max_len=prefix + own, tokens=sequences * new if tokens is None else tokens, q=P, out=P,
                     q_start=P, q_token_stride=heads * group * D, q_head_stride=D, out_token_stride=heads * group * D, out_head_stride=D)
    g = szo.AttnGroups(groups=groups, max_sequences=sequences // groups if most is None else most, max_shared=prefix, group_start=P, shared=P)
    return szo.szo_attn_shared_plan(d, g)


@pytest.mark.parametrize("prefix", [1024, 4096])
def test_groups_of_one_have_nothing_to_share(prefix):
    assert plan(64, 64, prefix, 100) == (0, 0, 0, 0) and plan(1, 64, prefix, 100, most=0) == (0, 0, 0, 0)
    assert plan(32, 64, prefix, 100)[0] == 1


def test_a_window_that_has_left_the_prefix():
    assert plan(1, 64, 8192, 200)[0] == plan(1, 64, 8192, 200, window=1024)[0] == 1
    assert plan(1, 64, 8192, 200, window=100) == (0, 0, 0, 0)                # half of the own tokens are as many
    assert plan(1, 64, 8192, 2000, window=1024) == (0, 0, 0, 0)
    assert plan(1, 64, 8192, 60, window=31) == (0, 0, 0, 0)
    assert plan(1, 64, 1024, 100, window=(1 << 31) - 1)[0] == 1


def test_sequences_that_fill_tiles_by_themselves():
    assert plan(1, 64, 1000, 500, new=64)[0] == 1
    assert plan(1, 64, 1000, 500, new=65) == (0, 0, 0, 0) and plan(1, 64, 1000, 500, new=500) == (0, 0, 0, 0)
    assert plan(1, 64, 1000, 500, new=500, tokens=563)[0] == 1               # one long prompt beside 63 continuations


def test_every_group_has_a_tile():
    """64 groups of four sequences are 512 tiles for eight key heads, which fill the chip's waves without parts: 256 rows alone would be 64 tiles."""
    for groups, sequences, parts in ((64, 256, 1), (32, 64, 1), (16, 64, 2), (8, 64, 4), (1, 64, 4)):
        assert plan(groups, sequences, 1024, 100)[3] == parts, groups


def test_more_tiles_than_a_launch_that_joins_their_parts_can_count():
    """Threads of a launch are counted in 32 bits: eight workgroups of 256 join a tile's parts at a head dimension of 256."""
    def call(groups):
        cache = szo.KvCache(pages=1000, page_tokens=32, kv_heads=1, head_dim=256, sequences=128, max_pages=1000, k=P, v=P, k_exp=P, v_exp=P, page_table=P, lengths=P)
        d = szo.AttnDesc(cache=cache, q_heads=1, type=szo.BF16, causal=1, scale=1.0, max_q=1, max_len=1 << 20, tokens=128, q=P, out=P, q_start=P, q_token_stride=256, q_head_stride=256,
                         out_token_stride=256, out_head_stride=256)
        plan = (C.c_int32 * 4)()
        return szo.lib.szo_attn_shared_plan(C.byref(d), C.byref(szo.AttnGroups(groups=groups, max_sequences=2, max_shared=64, group_start=P, shared=P)), plan), plan[3]

    least = (1 << 32) // (256 * 8) - 128 // 32 - 2                           # tiles: of the rows, and two besides those of the groups
    assert call(least - 1) == (szo.OK, 2)
    assert call(least)[0] == szo.EUNSUPPORTED
