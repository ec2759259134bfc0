"""Sequences that share a prefix and name its pages only where they see them: pages behind a sequence's length, or that its window has left, need not be there."""
import functools

import numpy as np
import pytest
import torch

from oracle import decoder as od
from test_gpu_attn_shared import Shared

pytestmark = pytest.mark.gpu
PAGE = 32


def leave(s, lengths, new, window, page=PAGE):
    """Takes away every page of which a sequence's queries see no token."""
    for i, (n, m) in enumerate(zip(lengths, new)):
        s.b.table[i, -(-n // page):] = -1
        if window:
            s.b.table[i, :max(0, n - m - window + 1) // page] = -1


# lengths, shared, new tokens, window
CASES = [([50, 131, 130], 96, [1, 1, 1], 0),                  # the first sequence ends inside the prefix
         ([131, 50, 130], 96, [3, 2, 4], 0),
         ([400, 270, 300], 256, [1, 1, 1], 100),              # the first one's window has left the prefix, others see its end
         ([230, 300, 260], 256, [1, 1, 1], 64),               # none sees all of it that the others see
         ([300, 230, 40, 260], 256, [1, 5, 3, 2], 90),
         ([64, 33, 96, 65, 131], 96, [1, 2, 1, 3, 2], 50),
         ([600, 520, 290, 40, 1, 450], 512, [20, 40, 7, 9, 1, 11], 200)]


@pytest.mark.parametrize("hint", [600, 1 << 17])
@pytest.mark.parametrize("D,heads,group,kind", [(64, 1, 1, "bf16"), (128, 2, 4, "f16"), (256, 1, 2, "bf16")])
@pytest.mark.parametrize("lengths,shared,new,window", CASES)
def test_pages_are_read_from_a_sequence_that_sees_them(monkeypatch, lengths, shared, new, window, D, heads, group, kind, hint):
    s = Shared(lengths, [0, len(lengths)], [shared], heads, D, PAGE)
    leave(s, lengths, new, window)
    s.check(monkeypatch, lengths, new, group, kind, window=window, max_len=hint)


@pytest.mark.parametrize("page", [64, 96])
def test_pages_of_several_blocks(monkeypatch, page):
    lengths, new = [700, 390, 200, 480, 100], [2, 1, 3, 1, 1]
    s = Shared(lengths, [0, 5], [384], 2, 64, page)
    leave(s, lengths, new, 150, page)
    s.check(monkeypatch, lengths, new, 4, "bf16", window=150)


@functools.lru_cache(maxsize=1)
def _many(sequences, D, heads):
    """Lengths from inside the prefix to far behind it, so that most tiles have sequences that see other pages than the next."""
    lengths = [61 + i * 37 % 230 for i in range(sequences)]
    return lengths, Shared(lengths, [0, sequences], [128], heads, D, PAGE)


def many(monkeypatch, sequences, D, heads, new, window):
    """One filling of a cache serves all tests of its size: only the tables are theirs."""
    lengths, s = _many(sequences, D, heads)
    monkeypatch.setattr(s.b, "table", s.b.table.copy())
    leave(s, lengths, [new] * sequences, window)
    return lengths, s


@pytest.mark.parametrize("window,new", [(20, 40), (33, 1), (64, 1), (64, 7), (150, 1), (150, 40), (1000, 1)])
def test_many_sequences_with_a_window(monkeypatch, window, new):
    lengths, s = many(monkeypatch, 300, 64, 8, new, window)
    plan = []
    s.check(monkeypatch, lengths, [new] * 300, 1, "bf16", window=window, max_len=max(lengths), max_shared=max(lengths), plan=plan)
    assert plan[0][0] == 1


# head_dim, key heads, group, sequences, new tokens, hint of lengths and of the prefix -> what the plan says, with a window of 150 and without
WAYS = [(64, 8, 2, 70, 60, 300, (1, 4, 1, 1)), (128, 8, 4, 40, 10, 300, (1, 1, 4, 1)), (128, 8, 4, 64, 1, 300, (1, 1, 4, 4)), (64, 8, 4, 256, 1, 3000, (1, 1, 8, 1)),
        (128, 8, 4, 64, 1, 6000, (1, 1, 8, 4)), (256, 8, 2, 64, 1, 600, (1, 1, 4, 8))]


@pytest.mark.parametrize("window", [0, 150])
@pytest.mark.parametrize("D,heads,group,sequences,new,hint,want", WAYS)
def test_every_way_that_sizes_choose(monkeypatch, D, heads, group, sequences, new, hint, want, window):
    lengths, s = many(monkeypatch, sequences, D, heads, new, window)
    plan = []
    s.check(monkeypatch, lengths, [new] * sequences, group, "bf16", window=window, max_len=hint, max_shared=hint, plan=plan)
    assert plan == [want]


def test_a_copy_of_a_page_that_holds_less_of_it(monkeypatch):
    """The first sequence has a copy of the prefix's last page that ends with its own length; what lies behind it is NaN."""
    lengths, new = [75, 140, 131], [1, 2, 1]
    s = Shared(lengths, [0, 3], [96], 2, 64, PAGE)
    spare = next(p for p in range(len(s.b.codes[0])) if p not in s.b.table)
    last = s.b.table[1, 2]
    for i in range(2):
        s.b.codes[i][spare] = s.b.codes[i][last]
        s.b.codes[i][spare][..., od.places(64, bool(i))[75 - 64:].ravel()] = 0x7F
        s.b.exps[i][spare] = s.b.exps[i][last]
        s.b.dev[i].copy_(torch.from_numpy(s.b.codes[i]))
        s.b.dev[2 + i].copy_(torch.from_numpy(s.b.exps[i]))
    s.b.table[0, 2] = spare
    got = s.check(monkeypatch, lengths, new, 4, "bf16")
    assert np.isfinite(got).all()
