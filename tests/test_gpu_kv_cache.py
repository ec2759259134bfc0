"""Quantising a cache as it is written and reading it back, bit for bit against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2406_02913_amd import szo

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Both:
    """The library's cache and the oracle's, of the same random bytes; tokens go to both."""

    def __init__(self, lengths, heads, D, page, seed=0, spare=2):
        self.rng = np.random.default_rng(seed)
        self.most = max(1, max(-(-n // page) for n in lengths))
        pages = len(lengths) * self.most + spare
        self.table = self.rng.permutation(pages)[:len(lengths) * self.most].reshape(len(lengths), self.most).astype(np.int32)
        shape = (pages, heads, page // 32, 32 * D)
        self.codes = [self.rng.integers(0, 256, shape).astype(np.uint8) for _ in range(2)]
        self.exps = [self.rng.integers(95, 130, shape[:3]).astype(np.uint8) for _ in range(2)]
        self.dev = [torch.from_numpy(a.copy()).to(DEV) for a in self.codes + self.exps]
        self.heads, self.D = heads, D
        self.lengths = torch.zeros(len(lengths), dtype=torch.int32, device=DEV)

    def cache(self):
        return szo.make_kv_cache(*self.dev, torch.from_numpy(self.table).to(DEV), self.lengths)

    def write(self, lengths, new, kind="f32", change=None, strided=False):
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        x = self.rng.standard_normal((2, start[-1], self.heads, self.D)) * np.exp(self.rng.standard_normal((2, start[-1], self.heads, 1)))
        if change:
            change(x)
        t = torch.from_numpy(x).to(TYPES[kind])
        if strided:                               # odd addresses and strides
            wide = torch.zeros(2, start[-1], self.heads, self.D + 3, dtype=t.dtype)
            wide[..., 1:self.D + 1] = t
            dev = wide.to(DEV)[..., 1:self.D + 1]
        else:
            dev = t.to(DEV)
        self.lengths.copy_(torch.from_numpy(np.asarray(lengths, dtype=np.int32)))
        szo.szo_kv_cache_write(self.cache(), szo.make_kv_tokens(dev[0], dev[1], torch.from_numpy(start).to(DEV), int(max(new))))
        for i in range(2):
            od.cache_write(self.codes[i], self.exps[i], bool(i), self.table, lengths, start, t[i].float().numpy())
        return t

    def same(self):
        got = [a.cpu().numpy() for a in self.dev]
        for i in range(2):
            assert np.array_equal(got[2 + i], self.exps[i])
            values = od.e4m3_values()
            assert np.array_equal(values[got[i]], values[self.codes[i]], equal_nan=True)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,heads,page", [(64, 3, 32), (96, 1, 64), (128, 2, 64), (256, 1, 96)])
def test_prompts_of_all_lengths(D, heads, page, kind):
    lengths = [1, 31, 32, 33, 64, 97, 0]
    b = Both(lengths, heads, D, page)
    b.write(lengths, lengths, kind)
    b.same()


@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_appended_tokens_move_the_exponents(D):
    b = Both([70, 45], 2, D, 64)
    b.write([5, 31], [5, 31], "bf16")
    at = np.array([5, 31])
    for step, (n, m) in enumerate([(1, 1), (1, 1), (3, 0), (0, 7), (30, 4), (1, 1)]):
        at = at + [n, m]
        b.write(at, [n, m], "bf16", change=lambda x: x.__imul__(3.0 ** step), strided=step % 2 == 1)
        b.same()


def test_blocks_of_zeros_of_huge_and_of_tiny_values():
    b = Both([40, 40, 40], 1, 64, 32)

    def change(x):
        x[:, :40] = 0
        x[:, 40:80] *= 1e30
        x[:, 80:] *= 1e-30

    b.write([40] * 3, [40] * 3, "f32", change)
    b.same()
    b.write([42] * 3, [2] * 3, "f32", lambda x: x.__imul__(1e6))       # every exponent but the huge one moves, by up to 150 places
    b.same()


def test_values_that_are_not_finite_become_nan_and_leave_the_exponent():
    b = Both([34], 2, 64, 64)

    def change(x):
        x[0, 3, 0, 5], x[1, 7, 1, 63], x[0, 20, 1, 0] = np.nan, np.inf, -np.inf

    b.write([30], [30], "f32", change)
    b.same()
    b.write([34], [4], "f32", lambda x: x.__imul__(100.0))
    b.same()


def test_halfway_values_round_to_even():
    b = Both([32], 1, 64, 32)

    def change(x):
        x[...] = 0
        x[:, 0, 0, 0] = 448
        x[:, 1, 0, :32] = np.linspace(16, 32, 33)[:32] + 0.0
        x[:, 2, 0, :32] = (np.arange(32) + 0.5) * 2.0 ** -9

    b.write([32], [32], "f32", change)
    b.same()


def test_pages_outside_the_cache_are_left_out_and_read_as_zeros():
    b = Both([100, 100], 2, 64, 32)
    b.table[0, 1], b.table[1, 0] = -1, 10 ** 6
    b.write([100, 100], [100, 100])
    b.same()
    k = torch.full((200, 2, 64), 7.0, device=DEV)
    v = torch.full((200, 2, 64), 7.0, device=DEV)
    start = torch.tensor([0, 100, 200], dtype=torch.int32, device=DEV)
    szo.szo_kv_cache_read(b.cache(), szo.make_kv_tokens(k, v, start, 100))
    for i, t in enumerate((k, v)):
        for s in range(2):
            want, _ = od.cache_dense(b.codes[i], b.exps[i], bool(i), b.table, [100, 100], s)
            assert np.array_equal(t[100 * s:100 * s + 100].cpu().numpy(), want)
    # more tokens than the table has places for
    b.lengths.fill_(150)
    k.fill_(7), v.fill_(7)
    szo.szo_kv_cache_read(b.cache(), szo.make_kv_tokens(k, v, start, 100))
    assert (k[78:100] == 0).all() and (v[178:] == 0).all() and (k[:40] != 0).any()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,page", [(64, 32), (96, 96), (128, 64), (256, 32)])
def test_read_back(D, page, kind):
    lengths, new = [1, 33, 65, 130], [1, 2, 65, 50]
    b = Both(lengths, 2, D, page)
    b.write(lengths, lengths)
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    out = [torch.full((start[-1], 2, D + 5), 7.0, dtype=TYPES[kind], device=DEV)[..., 2:D + 2] for _ in range(2)]
    szo.szo_kv_cache_read(b.cache(), szo.make_kv_tokens(out[0], out[1], torch.from_numpy(start).to(DEV), max(new)))
    for i in range(2):
        for s in range(4):
            want, _ = od.cache_dense(b.codes[i], b.exps[i], bool(i), b.table, lengths, s)
            want = torch.from_numpy(want[lengths[s] - new[s]:]).to(TYPES[kind])       # exact but for fp16's smallest
            assert torch.equal(out[i][start[s]:start[s + 1]].cpu(), want)


def test_more_new_tokens_than_a_sequence_has():
    b = Both([20], 1, 64, 32)
    b.write([20], [30])                           # the first ten have no place
    b.same()


def test_offsets_beyond_32_bits():
    """Pages behind 4 GiB of codes."""
    pages, heads, D = 33000, 16, 128              # 128 KiB a page for each of keys and values
    k, v, ke, ve = szo.new_kv_cache(pages, 64, heads, D)
    table = torch.tensor([[pages - 1], [5]], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([40, 40], dtype=torch.int32, device=DEV)
    cache = szo.make_kv_cache(k, v, ke, ve, table, lengths)
    x = torch.randn(80, heads, D, device=DEV)
    start = torch.tensor([0, 40, 80], dtype=torch.int32, device=DEV)
    szo.szo_kv_cache_write(cache, szo.make_kv_tokens(x, x, start, 40))
    a, b = torch.empty_like(x), torch.empty_like(x)
    szo.szo_kv_cache_read(cache, szo.make_kv_tokens(a, b, start, 40))
    assert torch.equal(a, b) and (a - x).abs().max() < x.abs().max() / 16
    assert not k[6:pages - 1].any()


def test_on_another_stream():
    b = Both([50], 2, 128, 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.write([50], [50])
    torch.cuda.current_stream().wait_stream(s)
    b.same()
