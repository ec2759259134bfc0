"""Sizes of workspaces and bounds that the calls between the linear layers keep to: on the host, no kernel is launched."""
import pytest
import torch

from paper_2406_02913_amd import szo
from test_decoder_refusals import P, attn, cache, grads, logp, qk, tokens


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("group,new", [(1, 1), (3, 1), (5, 1), (7, 1), (1, 3), (4, 1)])
def test_parts_of_a_cache_are_stored_at_multiples_of_16_bytes(D, group, new):
    """One sequence of one key head in some number of parts, at most 64: each is a whole number of 16 bytes and holds its rows' sums."""
    rows = group * new
    for length in (1200, 2000, 2500, 3300, 5000, 9000, 40000):
        d = attn(q_heads=group, max_q=new, tokens=new, max_len=length, cache=cache(kv_heads=1, sequences=1, head_dim=D, max_pages=1000, page_tokens=64),
                 q_token_stride=group * D, q_head_stride=D, out_token_stride=group * D, out_head_stride=D)
        size = szo.szo_attn_workspace_bytes(d)
        least = 4 * rows * (D + 2)                # numerators, maximum, denominator; one statistic more would still be a row's sums
        assert size > 16 and any(size % parts == 0 and size // parts % 16 == 0 and 0 <= size // parts - least < 16 + 4 * rows for parts in range(2, 65)), (length, size)


@pytest.mark.parametrize("scale", [2.4e38, 3.3e38])
def test_log_probabilities_refuse_a_scale_whose_product_by_log2_e_is_infinite(scale):
    assert szo.lib.szo_token_logprobs(logp(scale=scale), P, None) == szo.EINVAL
    assert szo.lib.szo_token_logprobs_bwd(logp(scale=scale), P, P, P, 10, None) == szo.EINVAL
    assert szo.lib.szo_token_logprobs(logp(scale=szo.MOST_SCALE, rows=0), P, None) == szo.OK


@pytest.mark.parametrize("scale", [2.4e38, -3.3e38])
def test_attention_refuses_a_scale_whose_product_by_log2_e_is_infinite(scale):
    assert szo.lib.szo_attn_cached(attn(scale=scale), P, None) == szo.EINVAL
    assert szo.lib.szo_attn_cached(attn(scale=-szo.MOST_SCALE, tokens=0), None, None) == szo.OK


@pytest.mark.parametrize("call", ["szo_kv_cache_write", "szo_kv_cache_read"])
@pytest.mark.parametrize("lengths", [None, P + 2])
def test_cache_calls_want_lengths_whatever_the_page_table_holds(call, lengths):
    """Without pages a read still asks every sequence's length."""
    for kw in (dict(max_pages=0), dict(max_pages=0, page_table=None), dict(pages=0, max_pages=0)):
        assert getattr(szo.lib, call)(cache(lengths=lengths, **kw), tokens(), None) == szo.EINVAL
    assert getattr(szo.lib, call)(cache(lengths=lengths, sequences=0, max_pages=0), tokens(), None) == szo.OK


@pytest.mark.parametrize("call", ["szo_kv_cache_write", "szo_kv_cache_read"])
def test_cache_calls_refuse_a_negative_number_of_rows(call):
    assert getattr(szo.lib, call)(cache(), tokens(tokens=-1), None) == szo.EINVAL


def test_new_tokens_that_no_grid_counts_are_refused():
    """A hint of any size is met by the rows that there are; what is left of it is counted in 64 bits."""
    most = 2 ** 63 - 1
    for new, rows in ((most, most), (most, 2 ** 31 - 1), (most - 7, 1 << 40), (1 << 40, most)):
        assert szo.lib.szo_kv_cache_read(cache(), tokens(max_new=new, tokens=rows), None) == szo.EUNSUPPORTED
        assert szo.lib.szo_kv_cache_write(cache(max_pages=1 << 20), tokens(max_new=new, tokens=rows), None) == szo.EUNSUPPORTED
    for call in (szo.lib.szo_kv_cache_read, szo.lib.szo_kv_cache_write):
        assert call(cache(), tokens(max_new=most, tokens=0), None) == szo.OK


class Room:
    """What the binding asks of a device tensor, without a device."""
    is_cuda = True

    def __init__(self, nbytes):
        self.nbytes = nbytes

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P


def decode(sequences, **kw):
    """One token each of sequences of up to 4000 tokens, 32 query and 8 key heads of 128."""
    return attn(q_heads=32, max_q=1, tokens=sequences, max_len=4000, q_token_stride=4096, out_token_stride=4096,
                cache=cache(kv_heads=8, sequences=sequences, max_pages=100, page_tokens=64), **kw)


def test_a_workspace_for_a_larger_batch_may_be_too_small_for_a_smaller_one_and_is_refused():
    size = {n: szo.szo_attn_workspace_bytes(decode(n)) for n in (8, 16, 64, 128)}
    assert size[8] > size[16] and size[64] > size[128]             # fewer sequences are split into more parts
    for n in size:
        for room in (size[n] - 1, size[128], 16):
            if room < size[n]:
                with pytest.raises(ValueError, match="workspace"):
                    szo.szo_attn_cached(decode(n), Room(room), stream=0)


def test_workspaces_of_log_probabilities_and_of_weight_gradients_are_checked():
    d = logp(rows=4, vocab=131072, row_stride=131072, top=5)
    size = szo.szo_logprobs_workspace_bytes(d)
    assert size > 16 and szo.szo_logprobs_workspace_bytes(logp(rows=600, vocab=131072, row_stride=131072, top=5)) == 16
    with pytest.raises(ValueError, match="workspace"):
        szo.szo_token_logprobs(d, Room(size - 1), stream=0)
    g = grads()
    g.shapes = (4, 2, 64), 1, szo.F32
    with pytest.raises(ValueError, match="workspace"):
        szo.szo_qk_norm_rope_bwd(qk(), g, Room(szo.szo_qk_workspace_bytes(qk()) - 1), stream=0)


def test_the_way_of_a_call_can_be_asked():
    assert szo.szo_attn_plan(decode(1))[2] > 1 and szo.szo_attn_plan(decode(128))[2] == 1
    assert szo.szo_attn_plan(attn(tokens=0)) == (0, 0, 0, 0)
    assert szo.lib.szo_attn_plan(attn(), None) == szo.EINVAL
    with pytest.raises(szo.SzoError):
        szo.szo_attn_plan(attn(type=szo.F32))


def fake(shape, dtype=torch.float32):
    """A tensor that says it is on the device; nothing is launched with it."""
    class On(torch.Tensor):
        is_cuda = True

    return torch.empty(shape, dtype=dtype).as_subclass(On)


def test_a_call_for_keys_alone_goes_by_the_type_of_its_output():
    d = szo.make_qk_desc(fake((4, 0, 64)), fake((4, 2, 64)), None, None, None, None, fake((4, 2, 64), torch.bfloat16), norm=True)
    assert (d.in_type, d.out_type) == (szo.F32, szo.BF16)
    d = szo.make_qk_desc(fake((4, 2, 64)), None, None, None, None, fake((4, 2, 64), torch.float16), norm=True)
    assert (d.in_type, d.out_type) == (szo.F32, szo.F16)


@pytest.mark.parametrize("shape", [(3, 1, 64), (5, 1, 64), (4, 1, 32), (4, 2, 64)])
def test_gradients_of_keys_have_the_tokens_and_features_of_the_queries(shape):
    """The call goes by the inputs' numbers of tokens, heads and features: buffers of others are refused."""
    d = qk()                                      # 4 tokens, 2 + 1 heads of 64
    q = fake((4, 2, 64))
    with pytest.raises(ValueError):
        szo.szo_qk_norm_rope_bwd(d, szo.make_qk_grads(q, fake(shape), q, fake(shape)), None, stream=0)
    with pytest.raises(ValueError):
        szo.make_qk_grads(q, fake((4, 1, 64)), q, fake((4, 3, 64)))
    with pytest.raises(ValueError):
        szo.make_qk_grads(fake((3, 2, 64)), None, q, None)
