"""What the calls between the linear layers refuse, and calls with nothing to do: decided on the host, no kernel is launched."""
import ctypes as C
import os
import subprocess

import pytest
import torch                                   # noqa: F401 -- before the library, as everywhere: both have to share one HIP runtime

from paper_2406_02913_amd import szo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000                                    # never dereferenced


def test_structures_match_the_header(tmp_path):
    kinds = {"szo_qk_desc": szo.QkDesc, "szo_qk_grads": szo.QkGrads, "szo_kv_cache": szo.KvCache, "szo_kv_tokens": szo.KvTokens,
             "szo_attn_desc": szo.AttnDesc, "szo_logprobs_desc": szo.LogprobsDesc}
    lines = [f'printf("{c} {n} %zu\\n", offsetof({c}, {n}));' for c, k in kinds.items() for n, _ in k._fields_]
    lines += [f'printf("{c} sizeof %zu\\n", sizeof({c}));' for c in kinds]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "szo.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")])
    for line in subprocess.check_output([str(tmp_path / "layout")], text=True).splitlines():
        c, n, at = line.split()
        assert int(at) == (C.sizeof(kinds[c]) if n == "sizeof" else getattr(kinds[c], n).offset), line


def qk(**kw):
    d = szo.QkDesc(tokens=4, q_heads=2, kv_heads=1, head_dim=64, rot_dim=64, in_type=szo.F32, out_type=szo.BF16, norm=1, interleaved=0, eps=1e-6, q=P, k=P,
                   q_token_stride=128, q_head_stride=64, k_token_stride=64, k_head_stride=64, q_weight=P, k_weight=P, positions=P, cos_table=P, sin_table=P,
                   table_rows=10, q_out=P, k_out=P, q_out_token_stride=128, q_out_head_stride=64, k_out_token_stride=64, k_out_head_stride=64)
    for n, v in kw.items():
        setattr(d, n, v)
    return d


def grads(**kw):
    g = szo.QkGrads(out_type=szo.BF16, q_out_grad=P, k_out_grad=P, q_out_token_stride=128, q_out_head_stride=64, k_out_token_stride=64, k_out_head_stride=64,
                    q_grad=P, k_grad=P, q_token_stride=128, q_head_stride=64, k_token_stride=64, k_head_stride=64, q_weight_grad=P, k_weight_grad=P)
    for n, v in kw.items():
        setattr(g, n, v)
    return g


BAD_QK = [dict(tokens=-1), dict(q_heads=-1), dict(rot_dim=72), dict(in_type=3), dict(out_type=-1), dict(norm=2), dict(interleaved=5), dict(eps=-1.0),
          dict(eps=float("nan")), dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(positions=None), dict(cos_table=None), dict(sin_table=None),
          dict(table_rows=-1), dict(q=P + 2), dict(q_out=P + 1), dict(q_weight=P + 2), dict(q_head_stride=32), dict(q_out_head_stride=8),
          dict(q_out_token_stride=16), dict(k_out_token_stride=0), dict(q_token_stride=-128), dict(reserved=1), dict(head_dim=0)]


@pytest.mark.parametrize("kw", BAD_QK)
def test_qk_norm_rope_refuses(kw):
    assert szo.lib.szo_qk_norm_rope(C.byref(qk(**kw)), None) == szo.EINVAL


@pytest.mark.parametrize("kw", [dict(head_dim=60, rot_dim=8), dict(head_dim=264, rot_dim=64), dict(rot_dim=4), dict(tokens=1 << 32)])
def test_qk_norm_rope_does_not_take(kw):
    assert szo.lib.szo_qk_norm_rope(C.byref(qk(**kw)), None) == szo.EUNSUPPORTED


@pytest.mark.parametrize("kw", [dict(q_out_grad=None), dict(q_grad=None), dict(k_grad=None), dict(out_type=7), dict(q_grad=P + 2), dict(q_token_stride=1),
                                dict(q_weight_grad=P + 1), dict(reserved=3), dict(k_out_head_stride=-1)])
def test_qk_norm_rope_backward_refuses(kw):
    assert szo.lib.szo_qk_norm_rope_bwd(C.byref(qk()), C.byref(grads(**kw)), P, None) == szo.EINVAL


def test_qk_norm_rope_backward_refuses_weights_without_room_or_norm():
    assert szo.lib.szo_qk_norm_rope_bwd(C.byref(qk()), C.byref(grads()), None, None) == szo.EINVAL
    assert szo.lib.szo_qk_norm_rope_bwd(C.byref(qk()), C.byref(grads()), P + 4, None) == szo.EINVAL
    assert szo.lib.szo_qk_norm_rope_bwd(C.byref(qk(norm=0)), C.byref(grads()), P, None) == szo.EINVAL
    assert szo.lib.szo_qk_norm_rope_bwd(None, C.byref(grads()), P, None) == szo.EINVAL
    assert szo.lib.szo_qk_norm_rope_bwd(C.byref(qk()), None, P, None) == szo.EINVAL


def cache(**kw):
    c = szo.KvCache(8, 64, 2, 128, 3, 4, P, P, P, P, P, P)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def tokens(**kw):
    t = szo.KvTokens(type=szo.F32, max_new=5, token_start=P, k=P, v=P, k_token_stride=256, k_head_stride=128, v_token_stride=256, v_head_stride=128)
    for n, v in kw.items():
        setattr(t, n, v)
    return t


BAD_CACHE = [dict(pages=-1), dict(page_tokens=48), dict(page_tokens=0), dict(kv_heads=-2), dict(sequences=-1), dict(max_pages=-1), dict(k=None), dict(v=P + 8),
             dict(k_exp=None), dict(page_table=None), dict(lengths=None), dict(lengths=P + 2), dict(head_dim=0)]


@pytest.mark.parametrize("call", ["szo_kv_cache_write", "szo_kv_cache_read"])
@pytest.mark.parametrize("kw", BAD_CACHE)
def test_cache_calls_refuse_a_cache(call, kw):
    assert getattr(szo.lib, call)(C.byref(cache(**kw)), C.byref(tokens()), None) == szo.EINVAL


@pytest.mark.parametrize("call", ["szo_kv_cache_write", "szo_kv_cache_read"])
@pytest.mark.parametrize("kw", [dict(type=9), dict(max_new=-1), dict(token_start=None), dict(k=None), dict(v=None), dict(k=P + 2), dict(k_token_stride=-1),
                                dict(reserved=1), dict(token_start=P + 1)])
def test_cache_calls_refuse_tokens(call, kw):
    assert getattr(szo.lib, call)(C.byref(cache()), C.byref(tokens(**kw)), None) == szo.EINVAL


def test_cache_limits():
    assert szo.lib.szo_kv_cache_write(C.byref(cache(head_dim=80)), C.byref(tokens()), None) == szo.EUNSUPPORTED
    assert szo.lib.szo_kv_cache_write(C.byref(cache(max_pages=1 << 26)), C.byref(tokens()), None) == szo.EUNSUPPORTED
    assert szo.lib.szo_kv_cache_read(C.byref(cache()), C.byref(tokens(k_token_stride=100)), None) == szo.EINVAL      # rows that are written overlap
    assert szo.lib.szo_kv_cache_read(C.byref(cache()), C.byref(tokens(v_head_stride=64)), None) == szo.EINVAL
    assert szo.lib.szo_kv_cache_write(C.byref(cache(sequences=0)), C.byref(tokens()), None) == szo.OK
    assert szo.lib.szo_kv_cache_write(C.byref(cache()), C.byref(tokens(max_new=0)), None) == szo.OK
    assert szo.lib.szo_kv_cache_write(None, C.byref(tokens()), None) == szo.EINVAL
    assert szo.lib.szo_kv_cache_write(C.byref(cache()), None, None) == szo.EINVAL


def attn(**kw):
    d = szo.AttnDesc(cache(), q_heads=4, type=szo.BF16, causal=1, window=0, scale=0.1, max_q=2, max_len=100, tokens=6, q=P, q_token_stride=512, q_head_stride=128,
                     q_start=P, out=P, out_token_stride=512, out_head_stride=128, lse=None)
    for n, v in kw.items():
        setattr(d, n, v)
    return d


@pytest.mark.parametrize("kw", [dict(type=szo.F32), dict(type=5), dict(causal=2), dict(window=-1), dict(scale=float("inf")), dict(scale=float("nan")), dict(max_q=-1),
                                dict(max_len=-1), dict(tokens=-1), dict(q_heads=3), dict(q_heads=-4), dict(q=None), dict(out=None), dict(q_start=None), dict(q=P + 1),
                                dict(lse=P + 2), dict(out_token_stride=64), dict(out_head_stride=64), dict(q_token_stride=-1), dict(reserved=2),
                                dict(cache=cache(k=None)), dict(cache=cache(page_tokens=33))])
def test_attention_refuses(kw):
    assert szo.lib.szo_attn_cached(C.byref(attn(**kw)), P, None) == szo.EINVAL


def test_attention_limits_and_nothing_to_do():
    assert szo.lib.szo_attn_cached(C.byref(attn(cache=cache(head_dim=32))), P, None) == szo.EUNSUPPORTED
    assert szo.lib.szo_attn_cached(C.byref(attn(tokens=1 << 33)), P, None) == szo.EUNSUPPORTED
    for kw in (dict(tokens=0), dict(max_q=0), dict(q_heads=0), dict(cache=cache(sequences=0))):
        assert szo.lib.szo_attn_cached(C.byref(attn(**kw)), None, None) == szo.OK
    long = attn(max_len=4096, cache=cache(max_pages=64))
    assert szo.lib.szo_attn_workspace_bytes(C.byref(long)) > 16
    assert szo.lib.szo_attn_cached(C.byref(long), None, None) == szo.EINVAL          # parts of the cache need room
    assert szo.lib.szo_attn_cached(C.byref(long), P + 4, None) == szo.EINVAL


def logp(**kw):
    d = szo.LogprobsDesc(rows=3, vocab=10, row_stride=10, type=szo.F32, top=2, scale=1.0, logits=P, targets=P, logp=P, entropy=P, stats=P, top_logp=P, top_index=P)
    for n, v in kw.items():
        setattr(d, n, v)
    return d


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(vocab=-1), dict(vocab=0), dict(type=4), dict(top=-1), dict(top=11), dict(scale=0.0), dict(scale=-1.0),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(logits=None), dict(logits=P + 2), dict(targets=P + 1), dict(row_stride=-3),
                                dict(loss_acc=P + 4), dict(loss_acc=P, logp=None), dict(reserved=1)])
def test_log_probabilities_refuse(kw):
    assert szo.lib.szo_token_logprobs(C.byref(logp(**kw)), P, None) == szo.EINVAL


def test_log_probabilities_limits():
    assert szo.lib.szo_token_logprobs(C.byref(logp(vocab=100, top=33)), P, None) == szo.EUNSUPPORTED
    assert szo.lib.szo_token_logprobs(C.byref(logp(vocab=(1 << 30) + 1)), P, None) == szo.EUNSUPPORTED
    assert szo.lib.szo_token_logprobs(C.byref(logp(rows=0)), P, None) == szo.OK
    assert szo.lib.szo_token_logprobs(None, P, None) == szo.EINVAL


@pytest.mark.parametrize("desc,args", [(dict(stats=None), (P, P, P, 10)), (dict(entropy=None), (P, P, P, 10)), ({}, (P, P, None, 10)), ({}, (P, P, P, 9)),
                                       ({}, (P + 1, P, P, 10)), ({}, (P, P + 2, P, 10)), ({}, (P, P, P + 1, 10))])
def test_gradient_of_log_probabilities_refuses(desc, args):
    assert szo.lib.szo_token_logprobs_bwd(C.byref(logp(**desc)), *args, None) == szo.EINVAL


def test_launches_that_cannot_be_counted_are_refused():
    """A launch counts its threads in 32 bits: more is refused by the call, not by the launch."""
    assert szo.lib.szo_qk_norm_rope(C.byref(qk(tokens=0x7FFFFFFF)), None) == szo.EUNSUPPORTED
    assert szo.lib.szo_token_logprobs(C.byref(logp(rows=1 << 25)), P, None) == szo.EUNSUPPORTED
    assert szo.lib.szo_token_logprobs_bwd(C.byref(logp(rows=1 << 25)), P, P, P, 10, None) == szo.EUNSUPPORTED
    assert szo.lib.szo_kv_cache_write(C.byref(cache(kv_heads=65536)), C.byref(tokens()), None) == szo.EUNSUPPORTED
