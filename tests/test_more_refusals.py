"""What norms around a block, attention behind shared prefixes and log probabilities without logits refuse, and calls with nothing to do: on the host, no kernel is launched."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2406_02913_amd import szo
from test_decoder_refusals import attn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000                                    # never dereferenced


def test_structures_match_the_header(tmp_path):
    kinds = {"szo_block_desc": szo.BlockDesc, "szo_block_grads": szo.BlockGrads, "szo_attn_groups": szo.AttnGroups, "szo_head_desc": szo.HeadDesc}
    lines = [f'printf("{c} {n} %zu\\n", offsetof({c}, {n}));' for c, k in kinds.items() for n, _ in k._fields_]
    lines += [f'printf("{c} sizeof %zu\\n", sizeof({c}));' for c in kinds]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "szo.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")])
    for line in subprocess.check_output([str(tmp_path / "layout")], text=True).splitlines():
        c, n, at = line.split()
        assert int(at) == (C.sizeof(kinds[c]) if n == "sizeof" else getattr(kinds[c], n).offset), line


# ---- norms around a block ------------------------------------------------------------------------
def block(**kw):
    d = szo.BlockDesc(tokens=4, width=64, y_type=szo.F32, h_type=szo.BF16, x_type=szo.BF16, norm=szo.NORM_LAYER, post=1, eps=1e-6, y_scale=1.0, h_scale=1.0, y=P, h=P,
                      post_weight=P, post_bias=P, pre_weight=P, pre_bias=P, gate=P, h_out=P, x_out=P, y_stride=64, h_stride=64, gate_stride=0, h_out_stride=64, x_out_stride=64)
    for n, v in kw.items():
        setattr(d, n, v)
    return d


def block_grads(**kw):
    g = szo.BlockGrads(x_out_grad=P, h_out_grad=P, y_grad=P, h_grad=P, gate_grad=P, post_weight_grad=P, post_bias_grad=P, pre_weight_grad=P, pre_bias_grad=P, x_out_stride=64,
                       h_out_stride=64, y_stride=64, h_stride=64)
    for n, v in kw.items():
        setattr(g, n, v)
    return g


BAD_BLOCK = [dict(tokens=-1), dict(width=0), dict(width=-8), dict(y_type=3), dict(h_type=-1), dict(x_type=7), dict(norm=2), dict(post=2), dict(eps=-1.0), dict(eps=float("nan")),
             dict(reserved=1), dict(y=None, h=None), dict(y=None), dict(y=P + 2), dict(h=P + 1), dict(gate=P + 2), dict(post_weight=P + 1), dict(pre_bias=P + 3), dict(y_stride=-1),
             dict(h_out_stride=63), dict(x_out_stride=0), dict(h_out=P + 1), dict(h_stride=1 << 41)]


@pytest.mark.parametrize("kw", BAD_BLOCK)
def test_block_norm_refuses(kw):
    assert szo.lib.szo_block_norm(C.byref(block(**kw)), None) == szo.EINVAL
    assert szo.lib.szo_block_norm(None, None) == szo.EINVAL


def test_block_norm_does_not_take_wide_rows_or_more_than_a_grid():
    assert szo.lib.szo_block_norm(C.byref(block(width=16385, y_stride=20000, h_stride=20000, h_out_stride=20000, x_out_stride=20000)), None) == szo.EUNSUPPORTED
    assert szo.lib.szo_block_norm(C.byref(block(tokens=1 << 40)), None) == szo.EUNSUPPORTED
    assert szo.lib.szo_block_norm(C.byref(block(tokens=0, y=None, h=None)), None) == szo.OK
    assert szo.lib.szo_block_norm(C.byref(block(h_out=None, x_out=None)), None) == szo.OK


@pytest.mark.parametrize("kw", [dict(x_out_grad=P + 1), dict(h_out_stride=-1), dict(y_stride=10), dict(h_grad=P + 1), dict(gate_grad=P + 2), dict(pre_weight_grad=P + 1),
                                dict(post_bias_grad=P + 2), dict(reserved=1)])
def test_block_norm_bwd_refuses(kw):
    assert szo.lib.szo_block_norm_bwd(C.byref(block()), C.byref(block_grads(**kw)), P, None) == szo.EINVAL


def test_block_norm_bwd_refuses_gradients_of_what_is_not_there_and_a_missing_workspace():
    call = szo.lib.szo_block_norm_bwd
    assert call(C.byref(block()), C.byref(block_grads()), None, None) == szo.EINVAL
    assert call(C.byref(block()), C.byref(block_grads()), P + 4, None) == szo.EINVAL
    assert call(C.byref(block()), None, P, None) == szo.EINVAL
    assert call(C.byref(block(post=0)), C.byref(block_grads()), P, None) == szo.EINVAL
    assert call(C.byref(block(h=None)), C.byref(block_grads()), P, None) == szo.EINVAL
    assert call(C.byref(block(gate=None)), C.byref(block_grads()), P, None) == szo.EINVAL
    assert call(C.byref(block(y=None, gate=None)), C.byref(block_grads(y_grad=None, gate_grad=None)), P, None) == szo.EINVAL
    assert call(C.byref(block(gate_stride=64)), C.byref(block_grads(gate_stride=63)), P, None) == szo.EINVAL


def test_sums_of_a_block_norm_fit_their_workspace():
    """One row of each wanted sum for every row of threads of every workgroup, for all widths."""
    for width in (1, 64, 511, 512, 513, 4096, 4097, 8192, 8200, 16384):
        for tokens in (1, 3, 100, 10000, 1 << 30):
            size = szo.szo_block_workspace_bytes(block(width=width, tokens=tokens))
            waves = -(-width // (512 if width <= 4096 else 1024))
            rows = max(1, 4 // waves)
            groups = min(-(-tokens // rows), 256 * max(1, (16 if width <= 4096 else 8) // (waves * rows)))
            assert size == 4 * 4 * width * groups * rows            # four sums in fp32: a gate that tokens share has none of its own


# ---- attention behind shared prefixes ------------------------------------------------------------
def groups(**kw):
    g = szo.AttnGroups(groups=1, max_sequences=2, max_shared=64, group_start=P, shared=P)
    for n, v in kw.items():
        setattr(g, n, v)
    return g


@pytest.mark.parametrize("kw", [dict(groups=-1), dict(max_sequences=-1), dict(max_shared=-1), dict(reserved=1), dict(group_start=None), dict(shared=None), dict(group_start=P + 2),
                                dict(shared=P + 1)])
def test_shared_attention_refuses(kw):
    assert szo.lib.szo_attn_shared(C.byref(attn(max_len=1 << 20)), C.byref(groups(**kw)), P, None) == szo.EINVAL


def test_shared_attention_refuses_what_attention_over_the_cache_does_and_a_missing_workspace():
    call = szo.lib.szo_attn_shared
    assert call(C.byref(attn(scale=float("nan"))), C.byref(groups()), P, None) == szo.EINVAL
    assert call(C.byref(attn()), None, P, None) == szo.EINVAL
    d = attn(max_len=1 << 20)
    assert szo.szo_attn_shared_plan(d, groups())[3] > 1
    assert call(C.byref(d), C.byref(groups()), None, None) == szo.EINVAL
    assert call(C.byref(d), C.byref(groups()), P + 8, None) == szo.EINVAL
    assert call(C.byref(attn(tokens=0)), C.byref(groups()), None, None) == szo.OK
    assert call(C.byref(attn(max_len=1 << 20)), C.byref(groups(groups=1 << 30)), P, None) == szo.EUNSUPPORTED
    assert szo.lib.szo_attn_shared_plan(C.byref(d), C.byref(groups()), None) == szo.EINVAL


# ---- log probabilities without logits ------------------------------------------------------------
def head(**kw):
    d = szo.HeadDesc(rows=5, vocab=100, width=128, type=szo.BF16, scale=1.0, x=P, weight=P, x_stride=128, weight_stride=128, targets=P, logp=P, stats=P)
    for n, v in kw.items():
        setattr(d, n, v)
    return d


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(vocab=-1), dict(width=-64), dict(type=szo.F32), dict(type=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                dict(scale=3e38), dict(reserved=1), dict(x=None), dict(weight=None), dict(x=P + 8), dict(weight=P + 2), dict(x_stride=-128), dict(weight_stride=64),
                                dict(targets=P + 2), dict(logp=P + 1), dict(stats=P + 2), dict(loss_acc=P + 4), dict(loss_acc=P, logp=None), dict(vocab=0)])
def test_head_refuses(kw):
    assert szo.lib.szo_head_logprobs(C.byref(head(**kw)), P, None) == szo.EINVAL


@pytest.mark.parametrize("kw", [dict(width=0), dict(width=96), dict(width=65600, x_stride=65600, weight_stride=65600), dict(vocab=(1 << 30) + 1), dict(rows=1 << 31), dict(x_stride=130),
                                dict(weight_stride=(1 << 22) + 8), dict(rows=1 << 30, vocab=1 << 30), dict(rows=(1 << 26) + 1, vocab=1)])
def test_head_does_not_take(kw):
    assert szo.lib.szo_head_logprobs(C.byref(head(**kw)), P, None) == szo.EUNSUPPORTED


def test_head_workspaces_and_gradients():
    fwd, bwd = szo.lib.szo_head_logprobs, szo.lib.szo_head_logprobs_bwd
    assert fwd(C.byref(head()), None, None) == szo.EINVAL and fwd(C.byref(head()), P + 8, None) == szo.EINVAL
    assert fwd(C.byref(head(rows=0, x=None)), None, None) == szo.OK
    assert bwd(C.byref(head()), P, P, 128, P, 128, None, None) == szo.EINVAL
    assert bwd(C.byref(head()), None, P, 128, P, 128, P, None) == szo.EINVAL
    assert bwd(C.byref(head(stats=None)), P, P, 128, P, 128, P, None) == szo.EINVAL
    assert bwd(C.byref(head()), P, P, 127, P, 128, P, None) == szo.EINVAL
    assert bwd(C.byref(head()), P, P, 128, P, 0, P, None) == szo.EINVAL
    assert bwd(C.byref(head()), P, P + 1, 128, None, 0, P, None) == szo.EINVAL
    assert bwd(C.byref(head()), P, None, 0, None, 0, P, None) == szo.OK
    # d for a piece of the vocabulary: 256 MiB at most, unless one tile of columns is more
    for rows, vocab in ((1, 1), (100, 32000), (4096, 32000), (8192, 131072), (100000, 50257)):
        d = head(rows=rows, vocab=vocab, width=64, x_stride=64, weight_stride=64)
        rows64 = -(-rows // 64) * 64
        d_bytes = max(256 << 20, rows64 * 256 * 2)
        sums = 256 * 4 * rows * 64
        assert szo.szo_head_bwd_workspace_bytes(d) <= d_bytes + rows64 * 128 + sums + 4 * rows + 1024


def test_binding_checks_shapes_and_types():
    x = torch.empty(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        szo.make_head_desc(x, x)                                       # not on the device
    with pytest.raises(ValueError):
        szo.make_block_desc(None, None)
    with pytest.raises(ValueError):
        szo.make_block_desc(x, x)
    with pytest.raises(ValueError):
        szo.make_attn_groups(torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), 1, 1)
