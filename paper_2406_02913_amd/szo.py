"""ctypes binding over libszo.so: same names as include/szo.h, argument
marshalling only.  Device arrays are torch tensors (PyTorch-ROCm is used for
device memory and streams, nothing else); host arrays are numpy arrays.

There is no fallback: if the native library is missing or fails to load, the
import raises.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# SZO_LIBRARY names another build of the same library (comparisons between builds); default: the in-tree one
LIB_PATH = os.environ.get("SZO_LIBRARY") or os.path.join(_HERE, "libszo.so")

OK, EINVAL, EUNSUPPORTED, ELAUNCH = 0, -1, -2, -3
TILE_F16, TILE_BF16 = 0, 1
TILE_ROWS, TILE_COLS = 64, 64
STEP_FUSED_LOSS = 1
STEP_ONE_DENSE_PASS = 2
STEP_SMALL_WORKSPACE = 4
FORMAT_UNIFORM, FORMAT_LUT = 0, 1
F32, BF16, F16 = 0, 1, 2                  # element types of the calls between the linear layers
KV_BLOCK = 32                             # tokens that share an exponent in the cache
LOGPROBS_MAX_TOP = 32
MOST_SCALE = 2.35e38                      # of logits and scores

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built: run `python -c 'import __graft_entry__ as g; g.build()'` "
                      "(or python paper_2406_02913_amd/build.py) first")
lib = C.CDLL(LIB_PATH)


class LinearDesc(C.Structure):
    _fields_ = [("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64),
                ("group", C.c_int32), ("tile_dtype", C.c_int32),
                ("nnz", C.c_int64), ("nnz_base", C.c_uint64),
                ("x", C.c_void_p), ("qweight", C.c_void_p), ("scales", C.c_void_p),
                ("tile_ptr", C.c_void_p), ("sp_idx", C.c_void_p), ("sp_val", C.c_void_p),
                ("y", C.c_void_p), ("target", C.c_void_p),
                ("lut", C.c_void_p), ("format", C.c_int32), ("reserved", C.c_int32),
                ("x_minus", C.c_void_p)]


def _fields(kind, names):
    return [(n, kind) for n in names.split()]


_I32, _I64, _PTR = C.c_int32, C.c_int64, C.c_void_p


class QkDesc(C.Structure):
    _fields_ = (_fields(_I64, "tokens") + _fields(_I32, "q_heads kv_heads head_dim rot_dim in_type out_type norm interleaved") + _fields(C.c_float, "eps") +
                _fields(_I32, "reserved") + _fields(_PTR, "q k") + _fields(_I64, "q_token_stride q_head_stride k_token_stride k_head_stride") +
                _fields(_PTR, "q_weight k_weight positions cos_table sin_table") + _fields(_I64, "table_rows") + _fields(_PTR, "q_out k_out") +
                _fields(_I64, "q_out_token_stride q_out_head_stride k_out_token_stride k_out_head_stride"))


class QkGrads(C.Structure):
    _fields_ = (_fields(_I32, "out_type reserved") + _fields(_PTR, "q_out_grad k_out_grad") +
                _fields(_I64, "q_out_token_stride q_out_head_stride k_out_token_stride k_out_head_stride") + _fields(_PTR, "q_grad k_grad") +
                _fields(_I64, "q_token_stride q_head_stride k_token_stride k_head_stride") + _fields(_PTR, "q_weight_grad k_weight_grad"))


class KvCache(C.Structure):
    _fields_ = _fields(_I32, "pages page_tokens kv_heads head_dim sequences max_pages") + _fields(_PTR, "k v k_exp v_exp page_table lengths")


class KvTokens(C.Structure):
    _fields_ = (_fields(_I32, "type reserved") + _fields(_I64, "max_new") + _fields(_PTR, "token_start k v") +
                _fields(_I64, "k_token_stride k_head_stride v_token_stride v_head_stride tokens"))


class AttnDesc(C.Structure):
    _fields_ = ([("cache", KvCache)] + _fields(_I32, "q_heads type causal window") + _fields(C.c_float, "scale") + _fields(_I32, "max_q max_len reserved") +
                _fields(_I64, "tokens") + _fields(_PTR, "q") + _fields(_I64, "q_token_stride q_head_stride") + _fields(_PTR, "q_start out") +
                _fields(_I64, "out_token_stride out_head_stride") + _fields(_PTR, "lse"))


class LogprobsDesc(C.Structure):
    _fields_ = (_fields(_I64, "rows vocab row_stride") + _fields(_I32, "type top") + _fields(C.c_float, "scale") + _fields(_I32, "reserved") +
                _fields(_PTR, "logits targets logp entropy stats top_logp top_index loss_acc") + _fields(C.c_double, "loss_scale"))


_P = C.POINTER
_SIGS = {
    "szo_linear_fwd": (C.c_int, [_P(LinearDesc), C.c_uint64, C.c_uint64, C.c_int, C.c_float, C.c_void_p]),
    "szo_mse_loss": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_double, C.c_void_p, C.c_void_p, C.c_void_p]),
    "szo_linear_fwd_mse": (C.c_int, [_P(LinearDesc), C.c_uint64, C.c_uint64, C.c_int, C.c_float, C.c_double,
                                      C.c_void_p, C.c_void_p, C.c_void_p]),
    "szo_spsa_g": (C.c_int, [C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p]),
    "szo_sparse_update": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_uint64, C.c_uint64, C.c_uint64,
                                     C.c_void_p, C.c_float, C.c_void_p]),
    "szo_zo_step": (C.c_int, [_P(LinearDesc), C.c_int, C.c_uint64, C.c_uint64, C.c_float, C.c_float,
                               C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]),
    "szo_zo_step_noalloc": (C.c_int, [_P(LinearDesc), C.c_int, C.c_uint64, C.c_uint64, C.c_float, C.c_float,
                                       C.c_void_p, C.c_void_p]),
    "szo_workspace_bytes": (C.c_size_t, []),
    "szo_step_workspace_bytes": (C.c_size_t, [_P(LinearDesc), C.c_int, C.c_int]),
    "szo_workspace_init": (C.c_int, [C.c_void_p, C.c_void_p]),
    "szo_num_tiles": (C.c_int64, [C.c_int64, C.c_int64]),
    "szo_mask_generate": (C.c_int, [C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_uint64, C.c_void_p]),
    "szo_tcsr_build": (C.c_int, [C.c_int64, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "szo_quantize_pack": (C.c_int, [C.c_void_p, C.c_int64, C.c_int64, C.c_int, C.c_void_p, C.c_int64,
                                     C.c_void_p, C.c_void_p, C.c_void_p]),
    "szo_quantize_pack_lut": (C.c_int, [C.c_void_p, C.c_int64, C.c_int64, C.c_void_p, C.c_int64,
                                         C.c_void_p, C.c_void_p, C.c_void_p]),
    "szo_qweight_bytes": (C.c_size_t, [C.c_int64, C.c_int64]),
    "szo_scales_count": (C.c_size_t, [C.c_int64, C.c_int64, C.c_int]),
    "szo_layout_weights": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int, C.c_void_p, C.c_void_p]),
    "szo_philox4x32_10": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "szo_debug_zbar": (C.c_int, [C.c_uint64, C.c_int64, C.c_uint64, C.c_uint64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "szo_activation_absmax": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]),
    "szo_choose_tile_dtype": (C.c_int, [C.c_float]),
    "szo_set_tile_config": (C.c_int, [C.c_int]),
    "szo_kernel_timing": (C.c_int, [C.c_int]),
    "szo_kernel_timing_read": (C.c_int, [C.c_void_p, C.c_void_p]),
    "szo_kernel_timing_read2": (C.c_int, [C.c_void_p, C.c_void_p]),
    "szo_qk_norm_rope": (C.c_int, [_P(QkDesc), C.c_void_p]),
    "szo_qk_norm_rope_bwd": (C.c_int, [_P(QkDesc), _P(QkGrads), C.c_void_p, C.c_void_p]),
    "szo_qk_workspace_bytes": (C.c_size_t, [_P(QkDesc)]),
    "szo_kv_cache_write": (C.c_int, [_P(KvCache), _P(KvTokens), C.c_void_p]),
    "szo_kv_cache_read": (C.c_int, [_P(KvCache), _P(KvTokens), C.c_void_p]),
    "szo_attn_cached": (C.c_int, [_P(AttnDesc), C.c_void_p, C.c_void_p]),
    "szo_attn_plan": (C.c_int, [_P(AttnDesc), C.c_void_p]),
    "szo_attn_workspace_bytes": (C.c_size_t, [_P(AttnDesc)]),
    "szo_token_logprobs": (C.c_int, [_P(LogprobsDesc), C.c_void_p, C.c_void_p]),
    "szo_logprobs_workspace_bytes": (C.c_size_t, [_P(LogprobsDesc)]),
    "szo_token_logprobs_bwd": (C.c_int, [_P(LogprobsDesc), C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "szo_last_hip_error": (C.c_int, []),
    "szo_version": (C.c_int, []),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(lib, _name)          # AttributeError here = header and library disagree
    _f.restype, _f.argtypes = _res, _args
EXPORTS = tuple(_SIGS)


class SzoError(RuntimeError):
    def __init__(self, fn, code):
        self.code = code
        names = {EINVAL: "SZO_EINVAL", EUNSUPPORTED: "SZO_EUNSUPPORTED", ELAUNCH: "SZO_ELAUNCH"}
        extra = f" (hip error {lib.szo_last_hip_error()})" if code == ELAUNCH else ""
        super().__init__(f"{fn} -> {names.get(code, code)}{extra}")


def _check(fn, rc):
    if rc != OK:
        raise SzoError(fn, rc)


def _dev(t):
    """Device pointer of a torch tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous device tensor")
    return t.data_ptr()


def _host(a, dtype):
    if a is None:
        return None, None
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data


def _stream(stream):
    """The handle of torch's current stream unless one is given.  torch.cuda.current_stream() builds a Stream object around it, which
    takes 2.7 us of the 7.2 that a single-layer call takes on the host; asked for the handle alone torch answers in 0.3."""
    if stream is not None:
        return stream
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(torch.cuda.current_device()) if raw else torch.cuda.current_stream().cuda_stream


def make_desc(M, N, K, group, nnz, nnz_base, x, qweight, scales, tile_ptr, sp_idx, sp_val,
              y=None, target=None, tile_dtype=TILE_F16, lut=None, x_minus=None):
    """With `lut` (device fp16 [N,16]) the layer is of the non-uniform format; scales may then be None.
    `x_minus` (device bf16 [M,K]): activations of the -eps forward of szo_zo_step, if they differ from x."""
    return LinearDesc(M, N, K, group, tile_dtype, nnz, nnz_base, _dev(x), _dev(qweight), _dev(scales),
                      _dev(tile_ptr), _dev(sp_idx), _dev(sp_val), _dev(y), _dev(target),
                      _dev(lut), FORMAT_UNIFORM if lut is None else FORMAT_LUT, 0, _dev(x_minus))


# ---- hot calls -------------------------------------------------------------------------------
def szo_linear_fwd(desc, seed, step, sign, eps, stream=None):
    _check("szo_linear_fwd", lib.szo_linear_fwd(C.byref(desc), seed, step, sign, eps, _stream(stream)))


def szo_mse_loss(y, target, count, scale, loss_acc, workspace, stream=None):
    _check("szo_mse_loss", lib.szo_mse_loss(_dev(y), _dev(target), count, scale, _dev(loss_acc),
                                            _dev(workspace), _stream(stream)))


def szo_linear_fwd_mse(desc, seed, step, sign, eps, scale, loss_acc, workspace, stream=None):
    _check("szo_linear_fwd_mse", lib.szo_linear_fwd_mse(C.byref(desc), seed, step, sign, eps, scale,
                                                        _dev(loss_acc), _dev(workspace), _stream(stream)))


def szo_spsa_g(loss_plus, loss_minus, eps, g, stream=None):
    _check("szo_spsa_g", lib.szo_spsa_g(_dev(loss_plus), _dev(loss_minus), eps, _dev(g), _stream(stream)))


def szo_sparse_update(sp_val, sp_idx, nnz, nnz_base, seed, step, g, lr, stream=None):
    _check("szo_sparse_update", lib.szo_sparse_update(_dev(sp_val), _dev(sp_idx), nnz, nnz_base, seed, step,
                                                      _dev(g), lr, _stream(stream)))


def desc_array(descs):
    arr = (LinearDesc * len(descs))(*descs)
    return arr


def szo_zo_step(descs, seed, step, eps, lr, scalars, workspace, flags=0, stream=None):
    """descs: a ctypes array from desc_array() (or a list of LinearDesc)."""
    if isinstance(descs, (list, tuple)):
        descs = desc_array(descs)
    _check("szo_zo_step", lib.szo_zo_step(descs, len(descs), seed, step, eps, lr, _dev(scalars),
                                          _dev(workspace), flags, _stream(stream)))


def szo_zo_step_noalloc(descs, seed, step, eps, lr, scalars, stream=None):
    """The fused-loss step without a workspace and without any allocation inside the library."""
    if isinstance(descs, (list, tuple)):
        descs = desc_array(descs)
    _check("szo_zo_step_noalloc", lib.szo_zo_step_noalloc(descs, len(descs), seed, step, eps, lr, _dev(scalars),
                                                          _stream(stream)))


def szo_workspace_bytes():
    return int(lib.szo_workspace_bytes())


def szo_step_workspace_bytes(descs=(), flags=STEP_FUSED_LOSS):
    """Without layers: what steps with STEP_SMALL_WORKSPACE and the loss calls need."""
    if isinstance(descs, (list, tuple)):
        descs = desc_array(descs)
    return int(lib.szo_step_workspace_bytes(descs, len(descs), flags))


def szo_workspace_init(workspace, stream=None):
    _check("szo_workspace_init", lib.szo_workspace_init(_dev(workspace), _stream(stream)))


def new_workspace(device="cuda", nbytes=None):
    """For any call, or of the size that szo_step_workspace_bytes() gives for some."""
    import torch
    ws = torch.empty(szo_workspace_bytes() if nbytes is None else nbytes, dtype=torch.uint8, device=device)
    szo_workspace_init(ws)
    return ws


# ---- between the linear layers ------------------------------------------------------------------
# A descriptor holds device pointers, so its tensors have to outlive it: it keeps them in `keep`.
def _type(t):
    import torch
    try:
        return {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}[t.dtype]
    except KeyError:
        raise ValueError(f"expected fp32, bf16 or fp16, got {t.dtype}") from None


def _strided(t, shape):
    """Pointer and the strides of tokens and heads of [tokens, heads, head_dim]; the last axis has to be contiguous."""
    if t is None:
        return None, 0, 0
    if not t.is_cuda or tuple(t.shape) != tuple(shape) or (t.shape[2] > 1 and t.stride(2) != 1):
        raise ValueError(f"expected a device tensor {tuple(shape)} with a contiguous last axis, got {tuple(t.shape)}, strides {t.stride()}")
    return t.data_ptr(), t.stride(0), t.stride(1)


def _typed(t, dtype, shape):
    """Pointer of a contiguous device tensor of the type and shape that a call reads or writes (None -> NULL)."""
    if t is not None and (t.dtype != dtype or tuple(t.shape) != tuple(shape)):
        raise ValueError(f"expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return _dev(t)


def _room(workspace, need):
    """Pointer of a workspace of at least as many bytes (None -> NULL: the call says whether it can do without)."""
    if workspace is not None and workspace.nbytes < need:
        raise ValueError(f"a workspace of {workspace.nbytes} bytes, this call needs {need}")
    return _dev(workspace)


def make_qk_desc(q, k, positions, cos_table, sin_table, q_out=None, k_out=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False, norm=None):
    """q [tokens, q_heads, head_dim] and k [tokens, kv_heads, head_dim] (or None), any strides with a contiguous last axis; tables fp32
    [rows, rot_dim / 2] (None: no rotation).  `norm` is on where a weight is given, unless said otherwise.  Without outputs: for the backward."""
    import torch
    T, heads, D = q.shape
    kv = 0 if k is None else k.shape[1]
    if k is not None and k.dtype != q.dtype or (q_out is not None and k_out is not None and q_out.dtype != k_out.dtype):
        raise ValueError("queries and keys are of one type, and so are their outputs")
    rows, rot = (0, 0) if cos_table is None else (cos_table.shape[0], 2 * cos_table.shape[1])
    out = q_out if q_out is not None else k_out if k_out is not None else q
    d = QkDesc(T, heads, kv, D, rot, _type(q), _type(out), int((q_weight is not None or k_weight is not None) if norm is None else norm), int(interleaved), eps, 0)
    d.q, d.q_token_stride, d.q_head_stride = _strided(q, (T, heads, D))
    d.k, d.k_token_stride, d.k_head_stride = _strided(k, (T, kv, D))
    d.q_weight, d.k_weight = _typed(q_weight, torch.float32, (D,)), _typed(k_weight, torch.float32, (D,))
    d.positions = _typed(positions, torch.int32, (T,))
    d.cos_table, d.sin_table = _typed(cos_table, torch.float32, (rows, rot // 2)), _typed(sin_table, torch.float32, (rows, rot // 2))
    d.table_rows = rows
    d.q_out, d.q_out_token_stride, d.q_out_head_stride = _strided(q_out, (T, heads, D))
    d.k_out, d.k_out_token_stride, d.k_out_head_stride = _strided(k_out, (T, kv, D))
    d.keep = (q, k, positions, cos_table, sin_table, q_out, k_out, q_weight, k_weight)
    return d


def make_qk_grads(q_out_grad, k_out_grad, q_grad, k_grad, q_weight_grad=None, k_weight_grad=None):
    import torch
    T, _, D = q_grad.shape
    if k_grad is not None and (k_grad.dtype != q_grad.dtype or k_out_grad.dtype != q_out_grad.dtype):
        raise ValueError("gradients of queries and keys are of one type")
    g = QkGrads(_type(q_out_grad), 0)
    g.q_out_grad, g.q_out_token_stride, g.q_out_head_stride = _strided(q_out_grad, q_grad.shape)
    g.q_grad, g.q_token_stride, g.q_head_stride = _strided(q_grad, q_grad.shape)
    if k_grad is not None:
        shape = (T, k_grad.shape[1], D)
        g.k_out_grad, g.k_out_token_stride, g.k_out_head_stride = _strided(k_out_grad, shape)
        g.k_grad, g.k_token_stride, g.k_head_stride = _strided(k_grad, shape)
    g.q_weight_grad, g.k_weight_grad = _typed(q_weight_grad, torch.float32, (D,)), _typed(k_weight_grad, torch.float32, (D,))
    g.shapes = tuple(q_grad.shape), (0 if k_grad is None else k_grad.shape[1]), _type(q_grad)
    g.keep = (q_out_grad, k_out_grad, q_grad, k_grad, q_weight_grad, k_weight_grad)
    return g


def szo_qk_norm_rope(desc, stream=None):
    _check("szo_qk_norm_rope", lib.szo_qk_norm_rope(C.byref(desc), _stream(stream)))


def szo_qk_norm_rope_bwd(desc, grads, workspace=None, stream=None):
    if grads.shapes != ((desc.tokens, desc.q_heads, desc.head_dim), desc.kv_heads, desc.in_type):
        raise ValueError("gradients of other shapes or another type than the inputs")
    need = lib.szo_qk_workspace_bytes(C.byref(desc)) if grads.q_weight_grad or grads.k_weight_grad else 0
    _check("szo_qk_norm_rope_bwd", lib.szo_qk_norm_rope_bwd(C.byref(desc), C.byref(grads), _room(workspace, need), _stream(stream)))


def szo_qk_workspace_bytes(desc):
    return int(lib.szo_qk_workspace_bytes(C.byref(desc)))


def new_kv_cache(pages, page_tokens, kv_heads, head_dim, device="cuda"):
    """(k, v, k_exp, v_exp) of an empty cache."""
    import torch
    shape = (pages, kv_heads, page_tokens // KV_BLOCK, KV_BLOCK * head_dim)
    return tuple(torch.zeros(s, dtype=torch.uint8, device=device) for s in (shape, shape, shape[:3], shape[:3]))


def make_kv_cache(k, v, k_exp, v_exp, page_table, lengths):
    """k, v u8 [pages, kv_heads, page_tokens / 32, 32 * head_dim]; exponents u8 without the last axis; page_table i32 [sequences, max_pages]; lengths i32
    [sequences], which a program updates in place as sequences grow."""
    import torch
    pages, heads, blocks, size = k.shape
    _typed(v, torch.uint8, k.shape)
    c = KvCache(pages, blocks * KV_BLOCK, heads, size // KV_BLOCK, page_table.shape[0], page_table.shape[1], _typed(k, torch.uint8, k.shape), _dev(v),
                _typed(k_exp, torch.uint8, k.shape[:3]), _typed(v_exp, torch.uint8, k.shape[:3]), _typed(page_table, torch.int32, page_table.shape),
                _typed(lengths, torch.int32, (page_table.shape[0],)))
    c.keep = (k, v, k_exp, v_exp, page_table, lengths)
    return c


def make_kv_tokens(k, v, token_start, max_new):
    """k, v [tokens, kv_heads, head_dim]: read by szo_kv_cache_write, written by szo_kv_cache_read."""
    import torch
    if k.dtype != v.dtype:
        raise ValueError("keys and values are of one type")
    t = KvTokens(_type(k), 0, max_new, _typed(token_start, torch.int32, token_start.shape))
    t.k, t.k_token_stride, t.k_head_stride = _strided(k, k.shape)
    t.v, t.v_token_stride, t.v_head_stride = _strided(v, k.shape)
    t.tokens = k.shape[0]
    t.shape = tuple(k.shape[1:]), token_start.shape[0]
    t.keep = (k, v, token_start)
    return t


def _same_cache(cache, tokens):
    if tokens.shape != ((cache.kv_heads, cache.head_dim), cache.sequences + 1):
        raise ValueError("tokens of other heads, another head_dim or another number of sequences than the cache")


def szo_kv_cache_write(cache, tokens, stream=None):
    _same_cache(cache, tokens)
    _check("szo_kv_cache_write", lib.szo_kv_cache_write(C.byref(cache), C.byref(tokens), _stream(stream)))


def szo_kv_cache_read(cache, tokens, stream=None):
    _same_cache(cache, tokens)
    _check("szo_kv_cache_read", lib.szo_kv_cache_read(C.byref(cache), C.byref(tokens), _stream(stream)))


def make_attn_desc(cache, q, out, q_start, max_q, max_len, scale, causal=True, window=0, lse=None):
    """cache from make_kv_cache(); q, out bf16 or fp16 [tokens, q_heads, head_dim]; lse fp32 [tokens, q_heads] or None."""
    import torch
    if out.dtype != q.dtype:
        raise ValueError("queries and output are of one type")
    T, heads, D = q.shape
    if D != cache.head_dim:
        raise ValueError(f"queries of head_dim {D}, a cache of {cache.head_dim}")
    d = AttnDesc(cache, heads, _type(q), int(causal), window, scale, max_q, max_len, 0, T)
    d.q, d.q_token_stride, d.q_head_stride = _strided(q, q.shape)
    d.q_start = _typed(q_start, torch.int32, (cache.sequences + 1,))
    d.out, d.out_token_stride, d.out_head_stride = _strided(out, q.shape)
    d.lse = _typed(lse, torch.float32, (T, heads))
    d.keep = (cache, q, out, q_start, lse)
    return d


def szo_attn_cached(desc, workspace=None, stream=None):
    """workspace: of szo_attn_workspace_bytes() for this very descriptor; fewer sequences or a longer max_len may need more than a larger batch did."""
    room = _room(workspace, lib.szo_attn_workspace_bytes(C.byref(desc)))
    _check("szo_attn_cached", lib.szo_attn_cached(C.byref(desc), room, _stream(stream)))


def szo_attn_workspace_bytes(desc):
    return int(lib.szo_attn_workspace_bytes(C.byref(desc)))


def szo_attn_plan(desc):
    """(tiles of rows side by side, waves that share a tile's cache, parts of the cache, codes pass the caches by)"""
    plan = (C.c_int32 * 4)()
    _check("szo_attn_plan", lib.szo_attn_plan(C.byref(desc), plan))
    return tuple(plan)


def make_logprobs_desc(logits, targets=None, logp=None, entropy=None, stats=None, top_logp=None, top_index=None, scale=1.0, loss_acc=None, loss_scale=1.0):
    """logits [rows, vocab], rows any distance apart; targets i32 [rows]; outputs that are None are not computed."""
    import torch
    R, V = logits.shape
    if not logits.is_cuda or (V > 1 and logits.stride(1) != 1):
        raise ValueError("expected device logits with contiguous rows")
    some = top_index if top_index is not None else top_logp
    top = 0 if some is None else some.shape[1]
    d = LogprobsDesc(R, V, logits.stride(0), _type(logits), top, scale, 0, logits.data_ptr(), _typed(targets, torch.int32, (R,)),
                     _typed(logp, torch.float32, (R,)), _typed(entropy, torch.float32, (R,)), _typed(stats, torch.float32, (R, 2)),
                     _typed(top_logp, torch.float32, (R, top)), _typed(top_index, torch.int32, (R, top)),
                     None if loss_acc is None else _typed(loss_acc, torch.float64, loss_acc.shape), loss_scale)
    d.keep = (logits, targets, logp, entropy, stats, top_logp, top_index, loss_acc)
    return d


def szo_token_logprobs(desc, workspace=None, stream=None):
    """workspace: of szo_logprobs_workspace_bytes() for this very descriptor; fewer rows may need more than many did."""
    room = _room(workspace, lib.szo_logprobs_workspace_bytes(C.byref(desc)))
    _check("szo_token_logprobs", lib.szo_token_logprobs(C.byref(desc), room, _stream(stream)))


def szo_logprobs_workspace_bytes(desc):
    return int(lib.szo_logprobs_workspace_bytes(C.byref(desc)))


def szo_token_logprobs_bwd(desc, grad_logp, grad_entropy, grad_logits, stream=None):
    """grad_logp, grad_entropy fp32 [rows] or None; grad_logits like the logits, or the logits themselves."""
    import torch
    R, V = desc.rows, desc.vocab
    if not grad_logits.is_cuda or tuple(grad_logits.shape) != (R, V) or _type(grad_logits) != desc.type or (V > 1 and grad_logits.stride(1) != 1):
        raise ValueError("expected a gradient of the logits' shape and type")
    _check("szo_token_logprobs_bwd", lib.szo_token_logprobs_bwd(C.byref(desc), _typed(grad_logp, torch.float32, (R,)), _typed(grad_entropy, torch.float32, (R,)),
                                                                grad_logits.data_ptr(), grad_logits.stride(0), _stream(stream)))


# ---- host set-up -----------------------------------------------------------------------------
def szo_num_tiles(N, K):
    return int(lib.szo_num_tiles(N, K))


def szo_mask_generate(N, K, nnz, kind, mask_seed):
    out = np.empty(nnz, dtype=np.uint32)
    _check("szo_mask_generate", lib.szo_mask_generate(N, K, nnz, kind, mask_seed, out.ctypes.data))
    return out


def szo_tcsr_build(N, K, flat_sorted):
    flat, fp = _host(flat_sorted, np.uint32)
    nnz = flat.size
    tile_ptr = np.empty(max(szo_num_tiles(N, K), 0) + 1, dtype=np.uint32)
    sp_idx = np.empty(nnz, dtype=np.uint32)
    perm = np.empty(nnz, dtype=np.uint32)
    _check("szo_tcsr_build", lib.szo_tcsr_build(N, K, fp, nnz, tile_ptr.ctypes.data, sp_idx.ctypes.data,
                                                perm.ctypes.data))
    return tile_ptr, sp_idx, perm


def szo_quantize_pack(W, group, mask_flat):
    W, wp = _host(W, np.float32)
    N, K = W.shape
    mask, mp = _host(mask_flat, np.uint32)
    q = np.empty((N, K // 2), dtype=np.uint8)
    scales = np.empty((N, K // group), dtype=np.uint16)
    sp_val = np.empty(mask.size, dtype=np.float32)
    _check("szo_quantize_pack", lib.szo_quantize_pack(wp, N, K, group, mp, mask.size, q.ctypes.data,
                                                      scales.ctypes.data, sp_val.ctypes.data))
    return q, scales.view(np.float16), sp_val


def szo_quantize_pack_lut(W, mask_flat):
    """-> (q u8 [N,K/2], lut fp16 [N,16], sp_val fp32 [nnz])."""
    W, wp = _host(W, np.float32)
    N, K = W.shape
    mask, mp = _host(mask_flat, np.uint32)
    q = np.empty((N, K // 2), dtype=np.uint8)
    lut = np.empty((N, 16), dtype=np.uint16)
    sp_val = np.empty(mask.size, dtype=np.float32)
    _check("szo_quantize_pack_lut", lib.szo_quantize_pack_lut(wp, N, K, mp, mask.size, q.ctypes.data,
                                                              lut.ctypes.data, sp_val.ctypes.data))
    return q, lut.view(np.float16), sp_val


def szo_qweight_bytes(N, K):
    return int(lib.szo_qweight_bytes(N, K))


def szo_scales_count(N, K, group):
    return int(lib.szo_scales_count(N, K, group))


def szo_layout_weights(q, scales, group):
    """Row-major host arrays -> (q_banded u8 [bytes], scales_banded fp16 [count]).
    scales None (non-uniform format): codes only, -> (q_banded, None)."""
    q, qp = _host(q, np.uint8)
    N, K = q.shape[0], q.shape[1] * 2
    if scales is None:
        qb = np.empty(szo_qweight_bytes(N, K), dtype=np.uint8)
        _check("szo_layout_weights", lib.szo_layout_weights(qp, None, N, K, 0, qb.ctypes.data, None))
        return qb, None
    sc, sp = _host(np.asarray(scales).view(np.uint16), np.uint16)
    qb = np.empty(szo_qweight_bytes(N, K), dtype=np.uint8)
    sb = np.empty(szo_scales_count(N, K, group), dtype=np.uint16)
    _check("szo_layout_weights", lib.szo_layout_weights(qp, sp, N, K, group, qb.ctypes.data, sb.ctypes.data))
    return qb, sb.view(np.float16)


def szo_philox4x32_10(ctr, key):
    c, cp = _host(ctr, np.uint32)
    k, kp = _host(key, np.uint32)
    out = np.empty(4, dtype=np.uint32)
    _check("szo_philox4x32_10", lib.szo_philox4x32_10(cp, kp, out.ctypes.data))
    return out


def szo_debug_zbar(nnz_base, nnz, seed, step, words_out=None, z_out=None, stream=None):
    _check("szo_debug_zbar", lib.szo_debug_zbar(nnz_base, nnz, seed, step, _dev(words_out), _dev(z_out),
                                                _stream(stream)))


def szo_activation_absmax(x, count, absmax_out, stream=None):
    _check("szo_activation_absmax", lib.szo_activation_absmax(_dev(x), count, _dev(absmax_out), _stream(stream)))


def szo_choose_tile_dtype(x_absmax):
    rc = lib.szo_choose_tile_dtype(x_absmax)
    if rc < 0:
        raise SzoError("szo_choose_tile_dtype", rc)
    return rc


def szo_set_tile_config(config):
    _check("szo_set_tile_config", lib.szo_set_tile_config(config))


def szo_kernel_timing(enable):
    _check("szo_kernel_timing", lib.szo_kernel_timing(1 if enable else 0))


def szo_kernel_timing_read():
    """(sum of the recorded forward-kernel durations in ms, number of launches)."""
    ms, n = C.c_double(0.0), C.c_int64(0)
    _check("szo_kernel_timing_read", lib.szo_kernel_timing_read(C.byref(ms), C.byref(n)))
    return ms.value, n.value


def szo_kernel_timing_read2():
    """((forward ms, forward launches), (sparse update ms, sparse update launches))."""
    ms, n = (C.c_double * 2)(), (C.c_int64 * 2)()
    _check("szo_kernel_timing_read2", lib.szo_kernel_timing_read2(ms, n))
    return (ms[0], n[0]), (ms[1], n[1])


def szo_last_hip_error():
    return int(lib.szo_last_hip_error())


def szo_version():
    return int(lib.szo_version())
