"""ctypes binding of libsgd (include/sgd.h, include/sgd_kernels.h).

Argument marshalling only: every step of the denoiser path runs in libsgd's
kernels.  The functions keep the C names; ``Denoiser`` is a small convenience
wrapper that builds the descriptor and weight structs from a config and a dict
of device tensors and keeps those tensors alive.

There is no fallback: if ``libsgd.so`` is missing or fails to load, every call
raises ``RuntimeError``.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libsgd.so")

# status codes (sgd_status)
SGD_OK = 0
SGD_ERR_ARG = -1
SGD_ERR_SHAPE = -2
SGD_ERR_SCHEDULE = -3
SGD_ERR_CACHE_INVALID = -4
SGD_ERR_CUDA = -5
SGD_ERR_DEVICE_TIMEOUT = -6
SGD_ERR_OOM = -7
SGD_ERR_STATE = -8
SGD_ERR_RANGE = -9
SGD_SELFTEST_TIMEOUT_CODE = 99  # status code recorded by sgd_selftest_wait_timeout

STEM = {"time_add": 0, "patch": 1, "patch_tokens": 2, "identity": 3, "embed": 4}
BLOCK = {"prenorm": 0, "adaln": 1, "xattn": 2}
NORM = {"rms": 0, "ln": 1, "ln_plain": 2}
MLP = {"swiglu": 0, "gelu_tanh": 1, "gelu_erf": 2, "geglu": 3}
HEAD = {"linear": 0, "adaln_linear": 1, "identity": 2, "logits": 3}
FLAG_SIMT_GEMM = 1
FLAG_MMA_SYNC_ATTENTION = 2
FLAG_GEMM_BK64 = 8
FLAG_PDL = 16
FLAG_FOLD_NORM = 32
FLAG_SERIAL = 64

EPI_F16, EPI_F32, EPI_DELTA, EPI_GATED, EPI_GELU, EPI_ROPE = range(6)
KERNEL_NAMES = ["gemm_tc", "gemm_simt", "attention", "norm", "frozen_run", "small"]

# every symbol include/*.h declares
EXPORTED = [
    "sgd_create", "sgd_set_schedule", "sgd_step", "sgd_step_host", "sgd_get_active_mask",
    "sgd_get_info", "sgd_reset", "sgd_check_device", "sgd_destroy", "sgd_last_error",
    "sgd_compile_schedule", "sgd_step_profile", "sgd_sampler_update", "sgd_kernel_gemm",
    "sgd_kernel_attention", "sgd_kernel_norm", "sgd_kernel_frozen_run", "sgd_kernel_status",
    "sgd_set_exec_mode", "sgd_step_host_async", "sgd_host_wait", "sgd_kernel_gemm_static_ws",
    "sgd_set_policy", "sgd_get_drift", "sgd_selftest_wait_timeout", "sgd_kernel_f16_clamped",
    "sgd_kernel_gemm_stat_slots", "sgd_kernel_attention_hs", "sgd_kernel_dependent_launches", "sgd_kernel_gemm_tile",
    "sgd_kernel_logprobs", "sgd_kernel_distill", "sgd_sampler_reveal", "sgd_kernel_sample", "sgd_kernel_embedding",
    "sgd_kernel_embedding_grad", "sgd_kernel_embedding_grad_workspace", "sgd_kernel_norm_grad", "sgd_kernel_norm_grad_workspace",
]
EXEC_JAGGED_GRAPH, EXEC_EAGER, EXEC_PADDED_GRAPH = 0, 1, 2
POLICY_STATIC, POLICY_DRIFT = 0, 1
DTYPES = {"float16": 0, "bfloat16": 1, "float32": 2}  # sgd_dtype, by torch's names
TAIL_RENORM, TAIL_BUCKET = 0, 1
TAIL = {"renorm": TAIL_RENORM, "bucket": TAIL_BUCKET}
MAX_ROW_BYTES, REVEAL_MAX_TOKENS = 3 << 20, 49152  # of a row of logits; of a sample that is revealed
MAX_SCALE = 2e38


class sgd_model_desc(C.Structure):
    _fields_ = [(n, C.c_int) for n in (
        "stem", "block", "norm", "mlp", "head", "n_blocks", "d", "n_heads", "d_head", "d_ff",
        "batch", "n_tokens", "n_prefix", "d_in", "d_out", "out_channels", "n_skips", "ctx_len",
        "d_ctx", "vocab", "n_classes", "t_freq", "rope")] + [
        ("rope_theta", C.c_float), ("eps", C.c_float), ("flags", C.c_int)]


class sgd_block_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in (
        "norm1_w", "norm1_b", "w_qkv", "w_o", "normx_w", "normx_b", "wx_q", "wx_kv", "wx_o",
        "norm2_w", "norm2_b", "w_1", "w_2", "w_mod")]


class sgd_weights(C.Structure):
    _fields_ = [("blocks", C.POINTER(sgd_block_weights)), ("w_stem", C.c_void_p),
                ("pos_emb", C.c_void_p), ("w_t1", C.c_void_p), ("w_t2", C.c_void_p),
                ("class_emb", C.c_void_p), ("skip_w", C.POINTER(C.c_void_p)),
                ("normf_w", C.c_void_p), ("normf_b", C.c_void_p), ("w_modf", C.c_void_p),
                ("w_head", C.c_void_p), ("embed", C.c_void_p)]


class sgd_cond(C.Structure):
    _fields_ = [("class_ids", C.c_void_p), ("ctx", C.c_void_p)]


class sgd_info(C.Structure):
    _fields_ = [("n_units", C.c_int), ("n_patterns", C.c_int), ("n_graphs", C.c_int),
                ("T", C.c_int), ("layer_steps", C.c_int64), ("cache_bytes", C.c_size_t),
                ("workspace_bytes", C.c_size_t), ("weight_bytes", C.c_size_t),
                ("policy", C.c_int), ("n_groups", C.c_int), ("graph_steps", C.c_int64),
                ("eager_steps", C.c_int64)]


class sgd_op_record(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("kernel", C.c_int), ("ms", C.c_float),
                ("flops", C.c_double), ("bytes", C.c_double)]


class sgd_epilogue_args(C.Structure):
    _fields_ = [("kind", C.c_int), ("alpha", C.c_float), ("out", C.c_void_p), ("ldo", C.c_int),
                ("h", C.c_void_p),
                ("ldh", C.c_int), ("cache", C.c_void_p), ("ld_cache", C.c_int),
                ("gate", C.c_void_p), ("ld_gate", C.c_int), ("rows_per_batch", C.c_int),
                ("act", C.c_int), ("rope_cos", C.c_void_p), ("rope_sin", C.c_void_p),
                ("rope_tokens", C.c_int), ("d_head", C.c_int), ("rope_cols", C.c_int),
                ("norm", C.c_int), ("rstat", C.c_void_p), ("stat_slots", C.c_int),
                ("stat_ld", C.c_int), ("norm_eps", C.c_float), ("colsum", C.c_void_p),
                ("colbias", C.c_void_p), ("h16", C.c_void_p), ("stat_out", C.c_void_p),
                ("stat_out_ld", C.c_int), ("stat_cnt", C.c_void_p), ("stat_final", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    """Load libsgd.so (raises if it is absent: there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"libsgd.so not built ({LIB_PATH}); run __graft_entry__.build()")
        L = C.CDLL(LIB_PATH)
        vp, i, i64, f = C.c_void_p, C.c_int, C.c_int64, C.c_float
        sig = {
            "sgd_create": (i, [C.POINTER(sgd_model_desc), C.POINTER(sgd_weights), C.POINTER(vp)]),
            "sgd_set_schedule": (i, [vp, i, i, vp, vp]),
            "sgd_step": (i, [vp, vp, vp, f, C.POINTER(sgd_cond), i, vp]),
            "sgd_step_host": (i, [vp, vp, vp, f, vp, vp, i, vp]),
            "sgd_get_active_mask": (i, [vp, i, vp, i]),
            "sgd_get_info": (i, [vp, C.POINTER(sgd_info)]),
            "sgd_reset": (i, [vp]),
            "sgd_check_device": (i, [vp, vp]),
            "sgd_destroy": (None, [vp]),
            "sgd_last_error": (C.c_char_p, []),
            "sgd_compile_schedule": (i, [i, i, vp, vp, vp, vp, vp]),
            "sgd_step_profile": (i, [vp, vp, vp, f, C.POINTER(sgd_cond), i, vp,
                                     C.POINTER(sgd_op_record), i, C.POINTER(C.c_int)]),
            "sgd_sampler_update": (i, [vp, vp, f, f, i64, vp]),
            "sgd_kernel_gemm": (i, [vp, i, vp, i, i, i, i, C.POINTER(sgd_epilogue_args), i, vp]),
            "sgd_kernel_gemm_static_ws": (i, [vp, i, vp, i, i, i, i, C.POINTER(sgd_epilogue_args), i, vp]),
            "sgd_kernel_attention": (i, [vp, i, vp, vp, i, vp, i, i, i, i, i, i, i, vp]),
            "sgd_kernel_attention_hs": (i, [vp, i, vp, vp, i, i, vp, i, i, i, i, i, i, i, vp]),
            "sgd_kernel_norm": (i, [vp, vp, i, i, i, vp, vp, vp, vp, i, i, f, vp]),
            "sgd_kernel_frozen_run": (i, [vp, C.POINTER(vp), i, i64, vp]),
            "sgd_kernel_status": (i, [C.POINTER(C.c_int)]),
            "sgd_kernel_f16_clamped": (i, [C.POINTER(C.c_int)]),
            "sgd_kernel_gemm_stat_slots": (i, [i, i, i, C.POINTER(sgd_epilogue_args), i, C.POINTER(C.c_int)]),
            "sgd_kernel_gemm_tile": (i, [i, i, i, C.POINTER(sgd_epilogue_args), i, C.POINTER(C.c_int),
                                         C.POINTER(C.c_int)]),
            "sgd_kernel_dependent_launches": (i, [C.POINTER(i64)]),
            "sgd_set_exec_mode": (i, [vp, i]),
            "sgd_step_host_async": (i, [vp, vp, vp, f, vp, vp, i, vp]),
            "sgd_host_wait": (i, [vp]),
            "sgd_set_policy": (i, [vp, i]),
            "sgd_selftest_wait_timeout": (i, [vp]),
            "sgd_get_drift": (i, [vp, i, vp, i]),
            "sgd_kernel_logprobs": (i, [vp, i, i64, i, i, f, vp, i, vp, i, vp, vp, i, vp, vp, vp]),
            "sgd_kernel_distill": (i, [vp, i, i64, i, i, f, vp, vp, i, vp, i, vp, vp, i, i64, vp]),
            "sgd_sampler_reveal": (i, [vp, vp, i64, vp, i64, i, vp, vp, vp, vp, i, i, i, vp]),
            "sgd_kernel_sample": (i, [vp, i, i64, i, i, f, i, C.c_double, C.c_double, vp, vp, i, vp, vp, vp]),
            "sgd_kernel_embedding": (i, [vp, i, i64, i, i, vp, i, f, vp, i, i64, vp]),
            "sgd_kernel_embedding_grad_workspace": (i, [i, i, i, C.POINTER(i64)]),
            "sgd_kernel_embedding_grad": (i, [vp, i, i64, vp, i, i, i, f, i, vp, i, i64, vp, i64, vp]),
            "sgd_kernel_norm_grad_workspace": (i, [i, i, i, C.POINTER(i64)]),
            "sgd_kernel_norm_grad": (i, [vp, vp, i, i, i, i, vp, vp, vp, i, i, f, vp, vp, vp, vp, vp, vp, i, vp, i64, vp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


class SgdError(RuntimeError):
    def __init__(self, code: int, where: str):
        msg = lib().sgd_last_error().decode(errors="replace")
        super().__init__(f"{where} failed with status {code}: {msg}")
        self.code = code


def check(code: int, where: str) -> int:
    if code != SGD_OK:
        raise SgdError(code, where)
    return code


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return stream if isinstance(stream, int) else stream.cuda_stream


# ---------------------------------------------------------------------------
# thin wrappers with the C names
# ---------------------------------------------------------------------------

def sgd_compile_schedule(T: int, lifetimes: Sequence[int], groups: Sequence[int]):
    """Host-only schedule compiler: (pattern_of_step[T], writes_at_step[T], n_patterns)."""
    S = np.ascontiguousarray(lifetimes, dtype=np.int32)
    G = np.ascontiguousarray(groups, dtype=np.int32)
    pos = np.zeros(T, np.int32)
    wr = np.zeros(T, np.int32)
    n = C.c_int32()
    check(lib().sgd_compile_schedule(T, len(S), S.ctypes.data, G.ctypes.data, pos.ctypes.data,
                                     wr.ctypes.data, C.byref(n)), "sgd_compile_schedule")
    return pos, wr, int(n.value)


def sgd_kernel_gemm(A, B, M, N, K, epi: sgd_epilogue_args, use_simt=False, lda=None, ldb=None,
                    stream=None):
    return check(lib().sgd_kernel_gemm(_ptr(A), lda or K, _ptr(B), ldb or K, M, N, K,
                                       C.byref(epi), int(use_simt), _stream(stream)),
                 "sgd_kernel_gemm")


def sgd_kernel_gemm_static_ws(A, B, M, N, K, epi: sgd_epilogue_args, variant=0, lda=None, ldb=None,
                              stream=None):
    """sgd_kernel_gemm that allocates no device memory (stream-K scratch in a fixed array)."""
    return check(lib().sgd_kernel_gemm_static_ws(_ptr(A), lda or K, _ptr(B), ldb or K, M, N, K,
                                                 C.byref(epi), int(variant), _stream(stream)),
                 "sgd_kernel_gemm_static_ws")


def sgd_kernel_attention(q, ldq, k, v, ldkv, o, ldo, batch, n_q, n_kv, n_heads, d_head,
                         impl=0, stream=None):
    return check(lib().sgd_kernel_attention(_ptr(q), ldq, _ptr(k), _ptr(v), ldkv, _ptr(o), ldo,
                                            batch, n_q, n_kv, n_heads, d_head, impl,
                                            _stream(stream)), "sgd_kernel_attention")


def sgd_kernel_attention_hs(q, ldq, k, v, ldkv, head_stride, o, ldo, batch, n_q, n_kv, n_heads,
                            d_head, impl=0, stream=None):
    return check(lib().sgd_kernel_attention_hs(_ptr(q), ldq, _ptr(k), _ptr(v), ldkv, head_stride,
                                               _ptr(o), ldo, batch, n_q, n_kv, n_heads, d_head,
                                               impl, _stream(stream)), "sgd_kernel_attention_hs")


def sgd_kernel_norm(h, out, rows, d, kind, g=None, b=None, shift=None, scale=None, ld_mod=0,
                    rows_per_batch=1, eps=1e-6, stream=None):
    return check(lib().sgd_kernel_norm(_ptr(h), _ptr(out), rows, d, kind, _ptr(g), _ptr(b),
                                       _ptr(shift), _ptr(scale), ld_mod, rows_per_batch, eps,
                                       _stream(stream)), "sgd_kernel_norm")


def sgd_kernel_frozen_run(h, caches, stream=None):
    arr = (C.c_void_p * len(caches))(*[c.data_ptr() for c in caches])
    return check(lib().sgd_kernel_frozen_run(_ptr(h), arr, len(caches), h.numel(),
                                             _stream(stream)), "sgd_kernel_frozen_run")


def sgd_kernel_status() -> int:
    st = C.c_int(0)
    check(lib().sgd_kernel_status(C.byref(st)), "sgd_kernel_status")
    return int(st.value)


def sgd_kernel_dependent_launches() -> int:
    n = C.c_int64(0)
    check(lib().sgd_kernel_dependent_launches(C.byref(n)), "sgd_kernel_dependent_launches")
    return int(n.value)


def sgd_kernel_gemm_tile(M, N, K, epi: "sgd_epilogue_args", variant=0):
    group, columns = C.c_int(0), C.c_int(0)
    check(lib().sgd_kernel_gemm_tile(M, N, K, C.byref(epi), int(variant), C.byref(group), C.byref(columns)),
          "sgd_kernel_gemm_tile")
    return int(group.value), int(columns.value)


def sgd_kernel_gemm_stat_slots(M, N, K, epi: "sgd_epilogue_args", variant=0) -> int:
    n = C.c_int(0)
    check(lib().sgd_kernel_gemm_stat_slots(M, N, K, C.byref(epi), int(variant), C.byref(n)),
          "sgd_kernel_gemm_stat_slots")
    return int(n.value)


def sgd_kernel_f16_clamped() -> int:
    st = C.c_int(0)
    check(lib().sgd_kernel_f16_clamped(C.byref(st)), "sgd_kernel_f16_clamped")
    return int(st.value)


def sgd_sampler_update(z, eps, alpha, beta, stream=None):
    return check(lib().sgd_sampler_update(_ptr(z), _ptr(eps), alpha, beta, z.numel(),
                                          _stream(stream)), "sgd_sampler_update")


# The operators on a token model's logits take tensors whose sizes are checked here, as the C side
# sees only pointers: shapes, types and devices (TypeError / ValueError), before anything is launched.

def _tensor(t, name, dtype, shape, device):
    """Address of `t` (or None): a dense tensor of this type, shape and device."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    raise ValueError(f"{name} must be contiguous")


_MOST = 2 ** 31 - 1  # rows, columns


def _too_many(name):
    raise ValueError(f"{name} has more rows or columns than a 32-bit integer holds")


def _id(value, name):
    """A token id or a size as the library has it: ctypes would cut one of more than 32 bits down to another."""
    if not -2 ** 31 <= value < 2 ** 31:
        raise ValueError(f"{name} must be a 32-bit integer")
    return value


def _rows(t, name):
    """(type, row stride) of a [rows, vocab] tensor on a CUDA device with dense rows."""
    kind = _dtypes().get(t.dtype)
    if kind is None:
        raise TypeError(f"{name} must be float16, bfloat16 or float32, not {t.dtype}")
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name} must be a 2-d tensor on a CUDA device")
    rows, vocab = t.shape
    if rows > _MOST or vocab > _MOST:
        _too_many(name)
    ld, step = t.stride()
    if step != 1 and vocab > 1:
        raise ValueError(f"the rows of {name} must be dense")
    return kind, ld if rows > 1 else max(ld, vocab)


_dtype_codes = None


def _dtypes():
    global _dtype_codes
    if _dtype_codes is None:
        import torch
        _dtype_codes = {getattr(torch, n): c for n, c in DTYPES.items()}
    return _dtype_codes


def _call_on(device, fn, name, stream, *args):
    """The library launches on the current device: that of the tensors, for the time of the call.  The
    current stream comes as its handle where torch has a call for that: making the stream's object takes
    longer than launching a small kernel."""
    import torch
    if stream is None:
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        stream = torch.cuda.current_stream(device) if raw is None else raw(device.index)
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, _stream(stream))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _stream(stream))
    return rc if rc == SGD_OK else check(rc, name)


def sgd_kernel_logprobs(logits, tokens=None, token_logprobs=None, entropy=None, top_ids=None, top_logprobs=None,
                        scale=1.0, row_ids=None, row_id=0, stream=None):
    """Log-probabilities of given tokens, entropy and likeliest tokens of logits [rows, vocab] (any row
    stride), into the output tensors that are given: token_logprobs float32 [rows, n] for tokens int32
    [rows, n], entropy float32 [rows], top_ids int32 and top_logprobs float32 [rows, k].  With row_ids
    (int32 [rows]) only rows whose entry is row_id are read and written."""
    import torch
    kind, ld = _rows(logits, "logits")
    rows, vocab = logits.shape
    device, i32, f32 = logits.device, torch.int32, torch.float32
    if (tokens is None) != (token_logprobs is None):
        raise ValueError("tokens and token_logprobs go together")
    n = k = 0
    if tokens is not None:
        if tokens.dim() != 2:
            raise ValueError("tokens must have the shape [rows, n]")
        n = tokens.shape[1]
    top = top_ids if top_ids is not None else top_logprobs
    if top is not None:
        if top.dim() != 2:
            raise ValueError("top_ids and top_logprobs must have the shape [rows, k]")
        k = top.shape[1]
    return _call_on(device, lib().sgd_kernel_logprobs, "sgd_kernel_logprobs", stream,
                    logits.data_ptr(), kind, ld, rows, vocab, scale,
                    _tensor(row_ids, "row_ids", i32, (rows,), device), _id(row_id, "row_id"),
                    _tensor(tokens, "tokens", i32, (rows, n), device), n,
                    _tensor(token_logprobs, "token_logprobs", f32, (rows, n), device),
                    _tensor(entropy, "entropy", f32, (rows,), device), k,
                    _tensor(top_ids, "top_ids", i32, (rows, k), device),
                    _tensor(top_logprobs, "top_logprobs", f32, (rows, k), device))


def sgd_kernel_sample(logits, uniforms, ids, logprobs=None, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, row_ids=None, row_id=0,
                      stream=None):
    """A token drawn from each row of logits [rows, vocab] (any row stride) by two numbers in [0, 1) a row (uniforms
    float32 [rows, 2]) into ids int32 [rows], and its log-probability (under softmax(scale * logits), whatever is filtered
    out) into logprobs float32 [rows]: from the top_k likeliest tokens (0: all) that have at least min_p times the
    likeliest one's probability, and of those from the likeliest that together have the share top_p.  scale is 1 /
    temperature.  With row_ids (int32 [rows]) only rows whose entry is row_id are read and written."""
    import torch
    kind, ld = _rows(logits, "logits")
    rows, vocab = logits.shape
    device, i32, f32 = logits.device, torch.int32, torch.float32
    return _call_on(device, lib().sgd_kernel_sample, "sgd_kernel_sample", stream,
                    logits.data_ptr(), kind, ld, rows, vocab, scale, _id(top_k, "top_k"), top_p, min_p,
                    _tensor(uniforms, "uniforms", f32, (rows, 2), device),
                    _tensor(row_ids, "row_ids", i32, (rows,), device), _id(row_id, "row_id"),
                    _tensor(ids, "ids", i32, (rows,), device), _tensor(logprobs, "logprobs", f32, (rows,), device))


def sgd_kernel_embedding(table, ids, out, scale=1.0, stream=None):
    """out [rows, d] = scale * table[ids] for table [vocab, d] and ids int32 [rows], table and out of any of the three types and
    any row stride; zeros where an id is not in the table (a Denoiser's stem takes the first or last row there)."""
    import torch
    kind, ld = _rows(table, "table")
    okind, ldo = _rows(out, "out")
    vocab, d = table.shape
    rows = out.shape[0]
    if out.shape[1] != d or out.device != table.device:
        raise ValueError("out must have the width and the device of table")
    return _call_on(table.device, lib().sgd_kernel_embedding, "sgd_kernel_embedding", stream,
                    table.data_ptr(), kind, ld, vocab, d, _tensor(ids, "ids", torch.int32, (rows,), table.device), rows, scale,
                    out.data_ptr(), okind, ldo)


def sgd_kernel_embedding_grad_workspace(rows, vocab, d) -> int:
    """Bytes of workspace of sgd_kernel_embedding_grad."""
    n = C.c_int64(0)
    check(lib().sgd_kernel_embedding_grad_workspace(_id(rows, "rows"), _id(vocab, "vocab"), _id(d, "d"), C.byref(n)), "sgd_kernel_embedding_grad_workspace")
    return int(n.value)


def _workspace(workspace, need, device, stream):
    """(workspace, bytes): the given one, or one of torch's allocator on the stream the call goes to."""
    import torch
    if workspace is None:
        if stream is None:
            with torch.cuda.device(device):
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
        else:
            # (an integer handle: torch's allocator has to know which stream uses the memory)
            # (and the default stream's handle is 0, of which ExternalStream makes another stream)
            st = stream
            if isinstance(stream, int):
                st = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
            with torch.cuda.device(device), torch.cuda.stream(st):
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
        return workspace, need
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"the workspace must be contiguous and on {device}")
    return workspace, workspace.numel() * workspace.element_size()


def sgd_kernel_embedding_grad(grad, ids, dtable, scale=1.0, accumulate=False, workspace=None, stream=None):
    """dtable [vocab, d] = (with accumulate: +=) scale * sum of grad [rows, d] over the rows of each token of ids int32 [rows];
    both of any of the three types and any row stride.  workspace: a tensor of sgd_kernel_embedding_grad_workspace bytes
    (None: allocated for the call)."""
    import torch
    kind, ld = _rows(grad, "grad")
    tkind, ldt = _rows(dtable, "dtable")
    rows, d = grad.shape
    vocab, device = dtable.shape[0], grad.device
    if dtable.shape[1] != d or dtable.device != device:
        raise ValueError("dtable must have the width and the device of grad")
    at = _tensor(ids, "ids", torch.int32, (rows,), device)
    need = sgd_kernel_embedding_grad_workspace(rows, vocab, d) if workspace is None else 0
    ws, n = _workspace(workspace, need, device, stream)
    return _call_on(device, lib().sgd_kernel_embedding_grad, "sgd_kernel_embedding_grad", stream,
                    grad.data_ptr(), kind, ld, at, rows, vocab, d, scale, int(accumulate), dtable.data_ptr(), tkind, ldt,
                    ws.data_ptr(), n)


def sgd_kernel_norm_grad_workspace(rows, d, rows_per_batch=0) -> int:
    """Bytes of workspace of sgd_kernel_norm_grad (rows_per_batch 0: without a modulation; any number from rows on: one sample)."""
    n = C.c_int64(0)
    check(lib().sgd_kernel_norm_grad_workspace(_id(rows, "rows"), _id(d, "d"), min(rows_per_batch, 2 ** 31 - 1), C.byref(n)), "sgd_kernel_norm_grad_workspace")
    return int(n.value)


def _modulation(t, name, samples, d, device):
    """(address, row stride) of a float32 [samples, d] tensor with dense rows (one part of a wider modulation, say)."""
    import torch
    if t.dtype is not torch.float32:
        raise TypeError(f"{name} must be torch.float32, not {t.dtype}")
    if t.shape != (samples, d) or t.device != device:
        raise ValueError(f"{name} must have the shape {(samples, d)} and be on {device}")
    if t.stride(1) != 1:
        raise ValueError(f"the rows of {name} must be dense")
    return t.data_ptr(), t.stride(0) if samples > 1 else max(t.stride(0), d)


def sgd_kernel_norm_grad(dout, h, kind, dh=None, g=None, b=None, scale=None, rows_per_batch=1, eps=1e-6, residual=None, dg=None,
                         db=None, dshift=None, dscale=None, workspace=None, stream=None):
    """Backward pass of sgd_kernel_norm on h float32 [rows, d]: from dout [rows, d] (any of the three types) the gradients
    that are given, dh float32 [rows, d] (plus residual float32 [rows, d], which may be dh), dg and db float32 [d] for
    g and b bfloat16 [d], dshift and dscale float32 [samples, d] (of one row stride) for the modulation scale float32 [samples, d]
    of rows_per_batch rows a sample.  workspace: a tensor of sgd_kernel_norm_grad_workspace bytes (None: allocated for
    the call)."""
    import torch
    bf16, f32 = torch.bfloat16, torch.float32
    if h.dim() != 2 or not h.is_cuda:
        raise ValueError("h must be a 2-d tensor on a CUDA device")
    shape, device = h.shape, h.device
    rows, d = shape
    if rows > _MOST or d > _MOST:
        _too_many("h")
    code = _dtypes().get(dout.dtype)
    if code is None:
        raise TypeError(f"dout must be float16, bfloat16 or float32, not {dout.dtype}")
    at_scale, ld, at_shift, at_dscale, ldd = None, 0, None, None, 0
    if scale is None and (dshift is not None or dscale is not None):
        raise ValueError("dshift and dscale need scale")
    if scale is not None:
        if rows_per_batch < 1:
            raise ValueError("rows_per_batch must be positive")
        rows_per_batch = min(rows_per_batch, max(rows, 1))  # (a longer period is one sample too, and may pass 32 bits)
        samples = -(-rows // rows_per_batch)
        at_scale, ld = _modulation(scale, "scale", samples, d, device)
        if dshift is not None:
            at_shift, ldd = _modulation(dshift, "dshift", samples, d, device)
        if dscale is not None:
            at_dscale, ld2 = _modulation(dscale, "dscale", samples, d, device)
            if dshift is not None and samples > 1 and ld2 != ldd:
                raise ValueError("dshift and dscale must have one row stride")
            ldd = max(ldd, ld2)
    args = (_tensor(h, "h", f32, shape, device), _tensor(dout, "dout", dout.dtype, shape, device), code, rows, d, kind,
            _tensor(g, "g", bf16, (d,), device), _tensor(b, "b", bf16, (d,), device), at_scale, ld, rows_per_batch, eps,
            _tensor(residual, "residual", f32, shape, device), _tensor(dh, "dh", f32, shape, device),
            _tensor(dg, "dg", f32, (d,), device), _tensor(db, "db", f32, (d,), device), at_shift, at_dscale, ldd)
    need = 0
    if workspace is None and (dg is not None or db is not None or ldd):
        need = sgd_kernel_norm_grad_workspace(rows, d, 0 if scale is None else rows_per_batch)
    ws, n = _workspace(workspace, need, device, stream) if need or workspace is not None else (None, 0)
    return _call_on(device, lib().sgd_kernel_norm_grad, "sgd_kernel_norm_grad", stream, *args, _ptr(ws), n)


def sgd_kernel_distill(logits, teacher_ids, teacher_logprobs, loss, grad=None, row_weight=None, tail=TAIL_BUCKET,
                       scale=1.0, stream=None):
    """Divergence of logits [rows, vocab] from the teacher's lists [rows, k] (sgd_kernel_logprobs' top_ids and
    top_logprobs), into loss float32 [rows] and, where given, its gradient [rows, vocab] of any of the
    three types (or logits itself)."""
    import torch
    kind, ld = _rows(logits, "logits")
    rows, vocab = logits.shape
    device, f32 = logits.device, torch.float32
    if teacher_ids.dim() != 2:
        raise ValueError("teacher_ids must have the shape [rows, k]")
    k = teacher_ids.shape[1]
    gkind = ldg = 0
    if grad is not None:
        gkind, ldg = _rows(grad, "grad")
        if grad.shape != logits.shape or grad.device != device:
            raise ValueError("grad must have the shape and the device of logits")
    return _call_on(device, lib().sgd_kernel_distill, "sgd_kernel_distill", stream,
                    logits.data_ptr(), kind, ld, rows, vocab, scale,
                    _tensor(teacher_ids, "teacher_ids", torch.int32, (rows, k), device),
                    _tensor(teacher_logprobs, "teacher_logprobs", f32, (rows, k), device), k,
                    _tensor(row_weight, "row_weight", f32, (rows,), device), tail,
                    _tensor(loss, "loss", f32, (rows,), device),
                    None if grad is None else grad.data_ptr(), gkind, ldg)


def _column(t, name, dtype, shape, device):
    """(address, stride) of a [batch, n_tokens] tensor whose positions are evenly spaced (a column of a
    [batch, n_tokens, k] one, say)."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape or t.device != device:
        raise ValueError(f"{name} must have the shape {tuple(shape)} and be on {device}")
    a, b = t.stride()
    if shape[1] <= 1:
        b = a
    if t.numel() > 1 and (b < 1 or shape[0] > 1 and a != b * shape[1]):
        raise ValueError(f"the positions of {name} must be evenly spaced")
    return t.data_ptr(), max(b, 1)


def sgd_sampler_reveal(ids, cand, score, n_reveal, ids_out, mask_id, lowest=False, window=None, n_left=None,
                       stream=None):
    """The masked positions of ids int32 [batch, n_tokens] with the best scores (n_reveal int32 [batch] of them;
    window int32 [batch, 2]: between these positions) take their candidates in ids_out (which may
    be ids); n_left int32 [batch]: masked positions that were not chosen (a candidate that is mask_id itself leaves its
    position masked, and chosen)."""
    import torch
    if ids.dim() != 2 or not ids.is_cuda:
        raise ValueError("ids must be a 2-d tensor on a CUDA device")
    device, shape, i32 = ids.device, ids.shape, torch.int32
    batch, n = shape
    pc, sc = _column(cand, "cand", i32, shape, device)
    ps, ss = _column(score, "score", torch.float32, shape, device)
    return _call_on(device, lib().sgd_sampler_reveal, "sgd_sampler_reveal", stream,
                    _tensor(ids, "ids", i32, shape, device), pc, sc, ps, ss, int(lowest),
                    _tensor(n_reveal, "n_reveal", i32, (batch,), device),
                    _tensor(window, "window", i32, (batch, 2), device),
                    _tensor(ids_out, "ids_out", i32, shape, device),
                    _tensor(n_left, "n_left", i32, (batch,), device), batch, n, _id(mask_id, "mask_id"))


def make_desc(cfg, flags: int = 0) -> sgd_model_desc:
    return sgd_model_desc(
        stem=STEM[cfg.stem], block=BLOCK[cfg.block], norm=NORM[cfg.norm], mlp=MLP[cfg.mlp],
        head=HEAD[cfg.head], n_blocks=cfg.n_blocks, d=cfg.d, n_heads=cfg.n_heads,
        d_head=cfg.d_head, d_ff=cfg.d_ff, batch=cfg.batch, n_tokens=cfg.n_tokens,
        n_prefix=cfg.n_prefix, d_in=cfg.d_in, d_out=cfg.d_out, out_channels=cfg.out_channels,
        n_skips=cfg.n_skips, ctx_len=cfg.ctx_len, d_ctx=cfg.d_ctx, vocab=cfg.vocab,
        n_classes=cfg.n_classes, t_freq=cfg.t_freq, rope=int(cfg.rope),
        rope_theta=cfg.rope_theta, eps=cfg.eps, flags=flags)


class Denoiser:
    """One libsgd context for a model config and its device weights."""

    def __init__(self, cfg, weights: Dict[str, "object"], flags: int = 0):
        self.cfg = cfg
        self._w = weights  # keep the tensors alive for the context's lifetime
        self.n_units = cfg.n_units
        blocks = (sgd_block_weights * cfg.n_blocks)()
        for b in range(cfg.n_blocks):
            for f, _ in sgd_block_weights._fields_:
                setattr(blocks[b], f, _ptr(weights.get(f"blocks.{b}.{f}")))
        self._blocks = blocks
        skips = (C.c_void_p * max(cfg.n_skips, 1))()
        for j in range(cfg.n_skips):
            skips[j] = _ptr(weights[f"skips.{j}.w"])
        self._skips = skips
        W = sgd_weights(blocks=blocks, skip_w=skips)
        for f in ("w_stem", "pos_emb", "w_t1", "w_t2", "class_emb", "normf_w", "normf_b",
                  "w_modf", "w_head", "embed"):
            setattr(W, f, _ptr(weights.get(f)))
        self._desc = make_desc(cfg, flags)
        h = C.c_void_p()
        check(lib().sgd_create(C.byref(self._desc), C.byref(W), C.byref(h)), "sgd_create")
        self.handle = h.value
        self.T = 0

    def close(self):
        if getattr(self, "handle", None):
            lib().sgd_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_schedule(self, T: int, lifetimes: Sequence[int], groups: Sequence[int]):
        S = np.ascontiguousarray(lifetimes, dtype=np.int32)
        G = np.ascontiguousarray(groups, dtype=np.int32)
        check(lib().sgd_set_schedule(self.handle, T, len(S), S.ctypes.data, G.ctypes.data),
              "sgd_set_schedule")
        self.T = T

    def _cond(self, class_ids=None, ctx=None) -> sgd_cond:
        return sgd_cond(class_ids=_ptr(class_ids), ctx=_ptr(ctx))

    def step(self, state, out, t: float, step: int, class_ids=None, ctx=None, stream=None):
        cond = self._cond(class_ids, ctx)
        return check(lib().sgd_step(self.handle, _ptr(state), _ptr(out), float(t),
                                    C.byref(cond), step, _stream(stream)), "sgd_step")

    def step_tokens(self, ids, ids_out, logits, t: float, step: int, cand, score, n_reveal, mask_id: int,
                    by: str = "confidence", scale: float = 1.0, window=None, n_left=None, stream=None, class_ids=None,
                    ctx=None, uniforms=None, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
        """One step of a masked-token trajectory (argmax remasking), queued on one stream: the denoiser on ids
        int32 [B, N] (with class_ids int32 [B] and ctx bf16 [B, L, d_ctx] as step takes them) into logits fp16 [B, N, V],
        the best token of every masked position into cand int32 [B, N] with its log-probability (by "confidence") or its
        row's entropy (by "entropy") in score float32 [B, N], and the n_reveal best of them revealed in ids_out
        (which may be ids).  What cand and score hold at other positions stays.  A position whose best token is
        mask_id itself counts as revealed in n_left, and stays masked.  With uniforms float32 [B, N, 2] candidates are drawn
        (sgd_kernel_sample, with scale, top_k, top_p and min_p) instead of the best.  The arguments are checked before
        the step is launched (TypeError / ValueError)."""
        import torch
        if by not in ("confidence", "entropy"):
            raise ValueError("by must be confidence or entropy")
        c = self.cfg
        if c.stem != "embed" or c.head != "logits":
            raise ValueError("step_tokens needs a token model (an embed stem and a logits head)")
        if c.d_out * 2 > MAX_ROW_BYTES or c.n_tokens > REVEAL_MAX_TOKENS:
            raise ValueError("the vocabulary or the sample is beyond what the operators on logits take")
        if not 0.0 < C.c_float(scale).value <= C.c_float(MAX_SCALE).value:
            raise ValueError("scale must be positive and at most 2e38")
        _id(mask_id, "mask_id")
        if uniforms is None and (top_k, top_p, min_p) != (0, 1.0, 0.0):
            raise ValueError("top_k, top_p and min_p go with uniforms: without, the best token is taken")
        if not (0 <= _id(top_k, "top_k") and 0.0 < top_p <= 1.0 and 0.0 <= min_p <= 1.0):
            raise ValueError("top_k must not be negative, top_p be above 0 and at most 1, min_p in 0..1")
        device, i32, f32 = ids.device, torch.int32, torch.float32
        shape = (c.batch, c.n_tokens)
        for x, name, dtype, of in ((ids, "ids", i32, shape), (ids_out, "ids_out", i32, shape), (cand, "cand", i32, shape),
                                   (score, "score", f32, shape), (logits, "logits", torch.float16, (*shape, c.d_out)),
                                   (n_reveal, "n_reveal", i32, (c.batch,))):
            if x is None:
                raise TypeError(f"{name} is needed")
            _tensor(x, name, dtype, of, device)
        _tensor(window, "window", i32, (c.batch, 2), device)
        _tensor(n_left, "n_left", i32, (c.batch,), device)
        _tensor(uniforms, "uniforms", f32, (*shape, 2), device)
        _tensor(class_ids, "class_ids", i32, (c.batch,), device)
        _tensor(ctx, "ctx", torch.bfloat16, (c.batch, c.ctx_len, c.d_ctx), device)
        if not ids.is_cuda:
            raise ValueError("ids must be on a CUDA device")
        self.step(ids, logits, t, step, class_ids=class_ids, ctx=ctx, stream=stream)
        rows = logits.view(-1, logits.shape[-1])
        which = dict(scale=scale, row_ids=ids.view(-1), row_id=mask_id, stream=stream)
        if uniforms is None:
            out = dict(top_logprobs=score.view(-1, 1)) if by == "confidence" else dict(entropy=score.view(-1))
            sgd_kernel_logprobs(rows, top_ids=cand.view(-1, 1), **out, **which)
        else:
            sgd_kernel_sample(rows, uniforms.view(-1, 2), cand.view(-1), logprobs=score.view(-1) if by == "confidence" else None,
                              top_k=top_k, top_p=top_p, min_p=min_p, **which)
            if by == "entropy":
                sgd_kernel_logprobs(rows, entropy=score.view(-1), **which)
        return sgd_sampler_reveal(ids, cand, score, n_reveal, ids_out, mask_id, lowest=by == "entropy", window=window,
                                  n_left=n_left, stream=stream)

    def step_host(self, state_host, out_host, t: float, step: int, class_ids_host=None,
                  ctx_host=None, stream=None):
        """Host (preferably pinned) torch tensors in and out; synchronous."""
        return check(lib().sgd_step_host(self.handle, _ptr(state_host), _ptr(out_host),
                                         float(t), _ptr(class_ids_host), _ptr(ctx_host), step,
                                         _stream(stream)), "sgd_step_host")

    def step_host_async(self, state_host, out_host, t: float, step: int, class_ids_host=None,
                        ctx_host=None, stream=None):
        """Queued host-buffer step; out_host is valid after host_wait()."""
        return check(lib().sgd_step_host_async(self.handle, _ptr(state_host), _ptr(out_host),
                                               float(t), _ptr(class_ids_host), _ptr(ctx_host),
                                               step, _stream(stream)), "sgd_step_host_async")

    def host_wait(self):
        return check(lib().sgd_host_wait(self.handle), "sgd_host_wait")

    def profile_step(self, state, out, t: float, step: int, class_ids=None, ctx=None,
                     stream=None, max_records: int = 4096) -> List[dict]:
        cond = self._cond(class_ids, ctx)
        recs = (sgd_op_record * max_records)()
        n = C.c_int(0)
        check(lib().sgd_step_profile(self.handle, _ptr(state), _ptr(out), float(t),
                                     C.byref(cond), step, _stream(stream), recs, max_records,
                                     C.byref(n)), "sgd_step_profile")
        return [dict(name=recs[i].name.decode(), kernel=KERNEL_NAMES[recs[i].kernel],
                     ms=recs[i].ms, flops=recs[i].flops, bytes=recs[i].bytes)
                for i in range(n.value)]

    def active_mask(self, step: int) -> np.ndarray:
        m = np.zeros(self.n_units, np.uint8)
        check(lib().sgd_get_active_mask(self.handle, step, m.ctypes.data, self.n_units),
              "sgd_get_active_mask")
        return m

    def info(self) -> dict:
        i = sgd_info()
        check(lib().sgd_get_info(self.handle, C.byref(i)), "sgd_get_info")
        return {f: getattr(i, f) for f, _ in sgd_info._fields_}

    def reset(self):
        check(lib().sgd_reset(self.handle), "sgd_reset")

    def set_exec_mode(self, mode: int):
        check(lib().sgd_set_exec_mode(self.handle, mode), "sgd_set_exec_mode")

    def set_policy(self, policy: int):
        """POLICY_STATIC (lifetimes) or POLICY_DRIFT (the input-aware baseline of App. B.1)."""
        check(lib().sgd_set_policy(self.handle, policy), "sgd_set_policy")

    def drift(self, step: int) -> np.ndarray:
        """Lagged drifts the drift policy ranked to choose `step`'s active groups."""
        n = self.info()["n_groups"]
        d = np.zeros(n, np.float64)
        check(lib().sgd_get_drift(self.handle, step, d.ctypes.data, n), "sgd_get_drift")
        return d

    def check_device(self, stream=None):
        return check(lib().sgd_check_device(self.handle, _stream(stream)), "sgd_check_device")
