"""Python binding of libsimsd.so (argument marshalling only).

Each function has the name of the C entry point it calls (include/simsd.h)
and takes torch CUDA tensors; it reads shapes and data pointers, passes them
with the current CUDA stream, and raises :class:`SimsdError` on a non-zero
status.  Every step of the computation runs in the library's kernels; there
is no fallback: if the library is missing or fails to load, the first call
raises.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_build", "libsimsd.so")

SIMSD_OK, SIMSD_ERR_INVALID_ARG, SIMSD_ERR_UNSUPPORTED, SIMSD_ERR_CUDA, SIMSD_ERR_DEVICE = 0, 1, 2, 3, 4
SIMSD_F32, SIMSD_BF16 = 0, 1
SECT_DATA, SECT_MASK, SECT_PAD = 0, 1, 255
EW_STEP_MAP, EW_PREFIX_LEN, EW_PAGE, EW_DRAFT, EW_TIMEOUT, EW_ACCEPT_LEN = 1, 2, 4, 8, 16, 32
EW_TOKENS, EW_SAMPLE = 64, 128
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
STEP_UNDRAFTED, STEP_DECODED = -1, -2

EXPORTED = ("simsd_build_mask", "simsd_verify_workspace_bytes", "simsd_verify_attention",
            "simsd_verify_attention_noalloc", "simsd_accept", "simsd_accept_workspace_bytes", "simsd_accept_ws",
            "simsd_accept_sampled", "simsd_accept_sampled_workspace_bytes", "simsd_accept_sampled_ws",
            "simsd_kv_commit", "simsd_plan_attention", "simsd_plan_accept",
            "simsd_rope_plan_init", "simsd_rope_rotate", "simsd_rope_append", "simsd_chunk_workspace_bytes",
            "simsd_chunk_attention", "simsd_sample",
            "simsd_check_error", "simsd_debug_expire_next_wait",
            "simsd_last_error", "simsd_version")
DEBUG_WAIT_ATTENTION, DEBUG_WAIT_ACCEPT = 1, 2


class SimsdError(RuntimeError):
    def __init__(self, status, where, detail=""):
        super().__init__(f"{where} failed with status {status}: {detail}")
        self.status = status


class RopePlan(ctypes.Structure):
    """simsd_rope_plan of the C ABI (host memory; fill it with
    :func:`simsd_rope_plan_init` and keep it)."""
    _fields_ = [("layout", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("turn", ctypes.c_uint64 * 64)]


_lib = None
_lock = threading.Lock()


def load_library(path: str = LIB_PATH):
    """Loads libsimsd.so once; raises if it is missing (build it with
    ``paper_2606_02544_gb300.build.build()``)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(path):
                raise RuntimeError(f"libsimsd.so not found at {path}; run paper_2606_02544_gb300.build.build()")
            lib = ctypes.CDLL(path)
            P, I, F, Z = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
            lib.simsd_build_mask.argtypes = [P, P, I, I, P, P, P, P, P, P]
            lib.simsd_verify_workspace_bytes.argtypes = [I, I, I, I, I, I, I, I]
            lib.simsd_verify_workspace_bytes.restype = Z
            lib.simsd_verify_attention.argtypes = [I, P, P, P, P, P, I, P, I, I, P, P, P, P, F, I, I, I, I, I, F,
                                                   P, P, Z, P, P]
            lib.simsd_verify_attention_noalloc.argtypes = [I, P, P, P, P, P, I, P, I, I, P, P, P, P, F, I, I, I, I,
                                                           I, F, P, P, P]
            lib.simsd_accept.argtypes = [P, P, I, I, I, P, P, P, P, P]
            lib.simsd_accept_workspace_bytes.argtypes = [I, I, I]
            lib.simsd_accept_workspace_bytes.restype = Z
            lib.simsd_accept_ws.argtypes = [P, P, I, I, I, P, P, P, P, Z, P, P]
            lib.simsd_accept_sampled.argtypes = [P, P, P, P, P, F, I, I, I, P, P, P, P]
            lib.simsd_accept_sampled_workspace_bytes.argtypes = [I, I, I]
            lib.simsd_accept_sampled_workspace_bytes.restype = Z
            lib.simsd_accept_sampled_ws.argtypes = [P, P, P, P, P, F, I, I, I, P, P, P, Z, P, P]
            lib.simsd_kv_commit.argtypes = [I, P, P, I, P, P, P, F, P, P, P, I, P, I, I, P, I, I, I, I, P, P]
            lib.simsd_check_error.argtypes = [P, P, P]
            lib.simsd_debug_expire_next_wait.argtypes = [I, ctypes.c_uint]
            lib.simsd_plan_attention.argtypes = [I, I, I, I, I, I, I, I, I, P, P]
            lib.simsd_plan_accept.argtypes = [I, I, I, I, I, P, P]
            D, S = ctypes.c_double, ctypes.c_int64
            lib.simsd_rope_plan_init.argtypes = [P, I, I, D, I, D, I, D, D]
            lib.simsd_rope_rotate.argtypes = [I, P, P, P, S, P, S, I, P, S, P, S, I, I, I, P]
            lib.simsd_rope_append.argtypes = [I, P, P, S, P, S, P, S, P, P, P, I, I, I, I, I, P, P, P, I, P, I, I,
                                              P, P]
            lib.simsd_chunk_workspace_bytes.argtypes = [I, I, I, I, I, I, I, I]
            lib.simsd_chunk_workspace_bytes.restype = Z
            lib.simsd_chunk_attention.argtypes = [I, P, S, P, P, P, P, P, I, P, I, I, I, I, I, I, I, I, I, F, P, P,
                                                  P, Z, P, P]
            lib.simsd_sample.argtypes = [I, P, S, I, I, P, P, P, P, P, P, P, P, P, P, P]
            lib.simsd_last_error.restype = ctypes.c_char_p
            for name in ("simsd_build_mask", "simsd_verify_attention", "simsd_verify_attention_noalloc",
                         "simsd_accept", "simsd_accept_sampled", "simsd_kv_commit", "simsd_check_error",
                         "simsd_debug_expire_next_wait", "simsd_version", "simsd_plan_attention",
                         "simsd_plan_accept", "simsd_rope_plan_init", "simsd_rope_rotate", "simsd_rope_append",
                         "simsd_chunk_attention", "simsd_sample"):
                getattr(lib, name).restype = ctypes.c_int
            _lib = lib
    return _lib


def _p(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _check(rc, where):
    if rc != SIMSD_OK:
        detail = load_library().simsd_last_error().decode(errors="replace")
        raise SimsdError(rc, where, detail)


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return SIMSD_BF16
    if t.dtype == torch.float32:
        return SIMSD_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def simsd_version() -> int:
    return load_library().simsd_version()


def simsd_plan_attention(dtype, Bt, gamma, Hq, Hkv, d, max_pages, page_size, num_sms):
    """The plan simsd_verify_attention takes on a GPU with num_sms SMs (no
    device needed): dict of kernel, nsplit, streamk, rows_blk, fuse and
    ws_bytes."""
    plan = (ctypes.c_int32 * 5)()
    ws = ctypes.c_size_t(0)
    rc = load_library().simsd_plan_attention(dtype, Bt, gamma, Hq, Hkv, d, max_pages, page_size, num_sms,
                                             ctypes.cast(plan, ctypes.c_void_p), ctypes.cast(ctypes.pointer(ws),
                                                                                            ctypes.c_void_p))
    _check(rc, "simsd_plan_attention")
    return {"kernel": plan[0], "nsplit": plan[1], "streamk": plan[2], "rows_blk": plan[3], "fuse": plan[4],
            "ws_bytes": ws.value}


def simsd_plan_accept(sampled, Bt, gamma, vocab, num_sms):
    """(parts, ws_bytes) of simsd_accept_ws (sampled False) or
    simsd_accept_sampled_ws (True) on a GPU with num_sms SMs."""
    parts = ctypes.c_int32(0)
    ws = ctypes.c_size_t(0)
    rc = load_library().simsd_plan_accept(int(bool(sampled)), Bt, gamma, vocab, num_sms,
                                          ctypes.cast(ctypes.pointer(parts), ctypes.c_void_p),
                                          ctypes.cast(ctypes.pointer(ws), ctypes.c_void_p))
    _check(rc, "simsd_plan_accept")
    return parts.value, ws.value


def simsd_build_mask(step_map, prefix_len, gamma, tau, section, rope_pos, mask_bits=None, err_word=None,
                     stream=None):
    Bt = prefix_len.shape[0]
    rc = load_library().simsd_build_mask(_p(step_map), _p(prefix_len), Bt, gamma, _p(tau), _p(section),
                                         _p(rope_pos), _p(mask_bits), _p(err_word), _stream(stream))
    _check(rc, "simsd_build_mask")


def simsd_verify_workspace_bytes(dtype_code, Bt, gamma, Hq, Hkv, d, max_pages, page_size) -> int:
    return int(load_library().simsd_verify_workspace_bytes(dtype_code, Bt, gamma, Hq, Hkv, d, max_pages, page_size))


def simsd_verify_attention(q, k_new, v_new, k_cache, v_cache, block_table, prefix_len, tau, section, out,
                           workspace=None, err_word=None, softmax_scale=0.0, rope_pos=None, rope_theta=0.0,
                           stream=None):
    """q/out [Bt][2g][Hq][d]; k_new/v_new [Bt][2g][Hkv][d];
    k_cache/v_cache [num_pages][Hkv][P][d]; block_table [Bt][max_pages].
    rope_pos [Bt][2g] (with rope_theta > 0): q and k_new are rotated first."""
    Bt, S, Hq, d = q.shape
    Hkv = k_new.shape[2]
    num_pages, _, P, _ = k_cache.shape
    max_pages = block_table.shape[1]
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = load_library().simsd_verify_attention(
        _dtype_code(q), _p(q), _p(k_new), _p(v_new), _p(k_cache), _p(v_cache), num_pages, _p(block_table),
        max_pages, P, _p(prefix_len), _p(tau), _p(section), _p(rope_pos), float(rope_theta), Bt, S // 2, Hq, Hkv,
        d, float(softmax_scale), _p(out), _p(workspace), ws_bytes, _p(err_word), _stream(stream))
    _check(rc, "simsd_verify_attention")


def simsd_verify_attention_noalloc(q, k_new, v_new, k_cache, v_cache, block_table, prefix_len, tau, section, out,
                                   err_word=None, softmax_scale=0.0, rope_pos=None, rope_theta=0.0, stream=None):
    """simsd_verify_attention without a workspace: the library's static
    device scratch is used instead (for callers that cannot allocate)."""
    Bt, S, Hq, d = q.shape
    Hkv = k_new.shape[2]
    num_pages, _, P, _ = k_cache.shape
    max_pages = block_table.shape[1]
    rc = load_library().simsd_verify_attention_noalloc(
        _dtype_code(q), _p(q), _p(k_new), _p(v_new), _p(k_cache), _p(v_cache), num_pages, _p(block_table),
        max_pages, P, _p(prefix_len), _p(tau), _p(section), _p(rope_pos), float(rope_theta), Bt, S // 2, Hq, Hkv,
        d, float(softmax_scale), _p(out), _p(err_word), _stream(stream))
    _check(rc, "simsd_verify_attention_noalloc")


def simsd_accept(logits, draft, accepted_len, out_tokens, row_argmax=None, err_word=None, stream=None):
    Bt, rows, V = logits.shape
    rc = load_library().simsd_accept(_p(logits), _p(draft), Bt, rows - 1, V, _p(accepted_len), _p(out_tokens),
                                     _p(row_argmax), _p(err_word), _stream(stream))
    _check(rc, "simsd_accept")


def simsd_accept_workspace_bytes(Bt, gamma, vocab) -> int:
    return int(load_library().simsd_accept_workspace_bytes(Bt, gamma, vocab))


def simsd_accept_ws(logits, draft, accepted_len, out_tokens, workspace=None, row_argmax=None, err_word=None,
                    stream=None):
    """simsd_accept with a caller workspace (uint8 device tensor of
    simsd_accept_workspace_bytes() bytes, or None when that is 0)."""
    Bt, rows, V = logits.shape
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = load_library().simsd_accept_ws(_p(logits), _p(draft), Bt, rows - 1, V, _p(accepted_len), _p(out_tokens),
                                        _p(row_argmax), _p(workspace), nbytes, _p(err_word), _stream(stream))
    _check(rc, "simsd_accept_ws")


def simsd_accept_sampled(target_logits, draft_logits, draft, u_accept, u_sample, accepted_len, out_tokens,
                         temperature=1.0, err_word=None, stream=None):
    """target_logits [Bt][g+1][V], draft_logits [Bt][g][V] fp32; draft [Bt][g];
    u_accept [Bt][g], u_sample [Bt] fp32 uniform draws."""
    Bt, rows, V = target_logits.shape
    rc = load_library().simsd_accept_sampled(_p(target_logits), _p(draft_logits), _p(draft), _p(u_accept),
                                             _p(u_sample), float(temperature), Bt, rows - 1, V, _p(accepted_len),
                                             _p(out_tokens), _p(err_word), _stream(stream))
    _check(rc, "simsd_accept_sampled")


def simsd_kv_commit(k_new, v_new, tau, section, accepted_len, k_cache, v_cache, block_table, prefix_len,
                    err_word=None, rope_pos=None, rope_theta=0.0, stream=None):
    """k_new/v_new [L][Bt][2g][Hkv][d]; k_cache/v_cache [L][num_pages][Hkv][P][d].
    rope_pos [Bt][2g] (with rope_theta > 0): committed keys are rotated."""
    L, Bt, S, Hkv, d = k_new.shape
    num_pages, P = k_cache.shape[1], k_cache.shape[3]
    rc = load_library().simsd_kv_commit(
        _dtype_code(k_new), _p(k_new), _p(v_new), L, _p(tau), _p(section), _p(rope_pos), float(rope_theta),
        _p(accepted_len), _p(k_cache),
        _p(v_cache), num_pages, _p(block_table), block_table.shape[1], P, _p(prefix_len), Bt, S // 2, Hkv, d,
        _p(err_word), _stream(stream))
    _check(rc, "simsd_kv_commit")


def simsd_debug_expire_next_wait(which, limit_us):
    """Test hook: the next attention (DEBUG_WAIT_ATTENTION) or acceptance
    (DEBUG_WAIT_ACCEPT) call of this thread waits for an arrival that never
    comes and gives up after limit_us."""
    _check(load_library().simsd_debug_expire_next_wait(int(which), int(limit_us)), "simsd_debug_expire_next_wait")


def simsd_check_error(err_word, stream=None):
    """Synchronises the stream; returns the device error word (int)."""
    w = ctypes.c_int32(0)
    rc = load_library().simsd_check_error(_p(err_word), ctypes.byref(w), _stream(stream))
    if rc not in (SIMSD_OK, SIMSD_ERR_DEVICE):
        _check(rc, "simsd_check_error")
    return int(w.value)


def simsd_accept_sampled_workspace_bytes(Bt, gamma, vocab) -> int:
    return int(load_library().simsd_accept_sampled_workspace_bytes(Bt, gamma, vocab))


def simsd_accept_sampled_ws(target_logits, draft_logits, draft, u_accept, u_sample, accepted_len, out_tokens,
                            workspace=None, temperature=1.0, err_word=None, stream=None):
    """simsd_accept_sampled with a caller workspace (uint8 device tensor of
    simsd_accept_sampled_workspace_bytes() bytes, or None when that is 0)."""
    Bt, rows, V = target_logits.shape
    nbytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    rc = load_library().simsd_accept_sampled_ws(_p(target_logits), _p(draft_logits), _p(draft), _p(u_accept),
                                                _p(u_sample), float(temperature), Bt, rows - 1, V, _p(accepted_len),
                                                _p(out_tokens), _p(workspace), nbytes, _p(err_word),
                                                _stream(stream))
    _check(rc, "simsd_accept_sampled_ws")


# ------------------------------------------------------------------ prompts
def _ptr(t):
    return None if t is None else t.data_ptr()


def _raw_stream(stream):
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _rows(t, name):
    """Token stride of a [T][H][d] tensor whose heads are dense."""
    T, H, d = t.shape
    s = t.stride()
    _need((s[2] == 1 or d == 1) and (s[1] == d or H == 1), f"{name}: the heads of a token must be dense")
    return s[0] if T > 1 else H * d


def _int32(t, n, name):
    _need(t.dtype == torch.int32 and t.numel() == n and t.is_contiguous(), f"{name}: {n} dense int32 wanted")


def _cache_sizes(k_cache, v_cache, block_table, Bt, Hkv, d, dtype):
    _need(k_cache.shape == v_cache.shape and k_cache.dim() == 4 and k_cache.shape[1] == Hkv
          and k_cache.shape[3] == d and k_cache.dtype == dtype and v_cache.dtype == dtype
          and k_cache.is_contiguous() and v_cache.is_contiguous(), "k_cache / v_cache: [num_pages][Hkv][P][d] wanted")
    _need(block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.shape[0] == Bt
          and block_table.is_contiguous(), "block_table: dense int32 [Bt][max_pages] wanted")
    return k_cache.shape[0], block_table.shape[1], k_cache.shape[2]


def simsd_rope_plan_init(layout, rot_dim, theta, scaling="none", factor=1.0, context=0, beta_fast=32.0,
                         beta_slow=1.0) -> RopePlan:
    """The rotation of a model's heads: layout "half" or "interleaved" over the
    first rot_dim components; scaling "none", "linear", "ntk" or "yarn" by
    ``factor`` (YaRN: over a trained ``context``).  Host only; keep the plan."""
    plan = RopePlan()
    rc = load_library().simsd_rope_plan_init(ctypes.addressof(plan), ROPE_LAYOUTS[layout], rot_dim, theta,
                                             ROPE_SCALINGS[scaling], factor, context, beta_fast, beta_slow)
    _check(rc, "simsd_rope_plan_init")
    return plan


def simsd_rope_rotate(plan, positions, q, q_out, k=None, k_out=None, stream=None):
    """q/q_out [T][Hq][d], k/k_out [T][Hkv][d] (token strides allowed, in place
    allowed); positions [T] int32."""
    T, Hq, d = q.shape
    _need(q_out.shape == q.shape and q_out.dtype == q.dtype, "q_out: shape and type of q wanted")
    _int32(positions, T, "positions")
    Hkv = ks = kos = 0
    if k is not None:
        Hkv, ks = k.shape[1], _rows(k, "k")
        _need(k.shape == (T, Hkv, d) and k_out is not None and k_out.shape == k.shape and k.dtype == q.dtype
              and k_out.dtype == q.dtype, "k / k_out: [T][Hkv][d] of q's type wanted")
        kos = _rows(k_out, "k_out")
    rc = load_library().simsd_rope_rotate(_dtype_code(q), ctypes.addressof(plan), positions.data_ptr(), q.data_ptr(),
                                          _rows(q, "q"), q_out.data_ptr(), _rows(q_out, "q_out"), Hq, _ptr(k), ks,
                                          _ptr(k_out) if k is not None else None, kos, Hkv, T, d,
                                          _raw_stream(stream))
    _check(rc, "simsd_rope_rotate")


def simsd_rope_append(plan, q, k, v, token_start, prefix_len, q_out, k_cache, v_cache, block_table, positions=None,
                      err_word=None, stream=None):
    """q [T][Hq][d], k/v [T][Hkv][d] (token strides allowed); token_start
    [Bt+1], prefix_len [Bt]; q_out [T][Hq][d] dense; k_cache/v_cache
    [num_pages][Hkv][P][d].  prefix_len is not advanced."""
    T, Hq, d = q.shape
    Hkv, Bt = k.shape[1], prefix_len.shape[0]
    _need(k.shape == (T, Hkv, d) and v.shape == k.shape and k.dtype == q.dtype and v.dtype == q.dtype,
          "k / v: [T][Hkv][d] of q's type wanted")
    _need(q_out.shape == q.shape and q_out.dtype == q.dtype and q_out.is_contiguous(), "q_out: dense, like q")
    _int32(token_start, Bt + 1, "token_start")
    _int32(prefix_len, Bt, "prefix_len")
    if positions is not None:
        _int32(positions, T, "positions")
    num_pages, max_pages, P = _cache_sizes(k_cache, v_cache, block_table, Bt, Hkv, d, q.dtype)
    rc = load_library().simsd_rope_append(
        _dtype_code(q), ctypes.addressof(plan), q.data_ptr(), _rows(q, "q"), k.data_ptr(), _rows(k, "k"),
        v.data_ptr(), _rows(v, "v"), token_start.data_ptr(), prefix_len.data_ptr(), _ptr(positions), T, Bt, Hq, Hkv,
        d, q_out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), num_pages, block_table.data_ptr(), max_pages, P,
        _ptr(err_word), _raw_stream(stream))
    _check(rc, "simsd_rope_append")


def simsd_chunk_workspace_bytes(dtype_code, T, Bt, Hq, Hkv, d, max_pages, page_size) -> int:
    return int(load_library().simsd_chunk_workspace_bytes(dtype_code, T, Bt, Hq, Hkv, d, max_pages, page_size))


def simsd_chunk_attention(q, token_start, prefix_len, k_cache, v_cache, block_table, out, lse=None, mask_block=1,
                          window=0, key_start=None, softmax_scale=0.0, workspace=None, err_word=None, stream=None):
    """q [T][Hq][d] (token stride allowed), rotated; the cache already holds the
    chunk's keys and values.  mask_block 1: causal, B: block-causal, 0: all;
    window > 0: that many rows back; key_start [Bt]: earlier rows hidden.
    out [T][Hq][d], lse [T][Hq] fp32."""
    T, Hq, d = q.shape
    Bt, Hkv = prefix_len.shape[0], k_cache.shape[1]
    _need(out.shape == q.shape and out.dtype == q.dtype and out.is_contiguous(), "out: dense, like q")
    _int32(token_start, Bt + 1, "token_start")
    _int32(prefix_len, Bt, "prefix_len")
    if key_start is not None:
        _int32(key_start, Bt, "key_start")
    if lse is not None:
        _need(lse.shape == (T, Hq) and lse.dtype == torch.float32 and lse.is_contiguous(),
              "lse: dense float32 [T][Hq] wanted")
    num_pages, max_pages, P = _cache_sizes(k_cache, v_cache, block_table, Bt, Hkv, d, q.dtype)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = load_library().simsd_chunk_attention(
        _dtype_code(q), q.data_ptr(), _rows(q, "q"), token_start.data_ptr(), prefix_len.data_ptr(), _ptr(key_start),
        k_cache.data_ptr(), v_cache.data_ptr(), num_pages, block_table.data_ptr(), max_pages, P, T, Bt, Hq, Hkv, d,
        mask_block, window, softmax_scale, out.data_ptr(), _ptr(lse), _ptr(workspace), ws_bytes, _ptr(err_word),
        _raw_stream(stream))
    _check(rc, "simsd_chunk_attention")


def simsd_sample(logits, u, token, temperature=None, top_k=None, top_p=None, min_p=None, kept=None, log_prob=None,
                 log_probs=None, err_word=None, stream=None):
    """logits [R][V] float32 or bfloat16 (row stride allowed); u, temperature,
    top_p, min_p [R] float32, top_k [R] int32; token/kept [R] int32,
    log_prob [R] and log_probs [R][V] float32 (outputs; all but token
    optional)."""
    R, V = logits.shape
    _need(logits.stride(1) == 1 or V == 1, "logits: dense rows wanted")
    for t, name in ((u, "u"), (temperature, "temperature"), (top_p, "top_p"), (min_p, "min_p"), (log_prob, "log_prob")):
        _need(t is None or (t.dtype == torch.float32 and t.numel() == R and t.is_contiguous()),
              f"{name}: {R} dense float32 wanted")
    for t, name in ((token, "token"), (top_k, "top_k"), (kept, "kept")):
        if t is not None:
            _int32(t, R, name)
    _need(log_probs is None or (log_probs.shape == (R, V) and log_probs.dtype == torch.float32
                                and log_probs.is_contiguous()), "log_probs: dense float32 [R][V] wanted")
    rc = load_library().simsd_sample(
        _dtype_code(logits), logits.data_ptr(), logits.stride(0) if R > 1 else V, R, V, u.data_ptr(),
        _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), token.data_ptr(), _ptr(kept), _ptr(log_prob),
        _ptr(log_probs), _ptr(err_word), _raw_stream(stream))
    _check(rc, "simsd_sample")
