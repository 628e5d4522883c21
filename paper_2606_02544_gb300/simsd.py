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
EW_POOL, EW_SEQ, EW_SHARED = 256, 512, 1024
MAX_PAGE_ARRAYS = 8
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
STEP_UNDRAFTED, STEP_DECODED = -1, -2

EXPORTED = ("simsd_build_mask", "simsd_verify_workspace_bytes", "simsd_verify_attention",
            "simsd_verify_attention_noalloc", "simsd_accept", "simsd_accept_workspace_bytes", "simsd_accept_ws",
            "simsd_accept_sampled", "simsd_accept_sampled_workspace_bytes", "simsd_accept_sampled_ws",
            "simsd_kv_commit", "simsd_plan_attention", "simsd_plan_accept",
            "simsd_rope_plan_init", "simsd_rope_rotate", "simsd_rope_append", "simsd_chunk_workspace_bytes",
            "simsd_chunk_attention", "simsd_chunk_attention_sinks", "simsd_rope_append_q4", "simsd_q4_expand",
            "simsd_chunk_q4_workspace_bytes", "simsd_chunk_attention_q4", "simsd_pages_extend",
            "simsd_pages_extend_granted", "simsd_pages_release", "simsd_pages_workspace_bytes", "simsd_pages_fork", "simsd_pages_compact",
            "simsd_sample", "simsd_check_error", "simsd_debug_expire_next_wait",
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


class _Q4Cache(ctypes.Structure):
    """simsd_q4_cache of the C ABI."""
    _fields_ = [("k_codes", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("v_scales", ctypes.c_void_p), ("k_unit", ctypes.c_float), ("v_unit", ctypes.c_float)]


class _PageArray(ctypes.Structure):
    """simsd_page_array of the C ABI."""
    _fields_ = [("base", ctypes.c_void_p), ("page_bytes", ctypes.c_int64), ("layer_bytes", ctypes.c_int64),
                ("layers", ctypes.c_int64)]


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
            lib.simsd_chunk_attention_sinks.argtypes = [I, P, S, P, P, P, P, P, I, P, I, I, I, I, I, I, I, I, I, I, F,
                                                        P, P, P, Z, P, P]
            lib.simsd_rope_append_q4.argtypes = [I, P, P, S, P, S, P, S, P, P, P, I, I, I, I, I, P, P, I, P, I, I,
                                                 P, P]
            lib.simsd_q4_expand.argtypes = [I, P, I, P, I, I, P, P, I, I, I, P, P, P, P]
            lib.simsd_chunk_q4_workspace_bytes.argtypes = [I, I, I, I, I, I, I, I, I]
            lib.simsd_chunk_q4_workspace_bytes.restype = Z
            lib.simsd_chunk_attention_q4.argtypes = [I, P, S, P, P, P, P, I, P, I, I, I, I, I, I, I, I, I, I, F, P, P,
                                                     P, Z, P, P]
            lib.simsd_pages_extend.argtypes = [P, P, P, P, I, I, I, I, P, P]
            lib.simsd_pages_extend_granted.argtypes = [P, P, P, P, I, I, I, I, P, P, P]
            lib.simsd_pages_release.argtypes = [P, P, P, I, P, P, I, I, I, I, P, P]
            lib.simsd_pages_workspace_bytes.argtypes = [I, I]
            lib.simsd_pages_workspace_bytes.restype = Z
            lib.simsd_pages_fork.argtypes = [P, I, P, P, I, P, P, P, I, I, I, I, P, Z, P, P]
            lib.simsd_pages_compact.argtypes = [P, I, P, P, I, I, I, P, P, Z, P, P]
            lib.simsd_sample.argtypes = [I, P, S, I, I, P, P, P, P, P, P, P, P, P, P, P]
            lib.simsd_last_error.restype = ctypes.c_char_p
            for name in ("simsd_build_mask", "simsd_verify_attention", "simsd_verify_attention_noalloc",
                         "simsd_accept", "simsd_accept_sampled", "simsd_kv_commit", "simsd_check_error",
                         "simsd_debug_expire_next_wait", "simsd_version", "simsd_plan_attention",
                         "simsd_plan_accept", "simsd_rope_plan_init", "simsd_rope_rotate", "simsd_rope_append",
                         "simsd_chunk_attention", "simsd_chunk_attention_sinks", "simsd_rope_append_q4",
                         "simsd_q4_expand", "simsd_chunk_attention_q4", "simsd_pages_extend",
                         "simsd_pages_extend_granted", "simsd_pages_release", "simsd_pages_fork", "simsd_pages_compact", "simsd_sample"):
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
# (These calls sit in decoding loops of a few microseconds, so their checks
# are written out, and no message is built unless one fails.)
_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32


def _ptr(t):
    return None if t is None else t.data_ptr()


def _wrong(what):
    raise ValueError(what)


_devices = torch.cuda.device_count()  # (with one, a tensor on a GPU is on the current one)


def _elsewhere():
    _wrong("tensors on the current CUDA device wanted")


def _device(t):
    """The device that the library will plan for and launch on, which has to
    be the tensor's."""
    dev = t.get_device()
    if dev < 0 or (_devices > 1 and dev != torch._C._cuda_getDevice()):
        _elsewhere()
    return dev


def _error_word(t, dev):
    if t is None:
        return None
    if t.dtype is not _I32 or t.get_device() != dev or t.numel() < 1:
        _wrong("err_word: int32 on the current CUDA device wanted")
    return t.data_ptr()


def _raw_stream(stream, dev):
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(dev)


def _code(dtype):
    if dtype is _BF16:
        return SIMSD_BF16
    if dtype is _F32:
        return SIMSD_F32
    raise TypeError(f"unsupported dtype {dtype}")


def _rows(t, H, d, name):
    """Token stride of a [T][H][d] tensor whose heads are dense."""
    s0, s1, s2 = t.stride()
    if (s2 != 1 and d > 1) or (s1 != d and H > 1):
        raise ValueError(f"{name}: the heads of a token must be dense")
    return s0 if t.shape[0] > 1 else H * d


def _dense_i32(t, n):
    return t.dtype is _I32 and t.numel() == n and t.is_contiguous()


def _cache_sizes(k_cache, v_cache, block_table, Bt, Hkv, d, dtype):
    N, h, P, dd = k_cache.shape
    if not (h == Hkv and dd == d and v_cache.shape == (N, h, P, d) and k_cache.dtype is dtype
            and v_cache.dtype is dtype and k_cache.is_contiguous() and v_cache.is_contiguous()):
        raise ValueError("k_cache / v_cache: dense [num_pages][Hkv][P][d] of q's type wanted")
    n, max_pages = block_table.shape
    if not (n == Bt and block_table.dtype is _I32 and block_table.is_contiguous()):
        raise ValueError("block_table: dense int32 [Bt][max_pages] wanted")
    return N, max_pages, P


def simsd_rope_plan_init(layout, rot_dim, theta, scaling="none", factor=1.0, context=0, beta_fast=32.0,
                         beta_slow=1.0) -> RopePlan:
    """The rotation of a model's heads: layout "half" or "interleaved" over the
    first rot_dim components; scaling "none", "linear", "ntk" or "yarn" by
    ``factor`` (YaRN: over a trained ``context``).  Host only; keep the plan."""
    if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
        _wrong(f"layout {sorted(ROPE_LAYOUTS)}, scaling {sorted(ROPE_SCALINGS)}")
    plan = RopePlan()
    rc = load_library().simsd_rope_plan_init(ctypes.addressof(plan), ROPE_LAYOUTS[layout], rot_dim, theta,
                                             ROPE_SCALINGS[scaling], factor, context, beta_fast, beta_slow)
    _check(rc, "simsd_rope_plan_init")
    return plan


def simsd_rope_rotate(plan, positions, q, q_out, k=None, k_out=None, stream=None):
    """q/q_out [T][Hq][d], k/k_out [T][Hkv][d] (token strides allowed, in place
    allowed); positions [T] int32."""
    T, Hq, d = q.shape
    dt = q.dtype
    if q_out.shape != (T, Hq, d) or q_out.dtype is not dt:
        _wrong("q_out: shape and type of q wanted")
    if not _dense_i32(positions, T):
        _wrong("positions: dense int32 [T] wanted")
    Hkv = ks = kos = 0
    kp = kop = None
    if k is not None:
        Hkv = k.shape[1]
        if (k_out is None or k.shape != (T, Hkv, d) or k_out.shape != (T, Hkv, d) or k.dtype is not dt
                or k_out.dtype is not dt):
            _wrong("k / k_out: [T][Hkv][d] of q's type wanted")
        ks, kos = _rows(k, Hkv, d, "k"), _rows(k_out, Hkv, d, "k_out")
        kp, kop = k.data_ptr(), k_out.data_ptr()
    dev = _device(q)
    if not (dev == positions.get_device() == q_out.get_device() and
            (k is None or dev == k.get_device() == k_out.get_device())):
        _elsewhere()
    rc = (_lib or load_library()).simsd_rope_rotate(
        _code(dt), ctypes.addressof(plan), positions.data_ptr(), q.data_ptr(), _rows(q, Hq, d, "q"),
        q_out.data_ptr(), _rows(q_out, Hq, d, "q_out"), Hq, kp, ks, kop, kos, Hkv, T, d, _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_rope_rotate")


def simsd_rope_append(plan, q, k, v, token_start, prefix_len, q_out, k_cache, v_cache, block_table, positions=None,
                      err_word=None, stream=None):
    """q [T][Hq][d], k/v [T][Hkv][d] (token strides allowed); token_start
    [Bt+1], prefix_len [Bt]; q_out [T][Hq][d] dense; k_cache/v_cache
    [num_pages][Hkv][P][d].  prefix_len is not advanced."""
    T, Hq, d = q.shape
    Tk, Hkv, dk = k.shape
    Bt, dt = prefix_len.shape[0], q.dtype
    if Tk != T or dk != d or v.shape != (T, Hkv, d) or k.dtype is not dt or v.dtype is not dt:
        _wrong("k / v: [T][Hkv][d] of q's type wanted")
    if q_out.shape != (T, Hq, d) or q_out.dtype is not dt or not q_out.is_contiguous():
        _wrong("q_out: dense, like q")
    if (token_start.dtype is not _I32 or token_start.numel() != Bt + 1 or not token_start.is_contiguous()
            or prefix_len.dtype is not _I32 or prefix_len.numel() != Bt or not prefix_len.is_contiguous()):
        _wrong("token_start / prefix_len: dense int32 [Bt+1] / [Bt] wanted")
    if positions is not None and not _dense_i32(positions, T):
        _wrong("positions: dense int32 [T] wanted")
    (qs, q1, q2), (ks, k1, k2), (vs, v1, v2) = q.stride(), k.stride(), v.stride()
    if (q1 != d and Hq > 1) or ((k1 != d or v1 != d) and Hkv > 1) or not (q2 == k2 == v2 == 1 or d == 1):
        _wrong("q / k / v: the heads of a token must be dense")
    if T <= 1:
        qs, ks, vs = Hq * d, Hkv * d, Hkv * d
    num_pages, max_pages, P = _cache_sizes(k_cache, v_cache, block_table, Bt, Hkv, d, dt)
    dev = _device(q)
    if not (dev == k.get_device() == v.get_device() == token_start.get_device() == prefix_len.get_device()
            == q_out.get_device() == k_cache.get_device() == v_cache.get_device() == block_table.get_device()
            and (positions is None or positions.get_device() == dev)):
        _elsewhere()
    rc = (_lib or load_library()).simsd_rope_append(
        _code(dt), ctypes.addressof(plan), q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs,
        token_start.data_ptr(), prefix_len.data_ptr(), _ptr(positions), T, Bt, Hq, Hkv, d, q_out.data_ptr(),
        k_cache.data_ptr(), v_cache.data_ptr(), num_pages, block_table.data_ptr(), max_pages, P,
        _error_word(err_word, dev), _raw_stream(stream, dev))
    if rc:
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
    Bt, Hkv, dt = prefix_len.shape[0], k_cache.shape[1], q.dtype
    if out.shape != (T, Hq, d) or out.dtype is not dt or not out.is_contiguous():
        _wrong("out: dense, like q")
    if not _dense_i32(token_start, Bt + 1) or not _dense_i32(prefix_len, Bt):
        _wrong("token_start / prefix_len: dense int32 [Bt+1] / [Bt] wanted")
    if key_start is not None and not _dense_i32(key_start, Bt):
        _wrong("key_start: dense int32 [Bt] wanted")
    if lse is not None and (lse.shape != (T, Hq) or lse.dtype is not _F32 or not lse.is_contiguous()):
        _wrong("lse: dense float32 [T][Hq] wanted")
    num_pages, max_pages, P = _cache_sizes(k_cache, v_cache, block_table, Bt, Hkv, d, dt)
    dev = _device(q)
    if not (dev == token_start.get_device() == prefix_len.get_device() == out.get_device() == k_cache.get_device()
            == v_cache.get_device() == block_table.get_device() and (lse is None or lse.get_device() == dev)
            and (key_start is None or key_start.get_device() == dev)
            and (workspace is None or workspace.get_device() == dev)):
        _elsewhere()
    ws = ws_bytes = 0
    if workspace is not None:
        ws, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = (_lib or load_library()).simsd_chunk_attention(
        _code(dt), q.data_ptr(), _rows(q, Hq, d, "q"), token_start.data_ptr(), prefix_len.data_ptr(),
        _ptr(key_start), k_cache.data_ptr(), v_cache.data_ptr(), num_pages, block_table.data_ptr(), max_pages, P, T,
        Bt, Hq, Hkv, d, mask_block, window, softmax_scale, out.data_ptr(), _ptr(lse), ws, ws_bytes,
        _error_word(err_word, dev), _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_chunk_attention")


# --------------------------------------------------------------- long caches
def _chunk_checks(q, token_start, prefix_len, block_table, out, lse, key_start, workspace):
    """What the calls of chunk attention over long caches check alike: the device, and the
    workspace's address and size."""
    T, Hq, d = q.shape
    Bt = prefix_len.shape[0]
    if out.shape != (T, Hq, d) or out.dtype is not q.dtype or not out.is_contiguous():
        _wrong("out: dense, like q")
    if not _dense_i32(token_start, Bt + 1) or not _dense_i32(prefix_len, Bt):
        _wrong("token_start / prefix_len: dense int32 [Bt+1] / [Bt] wanted")
    if key_start is not None and not _dense_i32(key_start, Bt):
        _wrong("key_start: dense int32 [Bt] wanted")
    if lse is not None and (lse.shape != (T, Hq) or lse.dtype is not _F32 or not lse.is_contiguous()):
        _wrong("lse: dense float32 [T][Hq] wanted")
    dev = _device(q)
    if not (dev == token_start.get_device() == prefix_len.get_device() == out.get_device()
            == block_table.get_device() and (lse is None or lse.get_device() == dev)
            and (key_start is None or key_start.get_device() == dev)
            and (workspace is None or workspace.get_device() == dev)):
        _elsewhere()
    if workspace is None:
        return dev, 0, 0
    if not workspace.is_contiguous():
        _wrong("workspace: dense tensor wanted")
    return dev, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def simsd_chunk_attention_sinks(q, token_start, prefix_len, k_cache, v_cache, block_table, out, window, sinks,
                                lse=None, mask_block=1, key_start=None, softmax_scale=0.0, workspace=None,
                                err_word=None, stream=None):
    """simsd_chunk_attention through a window of ``window`` rows beside which the
    first ``sinks`` rows (from key_start on) stay visible; the workspace is
    that of simsd_chunk_workspace_bytes."""
    T, Hq, d = q.shape
    Bt, Hkv, dt = prefix_len.shape[0], k_cache.shape[1], q.dtype
    num_pages, max_pages, P = _cache_sizes(k_cache, v_cache, block_table, Bt, Hkv, d, dt)
    dev, ws, ws_bytes = _chunk_checks(q, token_start, prefix_len, block_table, out, lse, key_start, workspace)
    if not dev == k_cache.get_device() == v_cache.get_device():
        _elsewhere()
    rc = (_lib or load_library()).simsd_chunk_attention_sinks(
        _code(dt), q.data_ptr(), _rows(q, Hq, d, "q"), token_start.data_ptr(), prefix_len.data_ptr(),
        _ptr(key_start), k_cache.data_ptr(), v_cache.data_ptr(), num_pages, block_table.data_ptr(), max_pages, P, T,
        Bt, Hq, Hkv, d, mask_block, window, sinks, softmax_scale, out.data_ptr(), _ptr(lse), ws, ws_bytes,
        _error_word(err_word, dev), _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_chunk_attention_sinks")


class Q4Cache:
    """A paged cache in 4 bits: k_codes/v_codes [num_pages][Hkv][P][d/2] and
    k_scales/v_scales [num_pages][Hkv][P][d/16], uint8 on one GPU, and the
    units of its keys and values.  Make it once and keep it: it holds the
    tensors, and the calls read their addresses from it."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales, k_unit=1.0, v_unit=1.0):
        N, H, P, half = k_codes.shape
        d = 2 * half
        for t, w in ((k_codes, half), (k_scales, d // 16), (v_codes, half), (v_scales, d // 16)):
            if t.shape != (N, H, P, w) or t.dtype is not torch.uint8 or not t.is_contiguous():
                _wrong("codes [num_pages][Hkv][P][d/2] and scales [num_pages][Hkv][P][d/16], dense uint8, wanted")
            if t.get_device() != k_codes.get_device() or t.get_device() < 0:
                _elsewhere()
        self.tensors = (k_codes, k_scales, v_codes, v_scales)
        self.num_pages, self.Hkv, self.P, self.d = N, H, P, d
        self.k_unit, self.v_unit = float(k_unit), float(v_unit)
        self.device_index = k_codes.get_device()
        self._c = _Q4Cache(*(t.data_ptr() for t in self.tensors), self.k_unit, self.v_unit)
        self._at = ctypes.addressof(self._c)

    @classmethod
    def zeros(cls, num_pages, Hkv, P, d, k_unit=1.0, v_unit=1.0, device="cuda"):
        """An empty cache (every row reads as zero)."""
        return cls(*(torch.zeros(num_pages, Hkv, P, w, dtype=torch.uint8, device=device)
                     for w in (d // 2, d // 16) * 2), k_unit, v_unit)


def _table(block_table, Bt):
    n, max_pages = block_table.shape
    if not (n == Bt and block_table.dtype is _I32 and block_table.is_contiguous()):
        _wrong("block_table: dense int32 [Bt][max_pages] wanted")
    return max_pages


def simsd_rope_append_q4(plan, q, k, v, token_start, prefix_len, q_out, cache, block_table, positions=None,
                         err_word=None, stream=None):
    """simsd_rope_append to a :class:`Q4Cache`: q [T][Hq][d] rotated to q_out,
    k [T][Hkv][d] rotated and v to the cache in 4 bits."""
    T, Hq, d = q.shape
    Tk, Hkv, dk = k.shape
    Bt, dt = prefix_len.shape[0], q.dtype
    if Tk != T or dk != d or v.shape != (T, Hkv, d) or k.dtype is not dt or v.dtype is not dt:
        _wrong("k / v: [T][Hkv][d] of q's type wanted")
    if q_out.shape != (T, Hq, d) or q_out.dtype is not dt or not q_out.is_contiguous():
        _wrong("q_out: dense, like q")
    if (token_start.dtype is not _I32 or token_start.numel() != Bt + 1 or not token_start.is_contiguous()
            or prefix_len.dtype is not _I32 or prefix_len.numel() != Bt or not prefix_len.is_contiguous()):
        _wrong("token_start / prefix_len: dense int32 [Bt+1] / [Bt] wanted")
    if positions is not None and not _dense_i32(positions, T):
        _wrong("positions: dense int32 [T] wanted")
    if cache.Hkv != Hkv or cache.d != d:
        _wrong("cache: k's heads and components wanted")
    (qs, q1, q2), (ks, k1, k2), (vs, v1, v2) = q.stride(), k.stride(), v.stride()
    if (q1 != d and Hq > 1) or ((k1 != d or v1 != d) and Hkv > 1) or not q2 == k2 == v2 == 1:
        _wrong("q / k / v: the heads of a token must be dense")
    if T <= 1:
        qs, ks, vs = Hq * d, Hkv * d, Hkv * d
    max_pages = _table(block_table, Bt)
    dev = _device(q)
    if not (dev == k.get_device() == v.get_device() == token_start.get_device() == prefix_len.get_device()
            == q_out.get_device() == cache.device_index == block_table.get_device()
            and (positions is None or positions.get_device() == dev)):
        _elsewhere()
    rc = (_lib or load_library()).simsd_rope_append_q4(
        _code(dt), ctypes.addressof(plan), q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs,
        token_start.data_ptr(), prefix_len.data_ptr(), _ptr(positions), T, Bt, Hq, Hkv, d, q_out.data_ptr(),
        cache._at, cache.num_pages, block_table.data_ptr(), max_pages, cache.P, _error_word(err_word, dev),
        _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_rope_append_q4")


def simsd_q4_expand(cache, block_table, first, last, k_cache, v_cache, err_word=None, stream=None):
    """Rows [first[b], last[b]) of each sequence, as a :class:`Q4Cache` holds
    them, written to k_cache / v_cache [num_pages][Hkv][P][d] (bf16 or fp32)."""
    Bt, dt = first.shape[0], k_cache.dtype
    if (first.dtype is not _I32 or last.dtype is not _I32 or first.numel() != Bt or last.numel() != Bt
            or not first.is_contiguous() or not last.is_contiguous()):
        _wrong("first / last: dense int32 [Bt] wanted")
    num_pages, P = cache.num_pages, cache.P
    if not (k_cache.shape == v_cache.shape == (num_pages, cache.Hkv, P, cache.d) and v_cache.dtype is dt
            and k_cache.is_contiguous() and v_cache.is_contiguous()):
        _wrong("k_cache / v_cache: dense, of one type, with the pages of the cache in 4 bits wanted")
    max_pages = _table(block_table, Bt)
    dev = _device(k_cache)
    if not (dev == v_cache.get_device() == block_table.get_device() == first.get_device() == last.get_device()
            == cache.device_index):
        _elsewhere()
    rc = (_lib or load_library()).simsd_q4_expand(
        _code(dt), cache._at, num_pages, block_table.data_ptr(), max_pages, P, first.data_ptr(),
        last.data_ptr(), Bt, cache.Hkv, cache.d, k_cache.data_ptr(), v_cache.data_ptr(), _error_word(err_word, dev),
        _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_q4_expand")


def simsd_chunk_q4_workspace_bytes(dtype_code, T, Bt, Hq, Hkv, d, max_pages, page_size, num_pages) -> int:
    return int(load_library().simsd_chunk_q4_workspace_bytes(dtype_code, T, Bt, Hq, Hkv, d, max_pages, page_size,
                                                             num_pages))


def simsd_chunk_attention_q4(q, token_start, prefix_len, cache, block_table, out, lse=None, mask_block=1, window=0,
                             sinks=0, key_start=None, softmax_scale=0.0, workspace=None, err_word=None, stream=None):
    """simsd_chunk_attention_sinks over a :class:`Q4Cache` (sinks = 0:
    simsd_chunk_attention); the workspace is that of
    simsd_chunk_q4_workspace_bytes."""
    T, Hq, d = q.shape
    Bt, dt = prefix_len.shape[0], q.dtype
    if cache.d != d:
        _wrong("cache: q's components wanted")
    max_pages = _table(block_table, Bt)
    dev, ws, ws_bytes = _chunk_checks(q, token_start, prefix_len, block_table, out, lse, key_start, workspace)
    if dev != cache.device_index:
        _elsewhere()
    rc = (_lib or load_library()).simsd_chunk_attention_q4(
        _code(dt), q.data_ptr(), _rows(q, Hq, d, "q"), token_start.data_ptr(), prefix_len.data_ptr(),
        _ptr(key_start), cache._at, cache.num_pages, block_table.data_ptr(), max_pages, cache.P, T, Bt, Hq,
        cache.Hkv, d, mask_block, window, sinks, softmax_scale, out.data_ptr(), _ptr(lse), ws, ws_bytes,
        _error_word(err_word, dev), _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_chunk_attention_q4")


class PageSet:
    """The arrays whose pages move together: tensors [num_pages][...] of four
    dimensions or [layers][num_pages][...] of five, at most 8, all with the
    same pages (k and v caches, or the four tensors of a :class:`Q4Cache`).
    Make it once and keep it."""

    def __init__(self, tensors):
        self.tensors = tuple(tensors)
        if len(self.tensors) > MAX_PAGE_ARRAYS:
            _wrong("at most 8 arrays")
        self._c = (_PageArray * max(1, len(self.tensors)))()
        self.num_pages = self.device_index = None
        for i, t in enumerate(self.tensors):
            if t.dim() not in (4, 5) or not t.is_contiguous():
                _wrong("dense tensors of pages [num_pages][Hkv][P][x], or [layers] of them, wanted")
            layers, pages = (1, t.shape[0]) if t.dim() == 4 else t.shape[:2]
            if self.num_pages not in (None, pages):
                _wrong("arrays of the same pages wanted")
            if self.device_index not in (None, t.get_device()) or t.get_device() < 0:
                _elsewhere()
            self.num_pages, self.device_index = pages, t.get_device()
            page = t.element_size() * t.shape[-3] * t.shape[-2] * t.shape[-1]
            self._c[i] = _PageArray(t.data_ptr(), page, page * pages, layers)
        self._at, self.count = ctypes.addressof(self._c), len(self.tensors)


# (The calls on pages take some microseconds on the GPU, so what is right is
# seen in one expression; _pages_wrong finds out what is not.)
def _pages_wrong(dev, block_table, refs, tables, pages=None, workspace=None):
    if block_table.dim() != 2 or block_table.dtype is not _I32 or not block_table.is_contiguous():
        _wrong("block_table: dense int32 [Bt][max_pages] wanted")
    for name, (t, n) in (tables | {"refs": (refs, refs.shape[0])}).items():
        if not _dense_i32(t, n):
            _wrong(f"{name}: dense int32 of {n} wanted")
    if pages is not None and pages.num_pages not in (None, refs.shape[0]):
        _wrong("refs: a count for every page of the arrays wanted")
    if workspace is not None and not workspace.is_contiguous():
        _wrong("workspace: dense tensor wanted")
    _elsewhere()


def _current(dev):
    return dev >= 0 and (_devices == 1 or dev == torch._C._cuda_getDevice())


def simsd_pages_extend(lens, add, block_table, refs, page_size, err_word=None, stream=None, granted=None):
    """Pages for the rows [lens[b], lens[b] + add[b]) that have none; granted
    [Bt] int32 out (simsd_pages_extend_granted): lens[b] where sequence b may
    go on, -1 where not."""
    Bt, max_pages = block_table.shape
    num_pages, dev = refs.shape[0], block_table.get_device()
    if not (lens.dtype is add.dtype is refs.dtype is block_table.dtype is _I32
            and lens.numel() == add.numel() == Bt and refs.numel() == num_pages
            and lens.is_contiguous() and add.is_contiguous() and refs.is_contiguous() and block_table.is_contiguous()
            and lens.get_device() == add.get_device() == refs.get_device() == dev and _current(dev)
            and (granted is None or granted.dtype is _I32 and granted.numel() == Bt and granted.is_contiguous()
                 and granted.get_device() == dev)):
        _pages_wrong(dev, block_table, refs, dict(lens=(lens, Bt), add=(add, Bt))
                     | ({} if granted is None else dict(granted=(granted, Bt))))
    args = (lens.data_ptr(), add.data_ptr(), block_table.data_ptr(), refs.data_ptr(), num_pages, Bt, max_pages, page_size)
    rest = (_error_word(err_word, dev), _raw_stream(stream, dev))
    lib = _lib or load_library()
    rc = (lib.simsd_pages_extend(*args, *rest) if granted is None
          else lib.simsd_pages_extend_granted(*args, granted.data_ptr(), *rest))
    if rc:
        _check(rc, "simsd_pages_extend")


def simsd_pages_release(block_table, refs, first, last, page_size, seq=None, err_word=None, stream=None):
    """Lets go of the pages that lie wholly within rows [first[i], last[i]) of
    sequence seq[i] (None: i)."""
    Bt, max_pages = block_table.shape
    num_pages, dev, n = refs.shape[0], block_table.get_device(), first.shape[0]
    if not (first.dtype is last.dtype is refs.dtype is block_table.dtype is _I32
            and last.numel() == first.numel() == n and refs.numel() == num_pages
            and first.is_contiguous() and last.is_contiguous() and refs.is_contiguous()
            and block_table.is_contiguous()
            and first.get_device() == last.get_device() == refs.get_device() == dev and _current(dev)
            and (n == Bt if seq is None else seq.dtype is _I32 and seq.numel() == n and seq.is_contiguous()
                 and seq.get_device() == dev)):
        n = Bt if seq is None else seq.shape[0]
        _pages_wrong(dev, block_table, refs, dict(first=(first, n), last=(last, n))
                     | ({} if seq is None else dict(seq=(seq, n))))
    if n == 0:  # (an empty tensor has no address, which would name all sequences)
        return
    rc = (_lib or load_library()).simsd_pages_release(
        None if seq is None else seq.data_ptr(), first.data_ptr(), last.data_ptr(), n, block_table.data_ptr(),
        refs.data_ptr(), num_pages, Bt, max_pages, page_size, _error_word(err_word, dev), _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_pages_release")


def simsd_pages_workspace_bytes(num_pages, pairs=0) -> int:
    return int(load_library().simsd_pages_workspace_bytes(num_pages, pairs))


def simsd_pages_fork(pages, src, dst, lens, block_table, refs, page_size, workspace, err_word=None, stream=None):
    """Sequence dst[i] becomes a copy of src[i]; pages: a :class:`PageSet`."""
    Bt, max_pages = block_table.shape
    num_pages, dev, n = refs.shape[0], block_table.get_device(), src.shape[0]
    if not (src.dtype is dst.dtype is lens.dtype is refs.dtype is block_table.dtype is _I32
            and src.numel() == dst.numel() == n and lens.numel() == Bt and refs.numel() == num_pages
            and src.is_contiguous() and dst.is_contiguous() and lens.is_contiguous() and refs.is_contiguous()
            and block_table.is_contiguous() and workspace.is_contiguous()
            and src.get_device() == dst.get_device() == lens.get_device() == refs.get_device()
            == workspace.get_device() == dev and _current(dev)
            and pages.num_pages in (num_pages, None) and pages.device_index in (dev, None)):
        _pages_wrong(dev, block_table, refs, dict(src=(src, n), dst=(dst, n), lens=(lens, Bt)), pages, workspace)
    rc = (_lib or load_library()).simsd_pages_fork(
        pages._at, pages.count, src.data_ptr(), dst.data_ptr(), n, lens.data_ptr(), block_table.data_ptr(),
        refs.data_ptr(), num_pages, Bt, max_pages, page_size, workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _error_word(err_word, dev), _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_pages_fork")


def simsd_pages_compact(pages, block_table, refs, live, workspace, err_word=None, stream=None):
    """Moves the live pages to the lowest ids; live [1] int32 out or None."""
    Bt, max_pages = block_table.shape
    num_pages, dev = refs.shape[0], block_table.get_device()
    if not (refs.dtype is block_table.dtype is _I32 and refs.numel() == num_pages
            and refs.is_contiguous() and block_table.is_contiguous() and workspace.is_contiguous()
            and refs.get_device() == workspace.get_device() == dev and _current(dev)
            and (live is None or live.dtype is _I32 and live.numel() == 1 and live.get_device() == dev)
            and pages.num_pages in (num_pages, None) and pages.device_index in (dev, None)):
        _pages_wrong(dev, block_table, refs, {} if live is None else dict(live=(live, 1)), pages, workspace)
    rc = (_lib or load_library()).simsd_pages_compact(
        pages._at, pages.count, block_table.data_ptr(), refs.data_ptr(), num_pages, Bt, max_pages,
        None if live is None else live.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _error_word(err_word, dev), _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_pages_compact")


def _row_f32(t, R, dev, name):
    if t is None:
        return None
    if t.dtype is not _F32 or t.numel() != R or not t.is_contiguous():
        _wrong(name + ": dense float32 [R] wanted")
    if t.get_device() != dev:
        _elsewhere()
    return t.data_ptr()


def _row_i32(t, R, dev, name):
    if t is None:
        return None
    if t.dtype is not _I32 or t.numel() != R or not t.is_contiguous():
        _wrong(name + ": dense int32 [R] wanted")
    if t.get_device() != dev:
        _elsewhere()
    return t.data_ptr()


def simsd_sample(logits, u, token, temperature=None, top_k=None, top_p=None, min_p=None, kept=None, log_prob=None,
                 log_probs=None, err_word=None, stream=None):
    """logits [R][V] float32 or bfloat16 (row stride allowed); u, temperature,
    top_p, min_p [R] float32, top_k [R] int32; token/kept [R] int32,
    log_prob [R] and log_probs [R][V] float32 (outputs; all but token
    optional)."""
    R, V = logits.shape
    s0, s1 = logits.stride()
    if s1 != 1 and V > 1:
        _wrong("logits: dense rows wanted")
    if log_probs is not None and (log_probs.shape != (R, V) or log_probs.dtype is not _F32
                                  or not log_probs.is_contiguous()):
        _wrong("log_probs: dense float32 [R][V] wanted")
    code, dev = _code(logits.dtype), logits.get_device()
    args = (_row_f32(u, R, dev, "u"), _row_f32(temperature, R, dev, "temperature"), _row_i32(top_k, R, dev, "top_k"),
            _row_f32(top_p, R, dev, "top_p"), _row_f32(min_p, R, dev, "min_p"), _row_i32(token, R, dev, "token"),
            _row_i32(kept, R, dev, "kept"), _row_f32(log_prob, R, dev, "log_prob"))
    _device(logits)
    if log_probs is not None and log_probs.get_device() != dev:
        _elsewhere()
    rc = (_lib or load_library()).simsd_sample(
        code, logits.data_ptr(), s0 if R > 1 else V, R, V, *args, _ptr(log_probs), _error_word(err_word, dev),
        _raw_stream(stream, dev))
    if rc:
        _check(rc, "simsd_sample")
