"""Python binding of the C-ABI library ``libmdi.so`` (see ``include/mdi.h``).

Argument marshalling only: every step of the decoding path runs in the CUDA
library.  There is no CPU fallback: loading fails loudly if the library has not
been built, and creating a context fails if there is no CUDA device.
"""
from __future__ import annotations

import ctypes
import os
from typing import Iterable, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmdi.so")

MDI_OK = 0
TRACE_WORDS = 128
KV_DEFAULT, KV_BF16, KV_F16, KV_F32, KV_I8, KV_E4M3 = 0, 1, 2, 3, 4, 5
STATUS_PAGE, STATUS_RANGE, STATUS_TIMEOUT = 1, 2, 4
ERR_ARG, ERR_SHAPE, ERR_OOM, ERR_CONTEXT, ERR_STATE, ERR_TIMEOUT, ERR_CUDA = -1, -2, -3, -4, -5, -6, -7
_ERR_NAMES = {ERR_ARG: "MDI_ERR_ARG", ERR_SHAPE: "MDI_ERR_SHAPE", ERR_OOM: "MDI_ERR_OOM", ERR_CONTEXT: "MDI_ERR_CONTEXT",
              ERR_STATE: "MDI_ERR_STATE", ERR_TIMEOUT: "MDI_ERR_TIMEOUT", ERR_CUDA: "MDI_ERR_CUDA"}

EXPORTS = ["mdi_create", "mdi_destroy", "mdi_load_weights", "mdi_prefill", "mdi_prefill_dev", "mdi_step",
           "mdi_generate", "mdi_generate_dev", "mdi_get_logits", "mdi_set_sampling", "mdi_set_teacher_tokens", "mdi_reset_sample",
           "mdi_get_stats", "mdi_get_partition_times", "mdi_get_trace", "mdi_memory_bytes", "mdi_sync", "mdi_last_error", "mdi_greedy_argmax_static",
           "mdi_kv_append", "mdi_kv_read", "mdi_attn_decode_workspace", "mdi_attn_decode", "mdi_attn_prompt"]


class MdiError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"{_ERR_NAMES.get(code, code)}: {text}")
        self.code = code


class ModelShape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in
                ("arch", "n_layer", "d_model", "n_head", "head_dim", "n_kv_head", "d_ff", "vocab", "n_ctx",
                 "weight_dtype", "tied_lm_head", "has_bias", "act")] + \
               [("norm_eps", ctypes.c_float), ("rope_theta", ctypes.c_float)]


class Options(ctypes.Structure):
    _fields_ = [("page_tokens", ctypes.c_int), ("kv_pool_tokens", ctypes.c_int), ("attn_splits", ctypes.c_int),
                ("rounds_per_graph", ctypes.c_int), ("kv_cache_dtype", ctypes.c_int), ("prefill_mode", ctypes.c_int), ("tc_min_group", ctypes.c_int), ("wait_limit_ms", ctypes.c_int), ("debug_withhold_handoff", ctypes.c_int),
                ("scheduler", ctypes.c_int), ("in_kernel_timing", ctypes.c_int), ("fused_blocks_per_head", ctypes.c_int),
                ("reserved0", ctypes.c_int), ("trace_slot", ctypes.c_int), ("td_b_kblocks", ctypes.c_int)]


class Stats(ctypes.Structure):
    _fields_ = [("n_partitions", ctypes.c_int), ("n_samples", ctypes.c_int), ("n_groups", ctypes.c_int),
                ("weight_bytes", ctypes.c_int64 * 16), ("kv_pool_bytes", ctypes.c_int64 * 16),
                ("kv_pages_in_use", ctypes.c_int64 * 16), ("tokens_generated", ctypes.c_int64),
                ("stage_steps", ctypes.c_int64), ("kernel_launches", ctypes.c_int64),
                ("last_prefill_ms", ctypes.c_float), ("last_generate_ms", ctypes.c_float),
                ("last_run_ms", ctypes.c_float), ("kv_element_bytes", ctypes.c_int)]


class Rows(ctypes.Structure):
    _fields_ = [("data_dev", ctypes.c_void_p), ("dtype", ctypes.c_int), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class KvCacheStruct(ctypes.Structure):
    _fields_ = [("pool_dev", ctypes.c_void_p), ("scale_dev", ctypes.c_void_p), ("page_table_dev", ctypes.c_void_p),
                ("page_table_stride", ctypes.c_int64)] + \
               [(n, ctypes.c_int) for n in ("n_pages", "n_slots", "pages_per_seq", "page_tokens", "n_kv_head", "head_dim", "dtype")]


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} has not been built (python -m paper_2505_18164_b200.build); "
                               "there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, ci = ctypes.c_void_p, ctypes.c_int
        L.mdi_create.argtypes = [ctypes.POINTER(ModelShape), ctypes.POINTER(ci), ci, ci, ctypes.POINTER(Options),
                                 ctypes.POINTER(vp)]
        L.mdi_destroy.argtypes = [vp]
        L.mdi_destroy.restype = None
        L.mdi_load_weights.argtypes = [vp, ctypes.c_char_p, vp, ctypes.c_size_t]
        L.mdi_prefill.argtypes = [vp, ci, vp, ci]
        L.mdi_prefill_dev.argtypes = [vp, ci, vp, ci]
        L.mdi_step.argtypes = [vp, ci, ci, vp, vp]
        L.mdi_generate.argtypes = [vp, ci, ci, vp]
        L.mdi_generate_dev.argtypes = [vp, ci, ci, vp]
        L.mdi_get_logits.argtypes = [vp, ci, vp]
        L.mdi_set_sampling.argtypes = [vp, ctypes.c_float, ci, ctypes.c_uint64]
        L.mdi_set_teacher_tokens.argtypes = [vp, ci, vp, ci]
        L.mdi_reset_sample.argtypes = [vp, ci]
        L.mdi_get_stats.argtypes = [vp, ctypes.POINTER(Stats)]
        L.mdi_get_partition_times.argtypes = [vp, ci, ctypes.POINTER(ctypes.c_double), ci]
        L.mdi_get_trace.argtypes = [vp, vp, ci]
        L.mdi_memory_bytes.argtypes = [vp, ci]
        L.mdi_memory_bytes.restype = ctypes.c_int64
        L.mdi_sync.argtypes = [vp]
        L.mdi_greedy_argmax_static.argtypes = [vp, ci, ci, vp, vp]
        i64, rows, cache = ctypes.c_int64, ctypes.POINTER(Rows), ctypes.POINTER(KvCacheStruct)
        L.mdi_kv_append.argtypes = [cache, ci, vp, vp, vp, ci, rows, rows, vp, vp]
        L.mdi_kv_read.argtypes = [cache, ci, vp, vp, vp, ci, rows, rows, vp, vp]
        L.mdi_attn_decode_workspace.argtypes = [cache, ci, ci, ci]
        L.mdi_attn_decode_workspace.restype = i64
        L.mdi_attn_decode.argtypes = [cache, ci, vp, vp, ci, ci, rows, rows, ctypes.c_float, vp, i64, vp, vp]
        L.mdi_attn_prompt.argtypes = [ci, vp, vp, ci, ci, ci, ci, ci, rows, rows, rows, rows, ctypes.c_float, vp, vp]
        L.mdi_last_error.argtypes = [vp]
        L.mdi_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _ptr(x) -> int:
    """Address of a numpy array (host) or torch tensor (host or device), or a raw integer address."""
    if x is None:
        return 0
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    return x.data_ptr()


def greedy_argmax_static(logits_dev, n_rows: int, n_cols: int, out_dev, stream: int = 0):
    """mdi_greedy_argmax_static: per-row argmax of device logits without any allocation (see mdi.h).
    ``logits_dev`` / ``out_dev``: device tensors or raw addresses; ``stream``: a cudaStream_t value."""
    rc = lib().mdi_greedy_argmax_static(_ptr(logits_dev), n_rows, n_cols, _ptr(out_dev), stream)
    if rc != MDI_OK:
        raise MdiError(rc, (lib().mdi_last_error(None) or b"").decode())


# ---- operators on the caller's device tensors (see the second half of mdi.h) ------------------------------------------
_ROW_DTYPES = {"torch.float32": 0, "torch.bfloat16": 1, "torch.float16": 2}
_ROW_CODES: dict = {}  # the same by the dtype objects met so far (their names are slow to look up)
_KV_DTYPES = {"torch.bfloat16": KV_BF16, "torch.float16": KV_F16, "torch.int8": KV_I8, "torch.float8_e4m3fn": KV_E4M3}


_INT32: set = set()


def _fail_arg(text: str):
    raise MdiError(ERR_ARG, text)


def _op_check(rc: int):
    if rc != MDI_OK:
        raise MdiError(rc, (lib().mdi_last_error(None) or b"").decode())


def _row_code(name: str, dtype) -> int:
    dt = _ROW_DTYPES.get(str(dtype))
    if dt is None:
        _fail_arg(f"{name}: dtype {dtype} is none of float32, bfloat16, float16")
    _ROW_CODES[dtype] = dt
    return dt


def _rows(name: str, t, rows: int, heads: int, head_dim: int) -> Rows:
    """A [rows][heads][head_dim] tensor (any strides but the last) as the library's row view."""
    dtype, shape = t.dtype, t.shape
    dt = _ROW_CODES.get(dtype)
    if dt is None:
        dt = _row_code(name, dtype)
    if len(shape) != 3 or shape[0] < rows or shape[1] != heads or shape[2] != head_dim:
        _fail_arg(f"{name}: shape {tuple(shape)}, expected [{rows}][{heads}][{head_dim}]")
    s0, s1, s2 = t.stride()
    if s2 != 1:
        _fail_arg(f"{name}: the elements of a head must be contiguous")
    return Rows(t.data_ptr(), dt, s0 if rows > 1 else heads * head_dim, s1 if heads > 1 else head_dim)


def _ints(name: str, t, n: int):
    """Address of a device tensor of at least n int32 values (None: 0)."""
    if t is None:
        return 0
    dtype = t.dtype
    if dtype not in _INT32:
        if str(dtype) != "torch.int32":
            _fail_arg(f"{name}: expected int32, not {dtype}")
        _INT32.add(dtype)
    if t.numel() < n or not t.is_contiguous():
        _fail_arg(f"{name}: expected a contiguous tensor of at least {n} elements")
    return t.data_ptr()


class KvCache:
    """A paged key/value cache over the caller's device tensors (mdi_kv_cache): ``pool`` [n_pages][2][n_kv_head][page_tokens]
    [head_dim] of float16, bfloat16, int8 or float8_e4m3fn; ``page_table`` int32 [n_slots][pages_per_seq]; ``scale`` float32
    [n_pages][2][n_kv_head][page_tokens] for the 8-bit types.  The tensors are kept alive by this object."""

    def __init__(self, pool, page_table, scale=None):
        dt = _KV_DTYPES.get(str(pool.dtype))
        if dt is None:
            _fail_arg(f"pool: dtype {pool.dtype} is none of float16, bfloat16, int8, float8_e4m3fn")
        if pool.dim() != 5 or pool.shape[1] != 2 or not pool.is_contiguous():
            _fail_arg("pool: expected a contiguous [n_pages][2][n_kv_head][page_tokens][head_dim] tensor")
        if str(page_table.dtype) != "torch.int32" or page_table.dim() != 2 or page_table.stride(1) != 1:
            _fail_arg("page_table: expected int32 [n_slots][pages_per_seq]")
        if dt in (KV_I8, KV_E4M3) and (scale is None or str(scale.dtype) != "torch.float32" or tuple(scale.shape) != tuple(pool.shape[:4])
                                       or not scale.is_contiguous()):
            _fail_arg("scale: 8-bit caches need a contiguous float32 [n_pages][2][n_kv_head][page_tokens] tensor")
        self.tensors = (pool, page_table, scale)
        self.n_slots, self.n_kv_head, self.head_dim = page_table.shape[0], pool.shape[2], pool.shape[4]
        self._lib = lib()
        self._c = KvCacheStruct(pool.data_ptr(), _ptr(scale) if scale is not None else 0, page_table.data_ptr(),
                                page_table.stride(0) if self.n_slots > 1 else max(page_table.shape[1], 1), pool.shape[0], self.n_slots, page_table.shape[1], pool.shape[3],
                                self.n_kv_head, self.head_dim, dt)


def kv_append(cache: KvCache, k, v, seq_start, pos, slots=None, status=None, stream: int = 0):
    """mdi_kv_append: rows seq_start[i] .. seq_start[i+1]-1 of ``k``, ``v`` ([rows][n_kv_head][head_dim]) go to positions pos[i] ..
    of sequence i's slot (``slots[i]``, or i)."""
    n_seq, n = seq_start.numel() - 1, k.shape[0]
    kr, vr = _rows("k", k, n, cache.n_kv_head, cache.head_dim), _rows("v", v, n, cache.n_kv_head, cache.head_dim)
    _op_check(cache._lib.mdi_kv_append(cache._c, n_seq, _ints("slots", slots, n_seq) if slots is not None else 0, _ints("seq_start", seq_start, n_seq + 1),
                                  _ints("pos", pos, n_seq), n, kr, vr, _ints("status", status, 1) if status is not None else 0, stream))


def kv_read(cache: KvCache, k_out, v_out, seq_start, pos=None, slots=None, status=None, stream: int = 0):
    """mdi_kv_read: the reverse of kv_append, into ``k_out``, ``v_out``; ``pos`` None reads every sequence from position 0."""
    n_seq, n = seq_start.numel() - 1, k_out.shape[0]
    kr, vr = _rows("k_out", k_out, n, cache.n_kv_head, cache.head_dim), _rows("v_out", v_out, n, cache.n_kv_head, cache.head_dim)
    _op_check(cache._lib.mdi_kv_read(cache._c, n_seq, _ints("slots", slots, n_seq) if slots is not None else 0, _ints("seq_start", seq_start, n_seq + 1),
                                _ints("pos", pos, n_seq), n, kr, vr, _ints("status", status, 1) if status is not None else 0, stream))


def attn_decode_workspace(cache: KvCache, n_head: int, max_len: int = 0, n_seq: Optional[int] = None) -> int:
    """Bytes of working memory of attn_decode for ``n_seq`` sequences (default: every slot)."""
    rc = lib().mdi_attn_decode_workspace(cache._c, cache.n_slots if n_seq is None else n_seq, n_head, max_len)
    if rc < 0:
        _op_check(rc)
    return rc


def attn_decode(cache: KvCache, q, out, lens, max_len: int = 0, scale: Optional[float] = None, workspace=None, slots=None,
                status=None, stream: int = 0):
    """mdi_attn_decode: one new token per sequence, ``q``, ``out`` [n_seq][n_head][head_dim], over the first lens[i] cached rows.
    ``scale``: default 1 / sqrt(head_dim).  ``workspace``: a device tensor of attn_decode_workspace() bytes."""
    n_seq, n_head = q.shape[0], q.shape[1]
    qr, orow = _rows("q", q, n_seq, n_head, cache.head_dim), _rows("out", out, n_seq, n_head, cache.head_dim)
    ws = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if workspace is not None else (0, 0)
    _op_check(cache._lib.mdi_attn_decode(cache._c, n_seq, _ints("slots", slots, n_seq) if slots is not None else 0, _ints("lens", lens, n_seq), max_len, n_head, qr, orow,
                                    cache.head_dim ** -0.5 if scale is None else scale, ws[0], ws[1], _ints("status", status, 1) if status is not None else 0, stream))


def attn_prompt(q, k, v, out, q_start, k_start, scale: Optional[float] = None, status=None, stream: int = 0):
    """mdi_attn_prompt: causal attention over packed sequences, ``q``, ``out`` [q rows][n_head][head_dim], ``k``, ``v`` [key
    rows][n_kv_head][head_dim]; ``q_start``, ``k_start`` int32 [n_seq + 1].  ``scale``: default 1 / sqrt(head_dim)."""
    n_seq, (nq, n_head, hd), (nk, n_kv) = q_start.numel() - 1, q.shape, k.shape[:2]
    r = [_rows("q", q, nq, n_head, hd), _rows("k", k, nk, n_kv, hd), _rows("v", v, nk, n_kv, hd), _rows("out", out, nq, n_head, hd)]
    _op_check(lib().mdi_attn_prompt(n_seq, _ints("q_start", q_start, n_seq + 1), _ints("k_start", k_start, n_seq + 1), nq, nk, n_head, n_kv, hd,
                                    r[0], r[1], r[2], r[3], hd ** -0.5 if scale is None else scale, _ints("status", status, 1) if status is not None else 0, stream))


class Context:
    """One model on one GPU: mdi_create ... mdi_destroy."""

    def __init__(self, shape, part_bounds: Sequence[int], n_samples: int, page_tokens: int = 0,
                 kv_pool_tokens: int = 0, attn_splits: int = 0, rounds_per_graph: int = 0, scheduler: int = 0,
                 kv_cache_dtype: int = 0, prefill_mode: int = 0, tc_min_group: int = 0,
                 wait_limit_ms: int = 0, debug_withhold_handoff: int = 0, in_kernel_timing: int = 0,
                 fused_blocks_per_head: int = 0, trace_slot: int = 0, td_b_kblocks: int = 0):
        self._h = None
        self.shape = shape
        self.K = len(part_bounds) - 1
        self.n_samples = n_samples
        cs = ModelShape(**{n: getattr(shape, n) for n, _ in ModelShape._fields_})
        bounds = (ctypes.c_int * len(part_bounds))(*part_bounds)
        opts = Options(page_tokens, kv_pool_tokens, attn_splits, rounds_per_graph, kv_cache_dtype, prefill_mode, tc_min_group,
                       wait_limit_ms, debug_withhold_handoff, scheduler, in_kernel_timing, fused_blocks_per_head,
                       0, trace_slot, td_b_kblocks)
        h = ctypes.c_void_p()
        rc = lib().mdi_create(ctypes.byref(cs), bounds, self.K, n_samples, ctypes.byref(opts), ctypes.byref(h))
        if rc != MDI_OK:
            raise MdiError(rc, (lib().mdi_last_error(None) or b"").decode())
        self._h = h

    def _check(self, rc: int):
        if rc != MDI_OK:
            raise MdiError(rc, (lib().mdi_last_error(self._h) or b"").decode())

    def close(self):
        if self._h and _lib is not None:
            _lib.mdi_destroy(self._h)
        self._h = None

    __del__ = close

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def load_weights(self, name: str, host: np.ndarray):
        host = np.ascontiguousarray(host)
        self._check(lib().mdi_load_weights(self._h, name.encode(), host.ctypes.data, host.nbytes))

    def load_all(self, named: Iterable):
        for name, a in (named.items() if hasattr(named, "items") else named):
            self.load_weights(name, a)

    def prefill(self, sample: int, prompt_host: np.ndarray):
        p = np.ascontiguousarray(prompt_host, np.int32)
        self._check(lib().mdi_prefill(self._h, sample, p.ctypes.data, p.size))

    def prefill_dev(self, sample: int, prompt_dev, n_prompt: int):
        self._check(lib().mdi_prefill_dev(self._h, sample, _ptr(prompt_dev), n_prompt))

    def step(self, partition: int, slot: int, act_in_dev, act_out_dev):
        self._check(lib().mdi_step(self._h, partition, slot, _ptr(act_in_dev), _ptr(act_out_dev)))

    def generate(self, n_samples: int, n_new_tokens: int, out_host: Optional[np.ndarray] = None) -> np.ndarray:
        if out_host is None:
            out_host = np.empty((n_samples, n_new_tokens), np.int32)
        assert out_host.dtype == np.int32 and out_host.size >= n_samples * n_new_tokens and out_host.flags.c_contiguous
        self._check(lib().mdi_generate(self._h, n_samples, n_new_tokens, out_host.ctypes.data))
        return out_host

    def generate_dev(self, n_samples: int, n_new_tokens: int, out_dev):
        self._check(lib().mdi_generate_dev(self._h, n_samples, n_new_tokens, _ptr(out_dev)))

    def get_logits(self, sample: int) -> np.ndarray:
        out = np.empty(self.shape.vocab, np.float32)
        self._check(lib().mdi_get_logits(self._h, sample, out.ctypes.data))
        return out

    def set_sampling(self, temperature: float, top_k: int, seed: int):
        self._check(lib().mdi_set_sampling(self._h, temperature, top_k, seed))

    def set_teacher_tokens(self, sample: int, tokens: Sequence[int]):
        t = np.ascontiguousarray(tokens, np.int32)
        self._check(lib().mdi_set_teacher_tokens(self._h, sample, t.ctypes.data, t.size))

    def reset_sample(self, sample: int):
        self._check(lib().mdi_reset_sample(self._h, sample))

    def stats(self) -> Stats:
        st = Stats()
        self._check(lib().mdi_get_stats(self._h, ctypes.byref(st)))
        return st

    def partition_times(self, partition: int):
        """(blocks in the partition's team, [12] mean milliseconds per category) of the last generate."""
        out = (ctypes.c_double * 12)()
        rc = lib().mdi_get_partition_times(self._h, partition, out, 12)
        if rc < 0:
            self._check(rc)
        return rc, list(out)

    def trace(self) -> np.ndarray:
        """[blocks][TRACE_WORDS] uint64 time stamps of the traced schedule slot ((ns << 4) | category, 0 = unused)."""
        buf = np.zeros(1024 * TRACE_WORDS, np.uint64)
        rc = lib().mdi_get_trace(self._h, buf.ctypes.data, buf.size)
        if rc < 0:
            self._check(rc)
        return buf[: rc * TRACE_WORDS].reshape(rc, TRACE_WORDS)

    def memory_bytes(self, partition: int) -> int:
        return lib().mdi_memory_bytes(self._h, partition)

    def sync(self):
        self._check(lib().mdi_sync(self._h))
