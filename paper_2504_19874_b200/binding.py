"""Python binding of include/tq.h.  Argument marshalling only: the calls a program makes again and again go through the
extension module _tqbind (csrc/tq_bind.cpp), set-up and size queries through ctypes."""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

TQ_MSE, TQ_PROD = 0, 1
TQ_F32, TQ_BF16 = 0, 1
TQ_ORTHOGONAL, TQ_GAUSSIAN = 0, 1
TQ_LAYOUT_CANONICAL, TQ_LAYOUT_NIBBLE = 0, 1
TQ_OP_QUANTIZE, TQ_OP_SCORE, TQ_OP_TOPK, TQ_OP_WSUM, TQ_OP_DEQUANTIZE = 0, 1, 2, 3, 4
TQ_I8, TQ_E4M3 = 0, 1
TQ_STATIC_SCRATCH_BYTES = 1 << 20

# TQ_LIB_VARIANT=debug loads libtq_debug.so, the build with device-side index checks (build.py --debug)
_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)),
                         "libtq_debug.so" if os.environ.get("TQ_LIB_VARIANT") == "debug" else "libtq.so")
_lib = None
_n = None        # the _tqbind module, bound to the loaded library

c_void_p, c_int, c_int64, c_size_t, c_u64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_uint64
_F = ctypes.POINTER(ctypes.c_float)

_SIGNATURES = {
    "tq_last_error": (ctypes.c_char_p, []),
    "tq_launch_count": (c_u64, []),
    "tq_codebook": (c_int, [c_int, c_int, _F, _F]),
    "tq_rotation": (c_int, [c_int, c_u64, c_int, _F]),
    "tq_idx_row_bytes": (c_size_t, [c_int, c_int]),
    "tq_qjl_row_bytes": (c_size_t, [c_int]),
    "tq_plan_create": (c_int, [c_int, c_int, c_int, _F, _F, _F, ctypes.POINTER(c_void_p)]),
    "tq_plan_destroy": (c_int, [c_void_p]),
    "tq_plan_status": (c_int, [c_void_p]),
    "tq_plan_set_layout": (c_int, [c_void_p, c_int]),
    "tq_plan_layout": (c_int, [c_void_p]),
    "tq_convert_layout": (c_int, [c_void_p, c_int64, c_void_p, c_void_p, c_int, c_int, c_void_p]),
    "tq_workspace_bytes": (c_size_t, [c_void_p, c_int, c_int64, c_int, c_int]),
    "tq_quantize_mse": (c_int, [c_void_p, c_void_p, c_int, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "tq_quantize_prod": (c_int, [c_void_p, c_void_p, c_int, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_void_p, c_size_t, c_void_p]),
    "tq_dequantize": (c_int, [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]),
    "tq_score": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                         c_void_p, c_int64, c_void_p, c_size_t, c_void_p]),
    "tq_score_static": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                c_void_p, c_int64, c_void_p]),
    "tq_score_static_max_queries": (c_int, [c_void_p]),
    "tq_query_bytes": (c_size_t, [c_void_p, c_int]),
    "tq_query_prepare": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int64, c_void_p, c_size_t, c_void_p]),
    "tq_score_prepared": (c_int, [c_void_p, c_void_p, c_int, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                  c_int64, c_void_p]),
    "tq_selftest_wait_timeout": (c_int, [c_void_p, ctypes.c_longlong, c_void_p]),
    "tq_entropy_lengths": (c_int, [c_int, c_int, _F, c_void_p]),
    "tq_entropy_workspace_bytes": (c_size_t, [c_int64]),
    "tq_entropy_measure": (c_int, [c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "tq_entropy_pack": (c_int, [c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "tq_entropy_unpack": (c_int, [c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p]),
    "tq_topk": (c_int, [c_void_p, c_void_p, c_int, c_int, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                        c_int, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "tq_select_topk": (c_int, [c_void_p, c_void_p, c_int, c_int64, c_int64, c_int, c_void_p, c_void_p, c_void_p]),
    "tq_softmax": (c_int, [c_void_p, c_void_p, c_int, c_int64, c_int64, ctypes.c_float, c_void_p, c_int64, c_void_p]),
    "tq_wsum": (c_int, [c_void_p, c_void_p, c_int, c_int64, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                        c_void_p, c_int64, c_void_p, c_size_t, c_void_p]),
    "tq_attend_decode_workspace_bytes": (c_size_t, [c_int, c_int, c_int64, c_int]),
    "tq_attend_decode": (c_int, [c_void_p, c_int, c_int, c_int64, c_int64, c_int, c_void_p, c_int, c_int64, ctypes.c_float,
                                 c_void_p, c_int64, c_void_p, c_size_t, c_void_p]),
    "tq_kv_append": (c_int, [c_void_p, c_int, c_int, c_int64, c_int64, c_void_p, c_void_p, c_int, c_int64, c_int64, c_void_p]),
    "tq_kv8_append": (c_int, [c_void_p, c_void_p, c_int64, c_int, c_int, c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_int64, c_void_p,
                              c_int64, c_int64, c_int, c_void_p]),
    "tq_kv8_attend_workspace_bytes": (c_size_t, [c_void_p, c_int, c_int64, c_int, c_int, c_int]),
    "tq_kv8_attend": (c_int, [c_void_p, c_void_p, c_int64, c_int, c_int, c_void_p, c_void_p, c_int64, c_int, c_void_p, c_int64, c_int64, c_int,
                              c_int, ctypes.c_float, c_void_p, c_int, c_void_p, c_int64, c_int64, c_void_p, c_void_p, c_size_t, c_void_p]),
    "tq_selftest_kv8_timeout": (c_int, [c_int]),
    "tq_kv8_select_workspace_bytes": (c_size_t, [c_void_p, c_int64, c_int]),
    "tq_kv8_select": (c_int, [c_void_p, c_void_p, c_int64, c_int, c_int, c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int, c_int,
                              c_int, c_int, c_int, c_void_p, c_void_p, c_size_t, c_void_p]),
    "tq_pages_workspace_bytes": (c_size_t, [c_int64, c_int]),
    "tq_pages_extend": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int, c_int, c_void_p, c_void_p, c_int, c_void_p, c_void_p, c_size_t,
                                c_void_p]),
    "tq_pages_fork": (c_int, [c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_void_p, c_void_p, c_void_p, c_int, c_void_p, c_void_p,
                              c_size_t, c_void_p]),
    "tq_pages_free": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int, c_int, c_void_p, c_void_p, c_int, c_void_p]),
    "tq_pages_compact": (c_int, [c_void_p, c_void_p, c_void_p, c_int64, c_int, c_int, c_void_p, c_void_p, c_size_t, c_void_p]),
    "tq_pages_copy": (c_int, [c_void_p, c_void_p, c_void_p, c_int, c_void_p]),
}


class KvGroup(ctypes.Structure):
    """struct tq_kv_group of include/tq.h (one channel group of a compressed KV layer), for programs that call
    lib().tq_attend_decode / tq_kv_append themselves; the functions below take mappings."""
    _fields_ = [(name, c_void_p) for name in ("plan_k", "plan_v", "k_idx", "k_qjl", "k_gamma", "k_norms", "v_idx", "v_norms",
                                              "k_channels", "v_channels")]


class Kv8(ctypes.Structure):
    """struct tq_kv8 of include/tq.h (a paged 8-bit KV cache), for programs that call lib() themselves; Kv8Cache owns one."""
    _fields_ = [(name, c_void_p) for name in ("k", "v", "k_scale", "v_scale", "k_bounds")] + [("pages", c_int64)] + [
        (name, c_int) for name in ("heads", "page_tokens", "d", "code_type")]


class TqError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"tq error {code}: {message}")
        self.code = code


def lib() -> ctypes.CDLL:
    """Loads libtq.so (built in-tree by paper_2504_19874_b200/build.py).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: run `python -m paper_2504_19874_b200.build` first "
                               "(there is no fallback path)")
        handle = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def _native():
    """The marshalling module, bound to the library that lib() loads."""
    global _n
    if _n is None:
        lib()
        try:
            from . import _tqbind
        except ImportError as e:
            raise RuntimeError("_tqbind.so is missing or does not load: run `python -m paper_2504_19874_b200.build` first "
                               f"(there is no fallback path): {e}") from e
        _tqbind.bind(_LIB_PATH)
        _n = _tqbind
    return _n


def _check(code: int):
    if code != 0:
        raise TqError(code, lib().tq_last_error().decode())


def _fptr(a: np.ndarray):
    return a.ctypes.data_as(_F)


def _dev(t):
    """Device pointer of a CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor (this library has no CPU path)")
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def tq_launch_count() -> int:
    return lib().tq_launch_count()


def tq_idx_row_bytes(d: int, bits: int) -> int:
    return lib().tq_idx_row_bytes(d, bits)


def tq_qjl_row_bytes(d: int) -> int:
    return lib().tq_qjl_row_bytes(d)


def tq_codebook(d: int, bits: int):
    """(centroids, boundaries) as float32 numpy arrays."""
    levels = 1 << min(max(bits, 0), 8)        # the library rejects bits outside 0..4
    c = np.zeros(levels, dtype=np.float32)
    t = np.zeros(max(levels - 1, 1), dtype=np.float32)
    _check(lib().tq_codebook(d, bits, _fptr(c), _fptr(t)))
    return c, t[:levels - 1]


def tq_rotation(d: int, seed: int, kind: int = TQ_ORTHOGONAL) -> np.ndarray:
    out = np.zeros((d, d), dtype=np.float32)
    _check(lib().tq_rotation(d, seed, kind, _fptr(out)))
    return out


class Plan:
    """Owner of a tq_plan handle (device copies of Pi, S', codebook for one (d, b, mode))."""

    def __init__(self, d: int, bits: int, mode: int, Pi, S, centroids):
        Pi = np.ascontiguousarray(Pi, dtype=np.float32)
        cent = np.ascontiguousarray(centroids, dtype=np.float32)
        Sp = None if S is None else np.ascontiguousarray(S, dtype=np.float32)
        if Pi.shape != (d, d) or (Sp is not None and Sp.shape != (d, d)):
            raise ValueError("Pi and S must be d x d")
        self.d, self.bits, self.mode = d, bits, mode
        self.mse_bits = bits - 1 if mode == TQ_PROD else bits
        if cent.size != (1 << max(self.mse_bits, 0)):
            raise ValueError("centroids must hold 2^b_m values")
        self.idx_row_bytes = tq_idx_row_bytes(d, self.mse_bits)
        self.qjl_row_bytes = tq_qjl_row_bytes(d)
        h = c_void_p()
        _check(lib().tq_plan_create(d, bits, mode, _fptr(Pi), None if Sp is None else _fptr(Sp), _fptr(cent),
                                    ctypes.byref(h)))
        self.handle = h.value

    def set_layout(self, layout: int) -> None:
        """TQ_LAYOUT_CANONICAL or TQ_LAYOUT_NIBBLE (TQ_PROD with b = 4 only): arrangement of the code rows."""
        _check(lib().tq_plan_set_layout(self.handle, layout))

    @property
    def layout(self) -> int:
        return lib().tq_plan_layout(self.handle)

    def close(self):
        if getattr(self, "handle", None):
            lib().tq_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def tq_plan_status(plan: Plan) -> None:
    """Synchronises and raises TqError(6) if a kernel of this plan gave up a bounded wait."""
    _check(lib().tq_plan_status(plan.handle))


def tq_convert_layout(plan: Plan, n: int, idx, qjl, src: int, dst: int) -> None:
    """Rewrites n rows of (idx, qjl) in place from layout `src` into layout `dst`."""
    _check(lib().tq_convert_layout(plan.handle, n, _dev(idx), _dev(qjl), src, dst, _stream()))


def tq_workspace_bytes(plan: Plan, op: int, n: int, nq: int = 0, k: int = 0) -> int:
    return lib().tq_workspace_bytes(plan.handle, op, n, nq, k)


def tq_quantize_mse(plan: Plan, X, idx, norms=None, scratch=None):
    _check((_n or _native()).quantize_mse(plan.handle, X, idx, norms, scratch))


def tq_quantize_prod(plan: Plan, X, idx, qjl, gamma, norms=None, scratch=None):
    _check((_n or _native()).quantize_prod(plan.handle, X, idx, qjl, gamma, norms, scratch))


def tq_dequantize(plan: Plan, n: int, idx, qjl, gamma, norms, Xhat):
    _check((_n or _native()).dequantize(plan.handle, n, idx, qjl, gamma, norms, Xhat))


def tq_score(plan: Plan, Q, n: int, idx, qjl, gamma, norms, scores, workspace):
    _check((_n or _native()).score(plan.handle, Q, n, idx, qjl, gamma, norms, scores, workspace))


def tq_score_static(plan: Plan, Q, n: int, idx, qjl, gamma, norms, scores):
    """tq_score for callers that cannot allocate device memory: the rotated-query workspace is an
    array built into the library (TQ_STATIC_SCRATCH_BYTES), shared by every call on the device."""
    _check((_n or _native()).score_static(plan.handle, Q, n, idx, qjl, gamma, norms, scores))


def tq_score_static_max_queries(plan: Plan) -> int:
    return lib().tq_score_static_max_queries(plan.handle)


def tq_query_bytes(plan: Plan, nq: int) -> int:
    return lib().tq_query_bytes(plan.handle, nq)


def tq_query_prepare(plan: Plan, Q, prepared):
    """Query-side work of tq_score (rotations, scan operand) into `prepared` (>= tq_query_bytes(plan, nq) bytes)."""
    _check((_n or _native()).query_prepare(plan.handle, Q, prepared))


def tq_score_prepared(plan: Plan, prepared, nq: int, n: int, idx, qjl, gamma, norms, scores):
    _check((_n or _native()).score_prepared(plan.handle, prepared, nq, n, idx, qjl, gamma, norms, scores))


def tq_selftest_wait_timeout(plan: Plan, limit_cycles: int = 20000) -> None:
    """Enqueues the library's bounded-wait self test; the next tq_plan_status(plan) must raise TqError(6)."""
    _check(lib().tq_selftest_wait_timeout(plan.handle, limit_cycles, _stream()))


def tq_topk(plan: Plan, Q, n: int, idx, qjl, gamma, norms, k: int, top_scores, top_ids, workspace):
    _check((_n or _native()).topk(plan.handle, Q, n, idx, qjl, gamma, norms, k, top_scores, top_ids, workspace))


def tq_wsum(plan: Plan, W, n: int, idx, qjl, gamma, norms, out, workspace):
    _check((_n or _native()).wsum(plan.handle, W, n, idx, qjl, gamma, norms, out, workspace))


def tq_softmax(s1, s2, scale: float, W):
    _check((_n or _native()).softmax(s1, s2, scale, W))


def tq_attend_decode_workspace_bytes(ngroups: int, heads: int, tokens: int, d: int) -> int:
    return lib().tq_attend_decode_workspace_bytes(ngroups, heads, tokens, d)


def tq_attend_decode(groups, heads: int, tokens: int, q_per_kv: int, Q, scale: float, out, workspace, head_stride=None):
    """groups: sequence of dicts with keys plan_k, plan_v (Plan) and k_idx, k_qjl, k_gamma, k_norms, v_idx,
    v_norms, k_channels, v_channels (CUDA tensors or None); rows of all heads head-major, head_stride rows
    per head (default: tokens)."""
    _check((_n or _native()).attend_decode(groups, heads, tokens, tokens if head_stride is None else head_stride, q_per_kv, Q, scale,
                                           out, workspace))


def tq_kv_append(groups, heads: int, head_stride: int, position: int, K, V):
    """Quantises one new token per KV head (K, V: [heads, head_dim]) into row `position` of every head."""
    _check((_n or _native()).kv_append(groups, heads, head_stride, position, K, V))


def tq_entropy_lengths(d: int, bits: int, centroids) -> np.ndarray:
    """Huffman code lengths of the 2^bits index values for the given codebook (uint8 array)."""
    cent = np.ascontiguousarray(centroids, dtype=np.float32)
    out = np.zeros(1 << bits, dtype=np.uint8)
    _check(lib().tq_entropy_lengths(d, bits, _fptr(cent), out.ctypes.data_as(c_void_p)))
    return out


def tq_entropy_pack(plan: Plan, lengths, n: int, idx):
    """(packed uint8 tensor, row_offsets int64 tensor of n + 1 byte offsets): the entropy-coded index rows."""
    ln = np.ascontiguousarray(lengths, dtype=np.uint8)
    got = (_n or _native()).entropy_pack(plan.handle, ln.ctypes.data, n, idx)
    if not isinstance(got, tuple):
        _check(got)
    return got


def tq_entropy_unpack(plan: Plan, lengths, n: int, packed, offsets, idx_out):
    ln = np.ascontiguousarray(lengths, dtype=np.uint8)
    _check((_n or _native()).entropy_unpack(plan.handle, ln.ctypes.data, n, packed, offsets, idx_out))


def tq_select_topk(cand_scores, cand_ids, k: int, top_scores, top_ids):
    _check((_n or _native()).select_topk(cand_scores, cand_ids, k, top_scores, top_ids))


_KV8_TYPES = {torch.int8: TQ_I8, torch.float8_e4m3fn: TQ_E4M3}


class Kv8Cache:
    """A paged 8-bit KV cache over tensors of the caller: k, v [pages, heads, page_tokens, d] of torch.int8 or torch.float8_e4m3fn,
    k_scale, v_scale [pages, heads] float32 and, for tq_kv8_select, k_bounds [pages, heads, 2, d] int8; all contiguous."""

    def __init__(self, k, v, k_scale, v_scale, k_bounds=None):
        if k.dim() != 4 or k.dtype not in _KV8_TYPES:
            raise ValueError("k must be [pages, heads, page_tokens, d] of torch.int8 or torch.float8_e4m3fn")
        pages, heads, page_tokens, d = k.shape
        wanted = [("k", k, k.shape, k.dtype), ("v", v, k.shape, k.dtype), ("k_scale", k_scale, (pages, heads), torch.float32),
                  ("v_scale", v_scale, (pages, heads), torch.float32)]
        if k_bounds is not None:
            wanted.append(("k_bounds", k_bounds, (pages, heads, 2, d), torch.int8))
        for name, t, shape, dtype in wanted:
            if not t.is_cuda or t.device != k.device:
                raise ValueError("expected CUDA tensors of one device (this library has no CPU path)")
            if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
        self.k, self.v, self.k_scale, self.v_scale, self.k_bounds = k, v, k_scale, v_scale, k_bounds
        self.pages, self.heads, self.page_tokens, self.d = pages, heads, page_tokens, d
        self._struct = Kv8(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                           None if k_bounds is None else k_bounds.data_ptr(), pages, heads, page_tokens, d, _KV8_TYPES[k.dtype])
        self.handle = ctypes.addressof(self._struct)
        self.device_index = k.device.index

    @classmethod
    def empty(cls, pages: int, heads: int, page_tokens: int, d: int, dtype=torch.int8, bounds: bool = True, device="cuda"):
        """A cache whose pages hold nothing yet."""
        new = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device=device)
        return cls(new(pages, heads, page_tokens, d, dtype=dtype), new(pages, heads, page_tokens, d, dtype=dtype),
                   new(pages, heads, dtype=torch.float32), new(pages, heads, dtype=torch.float32),
                   new(pages, heads, 2, d, dtype=torch.int8) if bounds else None)


def tq_kv8_append(cache: Kv8Cache, table, tokens, K, V, starts=None):
    """Quantises new tokens (rows of K, V: [n, heads, d]) into the pages behind the tokens[b] cached ones of every sequence."""
    _check((_n or _native()).kv8_append(cache, table, tokens, starts, K, V))


def tq_kv8_attend_workspace_bytes(cache: Kv8Cache, nseq: int, n: int, q_per_kv: int, max_queries: int = 1, nlist: int = 0) -> int:
    return lib().tq_kv8_attend_workspace_bytes(cache.handle, nseq, n, q_per_kv, max_queries, nlist)


def tq_kv8_attend(cache: Kv8Cache, table, tokens, Q, scale: float, out, workspace, lse=None, starts=None, max_queries=None, lists=None):
    """Attention of Q [n, heads * q_per_kv, d] over the sequences' caches (or, with lists [n, heads, nlist], over the listed pages).
    max_queries: the largest number of rows of a sequence; without it, all rows may be one sequence's (one each without starts)."""
    if max_queries is None:
        max_queries = 1 if starts is None else Q.shape[0]
    _check((_n or _native()).kv8_attend(cache, table, tokens, starts, Q, scale, out, lse, max_queries, lists, workspace))


def tq_selftest_kv8_timeout(on: bool) -> None:
    """While on, for the whole process, waits of the kernel for many queries run out at once: its rows must be NaN."""
    _check(lib().tq_selftest_kv8_timeout(int(on)))


def tq_kv8_select_workspace_bytes(cache: Kv8Cache, n: int, width: int) -> int:
    return lib().tq_kv8_select_workspace_bytes(cache.handle, n, width)


def tq_kv8_select(cache: Kv8Cache, table, tokens, Q, lists, workspace, starts=None, first: int = 1, last: int = 1):
    """The lists.shape[2] best pages of every row and KV head into lists [n, heads, k] (int32), for tq_kv8_attend."""
    _check((_n or _native()).kv8_select(cache, table, tokens, starts, Q, first, last, lists, workspace))


def tq_pages_workspace_bytes(pages: int, requests: int) -> int:
    return lib().tq_pages_workspace_bytes(pages, requests)


def tq_pages_extend(refs, table, tokens, next_tokens, page_tokens: int, spare, workspace):
    """Gives every row of the table the pages that next_tokens[b] need beyond those of tokens[b]."""
    _check((_n or _native()).pages_extend(refs, table, tokens, next_tokens, page_tokens, spare, workspace))


def tq_pages_fork(cache: Kv8Cache, refs, table, tokens, parents, children, spare, workspace):
    """Makes row children[f] a copy of row parents[f]: full pages shared, the last one in part copied."""
    _check((_n or _native()).pages_fork(cache, refs, table, tokens, parents, children, spare, workspace))


def tq_pages_free(refs, table, tokens, seqs):
    """The rows seqs give back their pages."""
    _check((_n or _native()).pages_free(refs, table, tokens, seqs))


def tq_pages_compact(cache: Kv8Cache, refs, table, spare, workspace):
    """Moves the pages in use to the front of the pool and renames them in refs and table."""
    _check((_n or _native()).pages_compact(cache, refs, table, spare, workspace))


def tq_pages_copy(cache: Kv8Cache, src, dst):
    """Page src[i] to page dst[i], in all arrays of the cache."""
    _check((_n or _native()).pages_copy(cache, src, dst))
