"""Python binding of libhardkv (Hard-KV decoding-time compression step on MI355X).

Argument marshalling only: every step runs in the HIP kernels of libhardkv.so.
Torch tensors provide device memory and the current stream; each wrapper passes
their device pointers to the C entry point of the same name (include/hardkv.h)
and raises HardKVError on a non-zero status.  There is no fallback: if the
library is missing, importing the entry points raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

__all__ = ["HardKVError", "lib", "PagedKV", "Allocator", "hk_score", "hk_calibrate",
           "hk_calibrate_solve_T", "hk_topp_select", "hk_compact", "hk_decode_attn",
           "hk_append_kv", "hk_workspace_size", "hk_status_string", "OP_SCORE", "OP_COMPACT",
           "OP_DECODE", "OP_APPEND", "FLAG_NOSPACE", "FLAG_NAN", "FLAG_RANGE", "LIB_PATH",
           "hk_timing_enable", "hk_timing_read", "TIMED_KERNELS", "hk_calibrate_topp",
           "hk_pool_max", "hk_score_rows", "hk_vote_topp", "hk_budget_plan", "hk_budget_select",
           "hk_compact_modes", "hk_calibrate_solve_T_gd", "hk_alloc_init", "hk_compress", "OP_COMPRESS", "BUDGET_KEEP", "BUDGET_SPARSE", "BUDGET_REWRITE",
           "hk_probe", "PROBE_EXP", "PROBE_MFMA", "PROBE_MIX", "PROBE_SPLIT", "PROBE_VALU",
           "PROBE_MFMA4", "hk_decode_plan",
           "hk_decode_attn_noalloc", "hk_decode_noalloc_scratch_bytes", "ERR_SCRATCH",
           "OP_SELECT", "hk_select_workspace_size", "select_workspace", "hk_topp_select_ws",
           "hk_calibrate_topp_ws", "Chunks", "OP_RESERVE", "OP_TRIM", "FLAG_CHUNK", "hk_reserve_slots",
           "hk_write_kv", "hk_chunk_attn_workspace_size", "chunk_attn_workspace", "hk_chunk_attn",
           "hk_verify_workspace_size", "verify_workspace", "hk_verify_draft", "hk_trim_slots"]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libhardkv.so")

HK_F32, HK_BF16 = 0, 1
OP_SCORE, OP_COMPACT, OP_DECODE, OP_APPEND, OP_COMPRESS, OP_SELECT = 0, 1, 2, 3, 4, 5
OP_RESERVE, OP_TRIM = 6, 7
FLAG_NOSPACE, FLAG_NAN, FLAG_RANGE, FLAG_CHUNK = 1, 2, 4, 8
ERR_SCRATCH = 7
BUDGET_KEEP, BUDGET_SPARSE, BUDGET_REWRITE = 0, 1, 2
PROBE_EXP, PROBE_MFMA, PROBE_MIX, PROBE_SPLIT, PROBE_VALU, PROBE_MFMA4 = 0, 1, 2, 3, 4, 5
EXPORTED = ["hk_score", "hk_calibrate", "hk_calibrate_solve_T", "hk_topp_select", "hk_compact",
            "hk_decode_attn", "hk_append_kv", "hk_workspace_size", "hk_status_string",
            "hk_timing_enable", "hk_timing_read", "hk_calibrate_topp", "hk_pool_max",
            "hk_score_rows", "hk_vote_topp", "hk_budget_plan", "hk_budget_select",
            "hk_compact_modes", "hk_calibrate_solve_T_gd", "hk_alloc_init", "hk_compress",
            "hk_probe", "hk_decode_plan", "hk_decode_attn_noalloc", "hk_decode_noalloc_scratch_bytes",
            "hk_select_workspace_size", "hk_topp_select_ws", "hk_calibrate_topp_ws",
            "hk_reserve_slots", "hk_write_kv", "hk_chunk_attn_workspace_size", "hk_chunk_attn",
            "hk_verify_workspace_size", "hk_verify_draft", "hk_trim_slots"]
# kernel ids of hk_timing_read, in header order
TIMED_KERNELS = ["score_pass1", "score_merge", "score_pass2", "calibrate", "topp", "solve_T",
                 "compact_gather", "compact_meta", "decode_split", "decode_merge", "append",
                 "calib_topp", "score_rows", "vote", "vote_count", "budget_plan", "budget_select",
                 "reserve", "write_kv", "chunk_attn", "chunk_merge", "verify", "trim"]


class HardKVError(RuntimeError):
    pass


class hk_dims(C.Structure):
    _fields_ = [("NS", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32),
                ("W", C.c_int32)]


class hk_paged_kv(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("page_table", C.c_void_p),
                ("page_mask", C.c_void_p), ("n_pages", C.c_void_p), ("num_pages", C.c_int32),
                ("max_pages", C.c_int32), ("dtype", C.c_int32)]


class hk_allocator(C.Structure):
    _fields_ = [("free_ids", C.c_void_p), ("free_top", C.c_void_p), ("capacity", C.c_int32)]


class hk_chunks(C.Structure):
    _fields_ = [("start", C.c_void_p), ("n_seq", C.c_int32), ("n_tokens", C.c_int32),
                ("max_len", C.c_int32), ("granted", C.c_void_p)]


_lib = None


def lib():
    """Load libhardkv.so (built in-tree by paper_2606_28831_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise HardKVError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2606_28831_amd.build` (no fallback exists)")
        L = C.CDLL(LIB_PATH)
        P, I32, SZ, F, D = C.c_void_p, C.c_int32, C.c_size_t, C.c_float, C.c_double
        L.hk_workspace_size.restype = SZ
        L.hk_workspace_size.argtypes = [I32, C.POINTER(hk_dims), I32]
        L.hk_status_string.restype = C.c_char_p
        L.hk_status_string.argtypes = [I32, I32]
        L.hk_score.restype = I32
        L.hk_score.argtypes = [C.POINTER(hk_dims), P, C.POINTER(hk_paged_kv), I32, F, P, P, P, P,
                               P, I32, P, P, SZ, P]
        L.hk_calibrate.restype = I32
        L.hk_calibrate.argtypes = [I32, I32, P, P, I32, C.POINTER(C.c_void_p),
                                   C.POINTER(C.c_void_p), C.POINTER(C.c_float), P, P, P]
        L.hk_topp_select.restype = I32
        L.hk_topp_select.argtypes = [I32, I32, P, P, P, D, I32, I32, P, P, P, P, P]
        L.hk_calibrate_solve_T.restype = I32
        L.hk_calibrate_solve_T.argtypes = [I32, I32, P, P, P, P, P, F, F, I32, P, P]
        L.hk_compact.restype = I32
        L.hk_compact.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_paged_kv), P, I32, I32,
                                 C.POINTER(hk_allocator), P, P, SZ, P]
        L.hk_decode_attn.restype = I32
        L.hk_decode_attn.argtypes = [C.POINTER(hk_dims), P, C.POINTER(hk_paged_kv), F, P, P, P,
                                     SZ, P]
        L.hk_append_kv.restype = I32
        L.hk_append_kv.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_paged_kv), P, P,
                                   C.POINTER(hk_allocator), P, P, SZ, P]
        L.hk_calibrate_topp.restype = I32
        L.hk_calibrate_topp.argtypes = [I32, I32, P, P, I32, C.POINTER(C.c_void_p),
                                        C.POINTER(C.c_void_p), C.POINTER(C.c_float), D, I32, I32,
                                        P, P, P, P, P, P, P]
        L.hk_select_workspace_size.restype = SZ
        L.hk_select_workspace_size.argtypes = [I32, I32]
        L.hk_topp_select_ws.restype = I32
        L.hk_topp_select_ws.argtypes = [I32, I32, P, P, P, D, I32, I32, P, P, P, P, P, SZ, P]
        L.hk_calibrate_topp_ws.restype = I32
        L.hk_calibrate_topp_ws.argtypes = [I32, I32, P, P, I32, C.POINTER(C.c_void_p),
                                           C.POINTER(C.c_void_p), C.POINTER(C.c_float), D, I32,
                                           I32, P, P, P, P, P, P, P, SZ, P]
        L.hk_pool_max.restype = I32
        L.hk_pool_max.argtypes = [I32, I32, P, P, P, I32, P, P]
        L.hk_score_rows.restype = I32
        L.hk_score_rows.argtypes = [C.POINTER(hk_dims), P, C.POINTER(hk_paged_kv), I32, F, P, P, P]
        L.hk_vote_topp.restype = I32
        L.hk_vote_topp.argtypes = [I32, I32, I32, P, P, P, D, P, P, P, P, P]
        L.hk_budget_plan.restype = I32
        L.hk_budget_plan.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_paged_kv), I32, I32, I32, P,
                                     P, P]
        L.hk_budget_select.restype = I32
        L.hk_budget_select.argtypes = [I32, I32, P, P, P, P, P, P, P, I32, P, P, P]
        L.hk_compact_modes.restype = I32
        L.hk_compact_modes.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_paged_kv), P, I32, P,
                                       C.POINTER(hk_allocator), P, P, C.c_size_t, P]
        L.hk_calibrate_solve_T_gd.restype = I32
        L.hk_calibrate_solve_T_gd.argtypes = [I32, I32, P, P, P, P, P, F, F, I32, F, P, P, P]
        L.hk_alloc_init.restype = I32
        L.hk_alloc_init.argtypes = [C.POINTER(hk_allocator), I32, I32, P]
        L.hk_compress.restype = I32
        L.hk_compress.argtypes = [C.POINTER(hk_dims), P, C.POINTER(hk_paged_kv), I32, I32, F, P, D,
                                  I32, I32, C.POINTER(hk_allocator), P, P, P, P, SZ, P]
        L.hk_decode_attn_noalloc.restype = I32
        L.hk_decode_attn_noalloc.argtypes = [C.POINTER(hk_dims), P, C.POINTER(hk_paged_kv), F, P, P, P]
        L.hk_decode_noalloc_scratch_bytes.restype = SZ
        L.hk_decode_noalloc_scratch_bytes.argtypes = [C.POINTER(hk_dims), I32]
        L.hk_decode_plan.restype = I32
        L.hk_decode_plan.argtypes = [C.POINTER(hk_dims), I32, C.POINTER(I32), C.POINTER(I32)]
        I64 = C.c_int64
        L.hk_reserve_slots.restype = I32
        L.hk_reserve_slots.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_paged_kv),
                                       C.POINTER(hk_chunks), C.POINTER(hk_allocator), P, P, P, SZ, P]
        L.hk_write_kv.restype = I32
        L.hk_write_kv.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_paged_kv), I32, I32, P, P, I64,
                                  I64, P, I64, I64, P]
        L.hk_chunk_attn_workspace_size.restype = SZ
        L.hk_chunk_attn_workspace_size.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_chunks), I32]
        L.hk_chunk_attn.restype = I32
        L.hk_chunk_attn.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_paged_kv), C.POINTER(hk_chunks),
                                    P, I64, F, P, P, P, SZ, P]
        L.hk_verify_workspace_size.restype = SZ
        L.hk_verify_workspace_size.argtypes = [I32, I32]
        L.hk_verify_draft.restype = I32
        L.hk_verify_draft.argtypes = [C.POINTER(hk_chunks), I32, I32, P, P, I64, P, I64, P, P, P, P,
                                      P, P, SZ, P]
        L.hk_trim_slots.restype = I32
        L.hk_trim_slots.argtypes = [C.POINTER(hk_dims), C.POINTER(hk_paged_kv), I32, P,
                                    C.POINTER(hk_allocator), P, SZ, P]
        L.hk_probe.restype = I32
        L.hk_probe.argtypes = [I32, I32, I32, P, P]
        L.hk_timing_enable.restype = I32
        L.hk_timing_enable.argtypes = [C.c_uint32]
        L.hk_timing_read.restype = I32
        L.hk_timing_read.argtypes = [I32, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        _lib = L
    return _lib


def _ptr(t):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor")
    if not t.is_contiguous():
        raise HardKVError("tensor arguments must be contiguous")
    return C.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _check(code: int, name: str):
    if code != 0:
        msg = lib().hk_status_string(code, 0).decode()
        raise HardKVError(f"{name}: {msg}")


def hk_status_string(code: int, flags: bool = False) -> str:
    return lib().hk_status_string(int(code), int(bool(flags))).decode()


def dims(NS, Hq, Hkv, D, W=0) -> hk_dims:
    return hk_dims(int(NS), int(Hq), int(Hkv), int(D), int(W))


class PagedKV:
    """Device tensors of one paged Cascade Cache plus its C descriptor."""

    def __init__(self, k_pool, v_pool, page_table, page_mask, n_pages):
        self.k_pool, self.v_pool = k_pool, v_pool
        self.page_table, self.page_mask, self.n_pages = page_table, page_mask, n_pages
        if k_pool.dtype == torch.bfloat16:
            dt = HK_BF16
        elif k_pool.dtype == torch.float32:
            dt = HK_F32
        else:
            raise HardKVError("cache dtype must be bfloat16 or float32")
        self.desc = hk_paged_kv(k_pool.data_ptr(), v_pool.data_ptr() if v_pool is not None else None,
                                page_table.data_ptr(), page_mask.data_ptr(), n_pages.data_ptr(),
                                k_pool.shape[0], page_table.shape[1], dt)
        self._sizes = None

    def sizes(self):
        """(heads, head size, device) that the tensors of desc hold, once they are found to agree."""
        if self._sizes is None:
            t, m, n, k, v = self.page_table, self.page_mask, self.n_pages, self.k_pool, self.v_pool
            of = lambda x: x is None or (x.is_contiguous() and x.get_device() == k.get_device())  # noqa: E731
            if not all(of(x) for x in (t, m, n, k, v)):
                raise HardKVError("a cache's tensors must be contiguous and on one device")
            if (t.dtype != torch.int32 or n.dtype != torch.int32 or m.dtype not in (torch.int16, torch.uint16)
                    or t.dim() != 2 or m.dim() != 2 or m.shape[1] != t.shape[1]):
                raise HardKVError("a cache's tables must be int32 [heads, pages], masks 16-bit [heads, pages], "
                                  "counts int32 [heads]")
            slots = k.shape[0] * 16
            if slots == 0 or k.numel() % slots or (v is not None and (v.dtype != k.dtype or v.numel() != k.numel())):
                raise HardKVError("a cache's pools must be [pages, 16, D], both in one type")
            self._sizes = min(t.shape[0], m.shape[0], n.numel()), k.numel() // slots, k.get_device()
        return self._sizes

    def rows(self, first_head: int, n_heads: int) -> "PagedKV":
        """A view of heads [first_head, first_head + n_heads) (e.g. one layer)."""
        sl = slice(first_head, first_head + n_heads)
        return PagedKV(self.k_pool, self.v_pool, self.page_table[sl], self.page_mask[sl],
                       self.n_pages[sl])

    @property
    def max_pages(self):
        return self.page_table.shape[1]


class Allocator:
    def __init__(self, free_ids, free_top):
        self.free_ids, self.free_top = free_ids, free_top
        self.desc = hk_allocator(free_ids.data_ptr(), free_top.data_ptr(), free_ids.shape[0])
        self._device = None

    def device(self):
        """The device of desc's tensors, once they are found to be what it says."""
        if self._device is None:
            ids, top = self.free_ids, self.free_top
            if (ids.dtype != torch.int32 or top.dtype != torch.int32 or ids.dim() != 1 or not ids.is_contiguous()
                    or top.numel() < 1 or ids.get_device() != top.get_device()):
                raise HardKVError("an allocator's stack and top must be contiguous int32, on one device")
            self._device = ids.get_device()
        return self._device


def hk_workspace_size(op: int, d: hk_dims, max_pages: int) -> int:
    return int(lib().hk_workspace_size(int(op), C.byref(d), int(max_pages)))


def workspace(op: int, d: hk_dims, max_pages: int, device) -> torch.Tensor:
    n = max(256, hk_workspace_size(op, d, max_pages))
    return torch.empty(n, dtype=torch.uint8, device=device)


def hk_score(d: hk_dims, q_obs, kv: PagedKV, L_dense: int, sm_scale: float, s_attn, cand_len,
             row_lse_in=None, row_lse_out=None, ref_slots=None, n_ref: int = 0, x_red=None,
             ws=None, stream=None):
    _check(lib().hk_score(C.byref(d), _ptr(q_obs), C.byref(kv.desc), int(L_dense),
                          float(sm_scale), _ptr(row_lse_in), _ptr(row_lse_out), _ptr(s_attn),
                          _ptr(cand_len), _ptr(ref_slots), int(n_ref), _ptr(x_red), _ptr(ws),
                          ws.numel() if ws is not None else 0, _stream(stream)), "hk_score")


def hk_calibrate(n_heads: int, S_max: int, cand_len, page_mask, xs, Ts, weights, c_out,
                 lse_out=None, stream=None):
    m = len(xs)
    xa = (C.c_void_p * m)(*[t.data_ptr() for t in xs])
    Ta = None
    if Ts is not None:
        Ta = (C.c_void_p * m)(*[(t.data_ptr() if t is not None else None) for t in Ts])
    wa = (C.c_float * m)(*[float(w) for w in weights])
    _check(lib().hk_calibrate(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask), m, xa,
                              Ta, wa, _ptr(c_out), _ptr(lse_out), _stream(stream)), "hk_calibrate")


def hk_topp_select(n_heads: int, S_max: int, cand_len, page_mask, c, p: float, sel_bits, k_out,
                   k_min: int = 1, k_max: int = 0, sel_mass=None, status=None, stream=None):
    _check(lib().hk_topp_select(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask), _ptr(c),
                                float(p), int(k_min), int(k_max), _ptr(sel_bits), _ptr(k_out),
                                _ptr(sel_mass), _ptr(status), _stream(stream)), "hk_topp_select")


def hk_calibrate_topp(n_heads: int, S_max: int, cand_len, page_mask, xs, Ts, weights, p: float,
                      sel_bits, k_out, c_out=None, lse_out=None, k_min: int = 1, k_max: int = 0,
                      sel_mass=None, status=None, stream=None):
    m = len(xs)
    xa = (C.c_void_p * m)(*[t.data_ptr() for t in xs])
    Ta = None
    if Ts is not None:
        Ta = (C.c_void_p * m)(*[(t.data_ptr() if t is not None else None) for t in Ts])
    wa = (C.c_float * m)(*[float(w) for w in weights])
    _check(lib().hk_calibrate_topp(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask), m,
                                   xa, Ta, wa, float(p), int(k_min), int(k_max), _ptr(c_out),
                                   _ptr(lse_out), _ptr(sel_bits), _ptr(k_out), _ptr(sel_mass),
                                   _ptr(status), _stream(stream)), "hk_calibrate_topp")


def hk_select_workspace_size(n_heads: int, S_max: int) -> int:
    return int(lib().hk_select_workspace_size(int(n_heads), int(S_max)))


def select_workspace(n_heads: int, S_max: int, device) -> torch.Tensor:
    """Workspace of hk_topp_select_ws / hk_calibrate_topp_ws for these sizes."""
    n = max(256, hk_select_workspace_size(n_heads, S_max))
    return torch.empty(n, dtype=torch.uint8, device=device)


def hk_topp_select_ws(n_heads: int, S_max: int, cand_len, page_mask, c, p: float, sel_bits, k_out,
                      ws, k_min: int = 1, k_max: int = 0, sel_mass=None, status=None, stream=None):
    _check(lib().hk_topp_select_ws(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask),
                                   _ptr(c), float(p), int(k_min), int(k_max), _ptr(sel_bits),
                                   _ptr(k_out), _ptr(sel_mass), _ptr(status), _ptr(ws),
                                   ws.numel() * ws.element_size(), _stream(stream)),
           "hk_topp_select_ws")


def hk_calibrate_topp_ws(n_heads: int, S_max: int, cand_len, page_mask, xs, Ts, weights, p: float,
                         sel_bits, k_out, ws, c_out=None, lse_out=None, k_min: int = 1,
                         k_max: int = 0, sel_mass=None, status=None, stream=None):
    m = len(xs)
    xa = (C.c_void_p * m)(*[t.data_ptr() for t in xs])
    Ta = None
    if Ts is not None:
        Ta = (C.c_void_p * m)(*[(t.data_ptr() if t is not None else None) for t in Ts])
    wa = (C.c_float * m)(*[float(w) for w in weights])
    _check(lib().hk_calibrate_topp_ws(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask),
                                      m, xa, Ta, wa, float(p), int(k_min), int(k_max),
                                      _ptr(c_out), _ptr(lse_out), _ptr(sel_bits), _ptr(k_out),
                                      _ptr(sel_mass), _ptr(status), _ptr(ws),
                                      ws.numel() * ws.element_size(), _stream(stream)),
           "hk_calibrate_topp_ws")


def hk_pool_max(n_heads: int, S_max: int, cand_len, page_mask, x, radius: int, x_out, stream=None):
    _check(lib().hk_pool_max(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask), _ptr(x),
                             int(radius), _ptr(x_out), _stream(stream)), "hk_pool_max")


def hk_calibrate_solve_T(n_heads: int, S_max: int, cand_len, page_mask, x, k, target_mass, T_out,
                         T_lo: float = 1e-4, T_hi: float = 1e4, iters: int = 40, stream=None):
    _check(lib().hk_calibrate_solve_T(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask),
                                      _ptr(x), _ptr(k), _ptr(target_mass), float(T_lo),
                                      float(T_hi), int(iters), _ptr(T_out), _stream(stream)),
           "hk_calibrate_solve_T")


def hk_calibrate_solve_T_gd(n_heads: int, S_max: int, cand_len, page_mask, x, k, target_mass,
                            T_out, T_init: float = 1.0, lr: float = 0.05, iters: int = 200,
                            tol: float = 0.0, loss_out=None, stream=None):
    _check(lib().hk_calibrate_solve_T_gd(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask),
                                         _ptr(x), _ptr(k), _ptr(target_mass), float(T_init),
                                         float(lr), int(iters), float(tol), _ptr(T_out),
                                         _ptr(loss_out), _stream(stream)), "hk_calibrate_solve_T_gd")


def hk_compress(d: hk_dims, q_obs, kv: PagedKV, L_dense: int, L_sparse: int, sm_scale: float,
                p: float, alloc: Allocator, k_out, ws, status=None, sel_bits_out=None,
                row_lse_in=None, k_min: int = 1, k_max: int = 0, stream=None):
    _check(lib().hk_compress(C.byref(d), _ptr(q_obs), C.byref(kv.desc), int(L_dense), int(L_sparse),
                             float(sm_scale), _ptr(row_lse_in), float(p), int(k_min), int(k_max),
                             C.byref(alloc.desc), _ptr(sel_bits_out), _ptr(k_out), _ptr(status),
                             _ptr(ws), ws.numel(), _stream(stream)), "hk_compress")


def hk_alloc_init(alloc: Allocator, first_free: int, num_pages: int, stream=None):
    _check(lib().hk_alloc_init(C.byref(alloc.desc), int(first_free), int(num_pages),
                               _stream(stream)), "hk_alloc_init")


def hk_compact(d: hk_dims, kv: PagedKV, sel_bits, L_dense: int, L_sparse: int, alloc: Allocator,
               status, ws, stream=None):
    _check(lib().hk_compact(C.byref(d), C.byref(kv.desc), _ptr(sel_bits), int(L_dense),
                            int(L_sparse), C.byref(alloc.desc), _ptr(status), _ptr(ws), ws.numel(),
                            _stream(stream)), "hk_compact")


def hk_decode_attn(d: hk_dims, q, kv: PagedKV, sm_scale: float, o, lse, ws, stream=None):
    _check(lib().hk_decode_attn(C.byref(d), _ptr(q), C.byref(kv.desc), float(sm_scale), _ptr(o),
                                _ptr(lse), _ptr(ws), ws.numel(), _stream(stream)), "hk_decode_attn")


def hk_decode_attn_noalloc(d: hk_dims, q, kv: PagedKV, sm_scale: float, o, lse, stream=None):
    """hk_decode_attn with the split states in the library's static scratch (no workspace)."""
    _check(lib().hk_decode_attn_noalloc(C.byref(d), _ptr(q), C.byref(kv.desc), float(sm_scale),
                                        _ptr(o), _ptr(lse), _stream(stream)), "hk_decode_attn_noalloc")


def hk_decode_noalloc_scratch_bytes(d: hk_dims, max_pages: int) -> int:
    return int(lib().hk_decode_noalloc_scratch_bytes(C.byref(d), int(max_pages)))


def hk_decode_plan(d: hk_dims, max_pages: int):
    """(n_split, pages_per_split) that hk_decode_attn uses for these dims and table width."""
    ns, pps = C.c_int32(0), C.c_int32(0)
    _check(lib().hk_decode_plan(C.byref(d), int(max_pages), C.byref(ns), C.byref(pps)),
           "hk_decode_plan")
    return ns.value, pps.value


def hk_append_kv(d: hk_dims, kv: PagedKV, k_new, v_new, alloc: Allocator, status, ws,
                 stream=None):
    _check(lib().hk_append_kv(C.byref(d), C.byref(kv.desc), _ptr(k_new), _ptr(v_new),
                              C.byref(alloc.desc), _ptr(status), _ptr(ws),
                              ws.numel() if ws is not None else 0, _stream(stream)), "hk_append_kv")


def hk_score_rows(d: hk_dims, q_obs, kv: PagedKV, L_dense: int, sm_scale: float, row_lse, a_rows,
                  stream=None):
    _check(lib().hk_score_rows(C.byref(d), _ptr(q_obs), C.byref(kv.desc), int(L_dense),
                               float(sm_scale), _ptr(row_lse), _ptr(a_rows), _stream(stream)),
           "hk_score_rows")


def hk_vote_topp(n_heads: int, R: int, S_max: int, cand_len, page_mask, a_rows, p: float, votes,
                 row_sel, row_k=None, status=None, stream=None):
    _check(lib().hk_vote_topp(int(n_heads), int(R), int(S_max), _ptr(cand_len), _ptr(page_mask),
                              _ptr(a_rows), float(p), _ptr(votes), _ptr(row_sel), _ptr(row_k),
                              _ptr(status), _stream(stream)), "hk_vote_topp")


def hk_budget_plan(d: hk_dims, kv: PagedKV, L_dense: int, L_lower: int, L_upper: int, head_mode,
                   k_cap, stream=None):
    _check(lib().hk_budget_plan(C.byref(d), C.byref(kv.desc), int(L_dense), int(L_lower),
                                int(L_upper), _ptr(head_mode), _ptr(k_cap), _stream(stream)),
           "hk_budget_plan")


def hk_budget_select(n_heads: int, S_max: int, cand_len, page_mask, sel_out, k_out, votes=None,
                     c=None, sel_in=None, head_mode=None, k_cap=None, n_sink: int = 0,
                     stream=None):
    _check(lib().hk_budget_select(int(n_heads), int(S_max), _ptr(cand_len), _ptr(page_mask),
                                  _ptr(votes), _ptr(c), _ptr(sel_in), _ptr(head_mode), _ptr(k_cap),
                                  int(n_sink), _ptr(sel_out), _ptr(k_out), _stream(stream)),
           "hk_budget_select")


def hk_compact_modes(d: hk_dims, kv: PagedKV, sel_bits, L_dense: int, head_mode, alloc: Allocator,
                     status, ws, stream=None):
    _check(lib().hk_compact_modes(C.byref(d), C.byref(kv.desc), _ptr(sel_bits), int(L_dense),
                                  _ptr(head_mode), C.byref(alloc.desc), _ptr(status), _ptr(ws),
                                  ws.numel(), _stream(stream)), "hk_compact_modes")


# ---------------------------------------------------------------- chunks of new tokens
# The wrappers below compare the tensors with the sizes given (a row too few would be read past
# its end, a pool of another head size past the pool's) and run on the tensors' own device, on its
# current stream unless one is given.
class Chunks:
    """The new tokens of a batch: sequence s has the token rows start[s] .. start[s + 1] of
    n_tokens (start: int32 device tensor of n_seq + 1 entries), at most max_len of them.
    granted: None, or an int32 device word that hk_reserve_slots sets to 1 or, where it refused, to
    0: hk_verify_draft then takes the chunks as empty, so that nothing is dropped that was not given."""

    def __init__(self, start, n_tokens: int, max_len: int, granted=None):
        if start.dtype != torch.int32 or start.dim() != 1 or not start.is_contiguous():
            raise HardKVError("chunk starts must be a contiguous int32 vector")
        self.start, self.n_tokens, self.max_len = start, int(n_tokens), int(max_len)
        self.n_seq = start.numel() - 1
        self.desc = hk_chunks(start.data_ptr(), self.n_seq, self.n_tokens, self.max_len)
        self.granted_by(granted)

    def granted_by(self, word):
        """The word that later calls set and read (None: none)."""
        if word is not None and (word.dtype != torch.int32 or word.numel() < 1 or word.device != self.start.device):
            raise HardKVError("granted must be an int32 word on the chunk starts' device")
        self.granted = word
        self.desc.granted = None if word is None else word.data_ptr()


def _need(ok: bool, what: str):
    if not ok:
        raise HardKVError(what)


def _kv_dtype(kv: PagedKV):
    return kv.k_pool.dtype


def _fits(d: hk_dims, kv: PagedKV, heads: int, alloc: Allocator = None):
    """The cache has the heads and the head size of d, and the allocator is beside it."""
    have, D, dev = kv.sizes()
    if have < heads:
        raise HardKVError("the cache has fewer rows than NS * Hkv")
    if D != d.D:
        raise HardKVError(f"the cache's head size is {D}, not {d.D}")
    if alloc is not None and alloc.device() != dev:
        raise HardKVError("the allocator is on another device than the cache")


def _status(status):
    return None if status is None else _vector(status, 1, torch.int32, "status")


def _run(name: str, t, tensors, stream, *args):
    """Call an entry point on the device that holds t and the tensors it works on."""
    dev = t.get_device()
    if dev < 0:
        raise HardKVError(f"{name}: tensors outside the GPU")
    for x in tensors:
        if x is not None and x.get_device() != dev:
            raise HardKVError(f"{name}: tensors on different devices")
    here = torch.cuda.current_device()
    if dev != here:
        with torch.cuda.device(t.device):
            _check(getattr(lib(), name)(*args, _stream(stream)), name)
        return
    # (the raw handle: torch's stream object takes longer than a launch)
    raw = torch._C._cuda_getCurrentRawStream(here) if stream is None else stream.cuda_stream
    _check(getattr(lib(), name)(*args, C.c_void_p(raw)), name)


def _vector(t, n: int, dtype, what: str):
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < n:
        raise HardKVError(f"{what} must be a contiguous {dtype} tensor of at least {n} entries")
    return C.c_void_p(t.data_ptr())


def _token_rows(t, n_tokens: int, heads: int, D: int, dtype, what: str):
    """(pointer, row stride) of a [..., tokens, heads, D] tensor whose rows are contiguous."""
    shape, stride = t.shape, t.stride()
    if (t.dtype != dtype or len(shape) < 3 or shape[-1] != D or shape[-2] != heads
            or shape[-3] < n_tokens):
        raise HardKVError(f"{what} must be [tokens, {heads}, {D}] in {dtype}")
    if stride[-1] != 1 or (heads > 1 and stride[-2] != D):
        raise HardKVError(f"{what}: the heads of a token must be contiguous")
    return C.c_void_p(t.data_ptr()), stride[-3] if n_tokens > 1 else max(stride[-3], heads * D)


def hk_reserve_slots(d: hk_dims, kv: PagedKV, chunks: Chunks, alloc: Allocator, ws, slot_map=None,
                     status=None, stream=None):
    _fits(d, kv, d.NS * d.Hkv, alloc)
    n = d.NS // max(chunks.n_seq, 1) * chunks.n_tokens * d.Hkv
    _run("hk_reserve_slots", kv.page_table, (chunks.start, slot_map, status, ws),
         stream, C.byref(d), C.byref(kv.desc),
         C.byref(chunks.desc), C.byref(alloc.desc),
         None if slot_map is None else _vector(slot_map, n, torch.int64, "slot_map"), _status(status),
         _ptr(ws), ws.numel())


def hk_write_kv(d: hk_dims, kv: PagedKV, n_tokens: int, slot_map, k_new, v_new, stream=None):
    """k_new, v_new: [tokens, Hkv, D], or [layers, tokens, Hkv, D] with the slot map of as many
    layers; views into larger tensors are fine as long as a token's heads are contiguous."""
    _need(k_new.dim() == v_new.dim() and k_new.dim() in (3, 4), "k_new and v_new must be 3- or 4-d")
    _fits(d, kv, 0)
    layers = k_new.shape[0] if k_new.dim() == 4 else 1
    _need(v_new.dim() == 3 or v_new.shape[0] == layers, "k_new and v_new differ in layers")
    kp, kr = _token_rows(k_new, n_tokens, d.Hkv, d.D, _kv_dtype(kv), "k_new")
    vp, vr = _token_rows(v_new, n_tokens, d.Hkv, d.D, _kv_dtype(kv), "v_new")
    _run("hk_write_kv", kv.k_pool, (slot_map, k_new, v_new), stream, C.byref(d), C.byref(kv.desc),
         layers, int(n_tokens),
         _vector(slot_map, layers * n_tokens * d.Hkv, torch.int64, "slot_map"), kp,
         k_new.stride(0) if layers > 1 else 0, kr, vp, v_new.stride(0) if layers > 1 else 0, vr)


def hk_chunk_attn_workspace_size(d: hk_dims, chunks: Chunks, max_pages: int) -> int:
    return int(lib().hk_chunk_attn_workspace_size(C.byref(d), C.byref(chunks.desc), int(max_pages)))


def chunk_attn_workspace(d: hk_dims, chunks: Chunks, max_pages: int, device) -> torch.Tensor:
    n = max(256, hk_chunk_attn_workspace_size(d, chunks, max_pages))
    return torch.empty(n, dtype=torch.uint8, device=device)


def hk_chunk_attn(d: hk_dims, kv: PagedKV, chunks: Chunks, q, sm_scale: float, o, ws, lse=None,
                  stream=None):
    T = chunks.n_tokens
    _fits(d, kv, d.NS * d.Hkv)
    qp, qr = _token_rows(q, T, d.Hq, d.D, _kv_dtype(kv), "q")
    _need(q.dim() == 3, "q must be 3-d")
    op = _vector(o, T * d.Hq * d.D, _kv_dtype(kv), "o")
    lp = None if lse is None else _vector(lse, T * d.Hq, torch.float32, "lse")
    _run("hk_chunk_attn", kv.k_pool, (chunks.start, q, o, lse, ws), stream,
         C.byref(d), C.byref(kv.desc), C.byref(chunks.desc), qp,
         qr, float(sm_scale), op, lp, _ptr(ws), 0 if ws is None else ws.numel())


def hk_verify_workspace_size(n_seq: int, V: int) -> int:
    return int(lib().hk_verify_workspace_size(int(n_seq), int(V)))


def verify_workspace(n_seq: int, V: int, device) -> torch.Tensor:
    n = max(256, hk_verify_workspace_size(n_seq, V))
    return torch.empty(n, dtype=torch.uint8, device=device)


def hk_verify_draft(chunks: Chunks, V: int, tokens, p, u, n_accept, next_token, n_drop, ws, q=None,
                    status=None, stream=None):
    T, B, i32 = chunks.n_tokens, chunks.n_seq, torch.int32
    dt = {torch.float32: HK_F32, torch.bfloat16: HK_BF16}.get(p.dtype)
    _need(dt is not None, "probabilities must be float32 or bfloat16")
    for t, what in ((p, "p"), (q, "q")):
        if t is not None and (t.dtype != p.dtype or t.dim() != 2 or t.shape[0] < T or t.shape[1] < V
                              or (t.stride(1) != 1 and V > 1)):
            raise HardKVError(f"{what} must be [tokens, V] with contiguous rows, both in one type")
    row = lambda t: 0 if t is None else (t.stride(0) if T > 1 else max(t.stride(0), V))  # noqa: E731
    _run("hk_verify_draft", p,
         (chunks.start, tokens, q, u, n_accept, next_token, n_drop, status, ws), stream,
         C.byref(chunks.desc), int(V), dt,
         _vector(tokens, T, i32, "tokens"), C.c_void_p(p.data_ptr()), row(p),
         None if q is None else C.c_void_p(q.data_ptr()), row(q),
         _vector(u, T, torch.float32, "u"), _vector(n_accept, B, i32, "n_accept"),
         _vector(next_token, B, i32, "next_token"), _vector(n_drop, B, i32, "n_drop"), _status(status),
         _ptr(ws), ws.numel())


def hk_trim_slots(d: hk_dims, kv: PagedKV, n_drop, alloc: Allocator, ws, stream=None):
    _fits(d, kv, d.NS * d.Hkv, alloc)
    n = n_drop.numel()
    _run("hk_trim_slots", kv.page_table, (n_drop, ws), stream, C.byref(d),
         C.byref(kv.desc), n,
         _vector(n_drop, n, torch.int32, "n_drop"), C.byref(alloc.desc), _ptr(ws), ws.numel())


def hk_timing_enable(kernels=None):
    """Time the launches of the named kernels (all of them for kernels=None; [] turns
    timing off)."""
    names = TIMED_KERNELS if kernels is None else kernels
    mask = 0
    for k in names:
        mask |= 1 << TIMED_KERNELS.index(k)
    _check(lib().hk_timing_enable(mask), "hk_timing_enable")


def hk_probe(kind: int, blocks: int, iters: int, out, stream=None):
    """One rate-probe launch (a PROBE_* kind); out: >= 256 * blocks floats."""
    _check(lib().hk_probe(int(kind), int(blocks), int(iters), _ptr(out), _stream(stream)),
           "hk_probe")


def hk_timing_read(kernel: str):
    """(summed ms, launches) of one timed kernel since the previous read; clears them."""
    ms, n = C.c_double(0.0), C.c_int64(0)
    _check(lib().hk_timing_read(TIMED_KERNELS.index(kernel), C.byref(ms), C.byref(n)),
           "hk_timing_read")
    return ms.value, n.value
