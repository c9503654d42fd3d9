"""Chaining of the C entry points into one compression step and one decode step.

Marshalling only: buffers are allocated once (static shapes) and every call goes to
libhardkv.  The compression step is Steps 2-3 of the continuous compression pipeline
(Sec. 3.1): score -> calibrate -> Top-p -> rewrite; the budgeted step adds Step 4
(hard budget with Cautious Update voting and attention sinks).
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

from . import (Allocator, Chunks, PagedKV, PagedKV8, OP_APPEND, OP_DECODE8, OP_COMPACT, OP_DECODE, OP_RESERVE, OP_SCORE, OP_TRIM,
               HardKVError, _fits, chunk_attn8_workspace, chunk_attn_workspace, dims, hk_chunk_attn8, hk_compact8,
               hk_decode_attn8, hk_read_kv8, hk_write_kv8, hk_append_kv, hk_chunk_attn, hk_reserve_slots,
               hk_trim_slots, hk_verify_draft, hk_write_kv, verify_workspace,
               hk_budget_plan, hk_budget_select, hk_calibrate, hk_calibrate_solve_T,
               hk_calibrate_solve_T_gd, hk_calibrate_topp_ws, hk_compact, hk_compact_modes, hk_decode_attn, hk_pool_max,
               hk_score, hk_score_rows, hk_vote_topp, select_workspace, workspace)


@dataclass
class CompressBuffers:
    s_attn: torch.Tensor
    s_pool: torch.Tensor | None
    x_red: torch.Tensor | None
    c: torch.Tensor
    c_attn: torch.Tensor | None
    cand_len: torch.Tensor
    row_lse: torch.Tensor
    sel_bits: torch.Tensor
    k: torch.Tensor
    sel_mass: torch.Tensor
    k_attn: torch.Tensor | None
    mass_attn: torch.Tensor | None
    T_red: torch.Tensor | None
    status: torch.Tensor
    ws_score: torch.Tensor
    ws_compact: torch.Tensor
    ws_select: torch.Tensor


def _shaped(t, shape, dtype, what: str):
    """t in a shape that can be cut by head or sequence: a contiguous one may come in any other."""
    if t.dtype != dtype:
        raise HardKVError(f"{what} must be {dtype}")
    if tuple(t.shape) == shape:
        return t
    if t.numel() != math.prod(shape) or not t.is_contiguous():
        raise HardKVError(f"{what} must be {list(shape)}")
    return t.view(shape)


class ScoringCopy:
    """K of an 8-bit cache read back in bf16 or fp32, a few sequences at a time, as the score passes
    take it: a paged cache of its own whose rows lie one after the other, at most max_bytes of it."""

    def __init__(self, NS, Hq, Hkv, D, W, kv: PagedKV8, dtype=torch.bfloat16, max_bytes: int = 1 << 30):
        _fits(dims(NS, Hq, Hkv, D, W), kv, NS * Hkv)
        dev, P = kv.k_pool.device, kv.max_pages
        row = P * 16 * D * dtype.itemsize * Hkv
        self.n = n = max(1, min(NS, max_bytes // row))
        self.kv, self.NS, self.Hq, self.Hkv, self.D, self.W, self.P = kv, NS, Hq, Hkv, D, W, P
        H, i32 = n * Hkv, torch.int32
        self.k = torch.zeros(H * P, 16, D, dtype=dtype, device=dev)
        self.table = torch.arange(H * P, dtype=i32, device=dev).view(H, P)
        self.mask = torch.zeros(H, P, dtype=kv.page_mask.dtype, device=dev)
        self.n_pages = torch.zeros(H, dtype=i32, device=dev)
        self.slot = torch.arange(16, dtype=torch.int64, device=dev)
        self.slot_map = torch.empty(H, P, 16, dtype=torch.int64, device=dev)
        self.q = torch.empty(W * n * Hq * D, dtype=dtype, device=dev)
        self.lse = torch.empty(W * n * Hq, dtype=torch.float32, device=dev)
        self.ws = workspace(OP_SCORE, dims(n, Hq, Hkv, D, W), P, dev)

    def takes(self, q_obs):
        """Refuse window queries that a copy in score_dtype would round."""
        dtype = self.k.dtype
        if q_obs.dtype != dtype and (q_obs.dtype, dtype) != (torch.bfloat16, torch.float32):
            raise HardKVError(f"window queries of {q_obs.dtype} over K read back in {dtype}: give their type as score_dtype")

    def groups(self, q_obs, stream=None):
        """For every few sequences: (their dims, first head, heads, sequences as a slice, queries, K)."""
        self.takes(q_obs)
        q_obs = _shaped(q_obs, (self.W, self.NS, self.Hq, self.D), q_obs.dtype, "window queries")
        for s0 in range(0, self.NS, self.n):
            ns = min(self.n, self.NS - s0)
            h0, H, sl = s0 * self.Hkv, ns * self.Hkv, slice(s0, s0 + ns)
            with torch.cuda.stream(stream):
                self.mask[:H].copy_(self.kv.page_mask[h0:h0 + H])
                self.n_pages[:H].copy_(self.kv.n_pages[h0:h0 + H])
                # 16 page + slot; below 0 past the rows' ends, where the table holds -1
                at = self.slot_map[:H]
                at.copy_(self.kv.page_table[h0:h0 + H, :, None].expand(H, self.P, 16))
                at.mul_(16).add_(self.slot)
                q = self.q[:self.W * ns * self.Hq * self.D].view(self.W, ns, self.Hq, self.D)
                q.copy_(q_obs[:, sl])
            n = H * self.P * 16
            hk_read_kv8(dims(1, 1, 1, self.D), self.kv, n, at, self.k.view(-1, 1, self.D), stream=stream)
            yield (dims(ns, self.Hq, self.Hkv, self.D, self.W), h0, H, sl, q,
                   PagedKV(self.k, None, self.table[:H], self.mask[:H], self.n_pages[:H]))

    def group_lse(self, sl):
        n = sl.stop - sl.start
        return self.lse[:self.W * n * self.Hq].view(self.W, n, self.Hq)


def _compact(d, kv, sel_bits, L_dense, L_sparse, alloc, status, ws, stream):
    run = hk_compact8 if isinstance(kv, PagedKV8) else hk_compact
    run(d, kv, sel_bits, L_dense, L_sparse, alloc, status, ws, stream=stream)


class Compressor:
    """One compression step over every head of a paged cache.

    An 8-bit cache (PagedKV8) is scored on copies of its K, read back in score_dtype, and rewritten as it
    lies.  score_dtype is the type of the window queries, or float32 for bfloat16 ones, whose K is then not
    rounded; others are refused.  K in bfloat16 moves a score by up to 2^-9 sm_scale sum |q k| against what
    hk_decode_attn8 sees: rows scored under its LSEs (row_lse_in) sum to 1 within e^ that.

    metric "attn": attention mass over the window, calibrated with T = 1.
    metric "attn+red": attention mass and key redundancy, each calibrated (the
    redundancy temperature solved once per head, on the first call), mixed 0.5/0.5.
    Calibration and Top-p run as one launch; keep_c=False leaves the calibrated
    probabilities on chip (buf.c / buf.c_attn are then not written).
    pool_radius: if set, the attention-mass scores are max-pooled along the sequence
    (Solution 1, SnapKV form) before calibration, into buf.s_pool.
    t_solver: "bisect" (App. D.1) or "gd" (Alg. 1, Adam on log T) for the redundancy
    temperature.
    """

    def __init__(self, NS, Hq, Hkv, D, W, kv: PagedKV, alloc: Allocator, p: float,
                 L_dense: int = 0, L_sparse: int = 0, metric: str = "attn", n_ref: int = 0,
                 k_max: int = 0, keep_c: bool = True, pool_radius: int | None = None,
                 t_solver: str = "bisect", score_dtype=torch.bfloat16):
        if t_solver not in ("bisect", "gd"):
            raise ValueError("t_solver must be 'bisect' or 'gd'")
        self.t_solver = t_solver
        self.d = dims(NS, Hq, Hkv, D, W)
        self.kv, self.alloc, self.p = kv, alloc, p
        self.L_dense, self.L_sparse = L_dense, L_sparse
        self.metric, self.n_ref, self.k_max, self.keep_c = metric, n_ref, k_max, keep_c
        self.pool_radius = pool_radius
        self.sm_scale = 1.0 / math.sqrt(D)
        dev = kv.k_pool.device
        H = NS * Hkv
        S = kv.max_pages * 16
        self.n_heads, self.S_max = H, S
        f32, i32 = torch.float32, torch.int32
        red = metric == "attn+red"
        self.copy = ScoringCopy(NS, Hq, Hkv, D, W, kv, score_dtype) if isinstance(kv, PagedKV8) else None
        self.buf = CompressBuffers(
            s_attn=torch.empty(H, S, dtype=f32, device=dev),
            s_pool=torch.empty(H, S, dtype=f32, device=dev) if pool_radius is not None else None,
            x_red=torch.empty(H, S, dtype=f32, device=dev) if red else None,
            c=torch.empty(H, S, dtype=f32, device=dev),
            c_attn=torch.empty(H, S, dtype=f32, device=dev) if red else None,
            cand_len=torch.empty(H, dtype=i32, device=dev),
            row_lse=torch.empty(W, NS, Hq, dtype=f32, device=dev),
            sel_bits=torch.empty(H, S // 32, dtype=i32, device=dev),
            k=torch.empty(H, dtype=i32, device=dev),
            sel_mass=torch.empty(H, dtype=f32, device=dev),
            k_attn=torch.empty(H, dtype=i32, device=dev) if red else None,
            mass_attn=torch.empty(H, dtype=f32, device=dev) if red else None,
            T_red=None,
            status=torch.zeros(1, dtype=i32, device=dev),
            ws_score=workspace(OP_SCORE, self.d, kv.max_pages, dev) if self.copy is None else self.copy.ws,
            ws_compact=workspace(OP_COMPACT, self.d, kv.max_pages, dev),
            ws_select=select_workspace(H, S, dev),
        )

    def score(self, q_obs, ref_slots=None, row_lse_in=None, stream=None):
        b = self.buf
        if self.copy is not None:
            if ref_slots is not None:
                ref_slots = _shaped(ref_slots, (self.n_heads, self.n_ref), torch.int32, "ref_slots")
            if row_lse_in is not None:
                row_lse_in = _shaped(row_lse_in, tuple(b.row_lse.shape), torch.float32, "row_lse_in")
            for d, h0, H, sl, q, kv in self.copy.groups(q_obs, stream):
                heads, lse = slice(h0, h0 + H), self.copy.group_lse(sl)
                if row_lse_in is not None:
                    with torch.cuda.stream(stream):
                        lse.copy_(row_lse_in[:, sl])
                hk_score(d, q, kv, self.L_dense, self.sm_scale, b.s_attn[heads], b.cand_len[heads],
                         row_lse_in=lse if row_lse_in is not None else None,
                         row_lse_out=lse if row_lse_in is None else None,
                         ref_slots=ref_slots[heads] if ref_slots is not None else None,
                         n_ref=self.n_ref if ref_slots is not None else 0,
                         x_red=b.x_red[heads] if ref_slots is not None else None, ws=b.ws_score, stream=stream)
                if row_lse_in is None:
                    with torch.cuda.stream(stream):
                        b.row_lse[:, sl].copy_(lse)
            return
        hk_score(self.d, q_obs, self.kv, self.L_dense, self.sm_scale, b.s_attn, b.cand_len,
                 row_lse_in=row_lse_in, row_lse_out=b.row_lse if row_lse_in is None else None,
                 ref_slots=ref_slots, n_ref=self.n_ref if ref_slots is not None else 0,
                 x_red=b.x_red if ref_slots is not None else None, ws=b.ws_score, stream=stream)

    def select(self, stream=None):
        b, H, S, pm = self.buf, self.n_heads, self.S_max, self.kv.page_mask
        s_attn = b.s_attn
        if self.pool_radius is not None:
            hk_pool_max(H, S, b.cand_len, pm, b.s_attn, self.pool_radius, b.s_pool, stream=stream)
            s_attn = b.s_pool
        if self.metric == "attn":
            xs, Ts, ws = [s_attn], None, [1.0]
        else:
            if b.T_red is None:
                # temperature of the redundancy metric, solved at the first compression only
                hk_calibrate_topp_ws(H, S, b.cand_len, pm, [s_attn], None, [1.0], self.p,
                                     b.sel_bits, b.k_attn, b.ws_select,
                                     c_out=b.c_attn if self.keep_c else None,
                                     sel_mass=b.mass_attn, status=b.status, stream=stream)
                b.T_red = torch.empty(H, dtype=torch.float32, device=b.c.device)
                solve = hk_calibrate_solve_T_gd if self.t_solver == "gd" else hk_calibrate_solve_T
                solve(H, S, b.cand_len, pm, b.x_red, b.k_attn, b.mass_attn, b.T_red, stream=stream)
            xs, Ts, ws = [s_attn, b.x_red], [None, b.T_red], [0.5, 0.5]
        hk_calibrate_topp_ws(H, S, b.cand_len, pm, xs, Ts, ws, self.p, b.sel_bits, b.k,
                             b.ws_select, c_out=b.c if self.keep_c else None, k_max=self.k_max,
                             sel_mass=b.sel_mass, status=b.status, stream=stream)

    def compact(self, stream=None):
        b = self.buf
        _compact(self.d, self.kv, b.sel_bits, self.L_dense, self.L_sparse, self.alloc, b.status,
                 b.ws_compact, stream)

    def step(self, q_obs, ref_slots=None, row_lse_in=None, stream=None):
        self.score(q_obs, ref_slots=ref_slots, row_lse_in=row_lse_in, stream=stream)
        self.select(stream=stream)
        self.compact(stream=stream)


class BudgetCompressor:
    """One compression step under the hard budget (Sec. 3.1 Step 4 and the budget
    thresholds of Sec. 3.3.1) with Cautious Update voting (Sec. 3.1):

      budget state (keep / sparse loading / rewrite, and the cap L_upper leaves)
      -> row LSEs of the window -> every row's own probabilities -> per-row Top-p votes
      -> selection ranked by votes under the cap, sinks kept -> mode-driven rewrite.

    rank_by_c: break ties in the votes by the window's calibrated mean attention (adds the
    attention-mass pass and the calibration); otherwise by recency.  The per-row
    probabilities take n_heads * G * W * S_max * 4 bytes (buf["a_rows"]).  8-bit caches and score_dtype
    as for Compressor.
    """

    def __init__(self, NS, Hq, Hkv, D, W, kv: PagedKV, alloc: Allocator, p: float,
                 L_lower: int, L_upper: int, L_dense: int = 0, n_sink: int = 0,
                 rank_by_c: bool = False, score_dtype=torch.bfloat16):
        self.copy = ScoringCopy(NS, Hq, Hkv, D, W, kv, score_dtype) if isinstance(kv, PagedKV8) else None
        self.d = dims(NS, Hq, Hkv, D, W)
        self.kv, self.alloc, self.p = kv, alloc, p
        self.L_lower, self.L_upper, self.L_dense, self.n_sink = L_lower, L_upper, L_dense, n_sink
        self.rank_by_c = rank_by_c
        self.sm_scale = 1.0 / math.sqrt(D)
        dev = kv.k_pool.device
        H, S, R = NS * Hkv, kv.max_pages * 16, Hq // Hkv * W
        self.n_heads, self.S_max, self.R = H, S, R
        f32, i32 = torch.float32, torch.int32
        self.buf = dict(
            head_mode=torch.empty(H, dtype=i32, device=dev),
            k_cap=torch.empty(H, dtype=i32, device=dev),
            cand_len=torch.empty(H, dtype=i32, device=dev),
            row_lse=torch.empty(W, NS, Hq, dtype=f32, device=dev),
            s_attn=torch.empty(H, S, dtype=f32, device=dev) if rank_by_c else None,
            c=torch.empty(H, S, dtype=f32, device=dev) if rank_by_c else None,
            a_rows=torch.empty(H, R, S, dtype=f32, device=dev),
            votes=torch.empty(H, S, dtype=torch.int16, device=dev),
            row_sel=torch.empty(H, R, S // 32, dtype=i32, device=dev),
            sel_bits=torch.empty(H, S // 32, dtype=i32, device=dev),
            k=torch.empty(H, dtype=i32, device=dev),
            status=torch.zeros(1, dtype=i32, device=dev),
            ws_score=workspace(OP_SCORE, self.d, kv.max_pages, dev) if self.copy is None else self.copy.ws,
            ws_compact=workspace(OP_COMPACT, self.d, kv.max_pages, dev),
        )

    def _rows(self, q_obs, stream):
        """Row LSEs, scores where they are needed, and every row's probabilities."""
        b = self.buf
        if self.copy is None:
            hk_score(self.d, q_obs, self.kv, self.L_dense, self.sm_scale, b["s_attn"], b["cand_len"],
                     row_lse_out=b["row_lse"], ws=b["ws_score"], stream=stream)
            hk_score_rows(self.d, q_obs, self.kv, self.L_dense, self.sm_scale, b["row_lse"],
                          b["a_rows"], stream=stream)
            return
        for d, h0, H, sl, q, kv in self.copy.groups(q_obs, stream):
            heads, lse = slice(h0, h0 + H), self.copy.group_lse(sl)
            hk_score(d, q, kv, self.L_dense, self.sm_scale, b["s_attn"][heads] if self.rank_by_c else None,
                     b["cand_len"][heads], row_lse_out=lse, ws=b["ws_score"], stream=stream)
            hk_score_rows(d, q, kv, self.L_dense, self.sm_scale, lse, b["a_rows"][heads], stream=stream)
            with torch.cuda.stream(stream):
                b["row_lse"][:, sl].copy_(lse)

    def select(self, q_obs, stream=None):
        if self.copy is not None:
            self.copy.takes(q_obs)
        b, H, S, pm = self.buf, self.n_heads, self.S_max, self.kv.page_mask
        hk_budget_plan(self.d, self.kv, self.L_dense, self.L_lower, self.L_upper, b["head_mode"],
                       b["k_cap"], stream=stream)
        self._rows(q_obs, stream)
        hk_vote_topp(H, self.R, S, b["cand_len"], pm, b["a_rows"], self.p, b["votes"],
                     b["row_sel"], status=b["status"], stream=stream)
        if self.rank_by_c:
            hk_calibrate(H, S, b["cand_len"], pm, [b["s_attn"]], None, [1.0], b["c"], stream=stream)
        hk_budget_select(H, S, b["cand_len"], pm, b["sel_bits"], b["k"], votes=b["votes"],
                         c=b["c"], head_mode=b["head_mode"], k_cap=b["k_cap"],
                         n_sink=self.n_sink, stream=stream)

    def compact(self, stream=None):
        b = self.buf
        if self.copy is not None:
            hk_compact8(self.d, self.kv, b["sel_bits"], self.L_dense, 0, self.alloc, b["status"],
                        b["ws_compact"], head_mode=b["head_mode"], stream=stream)
            return
        hk_compact_modes(self.d, self.kv, b["sel_bits"], self.L_dense, b["head_mode"], self.alloc,
                         b["status"], b["ws_compact"], stream=stream)

    def step(self, q_obs, stream=None):
        self.select(q_obs, stream=stream)
        self.compact(stream=stream)


class OneToken:
    """hk_append_kv's place for 8-bit caches: a chunk of one token per sequence, reserved and written."""

    def __init__(self, NS, kv: PagedKV8, d, alloc: Allocator, status):
        dev = kv.k_pool.device
        self.kv, self.d, self.alloc, self.status, self.NS = kv, d, alloc, status, NS
        self.chunks = Chunks(torch.arange(NS + 1, dtype=torch.int32, device=dev), NS, 1)
        self.slot_map = torch.empty(NS * d.Hkv, dtype=torch.int64, device=dev)
        self.ws = workspace(OP_RESERVE, d, kv.max_pages, dev)

    def append(self, k_new, v_new, stream=None):
        hk_reserve_slots(self.d, self.kv, self.chunks, self.alloc, self.ws, slot_map=self.slot_map,
                         status=self.status, stream=stream)
        hk_write_kv8(self.d, self.kv, self.NS, self.slot_map, k_new, v_new, stream=stream)


class Decoder:
    """One decode step of one layer: append the step's K/V, then attend.  An 8-bit cache (PagedKV8)
    takes K, V and q in bf16 or fp32."""

    def __init__(self, NS, Hq, Hkv, D, kv: PagedKV, alloc: Allocator):
        self.d = dims(NS, Hq, Hkv, D, 0)
        self.kv, self.alloc = kv, alloc
        self.sm_scale = 1.0 / math.sqrt(D)
        dev = kv.k_pool.device
        self.bits8 = isinstance(kv, PagedKV8)
        self.ws = workspace(OP_DECODE8 if self.bits8 else OP_DECODE, self.d, kv.max_pages, dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        if self.bits8:
            self.one = OneToken(NS, kv, self.d, alloc, self.status)
        else:
            self.ws_app = workspace(OP_APPEND, self.d, kv.max_pages, dev)

    def append(self, k_new, v_new, stream=None):
        if self.bits8:
            self.one.append(k_new, v_new, stream=stream)
            return
        hk_append_kv(self.d, self.kv, k_new, v_new, self.alloc, self.status, self.ws_app,
                     stream=stream)

    def attend(self, q, o, lse, stream=None):
        run = hk_decode_attn8 if self.bits8 else hk_decode_attn
        run(self.d, q, self.kv, self.sm_scale, o, lse, self.ws, stream=stream)


class ChunkDecoder:
    """Steps of several new tokens per sequence (prompts in chunks, drafts, single tokens beside
    them) over a cache of `layers` layers of B sequences, layers one after the other.

    append(): slots for a batch of chunks in every layer, and their K and V rows into the pool;
    reserve() and write() are its halves, for K and V that come layer by layer.
    attend(): one layer's causal attention of the chunks.
    trim(): the newest n_drop[s] tokens of every sequence taken back, in every layer.
    The buffers serve any chunks of at most max_tokens rows and max_len tokens a sequence.
    status collects FLAG_NOSPACE / FLAG_CHUNK: such a reserve() gave no slots (see hardkv.h).
    granted says on the device whether the last reserve() gave them; its chunks carry the word on to
    the Verifier, which drops nothing of refused chunks (one Chunks reserved by several decoders carries
    the last one's word: give each its own).  trim() itself always takes n_drop back.
    An 8-bit cache (PagedKV8) takes K, V, q and o in bf16 or fp32; write() quantises.
    """

    def __init__(self, B, Hq, Hkv, D, kv: PagedKV, alloc: Allocator, max_tokens: int, max_len: int,
                 layers: int = 1):
        self.B, self.layers, self.max_tokens, self.max_len = B, layers, max_tokens, max_len
        self.d_all, self.d = dims(layers * B, Hq, Hkv, D), dims(B, Hq, Hkv, D)
        self.kv, self.alloc = kv, alloc
        self.kv_layer = [kv.rows(l * B * Hkv, B * Hkv) for l in range(layers)] if layers > 1 else [kv]
        self.sm_scale = 1.0 / math.sqrt(D)
        dev = kv.k_pool.device
        self.ws_slots = workspace(OP_RESERVE, self.d_all, kv.max_pages, dev)
        self.ws_trim = workspace(OP_TRIM, self.d_all, kv.max_pages, dev)
        most = Chunks(torch.empty(B + 1, dtype=torch.int32), max_tokens, max_len)
        self.bits8 = isinstance(kv, PagedKV8)
        ws = chunk_attn8_workspace if self.bits8 else chunk_attn_workspace
        self.ws = ws(self.d, most, kv.max_pages, dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.granted = torch.ones(1, dtype=torch.int32, device=dev)

    def _fits(self, chunks: Chunks):
        if chunks.n_seq != self.B or chunks.n_tokens > self.max_tokens or chunks.max_len > self.max_len:
            raise HardKVError("the chunks are larger than the decoder was made for")

    def reserve(self, chunks: Chunks, slot_map, stream=None):
        """slot_map: [layers, n_tokens, Hkv] int64, written in full."""
        self._fits(chunks)
        chunks.granted_by(self.granted)
        hk_reserve_slots(self.d_all, self.kv, chunks, self.alloc, self.ws_slots, slot_map=slot_map,
                         status=self.status, stream=stream)

    def write(self, chunks: Chunks, slot_map, k_new, v_new, stream=None):
        """One layer ([tokens, Hkv, D], that layer's part of the slot map) or all of them
        ([layers, tokens, Hkv, D])."""
        run = hk_write_kv8 if self.bits8 else hk_write_kv
        run(self.d, self.kv, chunks.n_tokens, slot_map, k_new, v_new, stream=stream)

    def append(self, chunks: Chunks, k_new, v_new, slot_map, stream=None):
        self.reserve(chunks, slot_map, stream=stream)
        self.write(chunks, slot_map, k_new, v_new, stream=stream)

    def attend(self, chunks: Chunks, q, o, lse=None, layer: int = 0, stream=None):
        self._fits(chunks)
        run = hk_chunk_attn8 if self.bits8 else hk_chunk_attn
        run(self.d, self.kv_layer[layer], chunks, q, self.sm_scale, o, self.ws, lse=lse, stream=stream)

    def trim(self, n_drop, stream=None):
        if n_drop.numel() != self.B:
            raise HardKVError("n_drop must have one entry per sequence")
        hk_trim_slots(self.d_all, self.kv, n_drop, self.alloc, self.ws_trim, stream=stream)


class Verifier:
    """Drafted tokens of up to B sequences against the target's probabilities over V tokens."""

    def __init__(self, B: int, V: int, device):
        self.B, self.V = B, V
        self.ws = verify_workspace(B, V, device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def verify(self, chunks: Chunks, tokens, p, u, n_accept, next_token, n_drop, q=None, stream=None):
        if chunks.n_seq > self.B:
            raise HardKVError("more sequences than the verifier was made for")
        hk_verify_draft(chunks, self.V, tokens, p, u, n_accept, next_token, n_drop, self.ws, q=q,
                        status=self.status, stream=stream)


class DecodeLoop:
    """End-to-end decode loop over L independent attention layers sharing one page pool
    and one allocator (config-5 style).

    step():     append this step's K/V for every layer (Step 1, dense tier), then one paged
                decode-attention launch per layer, writing o and the row LSE.
    compress(): Steps 2-3 over every layer at once, with the window queries and the decode
                step's own LSEs (single-pass score).
    With max_tokens (and max_len) it also takes several new tokens per sequence at once:
    extend():   prompts in chunks, or the last token and its drafts: slots and K/V for every
                layer, then one chunk attention per layer;
    accept():   drafts against the target's probabilities, the rejected ones taken back in
                every layer.  After an extend() whose slots were refused (status) it takes
                nothing back and draws no token (-1): the cache stays as it was.
    Heads are ordered (layer, sequence, KV head); sequence index = layer * B + b.
    An 8-bit cache (PagedKV8) takes queries, K and V in bf16 or fp32, and o of extend() in the queries'
    type; compress() takes window queries as Compressor does (fp32 ones: score_dtype=torch.float32).
    """

    def __init__(self, L, B, Hq, Hkv, D, W, kv: PagedKV, alloc: Allocator, p: float,
                 L_dense: int, L_sparse: int = 0, keep_c: bool = True, max_tokens: int = 0,
                 max_len: int = 0, score_dtype=torch.bfloat16):
        self.L, self.B, self.Hq, self.Hkv, self.D, self.W = L, B, Hq, Hkv, D, W
        self.kv, self.alloc = kv, alloc
        self.NS = L * B
        dev = kv.k_pool.device
        self.d_all = dims(self.NS, Hq, Hkv, D, W)
        self.d_layer = dims(B, Hq, Hkv, D, W)
        self.layers = [kv.rows(l * B * Hkv, B * Hkv) for l in range(L)]
        self.sm_scale = 1.0 / math.sqrt(D)
        self.bits8 = isinstance(kv, PagedKV8)
        self.ws_dec = workspace(OP_DECODE8 if self.bits8 else OP_DECODE, self.d_layer, kv.max_pages, dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        if self.bits8:
            self.one = OneToken(self.NS, kv, self.d_all, alloc, self.status)
        else:
            self.ws_app = workspace(OP_APPEND, self.d_all, kv.max_pages, dev)
        self.o = torch.empty(self.NS, Hq, D, dtype=torch.float32, device=dev)
        self.comp = Compressor(self.NS, Hq, Hkv, D, W, kv, alloc, p, L_dense=L_dense,
                               L_sparse=L_sparse, metric="attn", keep_c=keep_c, score_dtype=score_dtype)
        self.chunked = None
        if max_tokens > 0:
            self.chunked = ChunkDecoder(B, Hq, Hkv, D, kv, alloc, max_tokens, max_len or max_tokens, layers=L)
            self.chunked.status = self.status
            self.slot_map = torch.empty(L * max_tokens * Hkv, dtype=torch.int64, device=dev)

    def extend(self, chunks, q, k, v, o, lse, stream=None):
        """q [L, tokens, Hq, D], k and v [L, tokens, Hkv, D] (views with contiguous heads will do),
        o [L, tokens, Hq, D] in the cache's type, lse [L, tokens, Hq] fp32."""
        if self.chunked is None:
            raise HardKVError("the loop was made without max_tokens")
        ch, n = self.chunked, self.L * chunks.n_tokens * self.Hkv
        ch.append(chunks, k, v, self.slot_map[:n], stream=stream)
        for l in range(self.L):
            ch.attend(chunks, q[l], o[l], lse[l], layer=l, stream=stream)

    def accept(self, verifier: Verifier, chunks, tokens, p, u, n_accept, next_token, n_drop, q=None,
               stream=None):
        if self.chunked is None:
            raise HardKVError("the loop was made without max_tokens")
        chunks.granted_by(self.chunked.granted)
        verifier.verify(chunks, tokens, p, u, n_accept, next_token, n_drop, q=q, stream=stream)
        self.chunked.trim(n_drop, stream=stream)

    def step(self, q_t, k_t, v_t, lse_t, stream=None):
        if self.bits8:
            self.one.append(k_t, v_t, stream=stream)
        else:
            hk_append_kv(self.d_all, self.kv, k_t, v_t, self.alloc, self.status, self.ws_app,
                         stream=stream)
        B, attend = self.B, hk_decode_attn8 if self.bits8 else hk_decode_attn
        for l, kv_l in enumerate(self.layers):
            attend(self.d_layer, q_t[l * B:(l + 1) * B], kv_l, self.sm_scale,
                   self.o[l * B:(l + 1) * B], lse_t[l * B:(l + 1) * B], self.ws_dec,
                   stream=stream)

    def compress(self, q_win, lse_win, stream=None):
        self.comp.step(q_win, row_lse_in=lse_win, stream=stream)

    def segment(self, q_seg, k_seg, v_seg, lse_seg, stream=None):
        """len(q_seg) decode steps, then one compression over the last W steps' queries
        and their decode LSEs (Sec. 3.1 Steps 1-3)."""
        if self.bits8:
            self.comp.copy.takes(q_seg)
        T = q_seg.shape[0]
        for t in range(T):
            self.step(q_seg[t], k_seg[t], v_seg[t], lse_seg[t], stream=stream)
        self.compress(q_seg[T - self.W:], lse_seg[T - self.W:], stream=stream)

    def capture_segment(self, q_seg, k_seg, v_seg, lse_seg):
        """Record one segment into a HIP graph (torch.cuda.CUDAGraph).  The graph keeps the
        buffers' addresses: refill q_seg / k_seg / v_seg in place and replay it.  Every step
        of a segment is a kernel launch on the capture stream with device-side metadata
        updates (no host synchronisation, no allocation, no memset), so one graph serves
        every segment.  Nothing runs at capture time."""
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.segment(q_seg, k_seg, v_seg, lse_seg)
        return g
