// 8-bit cache: attention of long chunks, bf16 queries (gfx950).
//
// A unit is TILE8_ROWS folded rows (see hk_attn8.hip) of a sequence and KV head: four waves of 32 rows
// against the same keys, 32 at a time.  The codes of a tile are converted once for all waves, by all of
// them, and lie in LDS as bf16: K by rows, V by dims, in the order of keys that the scores' registers
// have, so that both kinds of fragment are 16 bytes in a row.  While two tiles are computed, the next two are
// converted into the other buffers and two more are on their way into registers.  One tile a barrier took 1673
// us where two take 1575; converting between the two computations 1660 to 1720.
//
// Per wave and tile, 32x32x16 MFMAs: C[key][row] = K Q^T in bf16, then O^T[dim][row] += V^T P^T in fp16,
// which holds V's codes exactly and P to 2^-11 of a term.  Lane l holds row l % 32 and half hi = l / 32 of the
// contraction; register r of a score tile is key (r & 3) + 8 (r >> 2) + 4 hi.
//
// For P to be in fp16's range whatever V's scales are, the reference m follows what enters the product: with
// V's scale s = f 2^e, f in [1/2, 1), and y = x + e, P = exp2(y - m) f 2^10 is at most 2^14, and smaller terms
// keep their bits down to 2^-24 of the largest.  The softmax's sum takes exp2(y - m) 2^-e.  e is counted
// from that of the unit's first keys, so that y is about x; of scales below 2^-90 it counts as 0 (their V is
// below 2^-81, next to nothing).  Against P in two parts of bf16, 24 products a tile instead of 16: 1930 us and
// 1673.
//
// Measured: 8 prompts of 4096 tokens of 32 query heads, 8 KV heads of 128 dims, causal, 1570 to 1625
// us, 677 to 700 TFLOP/s; a bf16 matrix product of 8192^3 reaches 1236.  The matrix units work 29% of the
// cycles and the vector units 53%, 13.6 vector instructions a product of 32 cycles: conversions, scales,
// softmax.  A wave waits 33% of its time, and 231 registers leave no room for a third a SIMD.
#include "hk_attn8.h"

namespace hk {

constexpr int TILE8_ROWS = 128;

template <int F, int D>
__global__ __launch_bounds__(A8_NT, 2) void attn8_tile_kernel(Args8 a) {
#pragma clang fp contract(off)
  constexpr int KS = D / 16, DT = D / 32;
  constexpr int K_ROW = 2 * D + 16, V_ROW = 80;               // bytes; padded: no bank twice among 16 lanes
  constexpr int KW = D / 16;                                  // words of codes of a thread that brings K
  constexpr int K_TILE = 32 * K_ROW, TILE = K_TILE + D * V_ROW;
  constexpr int NT = 4;                                       // tiles in LDS: two computed, two converted
  __shared__ __align__(16) char s_tile[NT][TILE];
  __shared__ __align__(16) float s_scale[NT][4][32];          // K's scales times c2; V's: e, f 2^10, 2^-e
  __shared__ int s_base;                                      // what e is counted from
  __shared__ int s_odd[NT];                                   // whether an f is NaN or infinite
  __shared__ int s_sums[A8_NW];
  const int lane = threadIdx.x & 63, row32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool is_v = wave >= 2;
  // Waves 0 and 1 bring a page of K each, 2 and 3 one of V.  A thread has of K a quarter of row lane / 4, of V
  // dims 4 c .. 4 c + 3 of the eight keys 4 (lane % 2) + {0 .. 3, 8 .. 11}, c = lane / 2 (D 64: c below 16).
  const int my = wave & 1, part4 = lane & 3, c = lane >> 1;
  const bool brings = !is_v || c < D / 4;
  const uint32_t from = is_v ? (lane & 1) * 4 * D + 4 * c : (lane >> 2) * D + part4 * (D / 4);
  const int to = is_v ? K_TILE + 4 * c * V_ROW + (2 * my + (lane & 1)) * 16
                      : (16 * my + (lane >> 2)) * K_ROW + part4 * (D / 2);

  int u = a.n_units - 1 - (int)blockIdx.x, skip = 0, left = 1 << 30;
  if (a.first) {
    static_assert(sizeof(s_tile) >= (A8_UNITS + 1) * sizeof(int));
    const Run r = run_of_group<TILE8_ROWS, true>(a, reinterpret_cast<int*>(s_tile), s_sums);
    u = r.unit;
    skip = r.skip;
    left = r.left;
  }
  for (; left > 0 && u < a.n_units; ++u) {
    const Unit w = unit_of<TILE8_ROWS, true>(a, u);
    if (w.rows == 0) {
      if (!a.first) return;
      continue;
    }
    const int steps = steps_of(w), take = min(steps - skip, left);
    const int p0 = skip * A8_STEP, p1 = min(p0 + take * A8_STEP, w.pages);
    const int64_t state = take == steps ? -1 : (int64_t)(2 * blockIdx.x + (skip == 0)) * a.cap;
    left = a.first ? left - take : 0;
    skip = 0;
    const int32_t* trow = a.table + (size_t)w.h * a.max_pages;
    const uint16_t* mrow = a.masks + (size_t)w.h * a.max_pages;

    // rows past the chunk repeat its last one; they are not stored
    const int w0 = w.r0 + wave * 32, r = min(w0 + row32, w.rows - 1), tok = r / a.G, g = r - tok * a.G;
    const int seen = w.off + tok;                             // keys before this one are seen by the lane's row,
    const int seen_all = w.off + min(w0, w.rows - 1) / a.G;   // by every row of the wave,
    const int seen_any = w.off + (min(w0 + 32, w.rows) - 1) / a.G;   // by any of them
    bf16x8 qf[KS];
    {
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)(w.c.first + tok) * a.q_row + (w.kv * a.G + g) * D;
#pragma unroll
      for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(q + 16 * s + 8 * hi));
      // (waited for here, or every tile's first product would wait for all loads, those of the tiles to come too)
#pragma unroll
      for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s]));
    }
    float m = -INFINITY, off = 0.f, l = 0.f;                  // off: m, or 0 while there is none
    f32x16 acc[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;

    // Ids and masks come 32 tiles at a time: lane i holds those of page i % 2 of tile i / 2.
    const int tiles = p1 > p0 ? (p1 - p0 + 1) / 2 : 0;
    int ids = 0, masks = 0;
    uint32_t code[2][8];                                      // of two tiles; K: KW words; V: word of eight keys
    float scale[2] = {0.f, 0.f};
    int base = 0;
    uint32_t mask[2] = {0, 0}, next_mask[2] = {0, 0};         // of the tiles computed, and of those converted
    auto load = [&](int x, int i) {                           // (past the last tile: its pages again)
      if ((i & 31) == 0) {
        const int page = p0 + 2 * i + lane;
        ids = min(max(trow[min(page, p1 - 1)], 0), a.num_pages - 1);
        masks = page < p1 ? mrow[page] : 0;
      }
      const int e = 2 * (i & 31);
      const int id0 = __builtin_amdgcn_readlane(ids, e), id1 = __builtin_amdgcn_readlane(ids, e + 1);
      next_mask[x] = (uint32_t)__builtin_amdgcn_readlane(masks, e) | (uint32_t)__builtin_amdgcn_readlane(masks, e + 1) << 16;
      const char* page = (is_v ? a.v_pool : a.k_pool) + (size_t)(uint32_t)(my ? id1 : id0) * (HK_PAGE * D);
      if (!is_v) {
#pragma unroll
        for (int k = 0; k < KW / 4; ++k)
          *reinterpret_cast<u32x4*>(&code[x][4 * k]) = *reinterpret_cast<const u32x4*>(page + from + 16 * k);
      } else if (brings) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          code[x][j] = *reinterpret_cast<const uint32_t*>(page + from + (8 * (j >> 2) + (j & 3)) * D);
      }
      if (wave == 0) {
        const int id = (lane >> 4) & 1 ? id1 : id0;
        scale[x] = (lane >> 5 ? a.v_scale : a.k_scale)[(size_t)(uint32_t)id * HK_PAGE + (lane & 15)];
      }
    };
    auto convert = [&](int which, int buf, uint32_t mk) {
      if (!is_v) {
        char* at = s_tile[buf] + to;
#pragma unroll
        for (int k = 0; k < KW / 2; ++k)
          *reinterpret_cast<u32x4*>(at + 16 * k) =
              u32x4{Code<F>::template pair<0>(code[which][2 * k]), Code<F>::template pair<1>(code[which][2 * k]),
                    Code<F>::template pair<0>(code[which][2 * k + 1]), Code<F>::template pair<1>(code[which][2 * k + 1])};
      } else if (brings) {
        if (F == HK_E4M3 && mk != 0xffffffffu) {
          // a slot that is not valid may hold codes that stand for NaN
          const uint32_t bits = mk >> (16 * my + 4 * (lane & 1));
#pragma unroll
          for (int j = 0; j < 8; ++j) code[which][j] = (bits >> (8 * (j >> 2) + (j & 3))) & 1u ? code[which][j] : 0u;
        }
        char* at = s_tile[buf] + to;
        u32x4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[0][k] = Code<F>::template halves<0>(code[which][2 * k], code[which][2 * k + 1]);
          x[1][k] = Code<F>::template halves<1>(code[which][2 * k], code[which][2 * k + 1]);
          x[2][k] = Code<F>::template halves<2>(code[which][2 * k], code[which][2 * k + 1]);
          x[3][k] = Code<F>::template halves<3>(code[which][2 * k], code[which][2 * k + 1]);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) *reinterpret_cast<u32x4*>(at + d * V_ROW) = x[d];
      }
      if (wave == 0) {
        const int top = __builtin_amdgcn_frexp_expf(scale[which]), e = top < -90 ? 0 : min(max(top - base, -126), 126);
        const float f = __builtin_amdgcn_ldexpf(scale[which], 10 - (e + base));
        if (lane < 32) {
          s_scale[buf][0][lane] = scale[which] * a.c2;
        } else {
          s_scale[buf][1][lane - 32] = (float)e;
          s_scale[buf][2][lane - 32] = f;
          s_scale[buf][3][lane - 32] = __builtin_amdgcn_ldexpf(1.f, -e);
        }
        const bool odd = __any(lane >= 32 && !(fabsf(f) < INFINITY));
        if (lane == 0) s_odd[buf] = odd;
      }
    };
    auto compute = [&](int buf, int key, uint32_t valid, bool full) {
      f32x16 z = {};
      const char* k = s_tile[buf] + row32 * K_ROW + hi * 16;
#pragma unroll
      for (int s = 0; s < KS; ++s)
        z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(k + 32 * s)),
                                                    qf[s], z, 0, 0, 0);
      const float* sc = s_scale[buf][0] + 4 * hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 ks = *reinterpret_cast<const f32x4*>(sc + 8 * i), ev = *reinterpret_cast<const f32x4*>(sc + 32 + 8 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[4 * i + j] = fmaf(z[4 * i + j], ks[j], ev[j]);
      }
      const int n = seen - key;
      uint32_t vis = (valid & (n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u)) >> (4 * hi);
      if (!full) {
        asm volatile("" : "+v"(vis));         // (a branch, not selects in every tile)
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = (vis >> ((e & 3) + 8 * (e >> 2))) & 1u ? z[e] : -INFINITY;
      }
      float zm = z[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) zm = fmaxf(zm, z[e]);
      if (__builtin_expect(__any(zm > m + A8_SLACK), 0)) {
        zm = fmaxf(zm, __shfl_xor(zm, 32, 64));
        const float mn = fmaxf(m, ceilf(zm));
        const float alpha = m == -INFINITY ? 0.f : fast_exp2(m - mn);
        m = mn;
        off = mn == -INFINITY ? 0.f : mn;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
      }
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 f = *reinterpret_cast<const f32x4*>(sc + 64 + 8 * i), up = *reinterpret_cast<const f32x4*>(sc + 96 + 8 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = fast_exp2(z[4 * i + j] - off);
          sum[j & 1] = fmaf(p, up[j], sum[j & 1]);
          z[4 * i + j] = p * f[j];
        }
      }
      l += sum[0] + sum[1];
      if (!full && s_odd[buf]) {
        // a probability of 0 times a scale of NaN, or of a slot that holds anything
        asm volatile("" : "+v"(vis));
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = (vis >> ((e & 3) + 8 * (e >> 2))) & 1u ? z[e] : 0.f;
      }
      u32x4 pf[2];                                            // halves of the keys
#pragma unroll
      for (int e = 0; e < 8; ++e)
        pf[e >> 2][e & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{z[2 * e], z[2 * e + 1]}), f16x2));
      const char* v = s_tile[buf] + K_TILE + row32 * V_ROW + hi * 16;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const f16x8 vf = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(v + 32 * d * V_ROW + 32 * s));
          acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, __builtin_bit_cast(f16x8, pf[s]), acc[d], 0, 0, 0);
        }
    };

    if (tiles > 0) {
      load(0, 0);
      if (tiles > 1) load(1, 1);
      if (wave == 0) {
        const int e = lane >= 32 && (next_mask[0] >> (lane - 32)) & 1u ? __builtin_amdgcn_frexp_expf(scale[0]) : -1000;
        base = (int)wave_max((float)e);
        if (base < -90) base = 0;
        if (lane == 0) s_base = base;
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (x < tiles) convert(x, x, next_mask[x]);
        mask[x] = next_mask[x];
      }
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (2 + x < tiles) load(x, 2 + x);
      __syncthreads();
      base = s_base;
    }
    for (int i = 0; i < tiles; i += 2) {
      const int buf = i & 2;
      const uint32_t mk[2] = {next_mask[0], next_mask[1]};
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (i + 2 + x < tiles) convert(x, (buf ^ 2) + x, mk[x]);
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (i + 4 + x < tiles) load(x, i + 4 + x);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int key = (p0 + 2 * (i + x)) * HK_PAGE;
        if (i + x < tiles && key < seen_any && w0 < w.rows)
          compute(buf + x, key, mask[x], mask[x] == 0xffffffffu && key + 32 <= seen_all);
        mask[x] = mk[x];
      }
      __syncthreads();
    }

    l += __shfl_xor(l, 32, 64);
    if (w0 + row32 < w.rows) {
      // l is brought to [1/2, 1): scales far apart leave sums far apart
      const int up = __builtin_amdgcn_frexp_expf(l), down = base + Code<F>::F16_DOWN - 10 - up;
      l = __builtin_amdgcn_frexp_mantf(l);
      m = off + (float)up;                                    // (NaN keys alone leave a sum of NaN and no reference)
      const float inv = l == 0.f ? 0.f : 1.f / l;             // (a NaN stays one)
      const int64_t at = (int64_t)(w.c.first + tok) * a.Hq + w.kv * a.G + g, part = state + wave * 32 + row32;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int dim = 32 * d + 8 * j + 4 * hi;
          float x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) x[k] = __builtin_amdgcn_ldexpf(acc[d][4 * j + k] * inv, down);
          if (state >= 0) *reinterpret_cast<f32x4*>(a.part_o + part * D + dim) = f32x4{x[0], x[1], x[2], x[3]};
          else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + at * D + dim) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
        }
      if (hi == 0) {
        if (state >= 0) *reinterpret_cast<f32x2*>(a.part_ml + part * 2) = f32x2{l == 0.f ? -INFINITY : m, l};
        else if (a.lse) a.lse[at] = lse8(m, l);
      }
    }
  }
}

}  // namespace hk

using namespace hk;

int64_t hk_attn8_tile_units(int NS, int Hkv, int G, int n_tokens) {
  return ((int64_t)n_tokens * G / TILE8_ROWS + NS) * Hkv;
}
size_t hk_attn8_tile_ws(int D) { return states8_bytes(D, TILE8_ROWS); }

template <int F, int D>
static void launch_tile(const Args8& a, hipStream_t st) {
  const uint32_t groups = a.first ? A8_GROUPS<D> : (uint32_t)a.n_units;
  {
    TimedLaunch t(HK_TK_ATTN8, st);
    hipLaunchKernelGGL((attn8_tile_kernel<F, D>), dim3(groups), dim3(A8_NT), 0, st, a);
  }
  if (a.first && a.max_pages > A8_STEP) merge8<D, TILE8_ROWS, 2, true>(a, groups, st);
}

void hk_launch_attn8_tile(Args8 a, hk_dtype format, int D, void* ws, hipStream_t st) {
  const int64_t units = hk_attn8_tile_units(a.n_seq, a.Hkv, a.G, a.n_tokens);
  a.n_units = (int)units;
  a.cap = TILE8_ROWS;
  a.one_tile = 0;
  a.rows_from = A8_ROWS + 1;
  a.rows_to = INT32_MAX;
  carve8(a, planned8(units, true, a.max_pages), D, ws);
  if (format == HK_I8) D == 128 ? launch_tile<HK_I8, 128>(a, st) : launch_tile<HK_I8, 64>(a, st);
  else D == 128 ? launch_tile<HK_E4M3, 128>(a, st) : launch_tile<HK_E4M3, 64>(a, st);
}
