// 8-bit cache: attention of long chunks, bf16 queries (gfx950).
//
// A unit is TILE8_ROWS folded rows (see hk_attn8.hip) of a sequence and KV head: four waves of 32 rows
// against the same keys, 32 at a time.  The codes of a tile lie in LDS as bf16 (K, by rows) and fp16 (V, by dims,
// in the order of keys that the scores' registers have), so that both kinds of fragment are 16 bytes in a row.
// They are converted by all waves for all of them: while two tiles are computed, the next two are converted into
// the other buffers and two more are on their way into registers.  Or, for long chunks (READY), a launch
// before has converted every tile of a head once, and it goes from memory straight into LDS.
//
// Per wave and tile, 32x32x16 MFMAs: C[key][row] = K Q^T in bf16, then O^T[dim][row] += V^T P^T in fp16,
// which holds V's codes exactly and P to 2^-11 of a term.  Lane l holds row l % 32 and half hi = l / 32 of the
// contraction; register r of a score tile is key (r & 3) + 8 (r >> 2) + 4 hi.
//
// For P to be in fp16's range whatever V's scales are, the reference m follows what enters the product: with
// V's scale s = f 2^e, f in [1/2, 1), and y = x + e, P = exp2(y - m) f 2^10 is at most 2^14, and smaller terms
// keep their bits down to 2^-24 of the largest.  The softmax's sum takes exp2(y - m) 2^-e.  e is counted
// from that of the unit's first keys (READY: the head's), so that y is about x; of scales below 2^-90 it counts as 0
// (their V is below 2^-81, next to nothing).  Where a valid key has an e past FAR8 in size, that sum could leave the
// range, or lose keys whose V is small: 2^-e is NaN there, and a unit that finds its sum to be NaN is computed again
// with a reference of the sum's own, which follows x (a check in every tile instead: 1435 to 1495 us for 1400 to
// 1460 of the prompts below).
//
// Measured on 8 prompts of 4096 tokens of 32 query heads, 8 KV heads of 128 dims, causal: 1390 to 1510 us, 728 to
// 791 TFLOP/s, of which the conversion is 38; 1570 to 1625 with every unit converting its tiles, and 1136 without
// conversions and loads at all.  A bf16 matrix product of 8192^3 reaches 1236 TFLOP/s.  What bounds it is vector
// work beside MFMA: the matrix units are busy for 34% of the cycles and the vector units for 51% (28 and 52 with
// every unit converting), waves wait for 34% of theirs, at two a SIMD.  P in two parts of bf16, 24 products a tile
// instead of 16: 1930 us for 1673; one tile a barrier 1673 for 1575; converting between the computations of two
// tiles 1660 to 1720; two tiles in one softmax spill (1767); 64 rows a wave, at one wave a SIMD, 2745; eight waves
// of 256 rows 1629 to 1675.
#include <type_traits>

#include "hk_attn8.h"

namespace hk {

constexpr int TILE8_ROWS = 128;
// Where every e is within it, a key of 2^-58 and more of the sum is in the range of exp2(y - m): y is at least
// m - SLACK - 2 FAR8 - 58.
constexpr int FAR8 = 32;

// A converted tile: K by rows and V by dims, whose 16-byte pieces lie in turned orders so that 16 lanes of
// a fragment's read meet no bank twice; K's scales times c2, V's e, f 2^10 and 2^-e; `odd` and what e is counted from.
template <int D>
struct Ready8 {
  static constexpr int V = 64 * D, SCALES = 2 * V, ODD = SCALES + 512, BASE = ODD + 4, BYTES = SCALES + 1024;
  __device__ static __forceinline__ int k_at(int row, int piece) {
    return row * 2 * D + (piece ^ (D == 128 ? row & 15 : row >> 1 & 7)) * 16;
  }
  // rows of one dim % 4 lie side by side
  __device__ static __forceinline__ int v_at(int dim, int piece) {
    return V + ((dim & 3) * (D / 4) + (dim >> 2)) * 64 + ((piece ^ dim ^ (dim >> 2 & 2)) & 3) * 16;
  }
};
// V's scale as e, f 2^10 (see above)
__device__ __forceinline__ int v_exponent(float scale, int base) {
  const int top = __builtin_amdgcn_frexp_expf(scale);
  return top < -90 ? 0 : top - base;
}
// 2^-e of key i, NaN past FAR8; of a slot that is not valid, whose scale may be anything, in range: its p is 0
__device__ __forceinline__ float v_back(int e, int i, uint32_t mask) {
  float back = __builtin_amdgcn_ldexpf(1.f, -e);
  if (__builtin_expect(__any(fabsf((float)e) > FAR8), 0) && abs(e) > FAR8) back = (mask >> i) & 1u ? __builtin_nanf("") : 1.f;
  return back;
}
// of 32 keys, in lanes 32 .. 63
__device__ __forceinline__ int v_base(float scale, uint32_t mask) {
  const int lane = threadIdx.x & 63;
  const int e = lane >= 32 && (mask >> (lane - 32)) & 1u ? __builtin_amdgcn_frexp_expf(scale) : -1000;
  const int base = (int)wave_max((float)e);
  return base < -90 ? 0 : base;
}

// A tile a workgroup, of the heads whose chunks the tile kernel takes.
template <int F, int D>
__global__ __launch_bounds__(A8_NT) void attn8_convert_kernel(Args8 a) {
  using L = Ready8<D>;
  const int per = a.max_pages / 2, h = blockIdx.x / per, t = blockIdx.x - h * per;
  const int len = chunk_of(a.start, h / a.Hkv, a.n_tokens, a.max_len).len, n = min(max(a.n_pages[h], 0), a.max_pages);
  if (len * a.G < a.rows_from || 2 * t >= n) return;
  const int32_t* trow = a.table + (size_t)h * a.max_pages;
  const uint16_t* mrow = a.masks + (size_t)h * a.max_pages;
  const auto page = [&](int p) { return min(max(trow[min(p, n - 1)], 0), a.num_pages - 1); };
  const auto valid = [&](int p) { return p < n ? (uint32_t)mrow[p] : 0u; };
  const int id[2] = {page(2 * t), page(2 * t + 1)};
  const uint32_t mask = valid(2 * t) | valid(2 * t + 1) << 16;
  char* to = a.ready + (size_t)blockIdx.x * L::BYTES;
  const int i = threadIdx.x;
  if (i < 2 * D) {
    const int key = i / (D / 16), piece = i % (D / 16);
    const u32x4 w = *reinterpret_cast<const u32x4*>(a.k_pool + ((size_t)(uint32_t)id[key >> 4] * HK_PAGE + (key & 15)) * D + piece * 16);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      *reinterpret_cast<u32x4*>(to + L::k_at(key, 2 * piece + k)) =
          u32x4{Code<F>::template pair<0>(w[2 * k]), Code<F>::template pair<1>(w[2 * k]),
                Code<F>::template pair<0>(w[2 * k + 1]), Code<F>::template pair<1>(w[2 * k + 1])};
  }
  if (i < D) {
    // dims 4 c .. of the eight keys of piece p: 16 (p / 2) + 4 (p % 2) + {0 .. 3, 8 .. 11}
    const int c = i >> 2, p = i & 3, first = 4 * (p & 1);
    const char* from = a.v_pool + ((size_t)(uint32_t)id[p >> 1] * HK_PAGE + first) * D + 4 * c;
    const uint32_t bits = mask >> (16 * (p >> 1) + first);
    uint32_t code[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int key = 8 * (j >> 2) + (j & 3);
      code[j] = *reinterpret_cast<const uint32_t*>(from + key * D);
      // a slot that is not valid may hold codes that stand for NaN
      if (F == HK_E4M3) code[j] = (bits >> key) & 1u ? code[j] : 0u;
    }
    u32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[0][k] = Code<F>::template halves<0>(code[2 * k], code[2 * k + 1]);
      x[1][k] = Code<F>::template halves<1>(code[2 * k], code[2 * k + 1]);
      x[2][k] = Code<F>::template halves<2>(code[2 * k], code[2 * k + 1]);
      x[3][k] = Code<F>::template halves<3>(code[2 * k], code[2 * k + 1]);
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) *reinterpret_cast<u32x4*>(to + L::v_at(4 * c + d, p)) = x[d];
  }
  if (i >= A8_NT - 64) {
    const int lane = i & 63, slot = lane & 15;
    const bool second = lane & 16;
    const size_t begin = (size_t)(uint32_t)(second ? page(1) : page(0)) * HK_PAGE + slot;
    const int base = v_base(a.v_scale[begin], valid(0) | valid(1) << 16);
    const float scale = (lane >> 5 ? a.v_scale : a.k_scale)[(size_t)(uint32_t)id[second] * HK_PAGE + slot];
    const int e = v_exponent(scale, base);
    const float f = __builtin_amdgcn_ldexpf(scale, 10 - (e + base));
    float* out = reinterpret_cast<float*>(to + L::SCALES) + (lane & 31);
    if (lane < 32) {
      out[0] = scale * a.c2;
    } else {
      out[32] = (float)e;
      out[64] = f;
      out[96] = v_back(e, lane & 31, mask);
    }
    const bool odd = __any(lane >= 32 && !(fabsf(f) < INFINITY));
    if (lane == 0) *reinterpret_cast<u32x2*>(to + L::ODD) = u32x2{odd ? 1u : 0u, (uint32_t)base};
  }
}

template <int F, int D, bool READY>
__global__ __launch_bounds__(A8_NT, 2) void attn8_tile_kernel(Args8 a) {
#pragma clang fp contract(off)
  using L = Ready8<D>;
  constexpr int KS = D / 16, DT = D / 32;
  constexpr int K_ROW = 2 * D + 16, V_ROW = 80;               // bytes; padded: no bank twice among 16 lanes
  constexpr int KW = D / 16;                                  // words of codes of a thread that brings K
  constexpr int K_TILE = 32 * K_ROW, TILE = READY ? L::BYTES : K_TILE + D * V_ROW;
  constexpr int NT = 4;                                       // tiles in LDS: two computed, two converted
  __shared__ __align__(16) char s_tile[NT][TILE];
  __shared__ __align__(16) float s_scale[READY ? 1 : NT][4][32];   // K's scales times c2; V's: e, f 2^10, 2^-e
  __shared__ int s_base;                                      // what e is counted from
  __shared__ int s_odd[READY ? 1 : NT];                       // whether an f is NaN or infinite
  __shared__ int s_sums[A8_NW];
  __shared__ int s_again;                                     // the last unit with a sum of NaN
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

  // the lane's fragments: of K, dims 16 s + 8 hi on of row row32; of V, the keys of piece 2 s + hi of dim 32 d + row32
  const auto k_at = [&](int s) { return READY ? L::k_at(row32, 2 * s + hi) : row32 * K_ROW + hi * 16 + 32 * s; };
  const auto v_at = [&](int d, int s) {
    return READY ? L::v_at(32 * d + row32, 2 * s + hi) : K_TILE + (32 * d + row32) * V_ROW + hi * 16 + 32 * s;
  };

  int u = a.n_units - 1 - (int)blockIdx.x, skip = 0, left = 1 << 30;
  if (threadIdx.x == 0) s_again = -1;
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
    float ahead = 0.f;                                        // l's reference is off plus this whole number
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
        const int e = v_exponent(scale[which], base);
        const float f = __builtin_amdgcn_ldexpf(scale[which], 10 - (e + base));
        if (lane < 32) {
          s_scale[READY ? 0 : buf][0][lane] = scale[which] * a.c2;
        } else {
          s_scale[READY ? 0 : buf][1][lane - 32] = (float)e;
          s_scale[READY ? 0 : buf][2][lane - 32] = f;
          s_scale[READY ? 0 : buf][3][lane - 32] = v_back(e, lane - 32, mk);
        }
        const bool odd = __any(lane >= 32 && !(fabsf(f) < INFINITY));
        if (lane == 0) s_odd[READY ? 0 : buf] = odd;
      }
    };
    auto compute = [&](auto far, int buf, int key, uint32_t valid, bool full) {
      f32x16 z = {};
      const char* tile = s_tile[buf];
#pragma unroll
      for (int s = 0; s < KS; ++s)
        z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(tile + k_at(s))),
                                                    qf[s], z, 0, 0, 0);
      if constexpr (!READY) {
        // reads ahead of the products (left to the compiler, each waits for its own: 4 to 5% slower)
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          if (s < KS - 2) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      }
      const float* sc = (READY ? reinterpret_cast<const float*>(tile + L::SCALES) : s_scale[READY ? 0 : buf][0]) + 4 * hi;
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
      if (far.value || __builtin_expect(__any(zm > m + A8_SLACK), 0)) {
        zm = fmaxf(zm, __shfl_xor(zm, 32, 64));
        const float mn = fmaxf(m, ceilf(zm));
        const float alpha = m == -INFINITY ? 0.f : fast_exp2(m - mn);
        const float to = mn == -INFINITY ? 0.f : mn;
        if constexpr (far.value) ahead += off - to;
        else l *= alpha;
        m = mn;
        off = to;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
      }
      if constexpr (far.value) {
        // (y - off - e, in this order: of scores past 2^24 the first difference is exact, and P and l agree)
        const auto x = [&](int e) { return z[e] - off - sc[32 + (e & 3) + 8 * (e >> 2)]; };
        float zx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          zx = fmaxf(zx, x(e));
          if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
        zx = fmaxf(zx, __shfl_xor(zx, 32, 64));
        const float an = fmaxf(ahead, ceilf(zx)), less = an == -INFINITY ? 0.f : an;
        l *= ahead == -INFINITY ? 0.f : fast_exp2(ahead - an);      // (a sum of NaN stays one)
        ahead = an;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          l += fast_exp2(x(e) - less);
          if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
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
      if constexpr (!far.value) l += sum[0] + sum[1];
      if (!full && (READY ? *reinterpret_cast<const int*>(tile + L::ODD) : s_odd[READY ? 0 : buf])) {
        // a probability of 0 times a scale of NaN, or of a slot that holds anything
        asm volatile("" : "+v"(vis));
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = (vis >> ((e & 3) + 8 * (e >> 2))) & 1u ? z[e] : 0.f;
      }
      u32x4 pf[2];                                            // halves of the keys
#pragma unroll
      for (int e = 0; e < 8; ++e)
        pf[e >> 2][e & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{z[2 * e], z[2 * e + 1]}), f16x2));
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const f16x8 vf = __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4*>(tile + v_at(d, s)));
          acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, __builtin_bit_cast(f16x8, pf[s]), acc[d], 0, 0, 0);
        }
    };

    // a tile converted beforehand, straight into LDS
    const char* ready = nullptr;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_tile[0];
    if constexpr (READY) ready = a.ready + ((size_t)w.h * (a.max_pages / 2) + p0 / 2) * L::BYTES + lane * 16;
    auto request = [&](int x, int i, int buf) {
      if ((i & 31) == 0) {
        const int page = p0 + 2 * i + lane;
        masks = page < p1 ? mrow[page] : 0;
      }
      const int e = 2 * (i & 31);
      next_mask[x] = (uint32_t)__builtin_amdgcn_readlane(masks, e) | (uint32_t)__builtin_amdgcn_readlane(masks, e + 1) << 16;
      for (int j = wave; j < L::BYTES / 1024; j += A8_NW)
        direct_load(ready + (size_t)i * L::BYTES + j * 1024, lds + buf * L::BYTES + j * 1024);
    };
    if constexpr (READY) {
      if (tiles > 0) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (x < tiles) request(x, x, x);
          mask[x] = next_mask[x];
        }
        direct_wait<0>();
        __syncthreads();
        base = *reinterpret_cast<const int*>(s_tile[0] + L::BASE);
      }
      for (int i = 0; i < tiles; i += 2) {
        const int buf = i & 2;
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (i + 2 + x < tiles) request(x, i + 2 + x, (buf ^ 2) + x);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int key = (p0 + 2 * (i + x)) * HK_PAGE;
          if (i + x < tiles && key < seen_any && w0 < w.rows)
            compute(std::false_type{}, buf + x, key, mask[x], mask[x] == 0xffffffffu && key + 32 <= seen_all);
          mask[x] = next_mask[x];
        }
        direct_wait<0>();
        __syncthreads();
      }
    } else {
      if (tiles > 0) {
        load(0, 0);
        if (tiles > 1) load(1, 1);
        if (wave == 0) {
          base = v_base(scale[0], next_mask[0]);
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
            compute(std::false_type{}, buf + x, key, mask[x], mask[x] == 0xffffffffu && key + 32 <= seen_all);
          mask[x] = mk[x];
        }
        __syncthreads();
      }
    }

    // (a unit's waves read s_again before the barriers of the next one that could write it)
    if (tiles > 0) {
      if (__any(l != l) && lane == 0) s_again = u;
      __syncthreads();
    }
    if (tiles > 0 && __builtin_amdgcn_readfirstlane(s_again) == u) {
      m = -INFINITY;
      off = 0.f;
      l = 0.f;
      ahead = -INFINITY;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[d][e] = 0.f;
      for (int i = 0; i < tiles; ++i) {
        if constexpr (READY) {
          request(0, i, 0);
          direct_wait<0>();
        } else {
          load(0, i);
          convert(0, 0, next_mask[0]);
        }
        __syncthreads();
        const int key = (p0 + 2 * i) * HK_PAGE;
        compute(std::true_type{}, 0, key, next_mask[0], false);
        __syncthreads();
      }
    }

    l += __shfl_xor(l, 32, 64);
    if (w0 + row32 < w.rows) {
      // l is brought to [1/2, 1): scales far apart leave sums far apart
      const int up = __builtin_amdgcn_frexp_expf(l) + (ahead == -INFINITY ? 0 : (int)ahead);
      const int down = base + Code<F>::F16_DOWN - 10 - up;
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
// Where chunks may be long, a launch before converts every tile once for all of its head's units, into the
// workspace.  (32 / 8 heads of 128, without and with it: 8 prompts of 4096 tokens 1613 and 1438 us, of 1024 153 and
// 142, of 512 65 and 63, of 256 55 and 59; 2 chunks of 1024 tokens over 32000 1546 and 1502, of 512 781 and 775, of 128
// 221 and 269; 8 of 64 over 4000 81 and 113: the tile kernel then reads twice the bytes.)
constexpr int64_t READY_ROWS = 4096;
constexpr size_t READY_MOST = (size_t)1 << 29;   // bytes of tiles at most
static size_t ready_bytes(int D, int64_t heads, int max_pages, int64_t most) {
  const size_t all = (size_t)heads * (max_pages / 2) * (D == 128 ? Ready8<128>::BYTES : Ready8<64>::BYTES);
  return most >= READY_ROWS && all <= READY_MOST ? all : 0;
}
size_t hk_attn8_tile_ws(int D, int64_t heads, int max_pages, int64_t most) {
  return states8_bytes(D, TILE8_ROWS) + ready_bytes(D, heads, max_pages, most);
}

template <int F, int D>
static void launch_tile(const Args8& a, hipStream_t st) {
  const uint32_t groups = a.first ? A8_GROUPS<D> : (uint32_t)a.n_units;
  {
    TimedLaunch t(HK_TK_ATTN8, st);
    if (a.ready) {
      const uint32_t tiles = (uint32_t)((int64_t)a.n_seq * a.Hkv * (a.max_pages / 2));
      hipLaunchKernelGGL((attn8_convert_kernel<F, D>), dim3(tiles), dim3(A8_NT), 0, st, a);
      hipLaunchKernelGGL((attn8_tile_kernel<F, D, true>), dim3(groups), dim3(A8_NT), 0, st, a);
    } else {
      hipLaunchKernelGGL((attn8_tile_kernel<F, D, false>), dim3(groups), dim3(A8_NT), 0, st, a);
    }
  }
  if (a.first && a.max_pages > A8_STEP) merge8<D, TILE8_ROWS, 2, true>(a, groups, st);
}

void hk_launch_attn8_tile(Args8 a, hk_dtype format, int D, int64_t most, void* ws, hipStream_t st) {
  const int64_t units = hk_attn8_tile_units(a.n_seq, a.Hkv, a.G, a.n_tokens);
  a.n_units = (int)units;
  a.cap = TILE8_ROWS;
  a.one_tile = 0;
  a.rows_from = A8_ROWS + 1;
  a.rows_to = INT32_MAX;
  carve8(a, planned8(units, true, a.max_pages), D, ws);
  if (ready_bytes(D, (int64_t)a.n_seq * a.Hkv, a.max_pages, most)) a.ready = static_cast<char*>(ws) + states8_bytes(D, TILE8_ROWS);
  if (format == HK_I8) D == 128 ? launch_tile<HK_I8, 128>(a, st) : launch_tile<HK_I8, 64>(a, st);
  else D == 128 ? launch_tile<HK_E4M3, 128>(a, st) : launch_tile<HK_E4M3, 64>(a, st);
}
