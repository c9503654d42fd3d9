// a7: causal attention of chunks of new tokens over the paged cache (gfx950).
//
// The query rows of one KV head are folded: row r of a chunk is query head r % G of token r / G,
// and all of them read the same K and V.  Two kernels share the work by the folded rows of a
// sequence:
//   tile   more than SHORT_ROWS rows: a workgroup takes TILE_ROWS rows, its four waves 32 each, all
//          against the same K and V tiles in LDS;
//   short  up to SHORT_ROWS rows (drafts, single tokens): a workgroup takes the 32 rows, its four
//          waves take the pages in turn, every page read once by one wave, and meet at the end.
// Both may cut a row's pages into pieces for several workgroups; chunk_merge_kernel joins the
// pieces' states with the operator of App. F.  Work and pieces of a workgroup follow from the chunk
// starts and page counts in device memory.
//
// Arithmetic of a wave, per block of 32 keys: C[key][query] = K Q^T on MFMA, so that a lane holds
// 16 keys of one query and the softmax needs no cross-lane step but for a new reference; then
// O^T[dim][query] += V^T P^T, P going in as it lies: contraction order is free, so the keys keep the
// order of the score tile's registers, and V's columns come from LDS by transposing reads (bf16)
// or one value a lane (fp32).
//
// Softmax: one pass with a running reference m per query, a whole number that moves only when a
// score exceeds it by 2^CH_SLACK, so most blocks need no rescaling.  Probabilities are formed as
// exp2(z - m) 2^-bias (in the bf16 tile kernel, whose P keeps 8 bits and whose LSE is off by some 2^-20,
// as exp2(z - m - bias)), where 2^bias is at least 2^CH_SLACK times the keys of the row: sums of P V
// and their merge cannot pass the top of the fp32 range where the result does not.  At its other end
// that costs bits: V of 1e-32 is off by 4e-7 of its norm, 1e-34 by 2e-5, 1e-36 by 2e-3 (fp32).
// Precision: scores, sums and outputs in fp32; the LSE is of the unrounded P.
// Into the bf16 product P enters in the short kernel in two bf16 parts, to 2^-16 of each term: the
// output is then off by its own rounding and little else, and as the kernel is bound by memory the
// second product takes no time (64 sequences of 1 to 8 tokens over 784 to 5600: 175 us and 173,
// single tokens 163 and 162).  In the tile kernel P is rounded once, to 2^-8 of each term at most, and o is
// normalised by the sum of the rounded: over many keys it is off by 2.3e-3 of its norm instead of the
// 1.7e-3 of its own rounding, and by no more than that where one key or few have the weight.  That sum takes
// 1% to 2% at D 128 and 5% at 64 (8 prompts of 4096 1190 -> 1201 us, 656 -> 699; one chunk of 2048 over 28671
// 869 -> 890); a second part of P would take 31% (1173 -> 1542, 902 -> 1201).
#include <algorithm>
#include <type_traits>

#include "hk_chunk.h"

namespace hk {

constexpr float CH_SLACK = 12.f;
constexpr int SHORT_ROWS = 32;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------ LDS tiles
// A tile row is one key's K or V row.  Rows are padded so that the fragments' reads spread over the
// 64 banks, at offsets that are constants: K, 16 bytes of eight consecutive keys, by 16 bytes; V by
// 64 (bf16: 64 bytes of eight keys, two to a bank group at best) or 32 (fp32: 128 bytes of keys k
// and k + 4).
template <typename T, int D>
struct TileLayout {
  static constexpr int ES = sizeof(T);
  static constexpr int ROW = D * ES;          // bytes
  static constexpr int PIECES = ROW / 16;
  static constexpr int PAGE = HK_PAGE * ROW;
  static constexpr int LOADS = PAGE / 1024;   // 16-byte loads per lane of a wave for a page
  static constexpr int K_ROW = ROW + 16, V_ROW = ROW + (ES == 2 ? 64 : 32);
};

// One page's K or V rows on their way from memory to LDS: piece i * 64 + lane of the page.
template <typename T, int D>
struct PageRegs {
  using L = TileLayout<T, D>;
  u32x4 r[L::LOADS];
  __device__ __forceinline__ void load(const char* pool, int page) {
    const u32x4* src = reinterpret_cast<const u32x4*>(pool + (size_t)page * L::PAGE) + (threadIdx.x & 63);
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) r[i] = src[i * 64];
  }
  // rows whose mask bit is 0 become zeros: nothing they hold may meet a probability of 0
  __device__ __forceinline__ void clear(uint32_t mask) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i)
      if (!((mask >> ((i * 64 + lane) / L::PIECES)) & 1u)) r[i] = u32x4{0u, 0u, 0u, 0u};
  }
  // the page's rows that hold an infinite value or NaN, bit per row
  __device__ __forceinline__ uint32_t odd_rows() const {
    uint32_t rows = 0;
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) {
      bool odd = false;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t x = r[i][w];
        odd |= L::ES == 4 ? (x & 0x7f800000u) == 0x7f800000u
                          : (x & 0x7f800000u) == 0x7f800000u || (x & 0x7f80u) == 0x7f80u;
      }
      const unsigned long long b = __ballot(odd);
      if (b)
        for (int k = 0; k < 64 / L::PIECES; ++k)
          if ((b >> (k * L::PIECES)) & ((1ull << L::PIECES) - 1)) rows |= 1u << (i * (64 / L::PIECES) + k);
    }
    return rows;
  }
  // into rows of `stride` bytes from `to` on
  __device__ __forceinline__ void store(char* to, int stride) const {
    const int lane = threadIdx.x & 63;
    to += lane / L::PIECES * stride + lane % L::PIECES * 16;
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) *reinterpret_cast<u32x4*>(to + i * (64 / L::PIECES) * stride) = r[i];
  }
};

// ------------------------------------------------------------------ matrix products of a wave
// Fragment order: lane l holds query (or key, or dim) l % 32 and half hi = l / 32 of the contraction.
// Register r of a score tile is key (r & 3) + 8 (r >> 2) + 4 hi.
template <typename T, int D>
struct Mma;

template <int D>
struct Mma<uint16_t, D> {
  using L = TileLayout<uint16_t, D>;
  struct Query {
    bf16x8 f[D / 16];
  };
  __device__ static __forceinline__ void load_q(Query& q, const uint16_t* row) {
    const int hi = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      q.f[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(row + (2 * s + hi) * 8));
  }
  __device__ static __forceinline__ void scores(f32x16& z, const Query& q, const char* k) {
    const int lane = threadIdx.x & 63, key = lane & 31, hi = lane >> 5;
    z = f32x16{};
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const bf16x8 a = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(k + key * L::K_ROW + (2 * s + hi) * 16));
      z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q.f[s], z, 0, 0, 0);
    }
  }
  __device__ static __forceinline__ void values(f32x16 (&acc)[D / 32], const f32x16& p, const char* v) {
    const int lane = threadIdx.x & 63, hi = lane >> 5, g1 = (lane >> 4) & 1, i16 = lane & 15;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      __builtin_amdgcn_sched_barrier(0);        // (here and below: the fragments of one product at a time, 247
                                                // registers at D 128; without, 256 and spills)
      bf16x8 bp, low;                           // P = bp + low, to 2^-16 of it
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const f32x2 x = {p[8 * s + j], p[8 * s + j + 1]};
        const bf16x2 t = __builtin_convertvector(x, bf16x2);
        const bf16x2 r = __builtin_convertvector((f32x2{x[0] - (float)t[0], x[1] - (float)t[1]}), bf16x2);
        bp[j] = t[0];
        bp[j + 1] = t[1];
        low[j] = r[0];
        low[j + 1] = r[1];
      }
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        s16x4 a[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // sixteen lanes turn four keys x 16 dims: lane i supplies 4 dims of key i / 4
          const char* at = v + (16 * s + 8 * h + 4 * hi + (i16 >> 2)) * L::V_ROW + dt * 64 + g1 * 32 + (i16 & 3) * 8;
          a[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4*)(uintptr_t)(__attribute__((address_space(3))) const char*)at);
        }
        const bf16x8 av = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a[0], a[1], 0, 1, 2, 3, 4, 5, 6, 7));
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, low, acc[dt], 0, 0, 0);
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, bp, acc[dt], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  __device__ static __forceinline__ float value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
  __device__ static __forceinline__ void put4(uint16_t* to, float x, float y, float z, float w) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
    const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{z, w}), bf16x2));
    *reinterpret_cast<u32x2*>(to) = u32x2{a, b};
  }
};

template <int D>
struct Mma<float, D> {
  using L = TileLayout<float, D>;
  struct Query {
    f32x4 f[D / 8];
  };
  __device__ static __forceinline__ void load_q(Query& q, const float* row) {
    const int hi = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < D / 8; ++s) q.f[s] = *reinterpret_cast<const f32x4*>(row + (2 * s + hi) * 4);
  }
  __device__ static __forceinline__ void scores(f32x16& z, const Query& q, const char* k) {
    const int lane = threadIdx.x & 63, key = lane & 31, hi = lane >> 5;
    z = f32x16{};
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(k + key * L::K_ROW + (2 * s + hi) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) z = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], q.f[s][j], z, 0, 0, 0);
    }
  }
  __device__ static __forceinline__ void values(f32x16 (&acc)[D / 32], const f32x16& p, const char* v) {
    const int lane = threadIdx.x & 63, hi = lane >> 5, dim = lane & 31;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int key = (r & 3) + 8 * (r >> 2) + 4 * hi;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        const float a = *reinterpret_cast<const float*>(v + key * L::V_ROW + (32 * dt + dim) * 4);
        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[r], acc[dt], 0, 0, 0);
      }
    }
  }
  __device__ static __forceinline__ float value(float x) { return x; }
  __device__ static __forceinline__ void put4(float* to, float x, float y, float z, float w) {
    *reinterpret_cast<f32x4*>(to) = f32x4{x, y, z, w};
  }
};

// ------------------------------------------------------------------ the softmax state of a wave
// The reference of a query.  A probability's exponent is z c2 - off, off being m and the kernel's shift (0
// while there is no m), one fma an element: exact where m is below FAR, 2^24.  From there on the product's rounding, which
// the fma leaves out and m has, is a whole number and more, and would make a largest score's
// probability infinite or 0: such a query's scores are brought to (z c2 - m) / c2, each step rounded as
// m was, and have off = shift.
constexpr float FAR = 16777216.f;
struct Reference {
  float m, off;
  float limit;                                // a score above it: move (far: any score, for bring)
  __device__ __forceinline__ void init() {
    m = limit = -INFINITY;
    off = 0.f;
  }
  __device__ static __forceinline__ bool is_far(float m) { return fabsf(m) >= FAR && fabsf(m) < INFINITY; }
  // moved to mn; returns the factor of the sums so far.  shift: of the exponent, beside mn
  __device__ __forceinline__ float move(float mn, float shift) {
    const float alpha = m == -INFINITY ? 0.f : fast_exp2(m - mn);
    m = mn;
    off = mn == -INFINITY ? 0.f : is_far(mn) ? shift : mn + shift;
    limit = is_far(mn) ? -INFINITY : mn + CH_SLACK;
    return alpha;
  }
  __device__ __forceinline__ void bring(f32x16& z, float c2) const {
#pragma clang fp contract(off)
    if (!__any(is_far(m))) return;
    const float back = fminf(1.f / c2, 0x1.fffffep127f);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float x = z[r] * c2, y = x - m;
      z[r] = is_far(m) ? y * back : z[r];
    }
  }
  // what the state's sums are relative to
  __device__ __forceinline__ float whole(float bias) const { return m == -INFINITY ? 0.f : m + bias; }
};

// 32 queries; lane l holds query l % 32, and half of its keys.
template <typename T, int D>
struct State {
  using M = Mma<T, D>;
  f32x16 acc[D / 32];                         // O^T: register r is dim 32 dt + (r & 3) + 8 (r >> 2) + 4 hi
  Reference ref;
  float l;                                    // sum
  __device__ __forceinline__ void init() {
    ref.init();
    l = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[dt][r] = 0.f;
  }
  // 32 keys from LDS; vis: bit k, key k of them is seen by the lane's query (all: every bit of
  // every lane is 1).  odd: keys whose V row holds infinite values and is not seen by every query;
  // it is zeros in LDS and added here, at row(key), to the queries that see it: for the others
  // its product with a probability of 0 would be NaN.
  // down: 2^-bias.  It is a factor of the probabilities here, and no part of the exponent, which it would
  // bring to 17 and more, where its rounding is 2^-20: o of an fp32 cache was off by 3.7e-7 of its norm
  // over short rows and is by 1.9e-7.
  template <typename F>
  __device__ __forceinline__ void block(const typename M::Query& q, const char* k, const char* v, uint32_t vis, bool all,
                                        float c2, float down, uint32_t odd, F row) {
    const int hi = (threadIdx.x & 63) >> 5;
    f32x16 z;
    M::scores(z, q, k);
    if (!all) {
      uint32_t w = vis >> (4 * hi);
      asm volatile("" : "+v"(w));             // (a branch, not selects in every block)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!((w >> ((r & 3) + 8 * (r >> 2))) & 1u)) z[r] = -INFINITY;
    }
    float zm = z[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) zm = fmaxf(zm, z[r]);
    zm *= c2;
    if (__builtin_expect(__any(zm > ref.limit), 0)) {
      zm = fmaxf(zm, __shfl_xor(zm, 32, 64));
      const float alpha = ref.move(fmaxf(ref.m, ceilf(zm)), 0.f);
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[dt][r] *= alpha;
      ref.bring(z, c2);
    }
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      z[r] = fast_exp2(fmaf(z[r], c2, -ref.off)) * down;
      s[r & 3] += z[r];
    }
    l += (s[0] + s[1]) + (s[2] + s[3]);
    M::values(acc, z, v);
    while (odd) {
      const int key = __builtin_ctz(odd), reg = (key & 3) + 4 * (key >> 3), lane = threadIdx.x & 63;
      odd &= odd - 1;
      const T* vr = row(key);
      float p = z[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) p = reg == r ? z[r] : p;
      p = __shfl(p, (lane & 31) + 32 * ((key >> 2) & 1), 64);
      const bool sees = (vis >> key) & 1u;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = M::value(vr[32 * dt + (r & 3) + 8 * (r >> 2) + 4 * hi]);
          acc[dt][r] = sees ? fmaf(p, x, acc[dt][r]) : acc[dt][r];
        }
    }
  }
};

// log of l 2^ref.  The powers of two of both, 17 and more, cancel as whole numbers: beside the logarithm of
// all of l they left an error of 2^-19 (small LSEs by 1.4e-6).
__device__ __forceinline__ float lse_of(float ref, float l) {
  if (l == 0.f) return -INFINITY;
  return (ref + (float)__builtin_amdgcn_frexp_expf(l) + __log2f(__builtin_amdgcn_frexp_mantf(l))) * kLn2;
}

// Pages that the token last_token of a chunk sees.
__device__ __forceinline__ int tile_pages(int n, int end, int len, int last_token) {
  const int seen = max(end - len + last_token + 1, 0);
  return min(n, (seen + HK_PAGE - 1) / HK_PAGE);
}
__device__ __forceinline__ float bias_of(int pages) { return (float)(32 - __clz(pages * HK_PAGE)) + CH_SLACK; }
__device__ __forceinline__ float down_of(float bias) { return __uint_as_float((uint32_t)(127 - (int)bias) << 23); }

struct Args {
  const char *q, *k_pool, *v_pool;
  const int32_t *table, *n_pages, *start;
  const uint16_t* masks;
  int64_t q_row;                              // elements
  char* o;
  float *lse;
  float *short_o, *short_ml, *tile_o, *tile_ml;
  int32_t* short_first;                       // the short rows' first steps, their total, a workgroup's share
  int32_t* tile_split;                        // the tiles' pieces: see TileSplit
  int Hq, Hkv, G, max_pages, num_pages, n_seq, n_tokens, max_len;
  int n_tiles;                                // of a KV head, for the tile kernels
  float c2;
};

// One query's result of a tile kernel (lane: half of the dims): normalised into o, or state `at` of
// its pieces (at < 0: there is one piece).  l: sum of the probabilities, for the LSE and a piece's weight;
// of_o: of those in acc, as they were rounded (acc / of_o is a mean of V, with one key that key's V).
template <typename T, int D>
__device__ __forceinline__ void put_state(const Args& a, int64_t row, int64_t at, const f32x16 (&acc)[D / 32],
                                          float mb, float l, float of_o) {
  const int hi = (threadIdx.x & 63) >> 5;
  if (at >= 0) {
    const float up = sizeof(T) == 4 || l == 0.f ? 1.f : l / of_o;
    float* to = a.tile_o + at * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(to + 32 * dt + 8 * j + 4 * hi) =
            f32x4{acc[dt][4 * j] * up, acc[dt][4 * j + 1] * up, acc[dt][4 * j + 2] * up, acc[dt][4 * j + 3] * up};
    if (hi == 0) *reinterpret_cast<f32x2*>(a.tile_ml + at * 2) = f32x2{l == 0.f ? -INFINITY : mb, l};
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / of_o;   // (a NaN stays one)
  T* to = reinterpret_cast<T*>(a.o) + row * D;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      Mma<T, D>::put4(to + 32 * dt + 8 * j + 4 * hi, acc[dt][4 * j] * inv, acc[dt][4 * j + 1] * inv,
                      acc[dt][4 * j + 2] * inv, acc[dt][4 * j + 3] * inv);
  if (hi == 0 && a.lse) a.lse[row] = lse_of(mb, l);
}

// ------------------------------------------------------------------ tile kernels
constexpr int TILE_ROWS = 128, TILE_PAGES = 4, TILE_KEYS = TILE_PAGES * HK_PAGE;

// Tiles of TILE_ROWS folded rows are numbered over the batch: a sequence's begin at tiles_before, which
// leaves at most one of a sequence without rows.
__device__ __forceinline__ int tiles_before(const Args& a, int s) {
  return min(max(a.start[s], 0), a.n_tokens) * a.G / TILE_ROWS + s;
}

// TILE_ROWS folded rows of one sequence and KV head, and the pages of them that a workgroup takes.  No
// steps: there are no such rows.
struct Tile {
  Chunk c;
  int kv, rows, r0, end, pages, steps, p0, p1;
  const int32_t* trow;
  const uint16_t* mrow;
};
__device__ __forceinline__ Tile tile_of(const Args& a, int u, int kv) {
  Tile w;
  int s = 0;
  for (int hi = a.n_seq; hi - s > 1;) {
    const int mid = (s + hi) / 2;
    if (tiles_before(a, mid) <= u) s = mid;
    else hi = mid;
  }
  w.kv = kv;
  w.c = chunk_of(a.start, s, a.n_tokens, a.max_len);
  w.rows = w.c.len * a.G;
  w.r0 = (u - tiles_before(a, s)) * TILE_ROWS;
  w.steps = 0;
  if (w.rows <= SHORT_ROWS || w.r0 < 0 || w.r0 >= w.rows) return w;
  const int h = s * a.Hkv + kv, n = min(max(a.n_pages[h], 0), a.max_pages);
  w.trow = a.table + (size_t)h * a.max_pages;
  w.mrow = a.masks + (size_t)h * a.max_pages;
  w.end = row_end(n, n > 0 ? w.mrow[n - 1] : 0u);
  w.pages = tile_pages(n, w.end, w.c.len, (min(w.r0 + TILE_ROWS, w.rows) - 1) / a.G);
  w.steps = max((w.pages + TILE_PAGES - 1) / TILE_PAGES, 1);     // (rows without pages have empty results to write)
  w.p0 = 0;
  w.p1 = w.pages;
  return w;
}

// A launch of many tiles has a workgroup for each, the largest of a sequence first.  One of few
// (PLANNED) has at most TILE_WG workgroups, which see from the rows' lengths into how many pieces to
// split the tiles: pieces of one length, that of the longest tile over one of twelve numbers, so that
// the pieces of a KV head's tiles that run beside one another read the same pages.
constexpr int TILE_WG = 512, PLAN_TILES = 1024, PLAN_PIECES = 1536;
constexpr int N_SPLITS = 12, MAX_STATES = 64; // choices, and pieces of a row at most
// length of a piece, choice c: the longest tile over 1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48 or 64
__device__ __forceinline__ int piece_length(int most, int c) {
  const int n = c == 0 ? 1 : c & 1 ? 2 << (c >> 1) : 3 << ((c >> 1) - 1);
  return (most + n - 1) / n;
}
// What a piece costs beside its steps, in steps of its type: its start, or that and its state's way to
// the merge; and what a step costs where a CU has one workgroup, in tenths of one where it has two.
// From timings with every split forced (bf16, 32/8 heads over 20000: 1024 tokens in 1, 2, 3, 4 pieces
// 457, 359, 395, 385 us, 2560 in 1, 2, 3 1122, 977, 940; 256 in 4, 8 135, 132; fp32, 2 sequences over
// 2000: 1, 2, 4, 8 177, 100, 58, 40).  STATE 10, 14, 18: 256 tokens 108, 108, 115 us, 16 tokens 43, 39, 39.
template <typename T>
struct Cost;
template <>
struct Cost<uint16_t> {
  static constexpr int START = 7, STATE = 14, ALONE = 7;
};
template <>
struct Cost<float> {
  static constexpr int START = 2, STATE = 3, ALONE = 5;
};

struct TileSplit {                            // for the merge, by tile: its pieces and its rows
  int32_t at, used, first, rows, r0, kv;
};

template <int NT>
struct Planned {
  int first[PLAN_TILES + 1];                  // piece that a tile begins at
  int sum[NT / 64], most[NT / 64];
  int pieces[N_SPLITS], whole[N_SPLITS];      // by choice of their length; whole: nearly all of it
};
// Counts the pieces of all tiles (into s.first); returns their length in steps.  The lengths are tried
// side by side (one after the other, unrolled or not: 3 and 6 us more a launch).
template <typename T, int NT>
__device__ __forceinline__ int plan_tiles(const Args& a, Planned<NT>& s) {
  const int n = a.n_tiles * a.Hkv, per = (n + NT - 1) / NT, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int MOST = (PLAN_TILES + NT - 1) / NT;
  auto add = [](uint32_t p, uint32_t q) { return p + q; };
  int k[MOST], sum = 0, most = 0;
#pragma unroll
  for (int j = 0; j < MOST; ++j) {
    const int i = threadIdx.x * per + j;
    k[j] = j < per && i < n ? tile_of(a, i % a.n_tiles, i / a.n_tiles).steps : 0;
    if (j < per && i < n) s.first[i] = k[j];  // (until the pieces are counted)
    sum += k[j];
    most = max(most, k[j]);
  }
  if (threadIdx.x < N_SPLITS) s.pieces[threadIdx.x] = s.whole[threadIdx.x] = 0;
  sum = (int)wave_reduce_u32((uint32_t)sum, 0u, add);
  most = (int)wave_reduce_u32((uint32_t)most, 0u, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
  if (lane == 63) {
    s.sum[wave] = sum;
    s.most[wave] = most;
  }
  __syncthreads();
  sum = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    sum += s.sum[w];
    most = max(most, s.most[w]);
  }
  most = max(most, 1);
  constexpr int GROUPS = NT / N_SPLITS;       // a thread takes one length and every GROUPS-th tile
  if (threadIdx.x < GROUPS * N_SPLITS) {
    const int c = threadIdx.x % N_SPLITS, len = piece_length(most, c);
    const float inv = 1.f / (float)len;
    int pieces = 0, whole = 0;
    for (int i = threadIdx.x / N_SPLITS; i < n; i += GROUPS) {
      const int steps = s.first[i];
      int x = (int)((float)steps * inv), rest = steps - x * len;       // (x at most 64: off by one at most)
      if (rest < 0) --x, rest += len;
      if (rest >= len) ++x, rest -= len;
      pieces += x + (rest > 0);
      whole += x + (rest > len - len / 8);
    }
    atomicAdd(&s.pieces[c], pieces);
    atomicAdd(&s.whole[c], whole);
  }
  __syncthreads();
  // the cheapest, in tenths of a step: rounds of (nearly) whole pieces, or an even share of all steps,
  // and a quarter piece of unevenness where not all pieces run at once; lane c of 16 computes choice c
  const int c = min(lane & 15, N_SPLITS - 1), len = piece_length(most, c), pieces = s.pieces[c], whole = s.whole[c];
  const int extra = c ? Cost<T>::STATE : Cost<T>::START, rest = whole % TILE_WG;
  const int last = rest == 0 ? 0 : Cost<T>::ALONE + (10 - Cost<T>::ALONE) * max(rest - TILE_WG / 2, 0) / (TILE_WG / 2);
  const int rounds = (whole / TILE_WG * 10 + last) * (len + extra);
  const int share = (sum + extra * pieces) / (TILE_WG / 10) + (pieces > TILE_WG ? len * 10 / 4 : 0);
  const bool fits = c == 0 || pieces <= PLAN_PIECES;
  int best = fits ? min(max(rounds, share), (1 << 27) - 1) << 4 | c : 0x7fffffff;
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) best = min(best, __shfl_xor(best, o, 64));
  const int length = piece_length(most, best & 15);
  int x = 0;
#pragma unroll
  for (int j = 0; j < MOST; ++j) {
    k[j] = (k[j] + length - 1) / length;
    x += k[j];
  }
  int before = -x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) s.sum[wave] = x;
  __syncthreads();
  before += x;
  int total = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wave) before += s.sum[w];
    total += s.sum[w];
  }
#pragma unroll
  for (int j = 0; j < MOST; ++j) {
    const int i = threadIdx.x * per + j;
    if (j < per && i < n) s.first[i] = before;
    before += k[j];
  }
  if (threadIdx.x == 0) s.first[n] = total;
  __syncthreads();
  if (blockIdx.x == gridDim.x - 1)            // (often without a piece)
    for (int i = threadIdx.x; i < n; i += NT) {
      const Tile w = tile_of(a, i % a.n_tiles, i / a.n_tiles);
      reinterpret_cast<TileSplit*>(a.tile_split)[i] = {s.first[i], s.first[i + 1] - s.first[i], w.c.first, w.rows,
                                                       w.r0, w.kv};
    }
  return length;
}

// The pieces of a workgroup.  next(): the next one, or false.
template <typename T, int NT, bool PLANNED>
struct Pieces {
  const Args& a;
  Planned<NT>& s;
  int x, stop, stride, length;
  int64_t state;                              // of the piece's first row; -1: the piece is all of its tile
  __device__ __forceinline__ Pieces(const Args& args, Planned<NT>& lds) : a(args), s(lds), state(-1) {
    x = 0;
    if (PLANNED) {
      length = __builtin_amdgcn_readfirstlane(plan_tiles<T, NT>(a, s));
      const int total = __builtin_amdgcn_readfirstlane(s.first[a.n_tiles * a.Hkv]);
      // the workgroups of a die (every eighth) share an eighth of the pieces that lie behind one another
      const int b = blockIdx.x, dies = gridDim.x % 8 ? 1 : 8;
      x = total * (b % dies) / dies + b / dies;
      stop = total * (b % dies + 1) / dies;
      stride = gridDim.x / dies;
    }
  }
  __device__ __forceinline__ bool next(Tile& w) {
    if (!PLANNED) {
      if (x++) return false;
      w = tile_of(a, a.n_tiles - 1 - (int)(blockIdx.x / a.Hkv), blockIdx.x % a.Hkv);
      return w.steps > 0;
    }
    if (x >= stop) return false;
    int i = 0;                                // the last tile that begins at or before x
    for (int hi = a.n_tiles * a.Hkv; hi - i > 1;) {
      const int mid = (i + hi) / 2;
      if (s.first[mid] <= x) i = mid;
      else hi = mid;
    }
    i = __builtin_amdgcn_readfirstlane(i);
    const int split = x - __builtin_amdgcn_readfirstlane(s.first[i]);
    w = tile_of(a, i % a.n_tiles, i / a.n_tiles);
    state = w.steps > length ? (int64_t)x * TILE_ROWS : -1;
    w.p0 = __builtin_amdgcn_readfirstlane(split * length * TILE_PAGES);
    w.p1 = __builtin_amdgcn_readfirstlane(min(w.p0 + length * TILE_PAGES, w.pages));
    x += stride;
    return true;
  }
};

// fp32: four waves take 32 rows each; the next tile's pages load while a tile is computed.  Bound by
// the fp32 matrix rate, a sixteenth of bf16's (154 TFLOP/s in a large product): 16 sequences of up to
// 203 tokens over 2000, 32/8 heads of 64: 316 us, 97 TFLOP/s (tiles of 256 rows: 497); 4 prompts of 2000:
// 105 TFLOP/s, of 128 101, at one workgroup a CU.
template <int D, bool PLANNED>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void chunk_tile_f32_kernel(Args a) {
  using L = TileLayout<float, D>;
  using M = Mma<float, D>;
  constexpr int NW = 4, TP = TILE_PAGES, PPW = 2 * TP / NW;               // pages that a wave brings
  __shared__ __align__(16) char s_k[2][TILE_KEYS * L::K_ROW], s_v[2][TILE_KEYS * L::V_ROW];
  __shared__ __align__(8) uint16_t s_mask[2][TP], s_odd[2][TP];
  __shared__ Planned<256> s_plan;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Pieces<float, 256, PLANNED> pieces(a, s_plan);
  for (Tile w; pieces.next(w);) {
    if (PLANNED) __syncthreads();                                   // (the last piece's tiles are read)
    // rows past the chunk repeat its last one; they are not stored
    const int w0 = w.r0 + wave * 32, off = w.end - w.c.len + 1;
    const int r = min(w0 + (lane & 31), w.rows - 1), tok = r / a.G, g = r - tok * a.G;
    const int64_t row = (int64_t)(w.c.first + tok) * a.Hq + w.kv * a.G + g;
    const int seen = off + tok;                                  // keys before this one are seen by the lane's query,
    const int seen_all = off + min(w0, w.rows - 1) / a.G;        // by every query of the wave,
    const int tile_seen = off + w.r0 / a.G;                      // of the workgroup
    typename M::Query q;
    M::load_q(q, reinterpret_cast<const float*>(a.q) + (int64_t)(w.c.first + tok) * a.q_row + (w.kv * a.G + g) * D);
    const float bias = bias_of(w.pages);
    State<float, D> st;
    st.init();
    const int tiles = w.p1 > w.p0 ? (w.p1 - w.p0 + TP - 1) / TP : 0;
    PageRegs<float, D> rp[PPW];
    int id[PPW];
    uint32_t mask[PPW], next_mask[PPW];
    auto load_id = [&](int t) {
#pragma unroll
      for (int i = 0; i < PPW; ++i) {
        const int p = w.p0 + t * TP + (wave * PPW + i) % TP;
        next_mask[i] = p < w.p1 ? w.mrow[p] : 0u;
        id[i] = w.trow[min(p, w.p1 - 1)];
      }
    };
    auto load = [&] {
#pragma unroll
      for (int i = 0; i < PPW; ++i) {
        mask[i] = next_mask[i];
        rp[i].load((wave * PPW + i) / TP ? a.v_pool : a.k_pool, min(max(id[i], 0), a.num_pages - 1));
      }
    };
    auto row_at = [&](int p) {                                   // V row of key k of the 32 from page p on
      return [&, p](int k) {
        const int at = min(max(w.trow[min(p + k / HK_PAGE, w.p1 - 1)], 0), a.num_pages - 1);
        return reinterpret_cast<const float*>(a.v_pool) + ((size_t)at * HK_PAGE + k % HK_PAGE) * D;
      };
    };
    if (tiles > 0) {
      load_id(0);
      load();
      load_id(1);
    }
    for (int t = 0; t < tiles; ++t) {
      const int p = w.p0 + t * TP, buf = t & 1;
#pragma unroll
      for (int i = 0; i < PPW; ++i) {
        const int my = (wave * PPW + i) % TP, is_v = (wave * PPW + i) / TP;
        if (is_v) {
          uint32_t keep = mask[i], odd = 0;
          if ((p + my + 1) * HK_PAGE > tile_seen) {
            odd = rp[i].odd_rows() & keep;
            keep &= ~odd;
          }
          if (keep != 0xffffu) rp[i].clear(keep);
          if (lane == 0) {
            s_mask[buf][my] = (uint16_t)mask[i];
            s_odd[buf][my] = (uint16_t)odd;
          }
        }
        if (is_v) rp[i].store(s_v[buf] + my * HK_PAGE * L::V_ROW, L::V_ROW);
        else rp[i].store(s_k[buf] + my * HK_PAGE * L::K_ROW, L::K_ROW);
      }
      __syncthreads();
      if (t + 1 < tiles) {
        load();
        load_id(t + 2);
      }
      if (w0 < w.rows) {
        const uint64_t m64 = *reinterpret_cast<const uint64_t*>(s_mask[buf]);
        const uint64_t o64 = *reinterpret_cast<const uint64_t*>(s_odd[buf]);
#pragma unroll
        for (int hb = 0; hb < TILE_KEYS / 32; ++hb) {
          const int key = (p + 2 * hb) * HK_PAGE;
          const uint32_t valid = __builtin_amdgcn_readfirstlane((uint32_t)(m64 >> (32 * hb)));
          const uint32_t odd = __builtin_amdgcn_readfirstlane((uint32_t)(o64 >> (32 * hb)));
          const bool all = valid == 0xffffffffu && key + 32 <= seen_all;
          const int k = seen - key;
          const uint32_t vis = valid & (k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u);
          st.block(q, s_k[buf] + hb * 32 * L::K_ROW, s_v[buf] + hb * 32 * L::V_ROW, vis, all, a.c2, down_of(bias), odd,
                   row_at(p + 2 * hb));
        }
      }
    }
    const float l = st.l + __shfl_xor(st.l, 32, 64);
    if (w0 + (lane & 31) < w.rows)
      put_state<float, D>(a, row, pieces.state < 0 ? -1 : pieces.state + r - w.r0, st.acc, st.ref.whole(bias), l, l);
  }
}

// LDS tiles of the bf16 kernel: filled straight from memory, 1 KB an instruction, 16 bytes a lane in
// lane order, so a tile is made of 1 KB groups of rows (8 of D 64, 4 of D 128), 16 or 32 bytes apart.
// Within a group the row's 64-byte quarters come first, then the rows, then the 16-byte pieces (of D
// 64 swapped in pairs in rows 4 to 7): four lanes fetch 64 bytes of a row, the eight or sixteen keys
// of a K fragment's read lie in different banks, those of a V fragment's two to a bank at best, and
// every fragment's offset is a constant.
template <int D>
struct DirectTile {
  static constexpr int ROWS = 512 / D, GROUP = D == 128 ? 1040 : 1056, BYTES = 32 / ROWS * GROUP;
  static constexpr int LOADS = HK_PAGE / ROWS, QUARTER = ROWS * 64;
  // the row within a group and the byte within the row that a lane fetches
  __device__ static __forceinline__ int row(int lane) { return (lane >> 2) & (ROWS - 1); }
  __device__ static __forceinline__ int byte(int lane) {
    return lane / (4 * ROWS) * 64 + ((lane & 3) ^ (D == 64 ? (lane >> 4) & 1 : 0)) * 16;
  }
  // fragment s of key lane % 32, dims 16 s + 8 (lane / 32) ..: at k_lane + k_step(s)
  __device__ static __forceinline__ int k_lane(int lane) {
    const int key = lane & 31, hi = lane >> 5, swap = D == 64 ? (key >> 2) & 1 : 0;
    return key / ROWS * GROUP + key % ROWS * 64 + (hi ^ swap) * 16;
  }
  static constexpr int k_step(int s) { return (s >> 1) * QUARTER + (s & 1) * 32; }
  // transposing read h of the keys 16 s + 8 h + 4 (lane / 32) .. of dims 32 dt ..: v_lane + v_step
  __device__ static __forceinline__ int v_lane(int lane) {
    const int i = lane & 15, g = (lane >> 4) & 1, hi = lane >> 5;
    if (D == 128) return hi * GROUP + (i >> 2) * 64 + g * 32 + (i & 3) * 8;
    return (4 * hi + (i >> 2)) * 64 + g * 32 + (((i & 3) >> 1) ^ hi) * 16 + (i & 1) * 8;
  }
  static constexpr int v_step(int s, int h, int dt) { return (16 * s + 8 * h) / ROWS * GROUP + dt * QUARTER; }
};
static __device__ const u32x4 zero_row[1] = {};

// 1 KB from memory to LDS: lane l's 16 bytes at `from` (+ `at`) to `to` + 16 l.  It is on its way
// afterwards; direct_wait waits until `later` such loads or fewer are.
__device__ __forceinline__ void direct_load(const char* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "m0", "memory");
}
__device__ __forceinline__ void direct_load(const char* from, uint32_t at, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(at), "s"(from), "s"(to) : "m0", "memory");
}
template <int later>
__device__ __forceinline__ void direct_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(later) : "memory"); }

// bf16.  Four waves take 32 rows each against tiles of 32 keys.  A wave's tiles are a pipeline: the
// scores of the next tile run beside the exponentials of this one, its P V beside the next one's
// maximum; MFMAs and the vector work between them are laid out by hand.  Two workgroups a CU, for
// one's start, end and waits to be beside the other's work (measured against one of eight waves and
// tiles of 64 keys, 8 prompts of 4096 tokens, 32 / 8 heads: D 128 1152 us and 1172, D 64 697 and 786).
// Bound by the products (2048 cycles of each SIMD for 64 keys) beside as many cycles of exponentials,
// sums and maxima, which overlap in part, and LDS reads at half their rate: 880 to 980 TFLOP/s by the
// card, of 1231 in a large library product; the products alone run at 1363.  By counters, 8 prompts of
// 4096: MFMA busy for 44% of the SIMDs' cycles at 1.88 GHz, vector instructions for 43%, no LDS conflicts.
// Waves 0 and 1 bring a page of K each, three tiles ahead of the wait for it, waves 2 and 3 the pages
// of V.
template <int D, bool PLANNED>
__global__ __launch_bounds__(256, 2) void chunk_tile_bf16_kernel(Args a) {
  using L = DirectTile<D>;
  using M = Mma<uint16_t, D>;
  constexpr int KS = D / 16, DT = D / 32, VS = 2 * DT, AHEAD = 3;
  constexpr int PAGE = HK_PAGE * D * 2, PAGE_LDS = HK_PAGE / L::ROWS * L::GROUP;
  constexpr int NK = 4, NV = 5;                                  // tiles in LDS
  __shared__ __align__(16) char s_k[NK][L::BYTES], s_v[NV][L::BYTES];
  __shared__ uint32_t s_odd[NV][2];                              // odd rows of a tile's pages
  const int lane = threadIdx.x & 63, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);   // (conditions on it are scalar)
  __shared__ Planned<256> s_plan;
  Pieces<uint16_t, 256, PLANNED> pieces(a, s_plan);
  for (Tile w; pieces.next(w);) {
    if (PLANNED) __syncthreads();                                   // (the last piece's tiles are read)
    // rows past the chunk repeat its last one; they are not stored
    const int w0 = w.r0 + wave * 32, off = w.end - w.c.len + 1;
    const int r = min(w0 + (lane & 31), w.rows - 1), tok = r / a.G, g = r - tok * a.G;
    const int64_t row = (int64_t)(w.c.first + tok) * a.Hq + w.kv * a.G + g;
    const int seen = off + tok;                                  // keys before this one are seen by the lane's query,
    const int seen_all = off + min(w0, w.rows - 1) / a.G;        // by every query of the wave,
    const int tile_seen = off + w.r0 / a.G;                      // of the workgroup
    typename M::Query q;
    M::load_q(q, reinterpret_cast<const uint16_t*>(a.q) + (int64_t)(w.c.first + tok) * a.q_row + (w.kv * a.G + g) * D);
    const float bias = bias_of(w.pages), c2 = a.c2;
    const int tiles = w.p1 > w.p0 ? (w.p1 - w.p0 + 1) / 2 : 0;

    // At the middle of tile t a wave has the pages up to K of t + 4 or V of t + 3 requested, and the
    // slots of K of t + 1 and V of t - 1 are read by all: K of t + 5 and V of t + 4 take them.  Ids and
    // masks come 64 tiles at a time: lane i holds tile i's masks, and the id of K's page of tile i or
    // V's of tile i - 1.  V rows that are not valid are fetched as zeros.
    constexpr int LEAD = 5;
    const int my = wave & 1, is_v = wave >> 1;
    const char* pool = is_v ? a.v_pool : a.k_pool;
    const uint32_t lane_at = L::row(lane) * (D * 2) + L::byte(lane);
    int ids, next_ids;
    uint32_t masks, next_masks;
    auto load_ids = [&](int t) {
      const int p = w.p0 + 2 * (t + lane);
      next_masks = (p < w.p1 ? w.mrow[p] : 0u) | (p + 1 < w.p1 ? (uint32_t)w.mrow[p + 1] << 16 : 0u);
      next_ids = min(max(w.trow[min(max(p - 2 * is_v + my, w.p0), w.p1 - 1)], 0), a.num_pages - 1);
    };
    auto request = [&](int id, uint32_t mask, uint32_t to) {     // mask: of the page's rows
      const char* from = pool + (size_t)(uint32_t)id * PAGE;
      to += my * PAGE_LDS;
      if (is_v && mask != 0xffffu) {
#pragma unroll
        for (int j = 0; j < L::LOADS; ++j) {
          const bool valid = (mask >> (j * L::ROWS + L::row(lane))) & 1u;
          direct_load(valid ? from + j * 1024 + lane_at : reinterpret_cast<const char*>(zero_row), to + j * L::GROUP);
        }
      } else {
#pragma unroll
        for (int j = 0; j < L::LOADS; ++j) direct_load(from + j * 1024, lane_at, to + j * L::GROUP);
      }
    };
    // V's page of tile t is in LDS: rows that hold infinite values and are not seen by every query of
    // the workgroup become zeros.
    auto settle = [&](int t, uint32_t mask, int slot) {
      uint32_t odd = 0;
      if (mask != 0) {
        char* at = s_v[slot] + my * PAGE_LDS + lane * 16;
#pragma unroll
        for (int j = 0; j < L::LOADS; ++j) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(at + j * L::GROUP);
          bool bad = false;
#pragma unroll
          for (int k = 0; k < 4; ++k) bad |= (x[k] & 0x7f800000u) == 0x7f800000u || (x[k] & 0x7f80u) == 0x7f80u;
          if (__any(bad))
            for (int r = 0; r < L::ROWS; ++r)
              if (__any(bad && L::row(lane) == r)) {
                odd |= 1u << (j * L::ROWS + r);
                if (L::row(lane) == r) *reinterpret_cast<u32x4*>(at + j * L::GROUP) = u32x4{0u, 0u, 0u, 0u};
              }
        }
      }
      if (lane == 0) s_odd[slot][my] = odd;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    // some keys of tile t, by some query
    auto unseen = [&](int t) { return (w.p0 + 2 * t + 2) * HK_PAGE > tile_seen; };
    const uint32_t lds_k = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_k[0];
    const uint32_t lds_v = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_v[0];

    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[dt][e] = 0.f;
    Reference ref;
    ref.init();
    float l = 0.f, rounded[2] = {0.f, 0.f};                      // sums of P, and of P as it enters the product

    const int k_at = L::k_lane(lane), v_at = L::v_lane(lane);    // the lane's fragments within 32 keys
    auto k_frag = [&](const char* k, int s) {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(k + k_at + L::k_step(s)));
    };
    auto v_frag = [&](const char* v, int i) {                    // i = s * DT + dt
      s16x4 x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const char* at = v + v_at + L::v_step(i / DT, h, i % DT);
        x[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(uintptr_t)(__attribute__((address_space(3))) const char*)at);
      }
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    bf16x8 kf[AHEAD], vf[AHEAD];
    uint32_t bp[8];                                              // P of 32 keys, two a word
    f32x16 z[2];
    auto first_k = [&](const char* k) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) kf[i] = k_frag(k, i);
    };
    // Probabilities of zc's pairs of elements, in place, in three stages a slot apart: an exponential's
    // latency is behind an MFMA and another pair's work.  The empty asm statements keep what is computed
    // beside an MFMA in its place.
    float sum[2];
    uint32_t ones = 0x3f803f80;                                  // two bf16 of 1
    asm volatile("" : "+s"(ones));
    auto scale = [&](f32x16& zc, int k) {
      zc[2 * k] = fmaf(zc[2 * k], c2, -ref.off);
      zc[2 * k + 1] = fmaf(zc[2 * k + 1], c2, -ref.off);
    };
    auto raise = [&](f32x16& zc, int k) {
      zc[2 * k] = fast_exp2(zc[2 * k]);
      zc[2 * k + 1] = fast_exp2(zc[2 * k + 1]);
    };
    auto finish = [&](const f32x16& zc, int k) {
      sum[0] = k ? sum[0] + zc[2 * k] : zc[0];
      sum[1] = k ? sum[1] + zc[2 * k + 1] : zc[1];
      bp[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{zc[2 * k], zc[2 * k + 1]}), bf16x2));
      if (k & 1)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          rounded[i] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, bp[k - 1 + i]),
                                                       __builtin_bit_cast(bf16x2, ones), rounded[i], false);
      asm volatile("" : "+v"(bp[k]), "+v"(sum[0]), "+v"(sum[1]), "+v"(rounded[0]), "+v"(rounded[1]));
    };
    auto weigh = [&](f32x16& zc, int k) {
      if (k + 1 < 8) raise(zc, k + 1);
      if (k + 2 < 8) scale(zc, k + 2);
      finish(zc, k);
    };
    // scores of the block at k into zn, beside the probabilities of zc (into bp; the block at v is zc's)
    auto scores = [&](f32x16& zn, f32x16& zc, const char* k, const char* v) {
      scale(zc, 0);
      scale(zc, 1);
      raise(zc, 0);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        zn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % AHEAD], q.f[i], i ? zn : f32x16{}, 0, 0, 0);
        if (i + AHEAD < KS) kf[i % AHEAD] = k_frag(k, i + AHEAD);
        else vf[i + AHEAD - KS] = v_frag(v, i + AHEAD - KS);
#pragma unroll
        for (int e = i * 8 / KS; e < (i + 1) * 8 / KS; ++e) weigh(zc, e);
        __builtin_amdgcn_sched_barrier(0);
      }
      l += sum[0] + sum[1];
    };
    // acc += P V of the block at v, beside the maximum of zn, which it returns; the first fragments of
    // the scores after these come from k
    auto values = [&](const f32x16& zn, const char* v, const char* k) {
      float zm = -INFINITY;
#pragma unroll
      for (int i = 0; i < VS; ++i) {
        const int s = 4 * (i / DT);
        const bf16x8 b = __builtin_bit_cast(bf16x8, (u32x4{bp[s], bp[s + 1], bp[s + 2], bp[s + 3]}));
        acc[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i % AHEAD], b, acc[i % DT], 0, 0, 0);
        if (i + AHEAD < VS) vf[i % AHEAD] = v_frag(v, i + AHEAD);
        else kf[i + AHEAD - VS] = k_frag(k, i + AHEAD - VS);
#pragma unroll
        for (int e = i * 16 / VS; e < (i + 1) * 16 / VS; e += 2) {
          zm = fmaxf(fmaxf(zm, zn[e]), zn[e + 1]);
          asm volatile("" : "+v"(zm));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      return zm;
    };
    // keys of the 32 from page p on that the lane's query does not see: -inf
    auto hide = [&](f32x16& zn, int p, uint32_t valid) {
      const int key = p * HK_PAGE;
      if (valid == 0xffffffffu && key + 32 <= seen_all) return;
      const int k = seen - key;
      uint32_t x = (valid & (k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u)) >> (4 * hi);
      asm volatile("" : "+v"(x));                                // (a branch, not selects in every block)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!((x >> ((e & 3) + 8 * (e >> 2))) & 1u)) zn[e] = -INFINITY;
    };
    // a new reference where a score of zn has outgrown it (zm: the lane's largest)
    auto refer = [&](f32x16& zn, float zm) {
      zm *= c2;
      if (__builtin_expect(__any(zm > ref.limit), 0)) {
        zm = fmaxf(zm, __shfl_xor(zm, 32, 64));
        const float alpha = ref.move(fmaxf(ref.m, ceilf(zm)), bias);
        l *= alpha;
        rounded[0] *= alpha;
        rounded[1] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[dt][e] *= alpha;
        ref.bring(zn, c2);
      }
    };
    // rows of V with infinite values that not every query of the tile sees (zeros in LDS)
    auto add_odd = [&](uint32_t odd, int p, uint32_t valid) {
      while (odd) {
        const int key = __builtin_ctz(odd), reg = (key & 3) + 4 * (key >> 3);
        odd &= odd - 1;
        const int at = min(max(w.trow[min(p + key / HK_PAGE, w.p1 - 1)], 0), a.num_pages - 1);
        const uint16_t* vr = reinterpret_cast<const uint16_t*>(a.v_pool) + ((size_t)at * HK_PAGE + key % HK_PAGE) * D;
        uint32_t two = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) two = reg / 2 == e ? bp[e] : two;
        asm volatile("" : "+v"(two));
        float pr = __uint_as_float(reg & 1 ? two & 0xffff0000u : two << 16);
        pr = __shfl(pr, (lane & 31) + 32 * ((key >> 2) & 1), 64);
        const bool sees = ((valid >> key) & 1u) && p * HK_PAGE + key < seen;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = M::value(vr[32 * dt + (e & 3) + 8 * (e >> 2) + 4 * hi]);
            acc[dt][e] = sees ? fmaf(pr, x, acc[dt][e]) : acc[dt][e];
          }
      }
    };
    uint32_t valid[LEAD + 1];                                    // of tiles t .. t + LEAD
    int slot = 0;                                                // of V of tile t
    auto behind = [&](int n) { return slot + n >= NV ? slot + n - NV : slot + n; };
    auto turn = [&](int t) {
      if (t + LEAD - 1 < tiles) direct_wait<2 * L::LOADS>();
      else direct_wait<0>();
      if (is_v && unseen(t + 1) && t + 1 < tiles) settle(t + 1, (valid[1] >> (16 * my)) & 0xffffu, behind(1));
      asm volatile("s_barrier" ::: "memory");
      const int i = (t + LEAD) & 63;
      if (i == 0) {
        ids = next_ids;
        masks = next_masks;
        load_ids(t + LEAD + 64);
      }
      valid[LEAD] = __builtin_amdgcn_readlane(masks, i);
      if (t + LEAD - is_v < tiles)
        request(__builtin_amdgcn_readlane(ids, i), (valid[LEAD - 1] >> (16 * my)) & 0xffffu,
                is_v ? lds_v + behind(NV - 1) * L::BYTES : lds_k + ((t + 1) & (NK - 1)) * L::BYTES);
    };
    auto first_read = [&] {                                      // K of tile 0 is read: tile 4's takes its slot
      asm volatile("s_barrier" ::: "memory");
      if (NK < tiles && !is_v) request(__builtin_amdgcn_readlane(ids, NK), 0, lds_k);
    };
    auto advance = [&] {
#pragma unroll
      for (int i = 0; i < LEAD; ++i) valid[i] = valid[i + 1];
      slot = behind(1);
    };
    if (tiles > 0) {
      load_ids(0);
      ids = next_ids;
      masks = next_masks;
#pragma unroll
      for (int i = 0; i < LEAD; ++i) valid[i] = __builtin_amdgcn_readlane(masks, i);
#pragma unroll
      for (int i = 0; i < NK; ++i)
        if (i < tiles)
          request(__builtin_amdgcn_readlane(ids, i + is_v), (valid[i] >> (16 * my)) & 0xffffu,
                  is_v ? lds_v + i * L::BYTES : lds_k + i * L::BYTES);
      if (tiles >= NK) direct_wait<2 * L::LOADS>();
      else direct_wait<0>();
      load_ids(64);
      if (is_v && unseen(0)) settle(0, (valid[0] >> (16 * my)) & 0xffffu, 0);
      __syncthreads();
    }
    if (w0 >= w.rows) {                                          // a wave without rows brings its pages
      if (tiles > 0) first_read();
      for (int t = 0; t < tiles; ++t, advance()) turn(t);
      continue;
    }
    // the queries are here before the loop, where a wait for them would be one for the next tile too
#pragma unroll
    for (int i = 0; i < KS; ++i) asm volatile("" : "+v"(q.f[i]));
    if (tiles > 0) {
      first_k(s_k[0]);
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        z[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % AHEAD], q.f[i], i ? z[0] : f32x16{}, 0, 0, 0);
        if (i + AHEAD < KS) kf[i % AHEAD] = k_frag(s_k[0], i + AHEAD);
      }
      hide(z[0], w.p0, valid[0]);
      float zm = z[0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) zm = fmaxf(zm, z[0][e]);
      refer(z[0], zm);
      first_read();
      first_k(s_k[1]);
    }
    auto step = [&](int t, f32x16& zc, f32x16& zn) {
      __builtin_amdgcn_s_setprio(0);
      scores(zn, zc, s_k[(t + 1) & (NK - 1)], s_v[slot]);
      turn(t);
      __builtin_amdgcn_s_setprio(1);
      hide(zn, w.p0 + 2 * t + 2, valid[1]);
      const float zm = values(zn, s_v[slot], s_k[(t + 2) & (NK - 1)]);
      if (unseen(t)) {
        const uint32_t odd = __builtin_amdgcn_readfirstlane(s_odd[slot][0] | s_odd[slot][1] << 16);
        if (odd) add_odd(odd, w.p0 + 2 * t, valid[0]);
      }
      if (t + 1 < tiles) refer(zn, zm);
      advance();
    };
    for (int t = 0; t < tiles; t += 2) {
      step(t, z[0], z[1]);
      if (t + 1 < tiles) step(t + 1, z[1], z[0]);
    }
    l += __shfl_xor(l, 32, 64);
    float of_o = rounded[0] + rounded[1];
    of_o += __shfl_xor(of_o, 32, 64);
    if (w0 + (lane & 31) < w.rows)
      put_state<uint16_t, D>(a, row, pieces.state < 0 ? -1 : pieces.state + r - w.r0, acc, ref.whole(bias), l, of_o);
  }
}

// ------------------------------------------------------------------ short kernels
constexpr int SHORT_NT = 256, SHORT_NW = SHORT_NT / 64;

constexpr int SHORT_WG = 512;                 // workgroups of a launch: two a CU
constexpr int STEP_PAGES = 8;                 // pages of a step, two a wave

// A row of the short kernels: the chunk of head h's sequence, its folded rows (0: not a short one),
// and the pages and steps that its last token sees.
struct ShortRow {
  Chunk c;
  int rows, end, pages, steps;
};
__device__ __forceinline__ ShortRow short_row(const Args& a, int h) {
  ShortRow r;
  const int n = min(max(a.n_pages[h], 0), a.max_pages);
  r.c = chunk_of(a.start, h / a.Hkv, a.n_tokens, a.max_len);
  r.rows = r.c.len * a.G <= SHORT_ROWS ? r.c.len * a.G : 0;
  r.end = row_end(n, n > 0 ? a.masks[(size_t)h * a.max_pages + n - 1] : 0u);
  r.pages = tile_pages(n, r.end, r.c.len, r.c.len - 1);
  // (a row without pages still has its empty result to write)
  r.steps = r.rows > 0 ? max((r.pages + STEP_PAGES - 1) / STEP_PAGES, 1) : 0;
  return r;
}

// The steps of all rows lie behind one another, and every workgroup takes an equal run of them:
// rows of any mixture of lengths fill the chip evenly, and a launch has no idle workgroups.  Each
// workgroup sums the rows' steps itself.
struct ShortRuns {
  int total, share;
};
__device__ inline ShortRuns short_runs(const Args& a, int (&s_first)[SHORT_NT + 1]) {
  __shared__ int s_sum[SHORT_NW], s_most[SHORT_NW];
  const int heads = a.n_seq * a.Hkv, per = (heads + SHORT_NT - 1) / SHORT_NT;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = 0, most = 0;
  for (int h = threadIdx.x * per; h < min((int)(threadIdx.x + 1) * per, heads); ++h) {
    const int k = short_row(a, h).steps;
    sum += k;
    most = max(most, k);
  }
  int x = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  most = (int)wave_reduce_u32((uint32_t)most, 0u, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
  if (lane == 63) {
    s_sum[wave] = x;
    s_most[wave] = most;
  }
  __syncthreads();
  ShortRuns u = {0, 0};
  int before = x - sum;
#pragma unroll
  for (int w = 0; w < SHORT_NW; ++w) {
    if (w < wave) before += s_sum[w];
    u.total += s_sum[w];
    most = max(most, s_most[w]);
  }
  // a row is shared by MAX_STATES workgroups at most
  u.share = max((u.total + SHORT_WG - 1) / SHORT_WG, (most + MAX_STATES - 2) / (MAX_STATES - 1));
  s_first[threadIdx.x] = before;
  if (threadIdx.x == 0) s_first[SHORT_NT] = u.total;
  if (blockIdx.x == gridDim.x - 1) {          // for the merge
    int32_t* first = a.short_first;
    for (int h = threadIdx.x * per; h < min((int)(threadIdx.x + 1) * per, heads); ++h) {
      first[h] = before;
      before += short_row(a, h).steps;
    }
    if (threadIdx.x == 0) {
      first[heads] = u.total;
      first[heads + 1] = u.share;
    }
  }
  __syncthreads();
  return u;
}

// A workgroup's next piece of a row: head h, its steps [from, to).
struct Piece {
  int h, from, to;
  ShortRow row;
};
// The piece that begins at step x of the launch and ends before step `stop` at the latest.  The same
// in every lane.
__device__ inline Piece short_piece(const Args& a, const int (&s_first)[SHORT_NT + 1], int x, int stop) {
  const int heads = a.n_seq * a.Hkv, per = (heads + SHORT_NT - 1) / SHORT_NT, lane = threadIdx.x & 63;
  int t = 0;                                  // the last thread whose rows begin at or before x
  for (int hi = SHORT_NT; hi - t > 1;) {
    const int mid = (t + hi) / 2;
    if (s_first[mid] <= x) t = mid;
    else hi = mid;
  }
  int first = s_first[t];
  Piece p;
  for (int h0 = t * per;; h0 += 64) {
    const int h = h0 + lane;
    const bool mine = h < heads && h < (t + 1) * per;
    const ShortRow r = short_row(a, mine ? h : heads - 1);
    const int k = mine ? r.steps : 0;
    int y = k;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int z = __shfl_up(y, o, 64);
      if (lane >= o) y += z;
    }
    const unsigned long long in = __ballot(first + y > x);
    if (in || h0 + 64 >= heads) {
      const int l = __builtin_amdgcn_readfirstlane(in ? __builtin_ctzll(in) : 63);
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      p.h = min(h0 + l, heads - 1);
      p.from = x - of(first + y - k);
      p.row = {{of(r.c.first), of(r.c.len)}, of(r.rows), of(r.end), of(r.pages), of(r.steps)};
      break;
    }
    first += __shfl(y, 63, 64);
  }
  p.to = min(p.row.steps, p.from + stop - x);
  return p;
}

// The four waves' states, summed against one reference, are the workgroup's result: the row's where
// the piece is all of it, one of the row's states otherwise.  A workgroup has at most two states: of
// the row that it begins in the middle of (0), and of the one that it begins and does not end (1).
// s_o: 32 x (D / 2 + 4) floats a wave, used for one half of the dims after the other.
template <typename T, int D>
__device__ __forceinline__ void join_waves(const Args& a, const Piece& w, const f32x16 (&acc)[D / 32], float mb, float l,
                                           float* s_o, float (*s_m)[32], float (*s_l)[32]) {
  constexpr int HD = D / 2, OP = HD + 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hi = lane >> 5, kv = w.h % a.Hkv;
  l += __shfl_xor(l, 32, 64);
  __syncthreads();                            // (s_o may be the waves' tiles)
  if (hi == 0) {
    s_m[wave][lane] = l == 0.f ? -INFINITY : mb;
    s_l[wave][lane] = l;
  }
  __syncthreads();
  auto whole = [&](int q, float& m) {         // reference and sum of query q
    m = -INFINITY;
#pragma unroll
    for (int v = 0; v < SHORT_NW; ++v) m = fmaxf(m, s_m[v][q]);
    float x = 0.f;
#pragma unroll
    for (int v = 0; v < SHORT_NW; ++v) x += m == -INFINITY ? s_l[v][q] : s_l[v][q] * fast_exp2(s_m[v][q] - m);
    return x;                                 // (0 or NaN where there is no reference)
  };
  float M_;
  whole(lane & 31, M_);
  const float own = M_ == -INFINITY ? 0.f : fast_exp2(s_m[wave][lane & 31] - M_);
  // eight threads of a query's dims each
  const int qr = threadIdx.x >> 3, d0 = (threadIdx.x & 7) * (HD / 8);
  const float l_all = whole(qr, M_);
  const int tq = qr / a.G;
  const int64_t row = (int64_t)(w.row.c.first + tq) * a.Hq + kv * a.G + (qr - tq * a.G);
  const bool part = w.from > 0 || w.to < w.row.steps;
  const float inv = part ? 1.f : l_all == 0.f ? 0.f : 1.f / l_all;   // (a NaN stays one)
  const int64_t state = (int64_t)(2 * blockIdx.x + (w.from > 0 ? 0 : 1)) * SHORT_ROWS + qr;
  float* po = a.short_o + state * D;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half) __syncthreads();
#pragma unroll
    for (int dt = 0; dt < D / 64; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x16& x = acc[half * (D / 64) + dt];
        *reinterpret_cast<f32x4*>(s_o + (wave * 32 + (lane & 31)) * OP + 32 * dt + 8 * j + 4 * hi) =
            f32x4{x[4 * j] * own, x[4 * j + 1] * own, x[4 * j + 2] * own, x[4 * j + 3] * own};
      }
    __syncthreads();
    if (qr < w.row.rows)
#pragma unroll
      for (int d = 0; d < HD / 8; d += 4) {
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < SHORT_NW; ++v) t += *reinterpret_cast<const f32x4*>(s_o + (v * 32 + qr) * OP + d0 + d);
        t *= inv;
        const int at = half * HD + d0 + d;
        if (part) *reinterpret_cast<f32x4*>(po + at) = t;
        else Mma<T, D>::put4(reinterpret_cast<T*>(a.o) + row * D + at, t[0], t[1], t[2], t[3]);
      }
  }
  if (qr < w.row.rows && (threadIdx.x & 7) == 0) {
    if (part) *reinterpret_cast<f32x2*>(a.short_ml + state * 2) = f32x2{M_, l_all};
    else if (a.lse) a.lse[row] = lse_of(M_, l_all);
  }
  __syncthreads();                            // the next piece writes the tiles
}

// Pages go through a wave's own part of LDS, two of K and two of V a step, and are requested a step
// ahead.  Two workgroups a CU, but for fp32 of 128.  Bound by HBM reads: 64 sequences of 1 to 8 tokens over 784 to
// 5600, 32/8 heads of 128: 165 to 171 us, 850 MB by the counter at 5.0 TB/s; 164 without the products and
// the softmax, and no faster with twice the loads in flight or with more workgroups (1024: 178).  fp32,
// 16 sequences of 1 to 6 tokens over 2000: heads of 64 39 us, of 128, where a CU has one workgroup, 78.
template <typename T, int D>
__global__ __launch_bounds__(SHORT_NT, sizeof(T) * D <= 256 ? 2 : 1) void chunk_short_kernel(Args a) {
  using L = TileLayout<T, D>;
  using M = Mma<T, D>;
  constexpr int WP = STEP_PAGES / SHORT_NW;
  static_assert(WP == 2, "a wave's step is 32 keys");
  constexpr int WAVE = 32 * (L::K_ROW + L::V_ROW);
  static_assert(WAVE >= 32 * (D / 2 + 4) * 4, "the join's sums fit the tiles");
  __shared__ __align__(16) char s_buf[SHORT_NW * WAVE];
  __shared__ float s_m[SHORT_NW][32], s_l[SHORT_NW][32];
  __shared__ int s_first[SHORT_NT + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ShortRuns u = short_runs(a, s_first);
  char* my_k = s_buf + wave * WAVE;
  char* my_v = my_k + 32 * L::K_ROW;
  const int stop = min((int)(blockIdx.x + 1) * u.share, u.total);
  for (int x = blockIdx.x * u.share; x < stop;) {
    const Piece w = short_piece(a, s_first, x, stop);
    x += w.to - w.from;
    const int kv = w.h % a.Hkv, r = min(lane & 31, w.row.rows - 1), tok = r / a.G, off = w.row.end - w.row.c.len + 1;
    const int seen = off + tok, seen_all = off;
    const int32_t* trow = a.table + (size_t)w.h * a.max_pages;
    const uint16_t* mrow = a.masks + (size_t)w.h * a.max_pages;
    const int p0 = w.from * STEP_PAGES, p1 = min(w.to * STEP_PAGES, w.row.pages);
    typename M::Query q;
    M::load_q(q, reinterpret_cast<const T*>(a.q) + (int64_t)(w.row.c.first + tok) * a.q_row + (kv * a.G + (r - tok * a.G)) * D);
    const float bias = bias_of(w.row.pages);
    State<T, D> st;
    st.init();
    PageRegs<T, D> rk[WP], rv[WP];
    int id[WP];
    uint32_t mask[WP], next_mask[WP];
    auto page_id = [&](int p) { return min(max(trow[min(p, p1 - 1)], 0), a.num_pages - 1); };
    auto load_id = [&](int t) {
#pragma unroll
      for (int i = 0; i < WP; ++i) {
        const int p = p0 + t * STEP_PAGES + wave * WP + i;
        next_mask[i] = p < p1 ? mrow[p] : 0u;
        id[i] = page_id(p);
      }
    };
    auto load = [&] {
#pragma unroll
      for (int i = 0; i < WP; ++i) rk[i].load(a.k_pool, id[i]);
#pragma unroll
      for (int i = 0; i < WP; ++i) rv[i].load(a.v_pool, id[i]);
    };
    const int steps = p1 > p0 ? w.to - w.from : 0;
    if (steps > 0) {
      load_id(0);
      load();
    }
    for (int t = 0; t < steps; ++t) {
      // the wave's own region of LDS: its reads of the last step are done before these writes, in
      // the order of its instructions
      const int p = p0 + t * STEP_PAGES + wave * WP, key = p * HK_PAGE;
#pragma unroll
      for (int i = 0; i < WP; ++i) mask[i] = next_mask[i];
      load_id(t + 1);
      uint32_t odd = 0;
      const uint32_t valid = mask[0] | mask[1] << 16;
#pragma unroll
      for (int i = 0; i < WP; ++i) rk[i].store(my_k + i * HK_PAGE * L::K_ROW, L::K_ROW);
#pragma unroll
      for (int i = 0; i < WP; ++i) {
        uint32_t keep = mask[i];
        if ((p + i + 1) * HK_PAGE > seen_all) {
          const uint32_t o = rv[i].odd_rows() & keep;
          keep &= ~o;
          odd |= o << (16 * i);
        }
        if (keep != 0xffffu) rv[i].clear(keep);
        rv[i].store(my_v + i * HK_PAGE * L::V_ROW, L::V_ROW);
      }
      load();                                 // (past the last step its pages once more, with no valid slot)
      const bool all = valid == 0xffffffffu && key + 32 <= seen_all;
      const int k = seen - key;
      const uint32_t vis = valid & (k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u);
      __builtin_amdgcn_wave_barrier();
      st.block(q, my_k, my_v, vis, all, a.c2, down_of(bias), __builtin_amdgcn_readfirstlane(odd), [&](int j) {
        return reinterpret_cast<const T*>(a.v_pool) + ((size_t)page_id(p + j / HK_PAGE) * HK_PAGE + j % HK_PAGE) * D;
      });
      __builtin_amdgcn_wave_barrier();
    }
    join_waves<T, D>(a, w, st.acc, st.ref.whole(bias), st.l, reinterpret_cast<float*>(s_buf), s_m, s_l);
  }
}

// ------------------------------------------------------------------ merge
// D / 4 lanes per query: the states of its row's pieces, in their order.  Lanes read the references and
// sums of the pieces (at most 64) side by side, and four dims of eight pieces' outputs at a time.
// Bound by reading the states: 12 us for 30 MB.
constexpr int MERGE_NT = 256;
template <int D>
constexpr int MERGE_ROWS = MERGE_NT / (D / 4);                   // of a workgroup at a time

template <typename T, int D, typename F>
__device__ __forceinline__ void merge_states(const Args& a, int64_t row, int used, const float* o_states,
                                             const float* ml_states, F at) {
  constexpr int LANES = D / 4, PER = MAX_STATES / LANES, U = 8;
  const int lane = threadIdx.x % LANES;
  f32x2 ml[PER];
  float M_ = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int j = i * LANES + lane;
    ml[i] = f32x2{-INFINITY, 0.f};
    if (j < used) ml[i] = *reinterpret_cast<const f32x2*>(ml_states + at(j) * 2);
    M_ = fmaxf(M_, ml[i][0]);
  }
#pragma unroll
  for (int x = 1; x < LANES; x <<= 1) M_ = fmaxf(M_, __shfl_xor(M_, x, 64));
  // (no valid key anywhere: sums of 0, or NaN)
  auto factor = [&](float m) { return M_ == -INFINITY ? 1.f : fast_exp2(m - M_); };
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i * LANES + lane < used) l += ml[i][1] * factor(ml[i][0]);
#pragma unroll
  for (int x = 1; x < LANES; x <<= 1) l += __shfl_xor(l, x, 64);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < used; j0 += U) {
    f32x4 x[U];
    float m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t state = at(min(j0 + u, used - 1));
      x[u] = *reinterpret_cast<const f32x4*>(o_states + state * D + lane * 4);
      m[u] = ml_states[state * 2];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float f = factor(m[u]);
      if (j0 + u < used && f != 0.f)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(x[u][e], f, o[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;   // (a NaN stays one)
  Mma<T, D>::put4(reinterpret_cast<T*>(a.o) + row * D + lane * 4, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  if (lane == 0 && a.lse) a.lse[row] = lse_of(M_, l);
}

// Tiles in pieces: tile_y workgroups each; then the short rows of a head: MERGE_Y each.
constexpr int MERGE_Y = 4;
template <typename T, int D>
__global__ __launch_bounds__(MERGE_NT) void chunk_merge_kernel(Args a, int tile_wg, int tile_y) {
  int r = threadIdx.x / (D / 4);
  if ((int)blockIdx.x < tile_wg) {
    const TileSplit t = reinterpret_cast<const TileSplit*>(a.tile_split)[blockIdx.x / tile_y];
    if (t.used <= 1) return;                  // written as it is
    for (r += blockIdx.x % tile_y * MERGE_ROWS<D>; r < min(TILE_ROWS, t.rows - t.r0); r += tile_y * MERGE_ROWS<D>) {
      const int tok = (t.r0 + r) / a.G;
      const int64_t row = (int64_t)(t.first + tok) * a.Hq + t.kv * a.G + (t.r0 + r - tok * a.G);
      merge_states<T, D>(a, row, t.used, a.tile_o, a.tile_ml,
                         [&](int j) { return (int64_t)(t.at + j) * TILE_ROWS + r; });
    }
    return;
  }
  const int x = blockIdx.x - tile_wg, h = x / MERGE_Y, heads = a.n_seq * a.Hkv;
  const int first = a.short_first[h], steps = a.short_first[h + 1] - first, share = a.short_first[heads + 1];
  const Chunk c = chunk_of(a.start, h / a.Hkv, a.n_tokens, a.max_len);
  if (steps <= 0) return;
  const int w0 = first / share, used = (first + steps - 1) / share - w0 + 1;
  if (used <= 1) return;                      // written as it is
  for (r += x % MERGE_Y * MERGE_ROWS<D>; r < c.len * a.G; r += MERGE_Y * MERGE_ROWS<D>) {
    const int tok = r / a.G;
    const int64_t row = (int64_t)(c.first + tok) * a.Hq + (h % a.Hkv) * a.G + (r - tok * a.G);
    merge_states<T, D>(a, row, used, a.short_o, a.short_ml, [&](int j) {
      return (int64_t)(2 * (w0 + j) + (j == 0 ? 1 : 0)) * SHORT_ROWS + r;
    });
  }
}

// Workgroups of a call.  heads: of the short kernel, 0 where no row can be a short one; tiles: numbers
// of tiles of a KV head; pieces: most of them that a planned launch makes, 0 for one of many tiles.
// The host knows no lengths, so it numbers a tile more for every sequence: with 8 KV heads, batches of
// about 125 sequences have no pieces, whatever they hold (500 tokens over 20000 among 127 single tokens
// 2209 us, the single tokens alone 1795; among 31 638, and about 440 by that rate).
struct Plan {
  int heads, tiles, pieces;
};
static int most_pieces(long long tiles, int max_pages) {
  const int steps = std::max((max_pages + TILE_PAGES - 1) / TILE_PAGES, 1);
  return (int)std::min<long long>(tiles * std::min(steps, MAX_STATES), PLAN_PIECES);
}
static Plan plan(int NS, int Hq, int Hkv, int cost, int n_tokens, int max_len, int max_pages) {
  const int G = Hq / Hkv;
  const long long rows = (long long)n_tokens * G;
  const bool tiles = (long long)max_len * G > SHORT_ROWS && rows > SHORT_ROWS;
  Plan p;
  p.heads = G <= SHORT_ROWS ? NS * Hkv : 0;
  p.tiles = tiles ? (int)(rows / TILE_ROWS + NS) : 0;
  const long long all = (long long)p.tiles * Hkv;
  // (rows of fewer than two costs of a piece gain nothing by pieces)
  p.pieces = all <= PLAN_TILES && max_pages >= 2 * cost * TILE_PAGES ? most_pieces(all, max_pages) : 0;
  return p;
}

template <typename T, int D>
static void launch(const Args& a, hipStream_t st, const Plan& p) {
  constexpr bool bf = sizeof(T) == 2;
  {
    TimedLaunch t(HK_TK_CHUNK_ATTN, st);
    if (p.tiles > 0) {
      const dim3 grid(p.pieces ? std::min(p.pieces, TILE_WG) : p.tiles * a.Hkv), block(2 * TILE_ROWS);
      if constexpr (bf) {
        if (p.pieces) hipLaunchKernelGGL((chunk_tile_bf16_kernel<D, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((chunk_tile_bf16_kernel<D, false>), grid, block, 0, st, a);
      } else {
        if (p.pieces) hipLaunchKernelGGL((chunk_tile_f32_kernel<D, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((chunk_tile_f32_kernel<D, false>), grid, block, 0, st, a);
      }
    }
    if (p.heads > 0) hipLaunchKernelGGL((chunk_short_kernel<T, D>), dim3(SHORT_WG), dim3(SHORT_NT), 0, st, a);
  }
  const int tiles = p.pieces ? p.tiles * a.Hkv : 0;
  // (one prompt of 500 among 31 single tokens, 392 tiles: 143 us, with 2048 here 149; others equal)
  const int tile_y = std::max(std::min(8192 / std::max(tiles, 1), TILE_ROWS / MERGE_ROWS<D>), 4);
  if (tiles * tile_y + p.heads * MERGE_Y == 0) return;
  TimedLaunch t(HK_TK_CHUNK_MERGE, st);
  hipLaunchKernelGGL((chunk_merge_kernel<T, D>), dim3(tiles * tile_y + p.heads * MERGE_Y), dim3(MERGE_NT), 0, st, a,
                     tiles * tile_y, tile_y);
}

}  // namespace hk

using namespace hk;

// States (rows of D + 2 floats) of the short kernel's workgroups, two each, and of the tiles' pieces,
// what the pieces are, and the short rows' first steps.  Grows with the tokens and does not depend on the type.
static size_t short_states(const Plan& p) { return p.heads ? (size_t)2 * SHORT_WG * SHORT_ROWS : 0; }
size_t hk_chunk_attn_ws(int NS, int Hq, int Hkv, int D, int n_tokens, int max_len, int max_pages) {
  const Plan p = plan(NS, Hq, Hkv, 0, n_tokens, max_len, max_pages);
  const int pieces = most_pieces(std::min<long long>((long long)p.tiles * Hkv, PLAN_TILES), max_pages);
  const size_t rows = short_states(p) + (size_t)pieces * TILE_ROWS;
  return rows * (D + 2) * sizeof(float) + PLAN_TILES * sizeof(TileSplit) + ((size_t)NS * Hkv + 2) * sizeof(int32_t);
}

long long hk_chunk_attn_threads(int NS, int Hq, int Hkv, int n_tokens, int max_len, int max_pages) {
  const Plan p = plan(NS, Hq, Hkv, 0, n_tokens, max_len, max_pages);
  return (long long)p.tiles * Hkv * (2 * TILE_ROWS);
}

hipError_t hk_launch_chunk_attn(int NS, int Hq, int Hkv, int D, const hk_paged_kv* kv, const hk_chunks* ch,
                                const void* q, int64_t q_row, float sm_scale, void* o, float* lse, void* ws,
                                hipStream_t st) {
  const bool bf = kv->dtype == HK_BF16;
  const Plan p = plan(NS, Hq, Hkv, bf ? Cost<uint16_t>::STATE : Cost<float>::STATE, ch->n_tokens, ch->max_len, kv->max_pages);
  Args a;
  a.q = static_cast<const char*>(q);
  a.k_pool = static_cast<const char*>(kv->k_pool);
  a.v_pool = static_cast<const char*>(kv->v_pool);
  a.table = kv->page_table;
  a.n_pages = kv->n_pages;
  a.start = ch->start;
  a.masks = kv->page_mask;
  a.q_row = q_row;
  a.o = static_cast<char*>(o);
  a.lse = lse;
  a.n_tiles = p.tiles;
  const size_t ss = short_states(p), ts = (size_t)p.pieces * TILE_ROWS;
  a.short_o = static_cast<float*>(ws);
  a.tile_o = a.short_o + ss * D;
  a.short_ml = a.tile_o + ts * D;
  a.tile_ml = a.short_ml + ss * 2;
  a.tile_split = reinterpret_cast<int32_t*>(a.tile_ml + ts * 2);
  a.short_first = a.tile_split + PLAN_TILES * (sizeof(TileSplit) / sizeof(int32_t));
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.max_pages = kv->max_pages;
  a.num_pages = kv->num_pages;
  a.n_seq = NS;
  a.n_tokens = ch->n_tokens;
  a.max_len = ch->max_len;
  a.c2 = sm_scale * kLog2e;
  if (bf && D == 128) launch<uint16_t, 128>(a, st, p);
  else if (bf) launch<uint16_t, 64>(a, st, p);
  else if (D == 128) launch<float, 128>(a, st, p);
  else launch<float, 64>(a, st, p);
  return hipGetLastError();
}
