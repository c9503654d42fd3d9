// 8-bit cache: attention of single tokens and of chunks of new tokens over its pages (gfx950).
//
// The query rows of a KV head are folded: row r of a chunk is query head r % G of token r / G.  A
// workgroup takes ROWS of them and a range of the row's pages; its four waves take the range's pages
// two at a time in turn, every page read once, straight into registers, and meet at the end in LDS.
// attn8_merge_kernel joins the ranges of a row.
//
// With codes c and scales s of a key's row, a query's score is z = (q . ck) sk and its output
// sum p (sv cv) / sum p: the codes are exact in bf16 and go into the matrix products as they are, the
// scales are factors of the scores and of the probabilities, both in fp32.  Per block of 32 keys (two
// pages) and 16 rows, on 16x16x32 MFMAs:
//   scores  C[key][row] = K Q^T: lane l holds K's row l % 16 of a page, a quarter l / 16 of its dims (the
//           contraction's order is free, so that a lane loads 16 bytes in a row), and receives the four
//           keys 4 (l / 16) .. of row l % 16;
//   values  O^T[dim][row] += V^T P^T: the contraction runs over the keys in the order that the scores
//           lie in, so that P needs no move: lane l loads of those eight keys D / 16 dims from
//           l % 16 D / 16 on, and the conversion of its codes pairs the keys.
// q enters in one bf16 part, or for fp32 in three (exactly); P in two for bf16 results, to 2^-16 of a
// term, and in three for fp32 ones, to 2^-24.
//
// Softmax: one pass with a running reference m per row, a whole number that moves when a score exceeds
// it by 2^SLACK.  The sums of P V are kept smaller by 2^bias, at least their number of terms times
// 2^SLACK, so that they stay finite where the result does.
#include <algorithm>
#include <type_traits>

#include "hk_chunk.h"
#include "hk_kv8.h"

namespace hk {

constexpr int A8_NT = 256, A8_NW = 4;
constexpr float A8_SLACK = 4.f;
constexpr int A8_PPS = 128, A8_PPS_MIN = 8;   // pages of a range at most and at least
constexpr int A8_TARGET = 2048, A8_MOST = 4096;   // workgroups that a launch should have, and with ranges at most
constexpr int A8_ROWS = 32;                   // rows of a workgroup at most

struct Args8 {
  const void* q;
  int64_t q_row;                              // elements
  const char *k_pool, *v_pool;
  const float *k_scale, *v_scale;
  const int32_t *table, *n_pages, *start;     // start NULL: one token per sequence
  const uint16_t* masks;
  void* o;
  float *lse, *part_o, *part_ml;
  int Hq, Hkv, G, max_pages, num_pages, n_seq, n_tokens, max_len;
  int n_units, n_split, cap;                  // cap: rows of a unit in the workspace
  int one_tile;                               // no sequence has more rows than a workgroup
  float c2;
};

// ROWS folded rows of one sequence and KV head.
struct Unit {
  Chunk c;
  int h, kv, rows, r0, off, pages;            // off: keys before off + token are seen by that token
};
__device__ __forceinline__ int tiles8_before(const Args8& a, int rows, int s) {
  return min(max(a.start[s], 0), a.n_tokens) * a.G / rows + s;
}
// rows 0: there are none
template <int ROWS, bool CHUNK>
__device__ __forceinline__ Unit unit_of(const Args8& a, int u) {
  Unit w;
  w.kv = u % a.Hkv;
  const int tile = u / a.Hkv;
  int s = tile;
  w.r0 = 0;
  if (!CHUNK) {
    const int per = (a.G + ROWS - 1) / ROWS;
    s = tile / per;
    w.r0 = (tile - s * per) * ROWS;
    w.c = {s, 1};
  } else {
    if (!a.one_tile) {
      s = 0;
      for (int hi = a.n_seq; hi - s > 1;) {
        const int mid = (s + hi) / 2;
        if (tiles8_before(a, ROWS, mid) <= tile) s = mid;
        else hi = mid;
      }
      w.r0 = (tile - tiles8_before(a, ROWS, s)) * ROWS;
    }
    w.c = chunk_of(a.start, s, a.n_tokens, a.max_len);
  }
  w.rows = w.c.len * a.G;
  if (w.r0 < 0 || w.r0 >= w.rows) {
    w.rows = 0;
    return w;
  }
  w.h = s * a.Hkv + w.kv;
  const int n = min(max(a.n_pages[w.h], 0), a.max_pages);
  w.pages = n;
  w.off = 0;
  if (CHUNK) {
    const int end = row_end(n, n > 0 ? a.masks[(size_t)w.h * a.max_pages + n - 1] : 0u);
    w.off = end - w.c.len + 1;
    const int last = (min(w.r0 + ROWS, w.rows) - 1) / a.G;
    w.pages = min(n, (max(w.off + last, 0) + HK_PAGE - 1) / HK_PAGE);
  }
  return w;
}
// pages of a range, an even number: the row's pages spread over the launch's ranges
__device__ __forceinline__ int share8(const Args8& a, int pages) {
  const int even = ((pages + a.n_split - 1) / a.n_split + 1) & ~1;
  return max(even, A8_PPS_MIN);
}

// log of l 2^m; the powers of two of both cancel as whole numbers
__device__ __forceinline__ float lse8(float m, float l) {
  if (l == 0.f) return -INFINITY;
  return (m + (float)__builtin_amdgcn_frexp_expf(l) + __log2f(__builtin_amdgcn_frexp_mantf(l))) * kLn2;
}

// fp32 in N bf16 parts, of two values a word: N 1: exact ones, 2: to 2^-16, 3: all of its bits
template <int N>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&out)[N]) {
  if constexpr (N == 1) {
    out[0] = pack_bf16(x, y);
  } else if constexpr (N == 2) {
    out[0] = pack_bf16(x, y);
    out[1] = pack_bf16(x - bf16_lo(out[0]), y - bf16_hi(out[0]));
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      out[i] = high_halves(x, y);
      x -= bf16_lo(out[i]);
      y -= bf16_hi(out[i]);
    }
  }
}

// Codes of two pages on their way: see above for what a lane holds.
template <int D>
struct Block8 {
  static constexpr int KW = D / 16, VW = D / 64;          // words of a K row's quarter, of a V row's piece
  uint32_t k[2][KW], v[8][VW];
  f32x4 ks[2], vs[2];
  uint32_t mask;
  __device__ __forceinline__ void load(const Args8& a, int id0, int id1, uint32_t m) {
    const int lane = threadIdx.x & 63, i16 = lane & 15, qd = lane >> 4;
    mask = m;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const size_t page = (size_t)(t ? id1 : id0);
      const char* kp = a.k_pool + page * (HK_PAGE * D) + (i16 * D + qd * (D / 4));
#pragma unroll
      for (int i = 0; i < KW / 4; ++i) *reinterpret_cast<u32x4*>(&k[t][4 * i]) = reinterpret_cast<const u32x4*>(kp)[i];
      const char* vp = a.v_pool + page * (HK_PAGE * D) + (4 * qd * D + i16 * (D / 16));
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (VW == 2) *reinterpret_cast<u32x2*>(&v[4 * t + r][0]) = *reinterpret_cast<const u32x2*>(vp + r * D);
        else v[4 * t + r][0] = *reinterpret_cast<const uint32_t*>(vp + r * D);
      }
      ks[t] = *reinterpret_cast<const f32x4*>(a.k_scale + page * HK_PAGE + 4 * qd);
      vs[t] = *reinterpret_cast<const f32x4*>(a.v_scale + page * HK_PAGE + 4 * qd);
    }
  }
};

__device__ __forceinline__ f32x4 mma8(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// QP: bf16 parts of q (1: q is bf16), PP: of P (2: o is bf16, 3: fp32)
template <int F, int D, int NQ, int QP, int PP, bool CHUNK>
__global__ __launch_bounds__(A8_NT, QP == 3 && NQ == 2 ? 1 : 2) void attn8_kernel(Args8 a) {
#pragma clang fp contract(off)
  constexpr int ROWS = 16 * NQ, KS = D / 32, DT = D / 16;
  __shared__ f32x4 s_acc[2][NQ * DT][64];
  __shared__ float s_m[A8_NW][NQ][16], s_l[A8_NW][NQ][16];
  const int lane = threadIdx.x & 63, i16 = lane & 15, qd = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int u = blockIdx.x / a.n_split, split = blockIdx.x - u * a.n_split;
  const Unit w = unit_of<ROWS, CHUNK>(a, u);
  if (w.rows == 0) return;
  const int share = share8(a, w.pages), p0 = split * share, p1 = min(p0 + share, w.pages);
  if (p0 >= w.pages && split > 0) return;
  const int32_t* trow = a.table + (size_t)w.h * a.max_pages;
  const uint16_t* mrow = a.masks + (size_t)w.h * a.max_pages;

  u32x4 qf[NQ][QP][KS];
  int seen[NQ];                               // keys before this one are seen by the lane's row
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    const int r = min(w.r0 + 16 * nq + i16, w.rows - 1), tok = r / a.G, g = r - tok * a.G;
    seen[nq] = w.off + tok;
    const int64_t at = (int64_t)(w.c.first + tok) * a.q_row + (w.kv * a.G + g) * D + qd * (D / 4);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      if constexpr (QP == 1) {
        qf[nq][0][s] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + at + 8 * s);
      } else {
        const f32x4 x = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + at + 8 * s);
        const f32x4 y = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + at + 8 * s + 4);
        uint32_t part[4][QP];
        split_pair<QP>(x[0], x[1], part[0]);
        split_pair<QP>(x[2], x[3], part[1]);
        split_pair<QP>(y[0], y[1], part[2]);
        split_pair<QP>(y[2], y[3], part[3]);
#pragma unroll
        for (int i = 0; i < QP; ++i) qf[nq][i][s] = u32x4{part[0][i], part[1][i], part[2][i], part[3][i]};
      }
    }
  }
  const int seen_all = w.off + w.r0 / a.G;    // by every row of the workgroup
  const int bias = (int)A8_SLACK + 33 - __clz(max(p1 - p0, 1) * HK_PAGE);
  const float down = __uint_as_float((uint32_t)(127 - bias) << 23), back = __uint_as_float((uint32_t)(127 + bias) << 23);

  float m[NQ], l[NQ];
  f32x4 acc[NQ][DT];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    m[nq] = -INFINITY;
    l[nq] = 0.f;
#pragma unroll
    for (int j = 0; j < DT; ++j) acc[nq][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // P V of dims 4 j + 2 H and 4 j + 2 H + 1: the codes' pairs turned into pairs of keys
  auto values = [&](auto half, const Block8<D>& b, const u32x4 (&pf)[NQ][PP], int j) {
    constexpr int H = decltype(half)::value;
    u32x4 vf[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = b.v[2 * i][j], y = b.v[2 * i + 1][j];
      if constexpr (F == HK_I8) {
        vf[0][i] = high_halves(Code<F>::template value<2 * H>(x), Code<F>::template value<2 * H>(y));
        vf[1][i] = high_halves(Code<F>::template value<2 * H + 1>(x), Code<F>::template value<2 * H + 1>(y));
      } else {
        const uint32_t px = Code<F>::template pair<H>(x), py = Code<F>::template pair<H>(y);
        vf[0][i] = __builtin_amdgcn_perm(py, px, 0x05040100u);
        vf[1][i] = __builtin_amdgcn_perm(py, px, 0x07060302u);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
        for (int i = PP - 1; i >= 0; --i)
          acc[nq][4 * j + 2 * H + h] = mma8(vf[h], pf[nq][i], acc[nq][4 * j + 2 * H + h]);
  };
  // 32 keys from page p on
  auto compute = [&](Block8<D>& b, int p) {
    const bool full = b.mask == 0xffffffffu && (!CHUNK || (p + 2) * HK_PAGE <= seen_all);
    // the lane's keys 4 t + r: slot 4 qd + r of page t
    const uint32_t valid = ((b.mask >> (4 * qd)) & 15u) | ((b.mask >> (16 + 4 * qd)) & 15u) << 4;
    if (F == HK_E4M3 && b.mask != 0xffffffffu) {
      // a slot that is not valid may hold codes that stand for NaN
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < Block8<D>::VW; ++j) b.v[i][j] = (valid >> i) & 1u ? b.v[i][j] : 0u;
    }
    f32x4 z[NQ][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) z[nq][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        // (here and below: one product's codes converted at a time; without, D 128 spills)
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" : "+v"(b.k[t][2 * s]), "+v"(b.k[t][2 * s + 1]));
        const u32x4 kf = {Code<F>::template pair<0>(b.k[t][2 * s]), Code<F>::template pair<1>(b.k[t][2 * s]),
                          Code<F>::template pair<0>(b.k[t][2 * s + 1]), Code<F>::template pair<1>(b.k[t][2 * s + 1])};
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int i = QP - 1; i >= 0; --i) z[nq][t] = mma8(kf, qf[nq][i][s], z[nq][t]);
      }
    }
    u32x4 pf[NQ][PP];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      uint32_t vis = 0xffu;
      if (!full) {
        vis = valid;
        if (CHUNK) {
          const int k = seen[nq] - p * HK_PAGE - 4 * qd;        // of the lane's keys: 0 .. 3 and 16 .. 19
          vis &= (k >= 4 ? 15u : k <= 0 ? 0u : (1u << k) - 1u) |
                 (k >= 20 ? 15u : k <= 16 ? 0u : (1u << (k - 16)) - 1u) << 4;
        }
      }
      float x[8], zm = -INFINITY;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = z[nq][i >> 2][i & 3] * (b.ks[i >> 2][i & 3] * a.c2);
        if (!full) x[i] = (vis >> i) & 1u ? x[i] : -INFINITY;
        zm = fmaxf(zm, x[i]);
      }
      if (__any(zm > m[nq] + A8_SLACK)) {
        zm = fmaxf(zm, __shfl_xor(zm, 16, 64));
        zm = fmaxf(zm, __shfl_xor(zm, 32, 64));
        const float mn = fmaxf(m[nq], ceilf(zm));
        const float alpha = m[nq] == -INFINITY ? 0.f : fast_exp2(m[nq] - mn);
        m[nq] = mn;
        l[nq] *= alpha;
#pragma unroll
        for (int j = 0; j < DT; ++j) acc[nq][j] *= alpha;
      }
      const float off = m[nq] == -INFINITY ? 0.f : m[nq];
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = fast_exp2(x[i] - off);
        sum[i & 1] += x[i];
        x[i] *= b.vs[i >> 2][i & 3] * down;
        if (!full) x[i] = (vis >> i) & 1u ? x[i] : 0.f;         // (whatever the slot's scale is)
      }
      l[nq] += sum[0] + sum[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t part[PP];
        split_pair<PP>(x[2 * i], x[2 * i + 1], part);
#pragma unroll
        for (int j = 0; j < PP; ++j) pf[nq][j][i] = part[j];
      }
    }
#pragma unroll
    for (int j = 0; j < DT / 4; ++j) {
      // dims 4 j .. 4 j + 3 of the lane's D / 16
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(b.v[i][j]));
      values(std::integral_constant<int, 0>{}, b, pf, j);
      __builtin_amdgcn_sched_barrier(0);
      values(std::integral_constant<int, 1>{}, b, pf, j);
    }
  };

  // A wave's blocks are wave, wave + 4, ..; lane i holds id and mask of page i % 2 of its block i / 2.
  for (int from = p0; from < p1; from += 64 * A8_NW) {
    const int first = from + 2 * wave;
    const int n = min((p1 - first + 2 * A8_NW - 1) / (2 * A8_NW), 32);
    const int mine = first + 2 * A8_NW * (lane >> 1) + (lane & 1);
    const int id = min(max(trow[min(mine, p1 - 1)], 0), a.num_pages - 1);
    const int mk = mine < p1 ? mrow[mine] : 0;
    auto load = [&](Block8<D>& b, int i) {
      if (i >= n) return;
      b.load(a, __builtin_amdgcn_readlane(id, 2 * i), __builtin_amdgcn_readlane(id, 2 * i + 1),
             (uint32_t)__builtin_amdgcn_readlane(mk, 2 * i) | (uint32_t)__builtin_amdgcn_readlane(mk, 2 * i + 1) << 16);
    };
    if (n <= 0) continue;
    Block8<D> x, y;
    load(x, 0);
    for (int i = 0; i < n; i += 2) {
      load(y, i + 1);
      compute(x, first + 2 * A8_NW * i);
      if (i + 1 >= n) break;
      load(x, i + 2);
      compute(y, first + 2 * A8_NW * (i + 1));
    }
  }

  // the waves' states: to one reference, then 2 and 3 into 0 and 1, 1 into 0
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    l[nq] += __shfl_xor(l[nq], 16, 64);
    l[nq] += __shfl_xor(l[nq], 32, 64);
    if (qd == 0) {
      s_m[wave][nq][i16] = m[nq];
      s_l[wave][nq][i16] = l[nq];
    }
  }
  __syncthreads();
  float mt[NQ], lt[NQ];
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    mt[nq] = s_m[0][nq][i16];
#pragma unroll
    for (int i = 1; i < A8_NW; ++i) mt[nq] = fmaxf(mt[nq], s_m[i][nq][i16]);
    lt[nq] = 0.f;
#pragma unroll
    for (int i = 0; i < A8_NW; ++i) {
      const float mi = s_m[i][nq][i16];
      lt[nq] += s_l[i][nq][i16] * (mi == -INFINITY ? 0.f : fast_exp2(mi - mt[nq]));
    }
    const float f = m[nq] == -INFINITY ? 0.f : fast_exp2(m[nq] - mt[nq]);
#pragma unroll
    for (int j = 0; j < DT; ++j) acc[nq][j] *= f;
  }
#pragma unroll
  for (int to = 2; to >= 1; --to) {
    if (to == 1) __syncthreads();
    if (wave >= to && wave < 2 * to)
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
        for (int j = 0; j < DT; ++j) s_acc[wave - to][nq * DT + j][lane] = acc[nq][j];
    __syncthreads();
    if (wave < to)
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
        for (int j = 0; j < DT; ++j) acc[nq][j] += s_acc[wave][nq * DT + j][lane];
  }
  if (wave != 0) return;
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    const int row = 16 * nq + i16, r = w.r0 + row;
    if (r >= w.rows) continue;
    const float inv = lt[nq] == 0.f ? 0.f : 1.f / lt[nq];       // (a NaN stays one)
    const int tok = r / a.G, g = r - tok * a.G;
    const int64_t at = (int64_t)(w.c.first + tok) * a.Hq + w.kv * a.G + g;
    const int64_t pt = ((int64_t)blockIdx.x * a.cap + row);
    // the lane's dims: D / 4 from qd D / 4 on, (D / 16) r + j of them in acc[j][r]
    const auto put = [&](int i, float x0, float x1, float x2, float x3) {
      if (a.n_split > 1) {
        *reinterpret_cast<f32x4*>(a.part_o + pt * D + qd * (D / 4) + i) = f32x4{x0, x1, x2, x3};
      } else if constexpr (PP == 3) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + at * D + qd * (D / 4) + i) = f32x4{x0, x1, x2, x3};
      } else {
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + at * D + qd * (D / 4) + i) =
            u32x2{pack_bf16(x0, x1), pack_bf16(x2, x3)};
      }
    };
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < DT; j += 4) {
        const auto value = [&](int i) { return acc[nq][j + i][k] * inv * back; };
        put(DT * k + j, value(0), value(1), value(2), value(3));
      }
    if (qd == 0) {
      if (a.n_split > 1) *reinterpret_cast<f32x2*>(a.part_ml + pt * 2) = f32x2{lt[nq] == 0.f ? -INFINITY : mt[nq], lt[nq]};
      else if (a.lse) a.lse[at] = lse8(mt[nq], lt[nq]);
    }
  }
}

// The ranges' states (means of V, references, sums) to the row's: a workgroup takes a unit, a wave
// every fourth of its rows.
template <int D, int ROWS, int PP, bool CHUNK>
__global__ __launch_bounds__(A8_NT) void attn8_merge_kernel(Args8 a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, u = blockIdx.x;
  const Unit w = unit_of<ROWS, CHUNK>(a, u);
  if (w.rows == 0) return;
  const int share = share8(a, w.pages), used = max((w.pages + share - 1) / share, 1);
  constexpr int PER = D / 64;
  for (int row = wave; row < ROWS && w.r0 + row < w.rows; row += A8_NW) {
    const int64_t first = (int64_t)u * a.n_split * a.cap + row;
    const f32x2* ml = reinterpret_cast<const f32x2*>(a.part_ml) + first;
    float mt = -INFINITY, lt = 0.f;
    for (int i = lane; i < used; i += 64) mt = fmaxf(mt, ml[(int64_t)i * a.cap][0]);
    mt = wave_max(mt);
    for (int i = lane; i < used; i += 64) {
      const f32x2 x = ml[(int64_t)i * a.cap];
      lt += x[0] == -INFINITY ? 0.f : x[1] * fast_exp2(x[0] - mt);
    }
    lt = wave_sum(lt);
    const float inv = lt == 0.f ? 0.f : 1.f / lt;
    float o[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) o[j] = 0.f;
#pragma unroll 8
    for (int i = 0; i < used; ++i) {
      const f32x2 x = ml[(int64_t)i * a.cap];
      const float f = x[0] == -INFINITY ? 0.f : x[1] * fast_exp2(x[0] - mt) * inv;
      const float* from = a.part_o + (first + (int64_t)i * a.cap) * D + lane * PER;
#pragma unroll
      for (int j = 0; j < PER; ++j) o[j] = fmaf(f, from[j], o[j]);
    }
    const int r = w.r0 + row, tok = r / a.G, g = r - tok * a.G;
    const int64_t at = (int64_t)(w.c.first + tok) * a.Hq + w.kv * a.G + g;
    if constexpr (PP == 3) {
#pragma unroll
      for (int j = 0; j < PER; ++j) static_cast<float*>(a.o)[at * D + lane * PER + j] = o[j];
    } else {
#pragma unroll
      for (int j = 0; j < PER; ++j)
        static_cast<__bf16*>(a.o)[at * D + lane * PER + j] = (__bf16)o[j];
    }
    if (lane == 0 && a.lse) a.lse[at] = lse8(mt, lt);
  }
}

// ------------------------------------------------------------------ host
struct Plan8 {
  int nq, one_tile, cap, n_split;
  int64_t units;
};
inline Plan8 plan8(int NS, int Hkv, int G, const hk_chunks* ch, int max_pages) {
  Plan8 p;
  const int64_t most = ch ? (int64_t)ch->max_len * G : G;       // rows of a sequence at most
  p.nq = most <= 16 ? 1 : 2;
  const int rows = 16 * p.nq;
  p.one_tile = most <= rows;
  p.cap = (int)(most < rows ? most : rows);
  const int64_t tiles = !ch ? (int64_t)NS * ((G + rows - 1) / rows)
                            : p.one_tile ? NS : (int64_t)ch->n_tokens * G / rows + NS;
  p.units = tiles * Hkv;
  int pps = A8_PPS;
  while (pps > A8_PPS_MIN && p.units * ((max_pages + pps - 1) / pps) < A8_TARGET) pps >>= 1;
  const int64_t most_split = (A8_MOST + p.units - 1) / p.units;
  p.n_split = (int)std::min<int64_t>((max_pages + pps - 1) / pps, most_split);
  return p;
}

}  // namespace hk

using namespace hk;

static size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }

size_t hk_attn8_ws(int NS, int Hq, int Hkv, int D, const hk_chunks* ch, int max_pages) {
  const Plan8 p = plan8(NS, Hkv, Hq / Hkv, ch, max_pages);
  size_t states = p.n_split > 1 ? (size_t)p.units * p.n_split * p.cap : 0;
  if (ch && max_pages > A8_PPS_MIN) {
    // what any chunks of no more tokens, and none longer, can take: ranges are for fewer than MOST units,
    // and leave fewer than 2 MOST workgroups
    const int64_t units = ((int64_t)ch->n_tokens * (Hq / Hkv) / 16 + NS) * Hkv;
    const int64_t groups = std::min<int64_t>(2 * A8_MOST, units * ((max_pages + A8_PPS_MIN - 1) / A8_PPS_MIN));
    const int64_t rows = (int64_t)ch->max_len * (Hq / Hkv);
    states = (size_t)(groups * std::min<int64_t>(rows, A8_ROWS));
  }
  return 256 + align_up(states * D * 4) + align_up(states * 8);
}

double hk_attn8_groups(int NS, int Hq, int Hkv, const hk_chunks* ch, int max_pages) {
  const Plan8 p = plan8(NS, Hkv, Hq / Hkv, ch, max_pages);
  return (double)p.units * p.n_split;
}

template <int F, int D, int NQ, int QP, int PP, bool CHUNK>
static void launch8(const Args8& a, hipStream_t st) {
  {
    TimedLaunch t(HK_TK_ATTN8, st);
    hipLaunchKernelGGL((attn8_kernel<F, D, NQ, QP, PP, CHUNK>), dim3((uint32_t)a.n_units * a.n_split), dim3(A8_NT), 0, st, a);
  }
  if (a.n_split > 1) {
    TimedLaunch t(HK_TK_ATTN8_MERGE, st);
    hipLaunchKernelGGL((attn8_merge_kernel<D, 16 * NQ, PP, CHUNK>), dim3((uint32_t)a.n_units), dim3(A8_NT), 0, st, a);
  }
}
template <int F, int D, int NQ>
static void launch8_t(const Args8& a, bool chunk, bool bf, hipStream_t st) {
  if (chunk) bf ? launch8<F, D, NQ, 1, 2, true>(a, st) : launch8<F, D, NQ, 3, 3, true>(a, st);
  else bf ? launch8<F, D, NQ, 1, 3, false>(a, st) : launch8<F, D, NQ, 3, 3, false>(a, st);
}
template <int F>
static void launch8_f(const Args8& a, int D, int nq, bool chunk, bool bf, hipStream_t st) {
  if (D == 128) nq == 1 ? launch8_t<F, 128, 1>(a, chunk, bf, st) : launch8_t<F, 128, 2>(a, chunk, bf, st);
  else nq == 1 ? launch8_t<F, 64, 1>(a, chunk, bf, st) : launch8_t<F, 64, 2>(a, chunk, bf, st);
}

hipError_t hk_launch_attn8(int NS, int Hq, int Hkv, int D, const hk_paged_kv8* kv8, const hk_chunks* ch,
                           hk_dtype dtype, const void* q, int64_t q_row, float sm_scale, void* o, float* lse,
                           void* ws, hipStream_t st) {
  const hk_paged_kv& kv = kv8->kv;
  const Plan8 p = plan8(NS, Hkv, Hq / Hkv, ch, kv.max_pages);
  Args8 a{};
  a.q = q;
  a.q_row = q_row;
  a.k_pool = static_cast<const char*>(kv.k_pool);
  a.v_pool = static_cast<const char*>(kv.v_pool);
  a.k_scale = kv8->k_scale;
  a.v_scale = kv8->v_scale;
  a.table = kv.page_table;
  a.n_pages = kv.n_pages;
  a.masks = kv.page_mask;
  a.start = ch ? ch->start : nullptr;
  a.o = o;
  a.lse = lse;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up((size_t)p.units * p.n_split * p.cap * D * 4));
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.max_pages = kv.max_pages;
  a.num_pages = kv.num_pages;
  a.n_seq = NS;
  a.n_tokens = ch ? ch->n_tokens : NS;
  a.max_len = ch ? ch->max_len : 1;
  a.n_units = (int)p.units;
  a.n_split = p.n_split;
  a.cap = p.cap;
  a.one_tile = p.one_tile;
  a.c2 = sm_scale * kLog2e;
  if (kv.dtype == HK_I8) launch8_f<HK_I8>(a, D, p.nq, ch != nullptr, dtype == HK_BF16, st);
  else launch8_f<HK_E4M3>(a, D, p.nq, ch != nullptr, dtype == HK_BF16, st);
  return hipGetLastError();
}
