// 8-bit cache: attention of single tokens and of chunks of new tokens over its pages (gfx950).
//
// The query rows of a KV head are folded: row r of a chunk is query head r % G of token r / G.  Up to
// 32 of them are a unit.  The units' pages, in steps of eight, are one long list that the workgroups of
// a launch share evenly (two a CU, or three of D 64): a workgroup takes a run of steps, the end of one
// unit, whole units and the beginning of another.  Its four waves take a step's pages two at a time, every
// page read once, straight into LDS, and meet at a unit's end.  attn8_merge_kernel joins the units that
// were cut.  (A grid of units x equal parts of each, 512 heads of 784 to 5600 tokens: 6 parts 104 us, 2
// 102, 1 95, whose shortest units leave early.)
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
// q enters in one bf16 part, or for fp32 in three (exactly).  P enters in two parts for bf16 results, to
// 2^-16 of a term, which is 2^-8 of their own rounding, and in three for fp32 ones, to 2^-24.
//
// Softmax: one pass with a running reference m per row, a whole number that moves when a score exceeds
// it by 2^SLACK.  The sums of P V are kept smaller by 2^bias, at least their number of terms times
// 2^SLACK, so that they stay finite where the result does.
//
// What bounds it: reading the pages, masked slots in them included, at the rate of these loads.  Single tokens
// of 64 sequences of 784 to 5600 tokens, 32 / 8 heads of 128: 448 MB in 89 us, 5.0 TB/s, and 5 the merge
// (without products and softmax 82); their drafts of 1 to 8 tokens 108 (97 without) and 8.5.  One row of 131071
// tokens, 8 heads of 64, fp32 queries: 32 us, 4.8 TB/s.  More blocks on their way (4 at D 64), three or four
// waves a SIMD, 1024 or 1536 workgroups and loads past the caches were no faster; units' sizes kept for a run's
// later units neither (1%).
#include <algorithm>
#include <type_traits>

#include "hk_attn8.h"

namespace hk {

// A block of 32 keys in LDS: K codes of two pages, V codes, and 64 scales (K's, V's).  It is filled
// straight from memory, 1 KB of codes an instruction, 16 bytes a lane in lane order, so that every line
// is asked for once (a fragment's loads into registers ask for it twice; the second waits on the first,
// 42% of the time).  A lane may fetch any 16 bytes: rows lie in an order, and their 16-byte pieces in one
// of a row's own, in which the fragments' reads meet no bank twice.
template <int D>
struct Tile8 {
  static constexpr int ROWS = 1024 / D, PIECES = D / 16, PAGE = HK_PAGE * D;
  static constexpr int SCALES = 4 * PAGE, BYTES = SCALES + 256;
  static constexpr int LOADS = 4 * PAGE / 1024 + 1;
  // place of a key among the rows of its instruction, and what its pieces' places are changed by
  __device__ static __forceinline__ int place(int key) {
    return D == 128 ? (key & 3) * 2 + ((key >> 2) & 1) : (key & 3) * 4 + (key >> 2);
  }
  __device__ static __forceinline__ int turn(int key) { return D == 128 ? (key & 3) | (key >> 3) << 2 : key & 3; }
  __device__ static __forceinline__ int at(int key, int piece) {
    return (D == 128 ? (key >> 3) * 1024 : 0) + place(key) * D + (piece ^ turn(key)) * 16;
  }
  // the bytes of a page that a lane fetches with instruction g of it
  __device__ static __forceinline__ int source(int lane, int g) {
    const int pos = lane / PIECES;
    const int key = D == 128 ? 8 * g + (pos >> 1) + 4 * (pos & 1) : (pos >> 2) + 4 * (pos & 3);
    return key * D + (((lane % PIECES) ^ turn(key)) * 16);
  }
};

__device__ __forceinline__ f32x4 mma8(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int D>
constexpr int A8_DEPTH = D == 128 ? 2 : 3;   // blocks of a wave in LDS
// QP: bf16 parts of q (1: q is bf16), PP: of P (2: o is bf16, 3: fp32)
template <int F, int D, int NQ, int QP, int PP, bool CHUNK>
__global__ __launch_bounds__(A8_NT, 2) void attn8_kernel(Args8 a) {
#pragma clang fp contract(off)
  constexpr int ROWS = 16 * NQ, KS = D / 32, DT = D / 16;
  using L = Tile8<D>;
  constexpr int DEPTH = A8_DEPTH<D>;
  __shared__ __align__(16) char s_tiles[A8_NW * DEPTH * L::BYTES];
  f32x4 (*s_acc)[NQ * DT][64] = reinterpret_cast<f32x4 (*)[NQ * DT][64]>(s_tiles);   // at the end
  static_assert(sizeof(s_tiles) >= 2 * sizeof(*s_acc));
  __shared__ float s_m[A8_NW][NQ][16], s_l[A8_NW][NQ][16];
  const int lane = threadIdx.x & 63, i16 = lane & 15, qd = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t source[L::PAGE / 1024];
#pragma unroll
  for (int g = 0; g < L::PAGE / 1024; ++g) source[g] = L::source(lane, g);
  int k_at[KS / 2], v_at[4];                  // the lane's fragments within a page
#pragma unroll
  for (int i = 0; i < KS / 2; ++i) k_at[i] = L::at(i16, KS / 2 * qd + i);
#pragma unroll
  for (int r = 0; r < 4; ++r) v_at[r] = L::at(4 * qd + r, i16 * (D / 16) / 16) + i16 * (D / 16) % 16;

  int u = blockIdx.x, skip = 0, left = 1 << 30;   // unit, its steps that are another's, steps of the run
  if (a.first) {
    static_assert(sizeof(s_tiles) >= (A8_UNITS + 1) * sizeof(int));
    const Run r = run_of_group<ROWS, CHUNK>(a, reinterpret_cast<int*>(s_tiles), reinterpret_cast<int*>(s_m));
    u = r.unit;
    skip = r.skip;
    left = r.left;
  }
  for (; left > 0 && u < a.n_units; ++u) {
  const Unit w = unit_of<ROWS, CHUNK>(a, u);
  if (w.rows == 0) {
    if (!a.first) return;
    continue;                                 // (no steps)
  }
  const int steps = steps_of(w), take = min(steps - skip, left);
  const int p0 = skip * A8_STEP, p1 = min(p0 + take * A8_STEP, w.pages);
  const int64_t state = take == steps ? -1 : (int64_t)(2 * blockIdx.x + (skip == 0)) * a.cap;
  left = a.first ? left - take : 0;
  skip = 0;
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
  // (waited for here, or every block's first product would wait for all loads, those of the blocks to come too)
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
    for (int i = 0; i < QP; ++i)
#pragma unroll
      for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[nq][i][s]));
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

  // P V of dims 4 j + 2 H and 4 j + 2 H + 1 from the eight keys' words j: the codes' pairs turned into
  // pairs of keys
  auto values = [&](auto half, const uint32_t (&v)[8], const u32x4 (&pf)[NQ][PP], int j) {
    constexpr int H = decltype(half)::value;
    u32x4 vf[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = v[2 * i], y = v[2 * i + 1];
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
  // the block at `b`, from page p on, keys valid where the bits of mask are 1
  auto compute = [&](const char* b, int p, uint32_t mask) {
    const bool full = mask == 0xffffffffu && (!CHUNK || (p + 2) * HK_PAGE <= seen_all);
    // the lane's keys 4 t + r: slot 4 qd + r of page t
    const uint32_t valid = ((mask >> (4 * qd)) & 15u) | ((mask >> (16 + 4 * qd)) & 15u) << 4;
    f32x4 z[NQ][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) z[nq][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s2 = 0; s2 < KS / 2; ++s2) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(b + t * L::PAGE + k_at[s2]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4 kf = {Code<F>::template pair<0>(w[2 * h]), Code<F>::template pair<1>(w[2 * h]),
                            Code<F>::template pair<0>(w[2 * h + 1]), Code<F>::template pair<1>(w[2 * h + 1])};
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int i = QP - 1; i >= 0; --i) z[nq][t] = mma8(kf, qf[nq][i][2 * s2 + h], z[nq][t]);
        }
      }
    }
    const float* scales = reinterpret_cast<const float*>(b + L::SCALES) + 4 * qd;
    const f32x4 ks[2] = {*reinterpret_cast<const f32x4*>(scales), *reinterpret_cast<const f32x4*>(scales + 16)};
    f32x4 vs[2] = {*reinterpret_cast<const f32x4*>(scales + 32), *reinterpret_cast<const f32x4*>(scales + 48)};
    if (!full) {
      uint32_t w = valid;
      asm volatile("" : "+v"(w));             // (here and below: a branch, not selects in every block)
#pragma unroll
      for (int i = 0; i < 8; ++i) vs[i >> 2][i & 3] = (w >> i) & 1u ? vs[i >> 2][i & 3] : 0.f;
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
        x[i] = z[nq][i >> 2][i & 3] * (ks[i >> 2][i & 3] * a.c2);
      }
      if (!full) {
        asm volatile("" : "+v"(vis));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (vis >> i) & 1u ? x[i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) zm = fmaxf(zm, x[i]);
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
        x[i] *= vs[i >> 2][i & 3] * down;
      }
      if (CHUNK && !full) {
        // a later token's scale may be NaN, and its product with a probability of 0
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) odd |= x[i] != x[i];
        if (__any(odd)) {
          asm volatile("" : "+v"(vis));
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = (vis >> i) & 1u ? x[i] : 0.f;
        }
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
    uint32_t v[DT / 4][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const char* from = b + (2 + (i >> 2)) * L::PAGE + v_at[i & 3];
      if constexpr (D == 128) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(from);
        v[0][i] = x[0];
        v[1][i] = x[1];
      } else {
        v[0][i] = *reinterpret_cast<const uint32_t*>(from);
      }
    }
    if (F == HK_E4M3 && mask != 0xffffffffu) {
      // a slot that is not valid may hold codes that stand for NaN
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < DT / 4; ++j) v[j][i] = (valid >> i) & 1u ? v[j][i] : 0u;
    }
#pragma unroll
    for (int j = 0; j < DT / 4; ++j) {
      // dims 4 j .. 4 j + 3 of the lane's D / 16; one product's codes converted at a time (without, spills)
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(v[j][i]));
      values(std::integral_constant<int, 0>{}, v[j], pf, j);
      __builtin_amdgcn_sched_barrier(0);
      values(std::integral_constant<int, 1>{}, v[j], pf, j);
    }
  };

  // A wave's blocks are wave, wave + 4, .. of the range's; DEPTH of them are in LDS or on their way.
  // Ids and masks come 32 blocks at a time: lane i holds those of page i % 2 of block i / 2.
  char* mine = s_tiles + wave * (DEPTH * L::BYTES);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
  const int first = p0 + 2 * wave, n = p1 > first ? (p1 - first + 2 * A8_NW - 1) / (2 * A8_NW) : 0;
  int ids = 0, masks = 0;
  uint32_t queue[DEPTH];                      // masks of the blocks on their way
  auto request = [&](int i, int slot) {       // returns the block's mask
    if ((i & 31) == 0) {
      const int page = first + 2 * A8_NW * (i + (lane >> 1)) + (lane & 1);
      ids = min(max(trow[min(page, p1 - 1)], 0), a.num_pages - 1);
      masks = page < p1 ? mrow[page] : 0;
    }
    const uint32_t to = lds + slot * L::BYTES;
    const int e = 2 * (i & 31);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (what lay there has been read)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const size_t at = (size_t)(uint32_t)__builtin_amdgcn_readlane(ids, e + t) * L::PAGE;
#pragma unroll
      for (int g = 0; g < L::PAGE / 1024; ++g) {
        direct_load(a.k_pool + at, source[g], to + t * L::PAGE + g * 1024);
        direct_load(a.v_pool + at, source[g], to + (2 + t) * L::PAGE + g * 1024);
      }
    }
    const int id = (qd & 1) ? __builtin_amdgcn_readlane(ids, e + 1) : __builtin_amdgcn_readlane(ids, e);
    direct_load4(reinterpret_cast<const char*>((qd >> 1 ? a.v_scale : a.k_scale) + (size_t)(uint32_t)id * HK_PAGE + i16),
                 to + L::SCALES);
    return (uint32_t)__builtin_amdgcn_readlane(masks, e) | (uint32_t)__builtin_amdgcn_readlane(masks, e + 1) << 16;
  };
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d)
    if (d < n) queue[d] = request(d, d);
  for (int i0 = 0; i0 < n; i0 += DEPTH)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int i = i0 + d;
      if (i >= n) break;
      if (i + DEPTH - 1 < n) {
        queue[(d + DEPTH - 1) % DEPTH] = request(i + DEPTH - 1, (d + DEPTH - 1) % DEPTH);
        direct_wait<(DEPTH - 1) * L::LOADS>();
      } else {
        direct_wait<0>();
      }
      compute(mine + d * L::BYTES, first + 2 * A8_NW * i, queue[d]);
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
  if (wave == 0)
#pragma unroll
  for (int nq = 0; nq < NQ; ++nq) {
    const int row = 16 * nq + i16, r = w.r0 + row;
    if (r >= w.rows) continue;
    const float inv = lt[nq] == 0.f ? 0.f : 1.f / lt[nq];       // (a NaN stays one)
    const int tok = r / a.G, g = r - tok * a.G;
    const int64_t at = (int64_t)(w.c.first + tok) * a.Hq + w.kv * a.G + g;
    // the lane's dims: D / 4 from qd D / 4 on, (D / 16) r + j of them in acc[j][r]
    const auto put = [&](int i, float x0, float x1, float x2, float x3) {
      if (state >= 0) {
        *reinterpret_cast<f32x4*>(a.part_o + (state + row) * D + qd * (D / 4) + i) = f32x4{x0, x1, x2, x3};
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
      // (NaN keys alone leave a sum of NaN and no reference)
      const float ref = lt[nq] == 0.f ? -INFINITY : mt[nq] == -INFINITY ? 0.f : mt[nq];
      if (state >= 0) *reinterpret_cast<f32x2*>(a.part_ml + (state + row) * 2) = f32x2{ref, lt[nq]};
      else if (a.lse) a.lse[at] = lse8(mt[nq], lt[nq]);
    }
  }
  __syncthreads();                            // (the states in LDS are read)
  }
}

// ------------------------------------------------------------------ host
struct Plan8 {
  int nq, one_tile, cap;
  int64_t units;
  bool tiles;                                 // chunks of more than A8_ROWS rows go to the tile kernel
  bool planned, cut;                          // whether units can be cut
};
inline Plan8 plan8(int NS, int Hkv, int G, const hk_chunks* ch, bool bf, int max_pages) {
  Plan8 p;
  const int64_t most = ch ? (int64_t)ch->max_len * G : G;       // rows of a sequence at most
  p.nq = most <= 16 ? 1 : 2;
  const int rows = 16 * p.nq;
  p.tiles = ch && bf && most > rows;
  p.one_tile = most <= rows || p.tiles;
  p.cap = (int)(most < rows ? most : rows);
  const int64_t tiles = !ch ? (int64_t)NS * ((G + rows - 1) / rows)
                            : p.one_tile ? NS : (int64_t)ch->n_tokens * G / rows + NS;
  p.units = tiles * Hkv;
  p.planned = planned8(p.units, !p.one_tile, max_pages);
  p.cut = p.planned && max_pages > A8_STEP;
  return p;
}

}  // namespace hk

using namespace hk;

// tokens of a chunk at most
static int64_t longest(const hk_chunks& ch) { return std::min(ch.max_len, ch.n_tokens); }

// (any chunks of no more tokens, and none longer, take no more)
size_t hk_attn8_ws(int NS, int Hq, int Hkv, int D, const hk_chunks* ch, int max_pages) {
  const int G = Hq / Hkv;
  const bool long_ones = ch && (int64_t)ch->max_len * G > A8_ROWS;
  const size_t most = states8_bytes(D, plan8(NS, Hkv, G, ch, false, max_pages).cap);
  return long_ones ? std::max(most, hk_attn8_tile_ws(D, (int64_t)NS * Hkv, max_pages, longest(*ch) * G)) : most;
}

double hk_attn8_groups(int NS, int Hq, int Hkv, const hk_chunks* ch, int max_pages) {
  const Plan8 p = plan8(NS, Hkv, Hq / Hkv, ch, false, max_pages);
  return (double)p.units;
}

template <int F, int D, int NQ, int QP, int PP, bool CHUNK>
static void launch8(const Args8& a, bool cut, hipStream_t st) {
  const uint32_t groups = a.first ? A8_GROUPS<D> : (uint32_t)a.n_units;
  {
    TimedLaunch t(HK_TK_ATTN8, st);
    hipLaunchKernelGGL((attn8_kernel<F, D, NQ, QP, PP, CHUNK>), dim3(groups), dim3(A8_NT), 0, st, a);
  }
  if (cut) merge8<D, 16 * NQ, PP, CHUNK>(a, groups, st);
}
template <int F, int D, int NQ>
static void launch8_t(const Args8& a, bool chunk, bool bf, bool cut, hipStream_t st) {
  if (chunk) bf ? launch8<F, D, NQ, 1, 2, true>(a, cut, st) : launch8<F, D, NQ, 3, 3, true>(a, cut, st);
  else bf ? launch8<F, D, NQ, 1, 3, false>(a, cut, st) : launch8<F, D, NQ, 3, 3, false>(a, cut, st);
}
template <int F>
static void launch8_f(const Args8& a, int D, int nq, bool chunk, bool bf, bool cut, hipStream_t st) {
  if (D == 128) nq == 1 ? launch8_t<F, 128, 1>(a, chunk, bf, cut, st) : launch8_t<F, 128, 2>(a, chunk, bf, cut, st);
  else nq == 1 ? launch8_t<F, 64, 1>(a, chunk, bf, cut, st) : launch8_t<F, 64, 2>(a, chunk, bf, cut, st);
}

hipError_t hk_launch_attn8(int NS, int Hq, int Hkv, int D, const hk_paged_kv8* kv8, const hk_chunks* ch,
                           hk_dtype dtype, const void* q, int64_t q_row, float sm_scale, void* o, float* lse,
                           void* ws, hipStream_t st) {
  const hk_paged_kv& kv = kv8->kv;
  const bool bf = dtype == HK_BF16;
  const Plan8 p = plan8(NS, Hkv, Hq / Hkv, ch, bf, kv.max_pages);
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
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.max_pages = kv.max_pages;
  a.num_pages = kv.num_pages;
  a.n_seq = NS;
  a.n_tokens = ch ? ch->n_tokens : NS;
  a.max_len = ch ? ch->max_len : 1;
  a.n_units = (int)p.units;
  a.cap = p.cap;
  a.one_tile = p.one_tile;
  a.rows_from = 1;
  a.rows_to = p.tiles ? A8_ROWS : INT32_MAX;
  a.c2 = sm_scale * kLog2e;
  carve8(a, p.planned, D, ws);
  if (kv.dtype == HK_I8) launch8_f<HK_I8>(a, D, p.nq, ch != nullptr, bf, p.cut, st);
  else launch8_f<HK_E4M3>(a, D, p.nq, ch != nullptr, bf, p.cut, st);
  // (the launches follow one another: one workspace serves both)
  if (p.tiles) hk_launch_attn8_tile(a, kv.dtype, D, longest(*ch) * a.G, ws, st);
  return hipGetLastError();
}
