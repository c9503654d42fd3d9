// Attention over an 8-bit cache: arguments, units, runs of steps and states shared by its kernels (gfx950).
#pragma once

#include "hk_chunk.h"
#include "hk_kv8.h"

namespace hk {

constexpr int A8_NT = 256, A8_NW = 4;
constexpr float A8_SLACK = 4.f;
constexpr int A8_STEP = 2 * A8_NW;            // pages of a step
constexpr int A8_UNITS = 4096;                // units that a launch plans; one of more has a workgroup for each
template <int D>
constexpr int A8_GROUPS = D == 128 ? 512 : 768;   // workgroups that share the steps
constexpr int A8_ROWS = 32;                   // rows of a unit at most, but for the tile kernel's

struct Args8 {
  const void* q;
  int64_t q_row;                              // elements
  const char *k_pool, *v_pool;
  const float *k_scale, *v_scale;
  const int32_t *table, *n_pages, *start;     // start NULL: one token per sequence
  const uint16_t* masks;
  void* o;
  float *lse, *part_o, *part_ml;              // states: of workgroup b's first unit at 2 b, of its last at 2 b + 1
  char* ready;                                // tiles converted beforehand, or NULL
  int32_t* first;                             // step that a unit begins at, and the number of steps; NULL: not planned
  int Hq, Hkv, G, max_pages, num_pages, n_seq, n_tokens, max_len;
  int n_units, cap;                           // cap: rows of a unit in the workspace
  int rows_from, rows_to;                     // sequences of other numbers of rows are another launch's
  int one_tile;                               // none of these has more rows than a unit
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
  if (w.r0 < 0 || w.r0 >= w.rows || w.rows < a.rows_from || w.rows > a.rows_to) {
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
__device__ __forceinline__ int steps_of(const Unit& w) {
  return w.rows == 0 ? 0 : max((w.pages + A8_STEP - 1) / A8_STEP, 1);
}
// Workgroup b of n, at most one a step, has the steps [run_of(b), run_of(b + 1)) of total; group_of: that
// of step x.
__device__ __forceinline__ int run_of(int b, int n, int total) { return (int)((int64_t)total * b / n); }
__device__ __forceinline__ int group_of(int x, int n, int total) { return (int)(((int64_t)(x + 1) * n - 1) / total); }

// Of up to 64 units whose steps lane i holds for unit i: those before it, and the total.
__device__ __forceinline__ int scan_units(int steps, int* before) {
  const int lane = threadIdx.x & 63;
  int x = steps;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  *before = x - steps;
  return __builtin_amdgcn_readlane(x, 63);
}

// Steps before every unit into first (LDS), the total at first[n_units]; the last workgroup leaves them
// for the merge.
template <int ROWS, bool CHUNK>
__device__ __forceinline__ void plan_units(const Args8& a, int* first, int* sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (a.n_units + A8_NT - 1) / A8_NT, u0 = threadIdx.x * per;
  int mine = 0;
  for (int u = u0; u < min(u0 + per, a.n_units); ++u) {
    const int n = steps_of(unit_of<ROWS, CHUNK>(a, u));
    first[u] = n;
    mine += n;
  }
  int x = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  int before = x - mine;
#pragma unroll
  for (int i = 0; i < A8_NW; ++i) before += i < wave ? sums[i] : 0;
  for (int u = u0; u < min(u0 + per, a.n_units); ++u) {
    const int n = first[u];
    first[u] = before;
    before += n;
  }
  if (threadIdx.x == A8_NT - 1) first[a.n_units] = before;
  __syncthreads();
  if (blockIdx.x == gridDim.x - 1)
    for (int u = threadIdx.x; u <= a.n_units; u += A8_NT) a.first[u] = first[u];
}

// A workgroup's run: its first unit, the steps of it that are another workgroup's, and its own steps (0: none).
struct Run {
  int unit, skip, left;
};
template <int ROWS, bool CHUNK>
__device__ __forceinline__ Run run_of_group(const Args8& a, int* first, int* sums) {
  Run r{0, 0, 0};
  if (a.n_units <= 64) {
    // every wave by itself (a launch of few units is short: with the list in LDS it took a microsecond more)
    const int lane = threadIdx.x & 63;
    int before;
    const int total = scan_units(lane < a.n_units ? steps_of(unit_of<ROWS, CHUNK>(a, lane)) : 0, &before);
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x < 64) {
      if (lane < a.n_units) a.first[lane] = before;
      if (lane == 0) a.first[a.n_units] = total;
    }
    const int n = min((int)gridDim.x, total);
    if ((int)blockIdx.x >= n) return r;
    const int x = run_of(blockIdx.x, n, total);
    r.left = run_of(blockIdx.x + 1, n, total) - x;
    r.unit = 63 - __clzll(__ballot(lane < a.n_units && before <= x));
    r.skip = x - __builtin_amdgcn_readlane(before, r.unit);
    return r;
  }
  plan_units<ROWS, CHUNK>(a, first, sums);
  const int total = __builtin_amdgcn_readfirstlane(first[a.n_units]), n = min((int)gridDim.x, total);
  if ((int)blockIdx.x >= n) return r;
  const int x = run_of(blockIdx.x, n, total);
  r.left = run_of(blockIdx.x + 1, n, total) - x;
  int u = 0;                                  // the last unit that begins at or before x
  for (int hi = a.n_units; hi - u > 1;) {
    const int mid = (u + hi) / 2;
    if (first[mid] <= x) u = mid;
    else hi = mid;
  }
  r.unit = __builtin_amdgcn_readfirstlane(u);
  r.skip = __builtin_amdgcn_readfirstlane(x - first[u]);
  __syncthreads();                            // (the tiles take first's place)
  return r;
}

// log of l 2^m; the powers of two of both cancel as whole numbers
__device__ __forceinline__ float lse8(float m, float l) {
  if (l == 0.f) return -INFINITY;
  return (m + (float)__builtin_amdgcn_frexp_expf(l) + __log2f(__builtin_amdgcn_frexp_mantf(l))) * kLn2;
}

// fp32 in N bf16 parts, of two values a word: N 1: exact ones, 2: to 2^-16, 3: all of its bits but the last.
// What a part leaves is formed by one dot product a value (with 0 for the other of the word), exactly.
template <int N>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&out)[N]) {
  uint32_t minus_lo = 0x0000bf80u, minus_hi = 0xbf800000u;      // -1 and 0
  asm("" : "+s"(minus_lo), "+s"(minus_hi));   // (in registers: as a literal the pair is not what it says)
  const bf16x2 less_lo = __builtin_bit_cast(bf16x2, minus_lo), less_hi = __builtin_bit_cast(bf16x2, minus_hi);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    out[i] = pack_bf16(x, y);
    if (i + 1 < N) {
      const bf16x2 part = __builtin_bit_cast(bf16x2, out[i]);
      x = __builtin_amdgcn_fdot2_f32_bf16(part, less_lo, x, false);
      y = __builtin_amdgcn_fdot2_f32_bf16(part, less_hi, y, false);
    }
  }
}

// The states of a cut unit's parts (means of V, references, sums) to the row's: a wave takes R rows, whose
// loads are on their way at once, or WAVES of them share a row's parts.  D / 4 lanes load a state; 256 / D of
// them lie side by side.  512 units, up to 32 rows: a row a wave 10.7 us, four 8.6; 4 rows 5.0 and 5.9.
template <int D, int ROWS, int PP, bool CHUNK, int WAVES, int R>
__global__ __launch_bounds__(A8_NT) void attn8_merge_kernel(Args8 a, int n_groups) {
  constexpr int LPR = D / 4, SIDE = 64 / LPR, PER = R * A8_NW / WAVES;
  __shared__ float s_m[A8_NW], s_l[A8_NW];
  __shared__ f32x4 s_o[A8_NW][LPR];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per_unit = (a.cap + PER - 1) / PER, u = blockIdx.x / per_unit;
  const int row = (blockIdx.x - u * per_unit) * PER + wave / WAVES * R;
  const Unit w = unit_of<ROWS, CHUNK>(a, u);
  const int rows = min(min(a.cap, w.rows - w.r0) - row, R);      // of the wave
  if (w.rows == 0 || rows <= 0) return;       // (the waves of a row leave together)
  const int total = a.first[a.n_units], x0 = a.first[u], x1 = a.first[u + 1];
  const int n = min(n_groups, total), b0 = group_of(x0, n, total), used = group_of(x1 - 1, n, total) - b0 + 1;
  if (used < 2) return;                       // not cut
  const int per = (used + WAVES - 1) / WAVES, i0 = wave % WAVES * per, i1 = min(i0 + per, used);
  const auto state = [&](int i, int k) { return (int64_t)(2 * (b0 + i) + (i == 0)) * a.cap + row + min(k, rows - 1); };
  const f32x2* ml = reinterpret_cast<const f32x2*>(a.part_ml);
  // lane i has the weight of part i of 64; the first 64 (often all) are loaded once
  const auto load = [&](int i, int k) { return i < i1 ? ml[state(i, k)] : f32x2{-INFINITY, 0.f}; };
  f32x2 mine[R];
  float m[R], l[R];
  f32x4 o[R];
#pragma unroll
  for (int k = 0; k < R; ++k) mine[k] = load(i0 + lane, k);
  const auto weight = [&](f32x2 x, int k) { return x[0] == -INFINITY ? 0.f : x[1] * fast_exp2(x[0] - m[k]); };
#pragma unroll
  for (int k = 0; k < R; ++k) {
    m[k] = mine[k][0];
    for (int i = i0 + 64 + lane; i < i1; i += 64) m[k] = fmaxf(m[k], load(i, k)[0]);
    m[k] = wave_max(m[k]);
    l[k] = weight(mine[k], k);
    for (int i = i0 + 64 + lane; i < i1; i += 64) l[k] += weight(load(i, k), k);
    l[k] = wave_sum(l[k]);
    o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int side = lane / LPR, at = lane % LPR;
  for (int from = i0; from < i1; from += 64) {
    const int most = min(i1 - from, 64);
    float f[R];
#pragma unroll
    for (int k = 0; k < R; ++k) f[k] = weight(from == i0 ? mine[k] : load(from + lane, k), k) * (l[k] == 0.f ? 0.f : 1.f / l[k]);
    constexpr int U = 4 / R;                  // four loads on their way
    for (int j = 0; j < most; j += U * SIDE) {
      f32x4 x[R][U];
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int v = 0; v < U; ++v)
          x[k][v] = *reinterpret_cast<const f32x4*>(a.part_o + state(from + min(j + v * SIDE + side, most - 1), k) * D + 4 * at);
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int v = 0; v < U; ++v) {
          const int i = j + v * SIDE + side;
          const float g = __shfl(f[k], i & 63, 64);
          if (i < most) o[k] += g * x[k][v];
        }
    }
  }
#pragma unroll
  for (int k = 0; k < R; ++k)
#pragma unroll
    for (int d = LPR; d < 64; d <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[k][e] += __shfl_xor(o[k][e], d, 64);
  if constexpr (WAVES > 1) {
    if (lane == 0) {
      s_m[wave] = m[0];
      s_l[wave] = l[0];
    }
    if (lane < LPR) s_o[wave][lane] = o[0];
    __syncthreads();
    if (wave != 0) return;
    float mt = -INFINITY, lt = 0.f, part[WAVES];
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mt = fmaxf(mt, s_m[i]);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      part[i] = s_m[i] == -INFINITY ? 0.f : s_l[i] * fast_exp2(s_m[i] - mt);
      lt += part[i];
    }
    m[0] = mt;
    l[0] = lt;
    const float back = lt == 0.f ? 0.f : 1.f / lt;
    o[0] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (lane < LPR)
#pragma unroll
      for (int i = 0; i < WAVES; ++i) o[0] += part[i] * back * s_o[i][lane];
  }
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (k >= rows) break;
    const int r = w.r0 + row + k, tok = r / a.G, g = r - tok * a.G;
    const int64_t to = (int64_t)(w.c.first + tok) * a.Hq + w.kv * a.G + g;
    if (lane < LPR) {
      if constexpr (PP == 3) *reinterpret_cast<f32x4*>(static_cast<float*>(a.o) + to * D + 4 * lane) = o[k];
      else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + to * D + 4 * lane) = u32x2{pack_bf16(o[k][0], o[k][1]), pack_bf16(o[k][2], o[k][3])};
    }
    if (lane == 0 && a.lse) a.lse[to] = lse8(m[k], l[k]);
  }
}

inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }
constexpr size_t kFirst8 = (A8_UNITS + 1) * sizeof(int32_t);
inline size_t states8(int D, int cap) { return (size_t)2 * (D == 128 ? A8_GROUPS<128> : A8_GROUPS<64>) * cap; }
// of the steps' firsts and the states of cut units
inline size_t states8_bytes(int D, int cap) {
  return align_up(kFirst8) + align_up(states8(D, cap) * D * 4) + align_up(states8(D, cap) * 8);
}
// Units of tiles cost a search in the starts each, and every workgroup plans them all: past four a thread a
// workgroup for each unit is sooner done (7 fp32 prompts of 504 tokens, 2670 units: 210 us planned, 116 not;
// 14 of 1016 in bf16, 2700 tiles: 321 and 214).
inline bool planned8(int64_t units, bool tiles, int max_pages) {
  return units <= (tiles ? 4 * A8_NT : A8_UNITS) && units * (((int64_t)max_pages + A8_STEP - 1) / A8_STEP) < (1ll << 31);
}
inline void carve8(Args8& a, bool planned, int D, void* ws) {
  char* at = static_cast<char*>(ws);
  a.first = planned ? reinterpret_cast<int32_t*>(at) : nullptr;
  at += align_up(kFirst8);
  a.part_o = reinterpret_cast<float*>(at);
  a.part_ml = reinterpret_cast<float*>(at + align_up(states8(D, a.cap) * D * 4));
}

template <int D, int ROWS, int PP, bool CHUNK>
inline void merge8(const Args8& a, uint32_t groups, hipStream_t st) {
  TimedLaunch t(HK_TK_ATTN8_MERGE, st);
  const bool few = a.n_units * 32 <= A8_GROUPS<D>, many = a.cap > 16;   // units, of many parts; rows
  const int per = few ? 1 : many ? 4 * A8_NW : A8_NW;
  const uint32_t rows = (uint32_t)a.n_units * ((a.cap + per - 1) / per);
  const auto merge = few    ? attn8_merge_kernel<D, ROWS, PP, CHUNK, A8_NW, 1>
                     : many ? attn8_merge_kernel<D, ROWS, PP, CHUNK, 1, 4>
                            : attn8_merge_kernel<D, ROWS, PP, CHUNK, 1, 1>;
  hipLaunchKernelGGL(merge, dim3(rows), dim3(A8_NT), 0, st, a, (int)groups);
}

}  // namespace hk

// bf16 chunks of more than A8_ROWS rows of a KV head: units, workspace, launch
int64_t hk_attn8_tile_units(int NS, int Hkv, int G, int n_tokens);
// (heads * max_pages: of the tables; most: rows of a chunk at most)
size_t hk_attn8_tile_ws(int D, int64_t heads, int max_pages, int64_t most);
void hk_launch_attn8_tile(hk::Args8 a, hk_dtype format, int D, int64_t most, void* ws, hipStream_t st);
