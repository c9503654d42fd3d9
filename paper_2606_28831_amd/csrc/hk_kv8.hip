// 8-bit cache: rows quantised into the pool through a slot map, and read back (gfx950).
#include <type_traits>

#include "hk_kv8.h"

namespace hk {

constexpr int KV8_NT = 256;

struct Rows8 {
  const int64_t* slot_map;
  int64_t n_slots;
  int Hkv, n_layers, n_tokens;
  // token t of layer l: at t * row + l * layer elements
  int64_t k_layer, k_row, v_layer, v_row;
};
struct RowAt {
  int64_t slot, k, v;                         // elements; slot -1: none
};
__device__ __forceinline__ RowAt row_at(const Rows8& a, int64_t r, int D) {
  const int hk = (int)(r % a.Hkv);
  const int64_t t = r / a.Hkv % a.n_tokens, l = r / a.Hkv / a.n_tokens;
  int64_t slot = a.slot_map[r];
  if (slot < 0 || slot >= a.n_slots) slot = -1;
  return {slot, l * a.k_layer + t * a.k_row + (int64_t)hk * D, l * a.v_layer + t * a.v_row + (int64_t)hk * D};
}

// ------------------------------------------------------------------ write
// 16 bytes of a row, as fp32
template <typename T>
struct Piece;
template <>
struct Piece<uint16_t> {
  static constexpr int N = 8;
  u32x4 w;
  __device__ __forceinline__ float at(int i) const { return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]); }
  // the largest size, as bits: NaN and infinities are above every finite one
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(w[i] & 0x7fff0000u, (w[i] & 0x7fffu) << 16));
    return m;
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  u32x4 w;
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(w[i]); }
  __device__ __forceinline__ uint32_t largest() const {
    return max(max(w[0] & 0x7fffffffu, w[1] & 0x7fffffffu), max(w[2] & 0x7fffffffu, w[3] & 0x7fffffffu));
  }
};

// over groups of LANES lanes, in every lane
template <int LANES>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  v = max(v, dpp_u32<0xb1>(v, 0u));
  v = max(v, dpp_u32<0x4e>(v, 0u));
  v = max(v, dpp_u32<0x141>(v, 0u));
  if (LANES >= 16) v = max(v, dpp_u32<0x140>(v, 0u));
  if (LANES >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  return v;
}

// A thread takes 16 bytes of a K row and of its V row, both on their way at once; the threads of a row find
// its largest value by lane moves.  One pass: every value is read once and its code written once.  Memory
// bounds it: 8 prompts of 4096 tokens, 8 heads of 128, bf16, 201 MB in 23 us (part of it held by the caches;
// a large copy reads and writes 4.9 TB/s); a single token in 32 layers takes 3.5 us, a launch.
template <int F, typename T, int D>
__global__ __launch_bounds__(KV8_NT) void write_kv8_kernel(Rows8 a, const T* __restrict__ k_new,
                                                           const T* __restrict__ v_new, char* __restrict__ k_pool,
                                                           char* __restrict__ v_pool, float* __restrict__ k_scale,
                                                           float* __restrict__ v_scale) {
  constexpr int N = Piece<T>::N, LANES = D / N;
  const int64_t e = (int64_t)blockIdx.x * KV8_NT + threadIdx.x, r = e / LANES;
  if (r >= (int64_t)a.n_layers * a.n_tokens * a.Hkv) return;      // (whole rows)
  const int piece = (int)(e % LANES);
  const RowAt at = row_at(a, r, D);
  if (at.slot < 0) return;
  Piece<T> x[2];
  x[0].w = *reinterpret_cast<const u32x4*>(k_new + at.k + piece * N);
  x[1].w = *reinterpret_cast<const u32x4*>(v_new + at.v + piece * N);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t top = group_max<LANES>(x[i].largest());
    const bool fine = top < 0x7f800000u;
    const float big = fmaxf(__uint_as_float(top), KV8_LEAST), up = Code<F>::MOST / big;
    uint32_t c[N / 4];
#pragma unroll
    for (int j = 0; j < N / 4; ++j) {
      float y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = fine ? x[i].at(4 * j + k) * up : 0.f;
      c[j] = Code<F>::pack(y[0], y[1], y[2], y[3]);
    }
    char* to = (i ? v_pool : k_pool) + at.slot * D + piece * N;
    if constexpr (N == 8) *reinterpret_cast<u32x2*>(to) = u32x2{c[0], c[1]};
    else *reinterpret_cast<uint32_t*>(to) = c[0];
    if (piece == 0) (i ? v_scale : k_scale)[at.slot] = fine ? big / Code<F>::MOST : __builtin_nanf("");
  }
}

// ------------------------------------------------------------------ read
// A thread takes eight codes of a K row and, where V is asked for, of its V row, and writes 16 bytes (bf16) or
// 32 of each.  Memory bounds it: 32 sequences of up to 8192 tokens, 4 heads of 128, to bf16: 621 MB in 125 us,
// 5.0 TB/s.
template <int F, typename T, int D>
__global__ __launch_bounds__(KV8_NT) void read_kv8_kernel(Rows8 a, const char* __restrict__ k_pool,
                                                          const char* __restrict__ v_pool,
                                                          const float* __restrict__ k_scale,
                                                          const float* __restrict__ v_scale, T* __restrict__ k_out,
                                                          T* __restrict__ v_out) {
  constexpr int LANES = D / 8;
  const int64_t e = (int64_t)blockIdx.x * KV8_NT + threadIdx.x, r = e / LANES;
  if (r >= (int64_t)a.n_layers * a.n_tokens * a.Hkv) return;
  const int piece = (int)(e % LANES);
  const RowAt at = row_at(a, r, D);
  if (at.slot < 0) return;
  u32x2 w[2];
  float s[2];
  w[0] = *reinterpret_cast<const u32x2*>(k_pool + at.slot * D + piece * 8);
  s[0] = k_scale[at.slot];
  if (v_out) {
    w[1] = *reinterpret_cast<const u32x2*>(v_pool + at.slot * D + piece * 8);
    s[1] = v_scale[at.slot];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (i && !v_out) return;
    T* to = (i ? v_out + at.v : k_out + at.k) + piece * 8;
    float y[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      y[4 * h] = Code<F>::template value<0>(w[i][h]) * s[i];
      y[4 * h + 1] = Code<F>::template value<1>(w[i][h]) * s[i];
      y[4 * h + 2] = Code<F>::template value<2>(w[i][h]) * s[i];
      y[4 * h + 3] = Code<F>::template value<3>(w[i][h]) * s[i];
    }
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<u32x4*>(to) =
          u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
    } else {
      *reinterpret_cast<f32x4*>(to) = f32x4{y[0], y[1], y[2], y[3]};
      *reinterpret_cast<f32x4*>(to + 4) = f32x4{y[4], y[5], y[6], y[7]};
    }
  }
}

}  // namespace hk

using namespace hk;

namespace {
// f(format, row type, head size) as compile-time constants
template <typename F>
void dispatch(hk_dtype format, hk_dtype dtype, int D, F f) {
  using i8 = std::integral_constant<int, HK_I8>;
  using e4m3 = std::integral_constant<int, HK_E4M3>;
  using d64 = std::integral_constant<int, 64>;
  using d128 = std::integral_constant<int, 128>;
  auto by_d = [&](auto fmt, auto t) {
    if (D == 64) f(fmt, t, d64{});
    else f(fmt, t, d128{});
  };
  auto by_t = [&](auto fmt) {
    if (dtype == HK_BF16) by_d(fmt, uint16_t{});
    else by_d(fmt, float{});
  };
  if (format == HK_I8) by_t(i8{});
  else by_t(e4m3{});
}
uint32_t blocks_of(const Rows8& a, int lanes) {
  return (uint32_t)(((int64_t)a.n_layers * a.n_tokens * a.Hkv * lanes + KV8_NT - 1) / KV8_NT);
}
}  // namespace

hipError_t hk_launch_write_kv8(int Hkv, int D, const hk_paged_kv8* kv8, int n_layers, int n_tokens,
                               const int64_t* slot_map, hk_dtype dtype, const void* k_new, int64_t k_layer,
                               int64_t k_row, const void* v_new, int64_t v_layer, int64_t v_row, hipStream_t st) {
  const hk_paged_kv& kv = kv8->kv;
  const Rows8 a{slot_map, (int64_t)kv.num_pages * HK_PAGE, Hkv, n_layers, n_tokens, k_layer, k_row, v_layer, v_row};
  TimedLaunch t(HK_TK_WRITE_KV8, st);
  dispatch(kv.dtype, dtype, D, [&](auto f, auto x, auto d) {
    using T = decltype(x);
    constexpr int HD = decltype(d)::value;
    hipLaunchKernelGGL((write_kv8_kernel<decltype(f)::value, T, HD>), dim3(blocks_of(a, HD / Piece<T>::N)), dim3(KV8_NT),
                       0, st, a, static_cast<const T*>(k_new), static_cast<const T*>(v_new),
                       static_cast<char*>(kv.k_pool), static_cast<char*>(kv.v_pool), kv8->k_scale, kv8->v_scale);
  });
  return hipGetLastError();
}

hipError_t hk_launch_read_kv8(int Hkv, int D, const hk_paged_kv8* kv8, int n_layers, int n_tokens,
                              const int64_t* slot_map, hk_dtype dtype, void* k_out, int64_t k_layer, int64_t k_row,
                              void* v_out, int64_t v_layer, int64_t v_row, hipStream_t st) {
  const hk_paged_kv& kv = kv8->kv;
  const Rows8 a{slot_map, (int64_t)kv.num_pages * HK_PAGE, Hkv, n_layers, n_tokens, k_layer, k_row, v_layer, v_row};
  TimedLaunch t(HK_TK_READ_KV8, st);
  dispatch(kv.dtype, dtype, D, [&](auto f, auto x, auto d) {
    using T = decltype(x);
    constexpr int HD = decltype(d)::value;
    hipLaunchKernelGGL((read_kv8_kernel<decltype(f)::value, T, HD>), dim3(blocks_of(a, HD / 8)), dim3(KV8_NT), 0, st, a,
                       static_cast<const char*>(kv.k_pool), static_cast<const char*>(kv.v_pool), kv8->k_scale,
                       kv8->v_scale, static_cast<T*>(k_out), static_cast<T*>(v_out));
  });
  return hipGetLastError();
}
