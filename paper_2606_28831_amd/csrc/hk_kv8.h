// The 8-bit cache: formats, launchers and device helpers shared by its kernels (gfx950).
#pragma once

#include "hk_internal.h"

namespace hk {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A row x of D values is held as D codes and one fp32 scale:
//   a = max(max |x|, LEAST),  scale = a / MOST,  code = round(x (MOST / a)),
// every step rounded to fp32, codes to the nearest with ties to even; a row with an infinite value
// or NaN has codes 0 and the scale NaN.  Below LEAST the steps stay those of LEAST: neither quotient
// leaves the normal numbers.  Both kinds of code are exact in bf16 and in fp16.
constexpr float KV8_LEAST = 0x1p-100f;
template <int F>
struct Code;
template <>
struct Code<HK_I8> {
  static constexpr float MOST = 127.f;
  // codes of four values
  __device__ static __forceinline__ uint32_t pack(float a, float b, float c, float d) {
    const int x = (int)__builtin_rintf(a), y = (int)__builtin_rintf(b), z = (int)__builtin_rintf(c), w = (int)__builtin_rintf(d);
    return (uint32_t)(x & 255) | (uint32_t)(y & 255) << 8 | (uint32_t)(z & 255) << 16 | (uint32_t)w << 24;
  }
  template <int I>
  __device__ static __forceinline__ float value(uint32_t w) {
    return (float)(int8_t)(w >> (8 * I));
  }
  // codes 2 I and 2 I + 1 of w as two bf16
  template <int I>
  __device__ static __forceinline__ uint32_t pair(uint32_t w) {
    return __builtin_amdgcn_perm(__float_as_uint(value<2 * I + 1>(w)), __float_as_uint(value<2 * I>(w)), 0x07060302u);
  }
  // Codes I of a and of b as two fp16 times 2^-F16_DOWN.  A byte c + 128 alone in a half is the subnormal
  // (c + 128) 2^-24, so that one fma a pair brings codes to c 2^-9, exactly.
  static constexpr int F16_DOWN = 9;
  template <int I>
  __device__ static __forceinline__ uint32_t halves(uint32_t a, uint32_t b) {
    const uint32_t x = __builtin_amdgcn_perm(b ^ 0x80808080u, a ^ 0x80808080u, 0x0c040c00u + 0x00010001u * I);
    const f16x2 up = {(_Float16)32768.f, (_Float16)32768.f}, less = {(_Float16)-0.25f, (_Float16)-0.25f};
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, x), up, less));
  }
};
template <>
struct Code<HK_E4M3> {
  static constexpr float MOST = 448.f;
  __device__ static __forceinline__ uint32_t pack(float a, float b, float c, float d) {
    // (the quotients' roundings may leave a row's largest value one bit above MOST)
    const auto cut = [](float x) { return fminf(fmaxf(x, -MOST), MOST); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(cut(a), cut(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(cut(c), cut(d), w, true);
  }
  template <int I>
  __device__ static __forceinline__ float value(uint32_t w) {
    return __builtin_amdgcn_cvt_f32_fp8((int)w, I);
  }
  template <int I>
  __device__ static __forceinline__ uint32_t pair(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, I != 0));
  }
  static constexpr int F16_DOWN = 0;
  template <int I>
  __device__ static __forceinline__ uint32_t halves(uint32_t a, uint32_t b) {
    const uint32_t x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, I >= 2));
    const uint32_t y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, I >= 2));
    return __builtin_amdgcn_perm(y, x, I & 1 ? 0x07060302u : 0x05040100u);
  }
};

// the high halves of two words: the bf16 of two fp32 that are exact in bf16, or cut to it
__device__ __forceinline__ uint32_t high_halves(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

}  // namespace hk

hipError_t hk_launch_write_kv8(int Hkv, int D, const hk_paged_kv8* kv8, int n_layers, int n_tokens,
                               const int64_t* slot_map, hk_dtype dtype, const void* k_new, int64_t k_layer,
                               int64_t k_row, const void* v_new, int64_t v_layer, int64_t v_row, hipStream_t st);
hipError_t hk_launch_read_kv8(int Hkv, int D, const hk_paged_kv8* kv8, int n_layers, int n_tokens,
                              const int64_t* slot_map, hk_dtype dtype, void* k_out, int64_t k_layer, int64_t k_row,
                              void* v_out, int64_t v_layer, int64_t v_row, hipStream_t st);

// chunks NULL: one token per sequence, o in fp32
size_t hk_attn8_ws(int NS, int Hq, int Hkv, int D, const hk_chunks* ch, int max_pages);
// workgroups of its largest launch
double hk_attn8_groups(int NS, int Hq, int Hkv, const hk_chunks* ch, int max_pages);
hipError_t hk_launch_attn8(int NS, int Hq, int Hkv, int D, const hk_paged_kv8* kv8, const hk_chunks* ch,
                           hk_dtype dtype, const void* q, int64_t q_row, float sm_scale, void* o, float* lse,
                           void* ws, hipStream_t st);

hipError_t hk_launch_compact8(int n_heads, int D, const hk_paged_kv8* kv8, const uint32_t* sel_bits,
                              int L_dense, int L_sparse, const int32_t* head_mode, const hk_allocator* alloc,
                              int32_t* status, void* ws, hipStream_t st);
