// Chunks of new tokens: launchers and device helpers shared by the slot, attention and
// verification kernels (gfx950).
#pragma once

#include "hk_internal.h"

namespace hk {

// One past the highest valid slot of a row's newest page, or that page's first slot when none of
// its slots is valid; 0 for an empty row.  n: pages in use, newest: their last mask.
__device__ __forceinline__ int row_end(int n, uint32_t newest) {
  return n > 0 ? (n - 1) * HK_PAGE + (32 - __clz((int)(newest & 0xffffu))) : 0;
}

// Rows [first, first + len) of sequence s.  A chunk that is not what hk_chunks promises (start
// descending or outside the n_tokens rows, longer than max_len) is cut to the rows that exist.
struct Chunk {
  int first, len;
};
__device__ __forceinline__ Chunk chunk_of(const int32_t* __restrict__ start, int s, int n_tokens, int max_len) {
  const int a = min(max(start[s], 0), n_tokens), b = min(max(start[s + 1], a), n_tokens);
  return {a, min(b - a, max_len)};
}

}  // namespace hk

size_t hk_reserve_ws(int n_heads);
hipError_t hk_launch_reserve(int n_heads, int Hkv, const hk_paged_kv* kv, const hk_chunks* ch,
                             const hk_allocator* alloc, int64_t* slot_map, int32_t* status, void* ws,
                             hipStream_t st);
hipError_t hk_launch_write_kv(int Hkv, int D, const hk_paged_kv* kv, int n_layers, int n_tokens,
                              const int64_t* slot_map, const void* k_new, int64_t k_layer, int64_t k_row,
                              const void* v_new, int64_t v_layer, int64_t v_row, hipStream_t st);
size_t hk_trim_ws(int n_heads);
hipError_t hk_launch_trim(int n_heads, int Hkv, const hk_paged_kv* kv, int n_seq, const int32_t* n_drop,
                          const hk_allocator* alloc, void* ws, hipStream_t st);

size_t hk_chunk_attn_ws(int NS, int Hq, int Hkv, int D, int n_tokens, int max_len, int max_pages);
// threads of its largest launch at most
long long hk_chunk_attn_threads(int NS, int Hq, int Hkv, int n_tokens, int max_len, int max_pages);
hipError_t hk_launch_chunk_attn(int NS, int Hq, int Hkv, int D, const hk_paged_kv* kv, const hk_chunks* ch,
                                const void* q, int64_t q_row, float sm_scale, void* o, float* lse, void* ws,
                                hipStream_t st);

size_t hk_verify_ws(int n_seq, int V);
hipError_t hk_launch_verify(int n_seq, int V, hk_dtype dtype, const hk_chunks* ch, const int32_t* tokens,
                            const void* p, int64_t p_row, const void* q, int64_t q_row, const float* u,
                            int32_t* n_accept, int32_t* next_token, int32_t* n_drop, int32_t* status, void* ws,
                            hipStream_t st);
