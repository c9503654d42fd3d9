// Slots for chunks of new tokens: reserved at the rows' ends from the chunks' lengths, filled
// through the slot map, and taken back (gfx950).
//
// Reserving and trimming are two launches each.  Count: a wave takes 64 heads and leaves their
// row ends and, scanned over the wave, the pages each needs or frees; block 0 keeps the free
// stack's top.  Write: every workgroup scans the blocks' counts itself (at most 1024 of them), so
// the pops and pushes follow the head order with no workgroup waiting on another, decides success
// from the total, and takes its share of the work.  The second launch reads row ends from the
// first one's workspace, never from the masks and counts it changes.
// Bound by latency: two dependent launches of a few loads each.
#include "hk_chunk.h"

namespace hk {

constexpr int SL_HPB = 64;                    // heads per count block
constexpr int SL_NT = 256;
constexpr int SL_BLOCKS = 1024;               // count blocks of 65535 heads

// Workspace (int32): top snapshot, a "refuse" word per block, the blocks' page counts, then per
// head its page count, row end and pages of the block's earlier heads.
struct SlotWs {
  int32_t *top, *refuse, *count, *n, *end, *base;
};
__host__ __device__ inline SlotWs slot_ws(void* ws, int n_heads) {
  const int nblk = (n_heads + SL_HPB - 1) / SL_HPB;
  int32_t* w = static_cast<int32_t*>(ws);
  return {w, w + 1, w + 1 + nblk, w + 1 + 2 * nblk, w + 1 + 2 * nblk + n_heads, w + 1 + 2 * nblk + 2 * n_heads};
}

// inclusive sum over the wave's lanes
__device__ __forceinline__ int wave_scan(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}

// What precedes every count block, and the total: every thread of the workgroup calls it.
// s_before[SL_BLOCKS] receives the exclusive sums.  The total is 64-bit: a refused call's needs can
// pass 2^31; a granted one's sums are below the stack's size.
__device__ inline long long scan_blocks(const int32_t* __restrict__ count, int nblk, int32_t* s_before) {
  __shared__ long long s_wave[SL_NT / 64];
  constexpr int PER = SL_BLOCKS / SL_NT;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long mine[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = threadIdx.x * PER + i;
    mine[i] = b < nblk ? count[b] : 0;
    sum += mine[i];
  }
  long long x = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  long long before = x - sum, total = 0;
#pragma unroll
  for (int w = 0; w < SL_NT / 64; ++w) {
    if (w < wave) before += s_wave[w];
    total += s_wave[w];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    s_before[threadIdx.x * PER + i] = (int32_t)before;
    before += mine[i];
  }
  __syncthreads();
  return total;
}

// ------------------------------------------------------------------ reserve
__global__ __launch_bounds__(64) void reserve_count_kernel(
    int n_heads, int Hkv, int n_seq, const int32_t* __restrict__ start, int n_tokens, int max_len,
    const int32_t* __restrict__ n_pages, const uint16_t* __restrict__ masks, int max_pages,
    const int32_t* __restrict__ free_top, void* ws) {
  const SlotWs w = slot_ws(ws, n_heads);
  const int h = blockIdx.x * SL_HPB + threadIdx.x;
  int need = 0, n = 0, end = 0, refuse = 0;
  if (h < n_heads) {
    const int s = (h / Hkv) % n_seq;
    n = min(max(n_pages[h], 0), max_pages);
    end = row_end(n, n > 0 ? masks[(size_t)h * max_pages + n - 1] : 0u);
    const int a = start[s], b = start[s + 1];
    if (a < 0 || b < a || b > n_tokens || b - a > max_len) {
      refuse = HK_FLAG_CHUNK;
    } else {
      need = max(0, (end + (b - a) + HK_PAGE - 1) / HK_PAGE - n);
      if (n + need > max_pages) refuse = HK_FLAG_NOSPACE;
    }
  }
  const int x = wave_scan(need);
  if (h < n_heads) {
    w.n[h] = n;
    w.end[h] = end;
    w.base[h] = x - need;
  }
  refuse = (__any(refuse & HK_FLAG_CHUNK) ? HK_FLAG_CHUNK : 0) | (__any(refuse & HK_FLAG_NOSPACE) ? HK_FLAG_NOSPACE : 0);
  if (threadIdx.x == 63) {
    w.count[blockIdx.x] = x;
    w.refuse[blockIdx.x] = refuse;
    if (blockIdx.x == 0) *w.top = *free_top;
  }
}

// Workgroups below n_table take one (head, touched page) a thread: page i of a head is the i-th
// from the one that holds its row's end.  The others take one (layer, row, KV head) of the slot
// map a thread, from the workspace and the old pages alone.
__global__ __launch_bounds__(SL_NT) void reserve_write_kernel(
    int n_heads, int Hkv, int n_seq, const int32_t* __restrict__ start, int n_tokens, int max_len,
    int touched, uint32_t n_table, int32_t* __restrict__ table, uint16_t* __restrict__ masks,
    int32_t* __restrict__ n_pages, int max_pages, const int32_t* __restrict__ free_ids,
    int32_t* __restrict__ free_top, int capacity, int64_t* __restrict__ slot_map,
    int32_t* __restrict__ status, int32_t* __restrict__ granted, const void* ws) {
  __shared__ int32_t s_before[SL_BLOCKS];
  __shared__ int s_refuse;
  const SlotWs w = slot_ws(const_cast<void*>(ws), n_heads);
  const int nblk = (n_heads + SL_HPB - 1) / SL_HPB;
  if (threadIdx.x == 0) s_refuse = 0;
  __syncthreads();
  for (int b = threadIdx.x; b < nblk; b += SL_NT)
    if (w.refuse[b]) atomicOr(&s_refuse, w.refuse[b]);
  const long long total = scan_blocks(w.count, nblk, s_before);
  const int top = min(*w.top, capacity);
  int refuse = s_refuse;
  if (total > top) refuse |= HK_FLAG_NOSPACE;
  const bool ok = refuse == 0;
  const int first_pop = ok ? top - (int)total : 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (ok) *free_top = first_pop;
    else if (status) atomicOr(status, refuse);
    if (granted) *granted = ok;
  }
  if (blockIdx.x < n_table) {
    const size_t e = (size_t)blockIdx.x * SL_NT + threadIdx.x;
    const int h = (int)min(e / touched, (size_t)n_heads), i = (int)(e % touched);
    if (!ok || h >= n_heads) return;
    const Chunk c = chunk_of(start, (h / Hkv) % n_seq, n_tokens, max_len);
    const int n = w.n[h], end = w.end[h], to = end + c.len;
    const int page = end / HK_PAGE + i, lo = max(end - page * HK_PAGE, 0), hi = min(to - page * HK_PAGE, HK_PAGE);
    if (i == 0) n_pages[h] = max(n, (to + HK_PAGE - 1) / HK_PAGE);
    if (hi <= lo) return;
    const uint32_t bits = (1u << hi) - (1u << lo);
    const size_t at = (size_t)h * max_pages + page;
    if (page < n) {
      masks[at] = (uint16_t)(masks[at] | bits);
    } else {
      table[at] = free_ids[first_pop + s_before[h / SL_HPB] + w.base[h] + page - n];
      masks[at] = (uint16_t)bits;
    }
    return;
  }
  const size_t e = (size_t)(blockIdx.x - n_table) * SL_NT + threadIdx.x;
  const size_t rows = (size_t)n_tokens * Hkv;
  const int n_layers = n_heads / Hkv / n_seq;
  if (e >= rows * n_layers) return;
  const int l = (int)(e / rows), t = (int)(e % rows / Hkv), hk = (int)(e % Hkv);
  int64_t slot = -1;
  if (ok) {
    // the last sequence that starts at or before row t (chunks were found to be in order)
    int lo = 0, hi = n_seq;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (start[mid] <= t) lo = mid;
      else hi = mid;
    }
    const int i = t - start[lo];
    if (i >= 0 && t < start[lo + 1]) {
      const int h = (l * n_seq + lo) * Hkv + hk, j = w.end[h] + i, page = j / HK_PAGE, n = w.n[h];
      const int id = page < n ? table[(size_t)h * max_pages + page]
                              : free_ids[first_pop + s_before[h / SL_HPB] + w.base[h] + page - n];
      slot = (int64_t)id * HK_PAGE + j % HK_PAGE;
    }
  }
  slot_map[e] = slot;
}

// ------------------------------------------------------------------ write
// One 16-byte piece of a K row and the same of its V row per thread, loaded beside the slot.  A row
// without one (-1, or one outside the pool) is not written.  Bound by the copy.
__global__ __launch_bounds__(SL_NT) void write_kv_kernel(
    int Hkv, int pieces, int n_layers, int n_tokens, int64_t n_slots, const int64_t* __restrict__ slot_map,
    const char* __restrict__ k_new, int64_t k_layer, int64_t k_row, const char* __restrict__ v_new,
    int64_t v_layer, int64_t v_row, char* __restrict__ k_pool, char* __restrict__ v_pool) {
  const size_t e = (size_t)blockIdx.x * SL_NT + threadIdx.x, r = e / pieces;
  const int piece = (int)(e % pieces);
  if (r >= (size_t)n_layers * n_tokens * Hkv) return;
  const int hk = (int)(r % Hkv);
  const int64_t t = (int64_t)(r / Hkv % n_tokens), l = (int64_t)(r / Hkv / n_tokens);
  const int64_t slot = slot_map[r];
  const int64_t in = ((int64_t)hk * pieces + piece) * 16;
  const u32x4 k = *reinterpret_cast<const u32x4*>(k_new + l * k_layer + t * k_row + in);
  const u32x4 v = *reinterpret_cast<const u32x4*>(v_new + l * v_layer + t * v_row + in);
  if (slot < 0 || slot >= n_slots) return;
  const int64_t out = (slot * pieces + piece) * 16;
  *reinterpret_cast<u32x4*>(k_pool + out) = k;
  *reinterpret_cast<u32x4*>(v_pool + out) = v;
}

// ------------------------------------------------------------------ trim
// heads; 512 heads with cuts of up to 3000 tokens: a wave each 5.4 us, eight lanes each 11.2
constexpr int TRIM_FEW = 2048;
struct Cut {
  int keep, end;                              // pages that stay, and the row's end after the cut
};
__device__ __forceinline__ Cut cut_row(int n, int end, int drop) {
  if (drop <= 0) return {n, end};
  const int e = end - min(drop, end);
  return {(e + HK_PAGE - 1) / HK_PAGE, e};
}

__global__ __launch_bounds__(64) void trim_count_kernel(int n_heads, int Hkv, int n_seq,
                                                        const int32_t* __restrict__ n_drop,
                                                        const int32_t* __restrict__ n_pages,
                                                        const uint16_t* __restrict__ masks, int max_pages,
                                                        const int32_t* __restrict__ free_top, void* ws) {
  const SlotWs w = slot_ws(ws, n_heads);
  const int h = blockIdx.x * SL_HPB + threadIdx.x;
  int gone = 0;
  if (h < n_heads) {
    const int n = min(max(n_pages[h], 0), max_pages);
    const int end = row_end(n, n > 0 ? masks[(size_t)h * max_pages + n - 1] : 0u);
    gone = n - cut_row(n, end, n_drop[(h / Hkv) % n_seq]).keep;
    w.n[h] = n;
    w.end[h] = end;
  }
  const int x = wave_scan(gone);
  if (h < n_heads) w.base[h] = x - gone;
  if (threadIdx.x == 63) {
    w.count[blockIdx.x] = x;
    if (blockIdx.x == 0) *w.top = *free_top;
  }
}

// LANES lanes per head: a wave where heads are few, for long cuts; eight where they are many and
// cuts are a few pages (16384 heads, 8 tokens: 5.0 us, a wave each 9.4).  The stack holds every page
// of the pool (checked by the caller), so a push only misses where the tables list more pages than
// there are: such a page is not pushed.
template <int LANES>
__global__ __launch_bounds__(SL_NT) void trim_write_kernel(int n_heads, int Hkv, int n_seq,
                                                           const int32_t* __restrict__ n_drop,
                                                           int32_t* __restrict__ table,
                                                           uint16_t* __restrict__ masks,
                                                           int32_t* __restrict__ n_pages, int max_pages,
                                                           int32_t* __restrict__ free_ids,
                                                           int32_t* __restrict__ free_top, int capacity,
                                                           const void* ws) {
  __shared__ int32_t s_before[SL_BLOCKS];
  const SlotWs w = slot_ws(const_cast<void*>(ws), n_heads);
  const long long total = scan_blocks(w.count, (n_heads + SL_HPB - 1) / SL_HPB, s_before);
  const int top = max(*w.top, 0);
  if (blockIdx.x == 0 && threadIdx.x == 0) *free_top = (int)min(top + total, (long long)capacity);
  const int h = blockIdx.x * (SL_NT / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
  if (h >= n_heads) return;
  const int drop = n_drop[(h / Hkv) % n_seq];
  if (drop <= 0) return;
  const int n = w.n[h];
  const Cut c = cut_row(n, w.end[h], drop);
  int32_t* row = table + (size_t)h * max_pages;
  uint16_t* mrow = masks + (size_t)h * max_pages;
  const int to = top + s_before[h / SL_HPB] + w.base[h];
  for (int i = lane; i < n - c.keep; i += LANES) {
    if (to + i < capacity) free_ids[to + i] = row[c.keep + i];
    row[c.keep + i] = -1;
    mrow[c.keep + i] = 0;
  }
  if (lane == 0) {
    n_pages[h] = c.keep;
    if (c.end % HK_PAGE) mrow[c.keep - 1] = (uint16_t)(mrow[c.keep - 1] & ((1u << (c.end % HK_PAGE)) - 1u));
  }
}

}  // namespace hk

using namespace hk;

size_t hk_reserve_ws(int n_heads) {
  const size_t nblk = ((size_t)n_heads + SL_HPB - 1) / SL_HPB;
  return (1 + 2 * nblk + 3 * (size_t)n_heads) * sizeof(int32_t);
}
size_t hk_trim_ws(int n_heads) { return hk_reserve_ws(n_heads); }

hipError_t hk_launch_reserve(int n_heads, int Hkv, const hk_paged_kv* kv, const hk_chunks* ch,
                             const hk_allocator* alloc, int64_t* slot_map, int32_t* status, void* ws,
                             hipStream_t st) {
  const int nblk = (n_heads + SL_HPB - 1) / SL_HPB;
  // a chunk of max_len tokens touches at most this many pages
  const int touched = (ch->max_len + 2 * HK_PAGE - 2) / HK_PAGE;
  const size_t n_table = ((size_t)n_heads * touched + SL_NT - 1) / SL_NT;
  const size_t rows = (size_t)(n_heads / ch->n_seq) * ch->n_tokens;   // n_heads / n_seq = layers x KV heads
  const size_t n_map = slot_map ? (rows + SL_NT - 1) / SL_NT : 0;
  TimedLaunch t(HK_TK_RESERVE, st);
  hipLaunchKernelGGL(reserve_count_kernel, dim3(nblk), dim3(64), 0, st, n_heads, Hkv, ch->n_seq, ch->start,
                     ch->n_tokens, ch->max_len, kv->n_pages, kv->page_mask, kv->max_pages, alloc->free_top, ws);
  hipLaunchKernelGGL(reserve_write_kernel, dim3((uint32_t)(n_table + n_map)), dim3(SL_NT), 0, st, n_heads, Hkv,
                     ch->n_seq, ch->start, ch->n_tokens, ch->max_len, touched, (uint32_t)n_table, kv->page_table,
                     kv->page_mask, kv->n_pages, kv->max_pages, alloc->free_ids, alloc->free_top, alloc->capacity,
                     slot_map, status, ch->granted, ws);
  return hipGetLastError();
}

hipError_t hk_launch_write_kv(int Hkv, int D, const hk_paged_kv* kv, int n_layers, int n_tokens,
                              const int64_t* slot_map, const void* k_new, int64_t k_layer, int64_t k_row,
                              const void* v_new, int64_t v_layer, int64_t v_row, hipStream_t st) {
  const int es = kv->dtype == HK_BF16 ? 2 : 4, pieces = D * es / 16;
  const size_t n = (size_t)n_layers * n_tokens * Hkv * pieces;
  TimedLaunch t(HK_TK_WRITE_KV, st);
  hipLaunchKernelGGL(write_kv_kernel, dim3((uint32_t)((n + SL_NT - 1) / SL_NT)), dim3(SL_NT), 0, st, Hkv, pieces,
                     n_layers, n_tokens, (int64_t)kv->num_pages * HK_PAGE, slot_map,
                     static_cast<const char*>(k_new), k_layer * es, k_row * es, static_cast<const char*>(v_new),
                     v_layer * es, v_row * es, static_cast<char*>(kv->k_pool), static_cast<char*>(kv->v_pool));
  return hipGetLastError();
}

hipError_t hk_launch_trim(int n_heads, int Hkv, const hk_paged_kv* kv, int n_seq, const int32_t* n_drop,
                          const hk_allocator* alloc, void* ws, hipStream_t st) {
  const int nblk = (n_heads + SL_HPB - 1) / SL_HPB;
  TimedLaunch t(HK_TK_TRIM, st);
  hipLaunchKernelGGL(trim_count_kernel, dim3(nblk), dim3(64), 0, st, n_heads, Hkv, n_seq, n_drop, kv->n_pages,
                     kv->page_mask, kv->max_pages, alloc->free_top, ws);
  const auto write = n_heads <= TRIM_FEW ? trim_write_kernel<64> : trim_write_kernel<8>;
  const int per = SL_NT / (n_heads <= TRIM_FEW ? 64 : 8);
  hipLaunchKernelGGL(write, dim3((n_heads + per - 1) / per), dim3(SL_NT), 0, st, n_heads, Hkv, n_seq, n_drop,
                     kv->page_table, kv->page_mask, kv->n_pages, kv->max_pages, alloc->free_ids, alloc->free_top,
                     alloc->capacity, ws);
  return hipGetLastError();
}
