// Drafted tokens against the target's probabilities, with given random numbers (gfx950).
//
// Everything is decided on whole numbers: a probability x counts F(x) = floor(2^40 x), a random
// number u counts floor(2^24 u), so neither the order of a sum nor the launch's shape can move a
// token.  Draft x of row t is kept while floor(2^24 u_t) F(q_t[x]) < 2^24 F(p_{t-1}[x]); the token
// after the kept ones is the first v whose running sum of weights passes
// floor(2^24 u) sum / 2^24, the weights being max(0, F(p) - F(q)) behind a rejected draft and F(p)
// otherwise.
//
// Two launches: the weights' sums over pieces of the row (every workgroup finds its sequence's
// rejected draft itself), then per sequence the piece and the place within it.  Bound by HBM
// reads of one row of p and one of q per sequence (64 of 131072 values: 67 MB in 15.7 us), at few
// sequences by the latency of loads that wait for one another (32000 values of one sequence: 5.6 us
// and 7.5; one launch of one workgroup a sequence, its rows in registers: 15).
#include "hk_chunk.h"

namespace hk {

constexpr int VF_NT = 256;
constexpr int VF_PER = 16;                    // values of a piece per thread
constexpr int VF_PIECE = VF_NT * VF_PER;

__device__ __forceinline__ float prob(const float* p, size_t i) { return p[i]; }
__device__ __forceinline__ float prob(const uint16_t* p, size_t i) { return __uint_as_float((uint32_t)p[i] << 16); }

// floor(2^40 clamp(x, 0, 1)), NaN as 0: x 2^8 and its fraction's 2^32-fold are exact
__device__ __forceinline__ unsigned long long whole(float x) {
  const float t = fminf(fmaxf(x, 0.f), 1.f) * 256.f;
  const float hi = floorf(t);
  return ((unsigned long long)(uint32_t)hi << 32) | (uint32_t)((t - hi) * 4294967296.f);
}
// HK_FLAG_* bits of a probability
__device__ __forceinline__ int strange(float x) { return x != x ? HK_FLAG_NAN : (x < 0.f || x > 1.f) ? HK_FLAG_RANGE : 0; }
__device__ __forceinline__ uint32_t draw24(float u) {
  return (uint32_t)(fminf(fmaxf(u, 0.f), 0x1.fffffep-1f) * 16777216.f);   // NaN as 0
}

// The kept drafts of a chunk of at least one row: every lane of a wave calls it and has the count.
template <typename T>
__device__ __forceinline__ int kept_drafts(Chunk c, int V, const int32_t* __restrict__ tokens, const T* __restrict__ p,
                                           int64_t p_row, const T* __restrict__ q, int64_t q_row,
                                           const float* __restrict__ u) {
  const int lane = threadIdx.x & 63;
  for (int i0 = 1; i0 < c.len; i0 += 64) {
    const int i = i0 + lane;
    bool reject = i < c.len;
    if (reject) {
      const int64_t t = c.first + i;
      const int x = tokens[t];
      if (x >= 0 && x < V) {
        const unsigned long long P = whole(prob(p + (t - 1) * p_row, x));
        const unsigned long long Q = q ? whole(prob(q + t * q_row, x)) : 1ull << 40;
        // draw24(u) Q < 2^24 P: the left side is below 2^64, the right side reaches it at P = 2^40
        reject = !((P >> 40) || draw24(u[t]) * Q < P << 24);
      }
    }
    const unsigned long long b = __ballot(reject);
    if (b) return i0 - 1 + __builtin_ctzll(b);
  }
  return c.len - 1;
}

// floor(m total / 2^24), m of the random number: m (total >> 24) and the low part's product, both exact
__device__ __forceinline__ unsigned long long goal_of(float u, unsigned long long total) {
  const unsigned long long d = draw24(u);
  return d * (total >> 24) + ((d * (total & 0xffffffull)) >> 24);
}

// Weights of a thread's values of a piece: consecutive threads hold consecutive values, value j of
// a thread lies VF_NT further on than value j - 1.
template <typename T>
struct Row {
  const T *p, *q;                             // q null: none, or the one draft `gone` alone
  int gone, V;
  bool rejected;
  __device__ __forceinline__ void load(int i, float& a, float& b) const {
    a = i < V ? prob(p, i) : 0.f;
    b = q ? (i < V ? prob(q, i) : 0.f) : i == gone ? 1.f : 0.f;
  }
};

// p and q of a thread's values are loaded together, then weighed
template <typename T>
__device__ __forceinline__ Row<T> row_of(Chunk c, int kept, int V, const int32_t* tokens, const T* p, int64_t p_row,
                                         const T* q, int64_t q_row) {
  Row<T> r;
  const int64_t t = c.first + kept;
  r.rejected = kept < c.len - 1;
  r.p = p + t * p_row;
  r.q = r.rejected && q ? q + (t + 1) * q_row : nullptr;
  r.gone = r.rejected && !q ? tokens[t + 1] : -1;
  r.V = V;
  return r;
}

__device__ __forceinline__ unsigned long long over(unsigned long long a, unsigned long long b) { return a > b ? a - b : 0ull; }

// Sums over a thread's values of what the draft leaves, and of F(p).  Nearly all probabilities are
// below 2^-8: where all of a wave's are, F is their 2^40-fold in 32 bits (11 instructions a value
// against 45; 64 rows of 131072 values: 15.7 us against 19.3).
constexpr uint32_t SMALL = 0x3b800000u;       // bits of 2^-8: of anything else, NaN and less than 0 too, not less
template <int N>
__device__ __forceinline__ void weigh(const float (&a)[N], const float (&b)[N], unsigned long long& left,
                                      unsigned long long& plain, int& odd) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) top = max(top, max(__float_as_uint(a[j]), __float_as_uint(b[j])));
  left = plain = 0;
  odd = 0;
  if (!__any(top >= SMALL)) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t P = (uint32_t)(a[j] * 0x1p40f), Q = (uint32_t)(b[j] * 0x1p40f);
      plain += P;
      left += max(P, Q) - Q;
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const unsigned long long P = whole(a[j]);
    plain += P;
    left += over(P, whole(b[j]));
    odd |= strange(a[j]) | strange(b[j]);
  }
  odd = (__any(odd & HK_FLAG_NAN) ? HK_FLAG_NAN : 0) | (__any(odd & HK_FLAG_RANGE) ? HK_FLAG_RANGE : 0);
}

// The chunk of sequence s; an empty one where the batch's slots were refused.
__device__ __forceinline__ Chunk granted_chunk(const int32_t* __restrict__ start, int s, int n_tokens, int max_len,
                                               const int32_t* __restrict__ granted) {
  const int given = granted ? *granted : 1;
  Chunk c = chunk_of(start, s, n_tokens, max_len);
  if (given == 0) c.len = 0;
  return c;
}

template <typename T>
__global__ __launch_bounds__(VF_NT) void verify_mass_kernel(
    int n_seq, int V, const int32_t* __restrict__ start, int n_tokens, int max_len, const int32_t* __restrict__ granted,
    const int32_t* __restrict__ tokens, const T* __restrict__ p, int64_t p_row, const T* __restrict__ q,
    int64_t q_row, const float* __restrict__ u, int32_t* __restrict__ n_accept, int32_t* __restrict__ n_drop,
    int32_t* __restrict__ status, unsigned long long* __restrict__ mass) {
  __shared__ unsigned long long s_red[VF_NT / 64];
  const int s = blockIdx.y, piece = blockIdx.x;
  const Chunk c = granted_chunk(start, s, n_tokens, max_len, granted);
  const int kept = c.len > 0 ? kept_drafts(c, V, tokens, p, p_row, q, q_row, u) : 0;
  if (piece == 0 && threadIdx.x == 0) {
    n_accept[s] = kept;
    n_drop[s] = max(c.len - 1 - kept, 0);
  }
  if (c.len <= 0) return;
  const Row<T> r = row_of(c, kept, V, tokens, p, p_row, q, q_row);
  float a[VF_PER], b[VF_PER];
#pragma unroll
  for (int j = 0; j < VF_PER; ++j) r.load(piece * VF_PIECE + j * VF_NT + threadIdx.x, a[j], b[j]);
  unsigned long long left, plain;
  int odd;
  weigh(a, b, left, plain, odd);
  left = block_sum_u64<VF_NT>(left, s_red);
  plain = block_sum_u64<VF_NT>(plain, s_red);
  if (odd && status && (threadIdx.x & 63) == 0) atomicOr(status, odd);
  if (threadIdx.x == 0) {
    unsigned long long* m = mass + ((size_t)s * gridDim.x + piece) * 2;
    m[0] = left;
    m[1] = plain;
  }
}

// inclusive sum over the wave's lanes
__device__ __forceinline__ unsigned long long wave_scan_u64(unsigned long long x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned long long y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}

template <typename T>
__global__ __launch_bounds__(VF_NT) void verify_pick_kernel(
    int V, const int32_t* __restrict__ start, int n_tokens, int max_len, const int32_t* __restrict__ granted,
    const int32_t* __restrict__ tokens, const T* __restrict__ p, int64_t p_row, const T* __restrict__ q, int64_t q_row,
    const float* __restrict__ u, const int32_t* __restrict__ n_accept, const unsigned long long* __restrict__ mass, int pieces,
    int32_t* __restrict__ next_token) {
  __shared__ unsigned long long s_red[VF_NT / 64], s_before;
  __shared__ int s_piece;
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Chunk c = granted_chunk(start, s, n_tokens, max_len, granted);
  if (c.len <= 0) {
    if (threadIdx.x == 0) next_token[s] = -1;
    return;
  }
  const unsigned long long* m = mass + (size_t)s * pieces * 2;
  // at most VF_NT pieces of a row: one per thread
  const unsigned long long left = threadIdx.x < pieces ? m[2 * threadIdx.x] : 0ull;
  const unsigned long long plain = threadIdx.x < pieces ? m[2 * threadIdx.x + 1] : 0ull;
  const Row<T> r = row_of(c, n_accept[s], V, tokens, p, p_row, q, q_row);
  unsigned long long total = block_sum_u64<VF_NT>(left, s_red);
  const bool rest = r.rejected && total > 0;   // (not rejected: both sums are of F(p))
  if (!rest) total = block_sum_u64<VF_NT>(plain, s_red);
  if (total == 0) {
    if (threadIdx.x == 0) next_token[s] = -1;
    return;
  }
  const unsigned long long goal = goal_of(u[c.first], total);
  auto before = [&](unsigned long long x) {    // exclusive sum over the workgroup
    const unsigned long long y = wave_scan_u64(x);
    __syncthreads();
    if (lane == 63) s_red[wave] = y;
    __syncthreads();
    unsigned long long b = y - x;
    for (int w = 0; w < wave; ++w) b += s_red[w];
    return b;
  };
  {
    const unsigned long long x = rest ? left : plain, b = before(x);
    if (b <= goal && goal < b + x) {
      s_piece = threadIdx.x;
      s_before = b;
    }
  }
  __syncthreads();
  // within the piece a thread takes consecutive values; the one whose span holds the goal walks them
  const int first = s_piece * VF_PIECE + threadIdx.x * VF_PER;
  unsigned long long w[VF_PER], sum = 0;
  {
    float a[VF_PER], b[VF_PER];
#pragma unroll
    for (int j = 0; j < VF_PER; ++j) r.load(first + j, a[j], b[j]);
#pragma unroll
    for (int j = 0; j < VF_PER; ++j) {
      const unsigned long long P = whole(a[j]);
      w[j] = rest ? over(P, whole(b[j])) : P;
      sum += w[j];
    }
  }
  unsigned long long at = s_before + before(sum);
  if (at <= goal && goal < at + sum) {
    int v = first;
#pragma unroll
    for (int j = 0; j < VF_PER; ++j) {
      at += w[j];
      if (at <= goal) v = first + j + 1;
    }
    next_token[s] = v;
  }
}

template <typename T>
static void launch_verify(int n_seq, int V, const hk_chunks* ch, const int32_t* tokens, const void* p, int64_t p_row,
                          const void* q, int64_t q_row, const float* u, int32_t* n_accept, int32_t* next_token,
                          int32_t* n_drop, int32_t* status, void* ws, hipStream_t st) {
  const int pieces = (V + VF_PIECE - 1) / VF_PIECE;
  unsigned long long* mass = static_cast<unsigned long long*>(ws);
  hipLaunchKernelGGL(verify_mass_kernel<T>, dim3(pieces, n_seq), dim3(VF_NT), 0, st, n_seq, V, ch->start, ch->n_tokens,
                     ch->max_len, ch->granted, tokens, static_cast<const T*>(p), p_row, static_cast<const T*>(q), q_row, u,
                     n_accept, n_drop, status, mass);
  hipLaunchKernelGGL(verify_pick_kernel<T>, dim3(n_seq), dim3(VF_NT), 0, st, V, ch->start, ch->n_tokens, ch->max_len,
                     ch->granted, tokens, static_cast<const T*>(p), p_row, static_cast<const T*>(q), q_row, u, n_accept, mass,
                     pieces, next_token);
}

}  // namespace hk

using namespace hk;

size_t hk_verify_ws(int n_seq, int V) {
  return (size_t)n_seq * ((V + VF_PIECE - 1) / VF_PIECE) * 2 * sizeof(unsigned long long);
}

hipError_t hk_launch_verify(int n_seq, int V, hk_dtype dtype, const hk_chunks* ch, const int32_t* tokens,
                            const void* p, int64_t p_row, const void* q, int64_t q_row, const float* u,
                            int32_t* n_accept, int32_t* next_token, int32_t* n_drop, int32_t* status, void* ws,
                            hipStream_t st) {
  TimedLaunch t(HK_TK_VERIFY, st);
  if (dtype == HK_BF16)
    launch_verify<uint16_t>(n_seq, V, ch, tokens, p, p_row, q, q_row, u, n_accept, next_token, n_drop, status, ws, st);
  else
    launch_verify<float>(n_seq, V, ch, tokens, p, p_row, q, q_row, u, n_accept, next_token, n_drop, status, ws, st);
  return hipGetLastError();
}
