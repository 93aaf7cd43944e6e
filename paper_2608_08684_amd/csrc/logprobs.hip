// Log probabilities of given tokens from a row of logits, with the row's entropy, the
// token's rank and the best alternatives.
//
//   log p_tok = (x_tok - m) - log S,   S = sum_v e^(x_v - m),  m = max_v x_v
//   H = log S - T / S,                 T = sum_v (x_v - m) e^(x_v - m)
//   rank = 1 + #{v : x_v > x_tok, or x_v = x_tok and v < tok}
//
// Each logit is read once: a running (m, S, T) per thread, joined in a fixed order.
// The alternatives come out of the same pass by groups of consecutive logits (16 lanes
// times one 16-byte load): the n best logits, ordered by value and then by lower index,
// lie in the n groups whose largest logits come first in that order (each of those
// groups holds at least one logit that precedes any logit of another group), so only
// those groups are looked at again.
#include <math.h>

#include <algorithm>

#include "rk_internal.h"

namespace rk {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kLpThreads = 256;

template <typename T> struct Logit;
template <> struct Logit<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(v4u u, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(u[i]);
  }
};
template <> struct Logit<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(v4u u, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
};

// Running softmax sums relative to the maximum m; s and t are 0 while m is -inf.
struct Sums {
  float m, s, t;
  __device__ __forceinline__ void join(float m2, float s2, float t2) {
    const float M = fmaxf(m, m2);
    const float ref = M == -INFINITY ? 0.f : M;
    const float d1 = fmaxf(m - ref, -1.0e4f), d2 = fmaxf(m2 - ref, -1.0e4f);   // -inf: weight 0
    const float c1 = __builtin_amdgcn_exp2f(d1 * kLog2e), c2 = __builtin_amdgcn_exp2f(d2 * kLog2e);
    t = c1 * (t + d1 * s) + c2 * (t2 + d2 * s2);
    s = c1 * s + c2 * s2;
    m = M;
  }
};

// A row seen as 16-byte vectors: vector v holds logits v N - shift .. of the row.
template <typename T> struct RowView {
  static constexpr int N = Logit<T>::N;
  const T* row;
  const v4u* base;   // aligned address at or below the row's first logit
  int shift, vocab, n_vec;
  __device__ __forceinline__ RowView(const LogprobArgs& a, int64_t r) {
    row = (const T*)a.logits + r * a.row_stride;
    shift = (int)(((uintptr_t)row & 15) / sizeof(T));
    base = (const v4u*)((uintptr_t)row & ~(uintptr_t)15);
    vocab = a.vocab;
    n_vec = (int)(((int64_t)shift + vocab + N - 1) / N);
  }
  // vectors that reach outside the row are read logit by logit; what is outside is -inf
  __device__ __forceinline__ void load(int v, float* f) const {
    const int id = v * N - shift;
    if (id >= 0 && id <= vocab - N) {
      Logit<T>::get(base[v], f);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = id + e >= 0 && id + e < vocab ? Act<T>::load(row + id + e) : -INFINITY;
    }
  }
};

template <typename T, bool TOP>
__global__ __launch_bounds__(kLpThreads) void logprob_part_kernel(LogprobArgs a, int groups) {
  constexpr int N = Logit<T>::N, NW = kLpThreads / 64;
  __shared__ float sm[NW], ss[NW], st[NW];
  __shared__ int sc[NW];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t r = blockIdx.x / a.chunks;
  const int chunk = (int)(blockIdx.x - r * a.chunks);
  const RowView<T> x(a, r);
  const int tok = a.tokens ? a.tokens[r] : -1;
  float xt = INFINITY;   // no token: nothing is counted
  if (tok >= 0 && tok < x.vocab) {
    xt = Act<T>::load(x.row + tok);
    if (xt != xt) xt = -INFINITY;
  }
  Sums q{-INFINITY, 0.f, 0.f};
  int count = 0;
  const int v0 = chunk * a.chunk_groups * 16, v1 = min(x.n_vec, v0 + a.chunk_groups * 16);
  const int whole = (v1 - v0 + kLpThreads - 1) / kLpThreads * kLpThreads;
  for (int i = tid; i < whole; i += kLpThreads) {
    const int v = v0 + i;
    float f[N];
    if (v < v1) {
      x.load(v, f);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = -INFINITY;
    }
    float vm = f[0];
#pragma unroll
    for (int e = 1; e < N; ++e) vm = fmaxf(vm, f[e]);
    if (vm > q.m) q.join(vm, 0.f, 0.f);
    const float ref = q.m == -INFINITY ? 0.f : q.m;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float d = f[e] - ref, p = __builtin_amdgcn_exp2f(d * kLog2e);
      q.s += p;
      q.t = fmaf(p, fmaxf(d, -1.0e4f), q.t);
    }
    const int id = v * N - x.shift;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const bool before = id + e < tok;
      count += id + e >= 0 && v < v1 && (f[e] > xt || (before && (f[e] == xt || xt == -INFINITY)));
    }
    if (TOP) {
      float g = fmaxf(vm, -INFINITY);
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) g = fmaxf(g, __shfl_xor(g, d, 16));
      if ((lane & 15) == 0 && v < v1) a.group_max[r * groups + v / 16] = g;
    }
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    q.join(__shfl_xor(q.m, d, 64), __shfl_xor(q.s, d, 64), __shfl_xor(q.t, d, 64));
    count += __shfl_xor(count, d, 64);
  }
  if (lane == 0) { sm[w] = q.m; ss[w] = q.s; st[w] = q.t; sc[w] = count; }
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < NW; ++i) { q.join(sm[i], ss[i], st[i]); count += sc[i]; }
    a.part[r * a.chunks + chunk] = make_float4(q.m, q.s, q.t, __int_as_float(count));
  }
}

// Orders by value, then by lower index; NaN counts as -inf.
__device__ __forceinline__ uint64_t logit_key(float x, int id) {
  if (x != x) x = -INFINITY;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (uint64_t)(u >> 31 ? ~u : u | 0x80000000u) << 32 | (uint32_t)~id;
}

__device__ __forceinline__ uint64_t block_max(uint64_t k, uint64_t* red) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)k, d, 64);
    k = o > k ? o : k;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = k;
  __syncthreads();
  for (int i = 0; i < kLpThreads / 64; ++i) k = red[i] > k ? red[i] : k;
  return k;
}

template <typename T>
__global__ __launch_bounds__(kLpThreads) void logprob_join_kernel(LogprobArgs a, int groups) {
  constexpr int N = Logit<T>::N, GE = 16 * N;
  __shared__ uint64_t red[kLpThreads / 64];
  __shared__ int chosen[RK_MAX_TOP];
  const int tid = threadIdx.x;
  const int64_t r = blockIdx.x;
  const RowView<T> x(a, r);
  Sums q{-INFINITY, 0.f, 0.f};
  int count = 0;
  for (int c = 0; c < a.chunks; ++c) {
    const float4 p = a.part[r * a.chunks + c];
    q.join(p.x, p.y, p.z);
    count += __float_as_int(p.w);
  }
  // a row without a largest logit has no distribution
  const float log_s = q.m == -INFINITY || q.m == INFINITY ? NAN : logf(q.s);
  if (tid == 0) {
    const int tok = a.tokens ? a.tokens[r] : -1;
    const bool has = tok >= 0 && tok < x.vocab;
    if (a.logprob) a.logprob[r] = has ? (Act<T>::load(x.row + tok) - q.m) - log_s : 0.f;
    if (a.rank) a.rank[r] = has ? 1 + count : 0;
    if (a.entropy) a.entropy[r] = log_s - q.t / q.s;
  }
  if (a.n_top == 0) return;
  const int n_groups = (x.n_vec + 15) / 16, n_ch = min(n_groups, a.n_top);
  const float* gm = a.group_max + r * groups;
  uint64_t prev = ~0ull;
  for (int i = 0; i < n_ch; ++i) {
    uint64_t best = 0;
    for (int g = tid; g < n_groups; g += kLpThreads) {
      const uint64_t k = logit_key(gm[g], g);
      if (k < prev && k > best) best = k;
    }
    prev = block_max(best, red);
    if (tid == 0) chosen[i] = (int)~(uint32_t)prev;
  }
  __syncthreads();
  prev = ~0ull;
  for (int i = 0; i < a.n_top; ++i) {
    uint64_t best = 0;
    for (int c = tid; c < n_ch * GE; c += kLpThreads) {
      const int id = chosen[c / GE] * GE - x.shift + c % GE;
      if (id < 0 || id >= x.vocab) continue;
      const uint64_t k = logit_key(Act<T>::load(x.row + id), id);
      if (k < prev && k > best) best = k;
    }
    prev = block_max(best, red);
    if (tid == 0) {
      const int id = (int)~(uint32_t)prev;
      if (a.top_ids) a.top_ids[r * a.n_top + i] = id;
      if (a.top_logprobs) a.top_logprobs[r * a.n_top + i] = (Act<T>::load(x.row + id) - q.m) - log_s;
    }
  }
}

// Groups of a row, wherever it starts.
int logprob_groups(int vocab, bool bf16) {
  const int n = bf16 ? 8 : 4;
  return (int)(((int64_t)vocab + n - 1 + 16 * n - 1) / (16 * n));
}

// Workgroups per row: about 1024 in all, none with less than four loads per thread.
void logprob_chunks(int64_t n_rows, int vocab, bool bf16, int* chunks, int* chunk_groups) {
  const int groups = logprob_groups(vocab, bf16);
  const int64_t want = std::max<int64_t>(1, 1024 / std::max<int64_t>(n_rows, 1));
  const int64_t n = std::min<int64_t>(std::min<int64_t>(want, 64), (groups + 63) / 64);
  *chunk_groups = (int)((groups + n - 1) / n);
  *chunks = (groups + *chunk_groups - 1) / *chunk_groups;
}

hipError_t launch_logprobs(const LogprobArgs& a, bool bf16, hipStream_t s) {
  if (a.n_rows <= 0) return hipSuccess;
  const int groups = logprob_groups(a.vocab, bf16);
  const uint32_t blocks = (uint32_t)(a.n_rows * a.chunks);
#define RK_LOGPROBS(T)                                                                        \
  do {                                                                                        \
    if (a.n_top) logprob_part_kernel<T, true><<<blocks, kLpThreads, 0, s>>>(a, groups);       \
    else logprob_part_kernel<T, false><<<blocks, kLpThreads, 0, s>>>(a, groups);              \
    logprob_join_kernel<T><<<(uint32_t)a.n_rows, kLpThreads, 0, s>>>(a, groups);              \
  } while (0)
  if (bf16) RK_LOGPROBS(bf16_t); else RK_LOGPROBS(float);
#undef RK_LOGPROBS
  return hipGetLastError();
}

}  // namespace rk
