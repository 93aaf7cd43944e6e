// Log probabilities of given tokens from a row of logits, with the row's entropy, the
// token's rank and the best alternatives.  With a reference c:
//
//   S = sum_v e^(x_v - c),  T = sum_v (x_v - c) e^(x_v - c)
//   log p_tok = (x_tok - c) - log S,   H = log S - T / S
//   rank = 1 + #{v : x_v > x_tok, or x_v = x_tok and v < tok}
//
// The sums lose nothing with c below the maximum as long as nothing overflows, so c
// follows a thread's maximum when that has run 32 ahead, and at the end (log S keeps
// its digits next to 0).  The difference is formed before the factor log2(e) of the
// exponential: x log2(e) would overflow at the type's lowest value, a common mask.
//
// Each logit is read once: a running (c, S, T) per thread, joined in a fixed order.
// The alternatives come out of the same pass by groups of consecutive logits (16 lanes
// times one 16-byte load): the n best logits, ordered by value and then by lower index,
// lie in the n groups whose largest logits come first in that order (each of those
// groups holds at least one logit that precedes any logit of another group), so only
// those groups are looked at again, by one wave.
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

constexpr float kLazy = 32.f;

// Softmax sums relative to e^c; s and t are 0 while c is -inf.
struct Sums {
  float c, s, t;
  __device__ __forceinline__ float ref() const { return c == -INFINITY ? 0.f : c; }
  // moves the reference up to c2
  __device__ __forceinline__ void raise(float c2) {
    const float d = fmaxf(c - c2, -1.0e4f), f = __builtin_amdgcn_exp2f(d * kLog2e);   // -inf: weight 0
    t = f * fmaf(d, s, t);
    s *= f;
    c = c2;
  }
  __device__ __forceinline__ void join(Sums o) {
    const float m = fmaxf(c, o.c);
    if (m == -INFINITY) {   // nothing but -inf so far; a NaN has left its mark on the sums
      s += o.s;
      t += o.t;
      return;
    }
    raise(m);
    o.raise(m);
    s += o.s;
    t += o.t;
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
  // vectors v .. v + n - 1 lie whole within the row
  __device__ __forceinline__ bool inside(int v, int n) const {
    return v * N >= shift && (int64_t)(v + n) * N - shift <= vocab;
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

// Orders floats as unsigned numbers: NaN as -inf, -0 as 0; never 0.
__device__ __forceinline__ uint32_t order_bits(float x) {
  if (x != x) x = -INFINITY;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// Largest of a value over the wave (unsigned), by row shifts and broadcasts.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#define RK_STEP(ctrl, rows) \
  { const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false); x = o > x ? o : x; }
  RK_STEP(0x111, 0xf) RK_STEP(0x112, 0xf) RK_STEP(0x114, 0xf) RK_STEP(0x118, 0xf)   // row_shr 1, 2, 4, 8
  RK_STEP(0x142, 0xa) RK_STEP(0x143, 0xc)                                           // row_bcast 15, 31
#undef RK_STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// Largest over the 16 lanes of a row, in every one of them.
__device__ __forceinline__ float row_max(float x) {
#define RK_STEP(ctrl) \
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xf, 0xf, false)));
  RK_STEP(0x128) RK_STEP(0x124) RK_STEP(0x122) RK_STEP(0x121)   // row_ror 8, 4, 2, 1
#undef RK_STEP
  return x;
}

// The float of order_bits.
__device__ __forceinline__ float from_order(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

constexpr int kTopGroups = 4096;   // group keys held in LDS
constexpr int kTopList = 256;      // candidates held in LDS

struct TopShared {
  v4u keys[kTopGroups / 4];
  uint64_t list[kTopList];
  int chosen[RK_MAX_TOP];
  int n_chosen, count;
};

// One wave: groups of the n largest keys (ties to the lower group) into sh.chosen; the
// smallest key taken.  A search between the least of the lanes' best keys and the best
// of all: about ten steps of counting, whatever n is.  KEYS(i): keys 4 i .. 4 i + 3, 0
// past the last group.
template <typename Keys>
__device__ __forceinline__ uint32_t choose_groups(int n_groups, int n, TopShared& sh, Keys keys) {
  const int lane = threadIdx.x & 63, its = (n_groups + 255) / 256;
  uint32_t best = 0;
  for (int it = 0; it < its; ++it) {
    const v4u k = keys(it * 64 + lane);
    best = max(max(max(best, k[0]), max(k[1], k[2])), k[3]);
  }
  // n <= 64 lanes: at least n keys reach the least of the lanes' best
  uint32_t hi = wave_max(best), lo = max(~wave_max(~best), 1u);
  int above = 0;
  bool exact = false;
  if (n_groups == n) { lo = 1; exact = true; }
  while (!exact && lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    int c = 0;
    for (int it = 0; it < its; ++it) {
      const v4u k = keys(it * 64 + lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) c += __popcll(__ballot(k[e] >= mid));
    }
    if (c >= n) lo = mid; else hi = mid - 1;
    exact = c == n;
  }
  // keys above lo, and of those equal to it the first that are still wanted
  if (lane == 0) sh.n_chosen = 0;
  wave_sync();
  if (!exact)
    for (int it = 0; it < its; ++it) {
      const v4u k = keys(it * 64 + lane);
#pragma unroll
      for (int e = 0; e < 4; ++e) above += __popcll(__ballot(k[e] > lo));
    }
  int want = n - above;
  for (int it = 0; it < its; ++it) {
    const v4u k = keys(it * 64 + lane);
    int equal = 0, before = 0, all = 0;
    if (!exact) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint64_t b = __ballot(k[e] == lo);
        before += __popcll(b & ((1ull << lane) - 1));
        all += __popcll(b);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool tie = !exact && k[e] == lo;
      if (tie ? before + equal < want : k[e] >= lo && k[e] != 0) sh.chosen[atomicAdd(&sh.n_chosen, 1)] = (it * 64 + lane) * 4 + e;
      equal += tie;
    }
    want -= all;
  }
  wave_sync();
  return lo;
}

// One wave: the n_top best logits of row r, given the groups' keys, c and log S.
template <typename T>
__device__ __forceinline__ void top_of_row(const LogprobArgs& a, const RowView<T>& x, int64_t r,
                                           const uint32_t* group_keys, float c, float log_s, TopShared& sh) {
  constexpr int N = Logit<T>::N, PASSES = RK_MAX_TOP / 4;
  const int lane = threadIdx.x & 63;
  const int n_groups = (x.n_vec + 15) / 16, n_ch = min(n_groups, a.n_top);
  const auto load_keys = [&](int i) {   // rows of keys are padded to whole vectors
    v4u k = v4u{0, 0, 0, 0};
    if (4 * i < n_groups) {
      k = reinterpret_cast<const v4u*>(group_keys)[i];
#pragma unroll
      for (int e = 1; e < 4; ++e) k[e] = 4 * i + e < n_groups ? k[e] : 0u;
    }
    return k;
  };
  uint32_t tau;
  if (n_groups <= kTopGroups) {
    const int its = (n_groups + 255) / 256;
#pragma unroll 4
    for (int it = 0; it < its; ++it) sh.keys[it * 64 + lane] = load_keys(it * 64 + lane);
    wave_sync();
    tau = choose_groups(n_groups, n_ch, sh, [&](int i) { return sh.keys[i]; });
  } else {
    tau = choose_groups(n_groups, n_ch, sh, load_keys);
  }
  if (lane == 0) sh.count = 0;
  wave_sync();
  // ---- logits of those groups at or above the last group's best: n_top of them or more
  v4u raw[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int i = p * 4 + lane / 16, v = i < n_ch ? sh.chosen[i] * 16 + (lane & 15) : -1;
    if (v >= 0 && x.inside(v, 1)) raw[p] = x.base[v];
  }
  if (n_ch < a.n_top) tau = 1;   // every logit counts
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int i = p * 4 + lane / 16, v = i < n_ch ? sh.chosen[i] * 16 + (lane & 15) : x.n_vec;
    if (v < x.n_vec) {
      float f[N];
      if (x.inside(v, 1)) Logit<T>::get(raw[p], f); else x.load(v, f);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int id = v * N - x.shift + e;
        const uint32_t k = order_bits(f[e]);
        if (k >= tau && id >= 0 && id < x.vocab) {
          const int n = atomicAdd(&sh.count, 1);
          if (n < kTopList) sh.list[n] = (uint64_t)k << 32 | (uint32_t)~id;
        }
      }
    }
  }
  wave_sync();
  const int count = sh.count;
  auto put = [&](int i, uint64_t key) {
    if (a.top_ids) a.top_ids[r * a.n_top + i] = (int)~(uint32_t)key;
    if (a.top_logprobs) a.top_logprobs[r * a.n_top + i] = (from_order((uint32_t)(key >> 32)) - c) - log_s;
  };
  if (count <= kTopList) {
    // a candidate's place is the number of candidates before it
    for (int i = lane; i < count; i += 64) {
      const uint64_t mine = sh.list[i];
      int before = 0;
#pragma unroll 8
      for (int j = 0; j < count; ++j) before += sh.list[j] > mine;
      if (before < a.n_top) put(before, mine);
    }
  } else {
    // runs of large or equal logits: n_top times the next in order, over all of them
    uint64_t prev = ~0ull;
    for (int i = 0; i < a.n_top; ++i) {
      uint64_t next = 0;
      for (int q = lane; q < n_ch * 16 * N; q += 64) {
        const int id = sh.chosen[q / (16 * N)] * (16 * N) + q % (16 * N) - x.shift;
        if (id < 0 || id >= x.vocab) continue;
        const uint64_t k = (uint64_t)order_bits(Act<T>::load(x.row + id)) << 32 | (uint32_t)~id;
        if (k < prev && k > next) next = k;
      }
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)next, d, 64);
        next = o > next ? o : next;
      }
      prev = next;
      if (lane == 0) put(i, next);
    }
  }
}

// The outputs of a row from its sums (wave-uniform), by one wave.
template <typename T>
__device__ __forceinline__ void finish_row(const LogprobArgs& a, const RowView<T>& x, int64_t r, const Sums& q,
                                           int count, uint32_t* group_keys, TopShared* sh) {
  const float c = q.ref();
  // without a finite largest logit the row has no distribution: S is 0 or NaN
  const float log_s = q.s > 0.f ? logf(q.s) : NAN;
  if ((threadIdx.x & 63) == 0) {
    const int tok = a.tokens ? a.tokens[r] : -1;
    const bool has = tok >= 0 && tok < x.vocab;
    if (a.logprob) a.logprob[r] = has ? (Act<T>::load(x.row + tok) - c) - log_s : 0.f;
    if (a.rank) a.rank[r] = has ? 1 + count : 0;
    if (a.entropy) a.entropy[r] = log_s - q.t / q.s;
  }
  if (sh) top_of_row<T>(a, x, r, group_keys, c, log_s, *sh);
}

// One workgroup per (row, run of groups).  FUSED: the run is the whole row, whose
// outputs the workgroup's first wave then forms while the other workgroups of the CU
// read on; otherwise the runs' sums go to the joining kernel.
template <typename T, bool TOP, bool FUSED>
__global__ __launch_bounds__(kLpThreads) void logprob_kernel(LogprobArgs a, int groups) {
  constexpr int N = Logit<T>::N, NW = kLpThreads / 64, U = 4;
  __shared__ Sums sums[NW];
  __shared__ int counts[NW];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t r = FUSED ? blockIdx.x : blockIdx.x / a.chunks;
  const int chunk = FUSED ? 0 : (int)(blockIdx.x - r * a.chunks);
  const RowView<T> x(a, r);
  const int tok = a.tokens ? a.tokens[r] : -1;
  const bool has = tok >= 0 && tok < x.vocab;
  float xt = INFINITY;   // no token: nothing is counted
  if (has) {
    xt = Act<T>::load(x.row + tok);
    if (xt != xt) xt = -INFINITY;
  }
  // x >= xt is x > below, the next float down (xt = -inf is counted index by index)
  const int bits = __float_as_int(xt);
  const float below = xt == 0.f ? __int_as_float((int)0x80000001) : __int_as_float(bits < 0 ? bits + 1 : bits - 1);
  Sums q{-INFINITY, 0.f, 0.f};
  float largest = -INFINITY;
  int count = 0;   // wave-uniform
  const int v0 = chunk * a.chunk_groups * 16, v1 = min(x.n_vec, v0 + a.chunk_groups * 16);
  uint32_t* group_keys = a.group_keys + r * groups;
  for (int b = v0 + w * 64; b < v1; b += kLpThreads * U) {   // the wave's first vector of U passes
    float f[U][N];
    if (b + (U - 1) * kLpThreads + 64 <= v1 && x.inside(b, (U - 1) * kLpThreads + 64)) {
      v4u raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u] = x.base[b + u * kLpThreads + lane];
#pragma unroll
      for (int u = 0; u < U; ++u) Logit<T>::get(raw[u], f[u]);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = b + u * kLpThreads + lane;
        if (v < v1) {
          x.load(v, f[u]);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) f[u][e] = -INFINITY;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int vb = b + u * kLpThreads, v = vb + lane;
      if (vb >= v1) break;
      float vm = f[u][0];
#pragma unroll
      for (int e = 1; e < N; ++e) vm = fmaxf(vm, f[u][e]);
      largest = fmaxf(largest, vm);
      if (vm > q.c + kLazy) q.raise(vm);
      const float c = q.ref();
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = f[u][e] - c, p = __builtin_amdgcn_exp2f(d * kLog2e);
        q.s += p;
        q.t = fmaf(p, fmaxf(d, -1.0e4f), q.t);
      }
      if (has) {
        const int id0 = vb * N - x.shift;   // of the wave: 64 N consecutive logits
        if (xt != -INFINITY && (id0 > tok || id0 + 64 * N <= tok)) {
          const float thr = id0 > tok ? xt : below;
#pragma unroll
          for (int e = 0; e < N; ++e) count += __popcll(__ballot(f[u][e] > thr));
        } else {
          const int id = v * N - x.shift;
#pragma unroll
          for (int e = 0; e < N; ++e)
            count += __popcll(__ballot(id + e >= 0 && v < v1 &&
                                       (f[u][e] > xt || (id + e < tok && (f[u][e] == xt || xt == -INFINITY)))));
        }
      }
      if (TOP) {
        const float g = row_max(fmaxf(vm, -INFINITY));
        if ((lane & 15) == 0 && v < v1) group_keys[v / 16] = order_bits(g);
      }
    }
  }
  if (largest > q.c) q.raise(largest);
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1)
    q.join(Sums{__shfl_xor(q.c, d, 64), __shfl_xor(q.s, d, 64), __shfl_xor(q.t, d, 64)});
  if (lane == 0) { sums[w] = q; counts[w] = count; }
  __syncthreads();
  if (w != 0) return;
  q = sums[0];
  count = counts[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) { q.join(sums[i]); count += counts[i]; }
  if constexpr (FUSED) {
    if constexpr (TOP) {
      __shared__ TopShared sh;
      finish_row<T>(a, x, r, q, count, group_keys, &sh);
    } else {
      finish_row<T>(a, x, r, q, count, group_keys, nullptr);
    }
  } else if (lane == 0) {
    a.part[r * a.chunks + chunk] = make_float4(q.c, q.s, q.t, __int_as_float(count));
  }
}

// One wave per row: joins the sums of its runs and forms its outputs.
template <typename T, bool TOP>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a, int groups) {
  const int64_t r = blockIdx.x;
  const int lane = threadIdx.x;
  const RowView<T> x(a, r);
  Sums q{-INFINITY, 0.f, 0.f};
  int count = 0;
  if (lane < a.chunks) {   // at most 64
    const float4 p = a.part[r * a.chunks + lane];
    q = Sums{p.x, p.y, p.z};
    count = __float_as_int(p.w);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    q.join(Sums{__shfl_xor(q.c, d, 64), __shfl_xor(q.s, d, 64), __shfl_xor(q.t, d, 64)});
    count += __shfl_xor(count, d, 64);
  }
  if constexpr (TOP) {
    __shared__ TopShared sh;
    finish_row<T>(a, x, r, q, count, a.group_keys + r * groups, &sh);
  } else {
    finish_row<T>(a, x, r, q, count, nullptr, nullptr);
  }
}

// Groups of a row, wherever it starts, in whole vectors of keys.
int logprob_groups(int vocab, bool bf16) {
  const int n = bf16 ? 8 : 4;
  return (int)(((int64_t)vocab + n - 1 + 16 * n - 1) / (16 * n) + 3) / 4 * 4;
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
#define RK_LOGPROBS(T, TOP)                                                                   \
  do {                                                                                        \
    if (a.chunks == 1) {                                                                      \
      logprob_kernel<T, TOP, true><<<blocks, kLpThreads, 0, s>>>(a, groups);                  \
    } else {                                                                                  \
      logprob_kernel<T, TOP, false><<<blocks, kLpThreads, 0, s>>>(a, groups);                 \
      logprob_join_kernel<T, TOP><<<(uint32_t)a.n_rows, 64, 0, s>>>(a, groups);               \
    }                                                                                         \
  } while (0)
  if (bf16) { if (a.n_top) RK_LOGPROBS(bf16_t, true); else RK_LOGPROBS(bf16_t, false); }
  else { if (a.n_top) RK_LOGPROBS(float, true); else RK_LOGPROBS(float, false); }
#undef RK_LOGPROBS
  return hipGetLastError();
}

}  // namespace rk
