// Log probabilities of given tokens from a row of logits, with the row's entropy, the
// token's rank and the best alternatives.  With a reference c:
//
//   S = sum_v e^(x_v - c),  T = sum_v (x_v - c) e^(x_v - c)
//   log p_tok = (x_tok - c) - log S,   H = log S - T / S
//   rank = 1 + #{v : x_v > x_tok, or x_v = x_tok and v < tok}
//
// c is a thread's largest logit so far, moved up before a pass of four vectors is added.  S
// would lose nothing with c below it, but T, moved up by D at the end, would be left as the
// small difference of D S and T (the entropy 2e-6 off with D = 20).  The difference x - c is
// formed before the factor log2(e) of the exponential: x log2(e) would overflow at the type's
// lowest value, a common mask.
//
// A workgroup reads each logit of a row (of a part of a long row, where rows are few)
// once: a running (c, S, T) per thread, joined in a fixed order.  The alternatives come
// out of the same pass by groups of 16 vectors (4 lanes, 4 passes): if n groups have a
// logit that reaches a bound, the n best logits lie in the groups whose largest logit
// reaches it.  Only those are looked at again, shared out over the waves.  Where equal
// logits make them too many (a constant row, a mask that leaves fewer than n), the bound
// is the n-th largest of the groups' largest logits: the logits above it come from the
// groups above it, and the rest are the first logits of the row that equal it.
//
// The exponentials' arguments carry the rounding of their product with log2(e): results are
// 6e-8 .. 1e-7 off on a language model's logits, as far as fp32 sums are; making it good would
// take 4 more instructions a logit.
//
// Bound: memory for many fp32 rows, a chain of short sections for few.  With the 20 best: 1024
// rows of 128256 fp32 101 us (5.2 TB/s, a copy of as many bytes 106), 1500 of 128256 bf16 93
// (4.1 TB/s).  301 of 50257 bf16 20.4 us in a graph: 4.7 for a launch and the joins (a row of
// 500), 8.8 for S and T, 2.2 for the rank, 4.7 for the 20 best; the vector units are busy 6.7
// of them in the mean, 11 on the 45 of 256 CUs that have two rows.  16 of 32000 fp32, 5 best,
// 10.0: 4.1, 1.7, 1.1 and 3.1.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "rk_internal.h"

namespace rk {

constexpr float kLog2e = 1.4426950408889634f;

template <typename T> struct Logit;
template <> struct Logit<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ v4u none() { return v4u{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u}; }
  static __device__ __forceinline__ v4u put(const float* f) {
    return v4u{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
  static __device__ __forceinline__ void get(v4u u, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(u[i]);
  }
};
template <> struct Logit<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ v4u none() { return v4u{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
  static __device__ __forceinline__ v4u put(const float* f) {
    v4u u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (uint32_t)f2bf(f[2 * i]) | ((uint32_t)f2bf(f[2 * i + 1]) << 16);
    return u;
  }
  static __device__ __forceinline__ void get(v4u u, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
};

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
};

// A row, or a part of one, as 16-byte vectors: vector v holds logits v N - shift .. of it.
template <typename T> struct RowView {
  static constexpr int N = Logit<T>::N;
  const T* row;
  const v4u* base;   // aligned address at or below the row's first logit
  int shift, vocab, n_vec;
  __device__ __forceinline__ RowView(const T* first, int n) {
    row = first;
    shift = (int)(((uintptr_t)row & 15) / sizeof(T));
    base = (const v4u*)(row - shift);
    vocab = n;
    n_vec = (int)(((int64_t)shift + vocab + N - 1) / N);
  }
  // vectors v .. v + n - 1 lie whole within the row
  __device__ __forceinline__ bool inside(int v, int n) const {
    return v * N >= shift && (int64_t)(v + n) * N - shift <= vocab;
  }
  // vectors that reach outside the row are read logit by logit; what is outside is -inf
  __device__ __forceinline__ v4u load(int v) const {
    if (inside(v, 1)) return base[v];
    const int id = v * N - shift;
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = Act<T>::load(row + min(max(id + e, 0), vocab - 1));
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = id + e >= 0 && id + e < vocab ? f[e] : -INFINITY;
    return Logit<T>::put(f);
  }
};

// Orders floats as unsigned numbers: NaN as -inf, -0 as 0; never 0.
__device__ __forceinline__ uint32_t order_bits(float x) {
  if (x != x) x = -INFINITY;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// Folds a value over the wave by row shifts and broadcasts; every lane gets the result.
template <typename F>
__device__ __forceinline__ uint32_t wave_fold(uint32_t x, F f) {   // 0 is the identity of f
#define RK_STEP(ctrl, rows) x = f(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false));
  RK_STEP(0x111, 0xf) RK_STEP(0x112, 0xf) RK_STEP(0x114, 0xf) RK_STEP(0x118, 0xf)   // row_shr 1, 2, 4, 8
  RK_STEP(0x142, 0xa) RK_STEP(0x143, 0xc)                                           // row_bcast 15, 31
#undef RK_STEP
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  return wave_fold(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ int wave_count(int x) {
  return (int)wave_fold((uint32_t)x, [](uint32_t a, uint32_t b) { return a + b; });
}
__device__ __forceinline__ float wave_total(float x) {
  return __uint_as_float(wave_fold(__float_as_uint(x), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}

// Largest over each four lanes, in every one of them.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
#define RK_STEP(ctrl) \
  { const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, false); x = o > x ? o : x; }
  RK_STEP(0xb1) RK_STEP(0x4e)   // quad_perm 1 0 3 2, 2 3 0 1
#undef RK_STEP
  return x;
}

// The float of order_bits.
__device__ __forceinline__ float from_order(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

// The wave's sums, all moved to the largest reference.  (A lane that has met a NaN or an
// infinity holds a NaN sum, and that stays.)
__device__ __forceinline__ Sums wave_sums(Sums q) {
  const float m = from_order(wave_max(order_bits(q.c)));
  if (m > -INFINITY) q.raise(m);
  return Sums{m, wave_total(q.s), wave_total(q.t)};
}

__device__ __forceinline__ double wave_total(double x) {
#define RK_STEP(ctrl, rows)                                                                                   \
  {                                                                                                           \
    const uint64_t u = (uint64_t)__double_as_longlong(x);                                                     \
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, ctrl, rows, 0xf, false);             \
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), ctrl, rows, 0xf, false);     \
    x += __longlong_as_double((long long)((uint64_t)hi << 32 | lo));                                          \
  }
  RK_STEP(0x111, 0xf) RK_STEP(0x112, 0xf) RK_STEP(0x114, 0xf) RK_STEP(0x118, 0xf)
  RK_STEP(0x142, 0xa) RK_STEP(0x143, 0xc)
#undef RK_STEP
  const uint64_t u = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)u, 63);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), 63);
  return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}

// The same for beams, whose scores are compared with each other: the exponentials are fp32's, what
// is done with them is done in doubles (128 rows of 128256 fp32 logits: 14.7 us either way; the
// joining kernel takes 0.4 us more).  log S is then 1e-8 off in the mean, 7e-8 at most on a language
// model's logits, where fp32 sums left 8e-8 and 4e-7.  What remains is the exponentials', so that a
// row's largest logit, whose exponential is 1, adds nothing to it: with a token of probability
// 0.9999 it is 1e-12.  Exponentials in doubles too, 17 instructions of half rate a logit: 23 us.
struct BeamSums {
  float c;
  float t;
  double s;
  __device__ __forceinline__ float ref() const { return c == -INFINITY ? 0.f : c; }
  __device__ __forceinline__ void raise(float c2) {
    const float d = fmaxf(c - c2, -1.0e4f), f = __builtin_amdgcn_exp2f(d * kLog2e);
    t = f * fmaf(d, (float)s, t);
    s *= (double)f;
    c = c2;
  }
  // S: every exponent above is (1 + e) of what it should be, fp32's log2(e) being 1.9259630e-8
  // too small, so the sum is off by e T
  __device__ __forceinline__ double sum() const { return s + 1.9259630e-8 * 0.69314718055994531 * (double)t; }
  // as the workspace holds them
  __device__ __forceinline__ float4 packed() const {
    const uint64_t u = (uint64_t)__double_as_longlong(s);
    return make_float4(c, t, __uint_as_float((uint32_t)u), __uint_as_float((uint32_t)(u >> 32)));
  }
  static __device__ __forceinline__ BeamSums of(float4 f) {
    const uint64_t u = (uint64_t)__float_as_uint(f.w) << 32 | __float_as_uint(f.z);
    return {f.x, f.y, __longlong_as_double((long long)u)};
  }
};
__device__ __forceinline__ BeamSums wave_sums(BeamSums q) {
  const float m = from_order(wave_max(order_bits(q.c)));
  if (m > -INFINITY) q.raise(m);
  return BeamSums{m, wave_total(q.t), wave_total(q.s)};
}

constexpr int kPasses = 4;         // vectors in flight per lane
constexpr int kTopGroups = 4096;   // groups of a row or part: 65536 vectors
constexpr int kTopLook = 128;      // groups looked at again
constexpr int kTopList = 256;      // candidates held in LDS
constexpr int kMaxParts = 64;

template <int NT> struct TopShared {
  v4u keys[kTopGroups / 4];        // order of each group's largest logit, 0 for a group without logits
  uint32_t best[NT / 4];           // the largest key of each four lanes
  uint64_t list[kTopList];
  int chosen[kTopLook], n_chosen, n_list;
  uint32_t tau;                    // of the search over every key:
  int n_look, all;
};

// The workgroup: the n best logits of x, given the groups' keys; put(i, order, id) takes
// the i-th.  An earlier barrier has made keys and best visible and n_chosen, n_list 0.
template <typename T, int NT, typename Put>
__device__ __forceinline__ void top_logits(const RowView<T>& x, int n, int n_groups, TopShared<NT>& sh, Put put) {
  constexpr int N = Logit<T>::N, NW = NT / 64, NB = NT / 256;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint64_t lower = (1ull << lane) - 1;
  // ---- a bound that n or a few more of the best keys reach, by halving an interval (1:
  // there are no n of them, every logit is a candidate); the same in every wave
  uint32_t bound = 1;
  {
    uint32_t best[NB], top = 0;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      best[i] = sh.best[i * 64 + lane];
      top = max(top, best[i]);
    }
    // every lane's largest reaches the least of them: 64 keys, if no lane is without one
    uint32_t hi = wave_max(top);
    bound = max(~wave_max(~top), 1u);
    while (bound < hi) {
      const uint32_t mid = bound + (hi - bound + 1) / 2;
      int c = 0;
#pragma unroll
      for (int i = 0; i < NB; ++i) c += __popcll(__ballot(best[i] >= mid));
      if (c >= n) bound = mid; else hi = mid - 1;
      if (c >= n && c <= n + n / 8 + 1) break;
    }
  }
  for (int i0 = w * 64; i0 < n_groups / 4; i0 += NT) {
    const int i = i0 + lane;
    const v4u k = i < n_groups / 4 ? sh.keys[i] : v4u{0, 0, 0, 0};
    int mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) mine += k[e] >= bound;
    if (__ballot(mine > 0) == 0) continue;
    if (mine) {
      int at = atomicAdd(&sh.n_chosen, mine);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k[e] >= bound) {
          if (at < kTopLook) sh.chosen[at] = 4 * i + e;
          ++at;
        }
    }
  }
  __syncthreads();
  int n_ch = sh.n_chosen;
  bool all = true;   // the chosen groups have every logit of at least the bound, or else every one above it
  if (n_ch > kTopLook) {
    // ---- the n-th largest key itself, and the groups above it, with those equal to it if they fit
    if (w == 0) {
      const auto reaching = [&](uint32_t b) {
        int c = 0;
        for (int i = lane; i < n_groups / 4; i += 64) {
          const v4u k = sh.keys[i];
          c += (k[0] >= b) + (k[1] >= b) + (k[2] >= b) + (k[3] >= b);
        }
        return wave_count(c);
      };
      uint32_t lo = bound, hi = ~0u;
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        if (reaching(mid) >= n) lo = mid; else hi = mid - 1;
      }
      const bool fits = reaching(lo) <= kTopLook;
      const uint32_t from = fits ? lo : lo + 1;
      int taken = 0;
      for (int i0 = 0; i0 < n_groups / 4; i0 += 64) {
        const int i = i0 + lane;
        const v4u k = i < n_groups / 4 ? sh.keys[i] : v4u{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint64_t b = __ballot(k[e] >= from);
          if (k[e] >= from) sh.chosen[taken + __popcll(b & lower)] = 4 * i + e;
          taken += __popcll(b);
        }
      }
      if (lane == 0) { sh.n_look = taken; sh.tau = lo; sh.all = fits; }
    }
    __syncthreads();
    n_ch = sh.n_look;
    bound = sh.tau;
    all = sh.all;
  }
  const uint32_t from = all ? bound : bound + 1;
  // vector l of chosen group i
  const auto vector_of = [&](int i, int l) {
    const int g = sh.chosen[i], wave = g / 16;
    return wave / NW * (NT * kPasses) + (l / 4) * NT + wave % NW * 64 + g % 16 * 4 + l % 4;
  };
  // ---- the chosen groups' logits at or above `from`, four groups a step and wave
#pragma unroll 1
  for (int p = w; p * 4 < n_ch; p += NW) {
    const int i = p * 4 + lane / 16, v = i < n_ch ? vector_of(i, lane & 15) : x.n_vec;
    if (v < x.n_vec) {
      float f[N];
      Logit<T>::get(x.load(v), f);
      uint32_t hits = 0;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int id = v * N - x.shift + e;
        if (order_bits(f[e]) >= from && id >= 0 && id < x.vocab) hits |= 1u << e;
      }
      if (hits) {
        int at = atomicAdd(&sh.n_list, __popc(hits));
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (hits >> e & 1) {
            if (at < kTopList) sh.list[at] = (uint64_t)order_bits(f[e]) << 32 | (uint32_t)~(v * N - x.shift + e);
            ++at;
          }
      }
    }
  }
  __syncthreads();
  const int n_list = sh.n_list;
  if (n_list <= kTopList) {
    // a candidate's place is the number of candidates before it
    if (tid < n_list) {
      const uint64_t mine = sh.list[tid];
      int before = 0;
#pragma unroll 4
      for (int j = 0; j < n_list; ++j) before += sh.list[j] > mine;
      if (before < n) put(before, (uint32_t)(mine >> 32), (int)~(uint32_t)mine);
    }
  } else if (w == 0) {
    // runs of large logits: n times the next in order, over all of the groups
    uint64_t prev = ~0ull;
    for (int i = 0; i < min(n_list, n); ++i) {
      uint64_t next = 0;
      for (int q = lane; q < n_ch * 16 * N; q += 64) {
        const int id = vector_of(q / (16 * N), q / N % 16) * N + q % N - x.shift;
        if (id < 0 || id >= x.vocab) continue;
        const uint32_t o = order_bits(Act<T>::load(x.row + id));
        const uint64_t k = (uint64_t)o << 32 | (uint32_t)~id;
        if (o >= from && k < prev && k > next) next = k;
      }
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)next, d, 64);
        next = o > next ? o : next;
      }
      prev = next;
      if (lane == 0) put(i, (uint32_t)(next >> 32), (int)~(uint32_t)next);
    }
  }
  // ---- the first logits of the row that equal the bound, until there are n
  if (all || w != 0) return;
  int count = n_list;
  for (int v0 = 0; count < n && v0 < x.n_vec; v0 += 64) {
    const int v = v0 + lane;
    float f[N];
    Logit<T>::get(x.load(min(v, x.n_vec - 1)), f);
    uint64_t b[N];
    int at = count;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int id = v * N - x.shift + e;
      b[e] = __ballot(v < x.n_vec && id >= 0 && id < x.vocab && order_bits(f[e]) == bound);
      at += __popcll(b[e] & lower);
      count += __popcll(b[e]);
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (b[e] >> lane & 1) {
        if (at < n) put(at, bound, v * N - x.shift + e);
        ++at;
      }
  }
}

// Outputs of a row from its sums.
struct RowResult {
  float c, log_s, logprob, entropy;
  int rank;
  __device__ __forceinline__ RowResult(const LogprobArgs& a, int64_t r, Sums q, int count, bool has, float x_tok) {
    c = q.ref();
    // without a finite largest logit the row has no distribution: S is 0 or NaN
    log_s = q.s > 0.f ? logf(q.s) : NAN;
    logprob = has ? (x_tok - c) - log_s : 0.f;
    entropy = log_s - q.t / q.s;
    rank = has ? 1 + count : 0;
  }
  __device__ __forceinline__ void write(const LogprobArgs& a, int64_t r) const {
    if (a.logprob) a.logprob[r] = logprob;
    if (a.rank) a.rank[r] = rank;
    if (a.entropy) a.entropy[r] = entropy;
  }
  __device__ __forceinline__ void put(const LogprobArgs& a, int64_t r, int i, uint32_t k, int id) const {
    if (a.top_ids) a.top_ids[r * a.n_top + i] = id;
    if (a.top_logprobs) a.top_logprobs[r * a.n_top + i] = (from_order(k) - c) - log_s;
  }
};

// A beam that can go on.
__device__ __forceinline__ bool beam_open(const BeamArgs& b, int64_t r) {
  return b.scores[r] > -INFINITY && !(b.ended && b.ended[r]);
}

// BEAM: sums and best logits always go to the workspace, for the join over a group's beams.
template <typename T, int NT, bool TOP, bool BEAM = false>
__global__ __launch_bounds__(NT) void logprob_kernel(LogprobArgs a, BeamArgs beam) {
  constexpr int N = Logit<T>::N, NW = NT / 64, U = kPasses;
  using RowSums = std::conditional_t<BEAM, BeamSums, Sums>;
  __shared__ RowSums sums[NW];
  __shared__ int counts[NW];
  __shared__ std::conditional_t<TOP, TopShared<NT>, int> sh;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t r = blockIdx.x / a.parts;
  if (BEAM && !beam_open(beam, r)) return;
  const int part = (int)(blockIdx.x - r * a.parts), first = part * a.part_logits;
  const T* row = (const T*)a.logits + r * a.row_stride;
  const RowView<T> x(row + first, min(a.part_logits, a.vocab - first));
  int tok = a.tokens ? a.tokens[r] : -1;
  const bool has = tok >= 0 && tok < a.vocab;
  float xt = INFINITY;   // no token: nothing is counted
  if (has) xt = Act<T>::load(row + tok);
  const float x_tok = xt;
  if (xt != xt) xt = -INFINITY;
  tok -= first;          // of the part, maybe outside it
  // x >= xt is x > below, the next float down (xt = -inf is counted index by index)
  const int bits = __float_as_int(xt);
  const float below = xt == 0.f ? __int_as_float((int)0x80000001) : __int_as_float(bits < 0 ? bits + 1 : bits - 1);
  RowSums q{};                          // sums of nothing
  q.c = -INFINITY;
  float c = 0.f;                        // q.ref()
  int count = 0;                        // wave-uniform
  uint32_t best_key = 0;
  const auto load = [&](v4u* raw, int b) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int vb = b + u * NT;
      if (x.inside(vb, 64)) raw[u] = x.base[vb + lane];
      else if (vb + lane < x.n_vec) raw[u] = x.load(vb + lane);
      else raw[u] = Logit<T>::none();
    }
  };
  // the next passes' loads are out while these are added up
  v4u raw[U], next[U];
  load(raw, w * 64);
  for (int b0 = 0; b0 < x.n_vec; b0 += NT * U) {   // the first vector of U passes
    const int b = b0 + w * 64;                     // .. of this wave's
    if (b0 + NT * U < x.n_vec) load(next, b + NT * U);
    float best = -INFINITY;               // what is outside the row is -inf
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      Logit<T>::get(raw[u], f);
#pragma unroll
      for (int e = 0; e < N; ++e) best = fmaxf(best, f[e]);
    }
    if (best > q.c) {
      q.raise(best);
      c = q.ref();
    }
    // these passes' own sums: chains of 16 or 32 terms, then one of the passes (a chain of a
    // thread's 500 terms left the entropy 2e-6 off)
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int vb = b + u * NT;
      if (vb >= x.n_vec) break;
      float f[N];
      Logit<T>::get(raw[u], f);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float d = f[e] - c, p = __builtin_amdgcn_exp2f(d * kLog2e);
        if constexpr (BEAM) q.s += (double)p;
        else s += p;
        t = fmaf(p, fmaxf(d, -1.0e4f), t);
      }
      if (has) {
        const int id0 = vb * N - x.shift;   // of the wave: 64 N consecutive logits
        if (xt != -INFINITY && (id0 > tok || id0 + 64 * N <= tok)) {
          const float thr = id0 > tok ? xt : below;
#pragma unroll
          for (int e = 0; e < N; ++e) count += __popcll(__ballot(f[e] > thr));
        } else {
          const int id = (vb + lane) * N - x.shift;
#pragma unroll
          for (int e = 0; e < N; ++e)
            count += __popcll(__ballot(id + e >= 0 && id + e < x.vocab &&
                                       (f[e] > xt || (id + e < tok && (f[e] == xt || xt == -INFINITY)))));
        }
      }
    }
    if constexpr (!BEAM) q.s += s;
    q.t += t;
    if constexpr (TOP) {
      // a group holds logits if its first vector does
      uint32_t key = quad_max(order_bits(best));
      if ((b + lane) - lane % 4 >= x.n_vec) key = 0;
      best_key = max(best_key, key);
      if (lane % 4 == 0) reinterpret_cast<uint32_t*>(sh.keys)[b0 / 16 + w * 16 + lane / 4] = key;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = next[u];
  }
  q = wave_sums(q);
  if (lane == 0) { sums[w] = q; counts[w] = count; }
  if constexpr (TOP) {
    if (lane % 4 == 0) sh.best[w * 16 + lane / 4] = best_key;
    if (tid == 0) { sh.n_chosen = 0; sh.n_list = 0; }
  }
  __syncthreads();
  RowSums mine{};
  mine.c = -INFINITY;
  if (lane < NW) mine = sums[lane];
  q = wave_sums(mine);
  count = wave_count(lane < NW ? counts[lane] : 0);
  if (BEAM || a.parts > 1) {
    if (tid == 0) {
      if constexpr (BEAM) a.part[r * a.parts + part] = q.packed();
      else a.part[r * a.parts + part] = make_float4(q.c, q.s, q.t, __int_as_float(count));
    }
    if constexpr (TOP)
      top_logits<T, NT>(x, a.n_top, (x.n_vec + NT * U - 1) / (NT * U) * (NT / 4), sh, [&](int i, uint32_t k, int id) {
        a.part_top[(r * a.parts + part) * a.n_top + i] = (uint64_t)k << 32 | (uint32_t)~(id + first);
      });
    return;
  }
  if constexpr (!BEAM) {
    const RowResult res(a, r, q, count, has, x_tok);
    if (tid == 0) res.write(a, r);
    if constexpr (TOP)
      top_logits<T, NT>(x, a.n_top, (x.n_vec + NT * U - 1) / (NT * U) * (NT / 4), sh,
                        [&](int i, uint32_t k, int id) { res.put(a, r, i, k, id); });
  }
}

// Joins the parts of a row: their sums, and the first n_top of their n_top best logits each.
template <typename T>
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobArgs a) {
  __shared__ uint64_t list[kMaxParts * RK_MAX_TOP];
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t r = blockIdx.x;
  const int n = a.parts * a.n_top;
  for (int i = tid; i < n; i += 256) list[i] = a.part_top[r * n + i];
  const float4 p = lane < a.parts ? a.part[r * a.parts + lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  const int tok = a.tokens ? a.tokens[r] : -1;
  const bool has = tok >= 0 && tok < a.vocab;
  const float x_tok = has ? Act<T>::load((const T*)a.logits + r * a.row_stride + tok) : 0.f;
  const Sums q = wave_sums(Sums{p.x, p.y, p.z});
  const RowResult res(a, r, q, wave_count(__float_as_int(p.w)), has, x_tok);
  if (tid == 0) res.write(a, r);
  __syncthreads();
  for (int i = tid; i < n; i += 256) {
    const uint64_t mine = list[i];
    int before = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) before += list[j] > mine;
    if (before < a.n_top) res.put(a, r, before, (uint32_t)(mine >> 32), (int)~(uint32_t)mine);
  }
}

// Parts of a row of about 8 passes of a 1024-thread workgroup, while CUs are idle.
void logprob_parts(int64_t n_rows, int vocab, bool bf16, int* parts, int* part_logits) {
  const int n = bf16 ? 8 : 4;
  const int64_t vectors = ((int64_t)vocab + n - 1) / n;
  const int64_t room = 256 / std::max<int64_t>(n_rows, 1), must = (vectors + kTopGroups * 16 - 2) / (kTopGroups * 16 - 1);
  const int64_t want = std::max(must, std::min(room, vectors / (8 * 1024)));
  *parts = (int)std::max<int64_t>(1, std::min<int64_t>(want, kMaxParts));
  *part_logits = (int)((vectors + *parts - 1) / *parts * n);
}

// Threads per row: the widest workgroups for few rows, so that every CU of 256 has 16
// waves with four loads each in flight (301 rows of 50257 bf16: 20.4 us with 512 threads,
// 24.8 with 1024, 24.3 with 256; in two parts a row 23.8).
hipError_t launch_logprobs(const LogprobArgs& a, bool bf16, hipStream_t s) {
  if (a.n_rows <= 0) return hipSuccess;
  const int64_t blocks = a.n_rows * a.parts;
#define RK_LOGPROBS(T, TOP)                                                                     \
  do {                                                                                          \
    if (blocks <= 256) logprob_kernel<T, 1024, TOP><<<(uint32_t)blocks, 1024, 0, s>>>(a, BeamArgs{});      \
    else if (blocks <= 512) logprob_kernel<T, 512, TOP><<<(uint32_t)blocks, 512, 0, s>>>(a, BeamArgs{});   \
    else logprob_kernel<T, 256, TOP><<<(uint32_t)blocks, 256, 0, s>>>(a, BeamArgs{});                      \
    if (a.parts > 1) logprob_join_kernel<T><<<(uint32_t)a.n_rows, 256, 0, s>>>(a);              \
  } while (0)
  if (bf16) { if (a.n_top) RK_LOGPROBS(bf16_t, true); else RK_LOGPROBS(bf16_t, false); }
  else { if (a.n_top) RK_LOGPROBS(float, true); else RK_LOGPROBS(float, false); }
#undef RK_LOGPROBS
  return hipGetLastError();
}

// --------------------------------------------------------------------------- beams
// Of a group's candidates (beam b, token v) with score_b + (x_v - c_b) - log S_b the n_out best.
// A candidate of the group's n_out best is one of its own row's: logprob_kernel leaves each
// row's (each part's) best logits in falling order, and a workgroup per group merges these lists:
// lane l of its first wave holds the head of list l, and n_out times the best head is taken and
// its list moved on.  More than 64 lists (rows in many parts) are first cut to the 64 with the
// best heads: a list with n_out better heads beside it gives nothing.  Scores between beams are
// doubles, log S among them (BeamSums says how good it is); within a beam the logits decide.
// Bound: latency, a chain of loads, sums and n_out short steps: 7.4 us for the 8 best of 16 lists,
// 4.9 for the 4 best of 12.  The rows' kernel before it reads every logit once (128 rows of 128256
// fp32 in two parts: 14.7 us, 4.5 TB/s, in part out of the cache; 4 rows of 50257 bf16: 8.0).
// (lists: 256 where rows are split to fill the card, 17 a row of 2^22 fp32 logits)
constexpr int kMaxLists = 17 * RK_MAX_BEAMS;

// log of a positive finite sum, 2^e m: logf(m), and what m times e^-that is above 1
__device__ __forceinline__ double log_sum(double s) {
  const uint64_t u = (uint64_t)__double_as_longlong(s);
  const int e = (int)(u >> 52) - 1023;
  const double m = __longlong_as_double((long long)((u & 0xfffffffffffffull) | 0x3ff0000000000000ull));
  const double y = (double)logf((float)m), z = -0.5 * y;     // e^z, |z| < 0.35, by its series: squared, 2e-15 off
  double p = 1.0 / 39916800.0;
  p = fma(p, z, 1.0 / 3628800.0);
  p = fma(p, z, 1.0 / 362880.0);
  p = fma(p, z, 1.0 / 40320.0);
  p = fma(p, z, 1.0 / 5040.0);
  p = fma(p, z, 1.0 / 720.0);
  p = fma(p, z, 1.0 / 120.0);
  p = fma(p, z, 1.0 / 24.0);
  p = fma(p, z, 1.0 / 6.0);
  p = fma(p, z, 0.5);
  p = fma(p, z, 1.0);
  p = fma(p, z, 1.0);
  return e * 0.69314718055994530942 + (y + fma(m * p, p, -1.0));
}

// A candidate as a whole number that orders like its score, 0 for none; its logit's order with
// the complement of the token; its beam.
struct Candidate {
  uint64_t score, key;
  int beam;
  __device__ __forceinline__ void set(double s, uint64_t k, int b) {
    const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);   // -0 and 0 are one score
    score = s > -INFINITY ? (u >> 63 ? ~u : u | 0x8000000000000000ull) : 0;
    key = k;
    beam = b;
  }
  __device__ __forceinline__ double value() const {
    return __longlong_as_double((long long)(score >> 63 ? score & 0x7fffffffffffffffull : ~score));
  }
  __device__ __forceinline__ bool before(const Candidate& o) const {
    return score > o.score || (score == o.score && (beam < o.beam || (beam == o.beam && key > o.key)));
  }
};

__global__ __launch_bounds__(256) void beam_join_kernel(LogprobArgs a, BeamArgs p) {
  constexpr int NT = 256;
  __shared__ float4 sums[kMaxLists];
  __shared__ uint64_t list[64 * RK_MAX_TOP];     // the lists of the first wave's lanes
  __shared__ Candidate heads[kMaxLists];
  __shared__ int chosen[64];
  // a logit's score is its difference to ref, plus shift; -inf: no candidates
  __shared__ double ref[RK_MAX_BEAMS], shift[RK_MAX_BEAMS];
  __shared__ float score[RK_MAX_BEAMS];
  __shared__ uint8_t ended[RK_MAX_BEAMS];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int nb = p.n_beams, n = a.n_top, parts = a.parts, lists = nb * parts;
  const int64_t row0 = (int64_t)blockIdx.x * nb;
  const uint64_t* top = a.part_top + row0 * parts * n;
  // what closed beams would have in the workspace is whatever was there: not used
  if (tid < nb) {
    score[tid] = p.scores[row0 + tid];
    ended[tid] = p.ended ? p.ended[row0 + tid] : 0;
  }
  for (int i = tid; i < lists; i += NT) sums[i] = a.part[row0 * parts + i];
  if (lists <= 64)
    for (int i = tid; i < lists * n; i += NT) list[i] = top[i];
  __syncthreads();
  if (parts > 1) {
    for (int b = w; b < nb; b += NT / 64) {
      const BeamSums q = wave_sums(lane < parts ? BeamSums::of(sums[b * parts + lane]) : BeamSums{-INFINITY, 0.f, 0.0});
      if (lane == 0) sums[b * parts] = q.packed();
    }
    __syncthreads();
  }
  if (tid < nb) {
    const BeamSums q = BeamSums::of(sums[tid * parts]);
    ref[tid] = q.ref();
    // without a finite largest logit S is 0 or NaN
    shift[tid] = q.s > 0.0 && q.s < INFINITY ? (double)score[tid] - log_sum(q.sum()) : -INFINITY;
  }
  __syncthreads();
  // candidate i of list l, whose key the lists have; the next in order has no better score
  const auto candidate = [&](int l, int i, uint64_t k) {
    Candidate c;
    const int b = l / parts;
    if (!(score[b] > -INFINITY)) c.set(-INFINITY, 0, b);
    else if (ended[b]) c.set(l - b * parts == 0 && i == 0 ? (double)score[b] : -INFINITY, (uint32_t)~p.end_token, b);
    else c.set(shift[b] > -INFINITY ? ((double)from_order((uint32_t)(k >> 32)) - ref[b]) + shift[b] : -INFINITY, k, b);
    return c;
  };
  const int held = min(lists, 64);                 // lists in hand
  int mine = lane;                                 // which one this lane has
  if (lists > 64) {
    for (int i = tid; i < lists; i += NT) heads[i] = candidate(i, 0, top[(int64_t)i * n]);
    __syncthreads();
    bool best[(kMaxLists + NT - 1) / NT];
#pragma unroll
    for (int q = 0; q < (kMaxLists + NT - 1) / NT; ++q) {
      const int i = q * NT + tid;
      int before = 64;
      if (i < lists) {
        const Candidate c = heads[i];
        before = 0;
        for (int j = 0; j < lists; ++j) before += heads[j].before(c) || (j < i && !c.before(heads[j]));
      }
      best[q] = before < 64;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < (kMaxLists + NT - 1) / NT; ++q)
      if (q * NT + tid < lists) heads[q * NT + tid].beam = best[q] ? 1 : 0;   // from here on: whether it is taken
    __syncthreads();
    if (w == 0) {   // in their order
      int taken = 0;
      for (int i0 = 0; i0 < lists; i0 += 64) {
        const bool t = i0 + lane < lists && heads[i0 + lane].beam;
        const uint64_t m = __ballot(t);
        if (t) chosen[taken + __popcll(m & ((1ull << lane) - 1))] = i0 + lane;
        taken += __popcll(m);
      }
    }
    __syncthreads();
    mine = chosen[lane];
    for (int i = tid; i < 64 * n; i += NT) list[i] = top[(int64_t)chosen[i / n] * n + i % n];
    __syncthreads();
  }
  if (w != 0) return;
  Candidate c;
  c.set(-INFINITY, 0, 0);
  int next = 0;
  if (lane < held) c = candidate(mine, 0, list[lane * n]);
  uint64_t ahead = lane < held ? list[lane * n + min(1, n - 1)] : 0;
  int parent = -1, token = -1;
  float value = -INFINITY;                         // of place `lane`
  for (int i = 0; i < p.n_out; ++i) {
    const uint32_t hi = wave_max((uint32_t)(c.score >> 32));
    if (hi == 0) break;                            // (a score's upper half is not 0)
    const bool up = (uint32_t)(c.score >> 32) == hi;
    uint64_t m = __ballot(up);
    if (m & (m - 1)) {
      const uint32_t lo = wave_max(up ? (uint32_t)c.score : 0);
      m = __ballot(up && (uint32_t)c.score == lo);
    }
    int win = __builtin_ctzll(m);
    if (m & (m - 1)) {   // equal scores: the lowest beam, in lanes as in lists; of its parts' the larger key
      m = __ballot((m >> lane & 1) && c.beam == __builtin_amdgcn_readlane(c.beam, win));
      uint64_t best = 0;
      for (; m; m &= m - 1) {
        const int l = __builtin_ctzll(m);
        const uint64_t k = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(c.key >> 32), l) << 32 |
                           (uint32_t)__builtin_amdgcn_readlane((int)c.key, l);
        if (k > best) { best = k; win = l; }
      }
    }
    const int b = __builtin_amdgcn_readlane(c.beam, win), t = ~__builtin_amdgcn_readlane((int)c.key, win);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)c.score, win);
    if (lane == i) {
      Candidate best;
      best.score = (uint64_t)hi << 32 | lo;
      parent = b;
      token = t;
      value = (float)best.value();
    }
    if (lane == win) {   // what comes after has been read since the list's last turn
      ++next;
      if (next < n) c = candidate(mine, next, ahead);
      else c.score = 0;
      ahead = list[lane * n + min(next + 1, n - 1)];
    }
  }
  if (lane < p.n_out) {
    const int64_t at = (int64_t)blockIdx.x * p.n_out + lane;
    p.parents[at] = parent;
    p.tokens[at] = token;
    p.scores_out[at] = value;
  }
}

// Parts of a row: as for the log probabilities, and with few rows shorter ones: there is a join
// behind them in any case (4 rows of 50257 bf16, 4 best: 9.4 us in one part, 7.8 in 3).
void beam_parts(int64_t n_rows, int vocab, bool bf16, int* parts, int* part_logits) {
  logprob_parts(n_rows, vocab, bf16, parts, part_logits);
  const int n = bf16 ? 8 : 4;
  const int64_t vectors = ((int64_t)vocab + n - 1) / n;
  const int64_t more = std::min<int64_t>(64 / std::max<int64_t>(n_rows, 1), vectors / 2048);
  if (more <= *parts) return;
  *parts = (int)more;
  *part_logits = (int)((vectors + more - 1) / more * n);
}

hipError_t launch_beam_select(const LogprobArgs& a, const BeamArgs& b, bool bf16, hipStream_t s) {
  if (a.n_rows <= 0) return hipSuccess;
  const int64_t blocks = a.n_rows * a.parts;
#define RK_BEAMS(T)                                                                                           \
  do {                                                                                                        \
    if (blocks <= 256) logprob_kernel<T, 1024, true, true><<<(uint32_t)blocks, 1024, 0, s>>>(a, b);           \
    else if (blocks <= 512) logprob_kernel<T, 512, true, true><<<(uint32_t)blocks, 512, 0, s>>>(a, b);        \
    else logprob_kernel<T, 256, true, true><<<(uint32_t)blocks, 256, 0, s>>>(a, b);                           \
  } while (0)
  if (bf16) RK_BEAMS(bf16_t); else RK_BEAMS(float);
#undef RK_BEAMS
  beam_join_kernel<<<(uint32_t)(a.n_rows / b.n_beams), 256, 0, s>>>(a, b);
  return hipGetLastError();
}

}  // namespace rk
