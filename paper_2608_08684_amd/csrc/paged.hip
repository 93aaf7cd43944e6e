// Paged key-value cache: append with the rotary embedding on the way, attention of one
// new token of each sequence over its pages, and the same over the pages that a bound
// on their keys' products ranks highest.
//
// Cache layout: k and v [n_pages, n_kv_heads, page_size, head_dim], so a page of one
// head is one contiguous block; bounds [n_pages, n_kv_heads, 2, head_dim], the least
// and the largest value of each channel over the page's keys.
#include <math.h>

#include <algorithm>

#include "rk_internal.h"

namespace rk {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;

constexpr float kLog2e = 1.4426950408889634f;

// 16 bytes of cache elements as floats and back (one rounding to nearest even)
template <typename T> struct Pack;
template <> struct Pack<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(v4u u, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ v4u put(const float* f) {
    v4u u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (uint32_t)f2bf(f[2 * i]) | ((uint32_t)f2bf(f[2 * i + 1]) << 16);
    return u;
  }
};
template <> struct Pack<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(v4u u, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(u[i]);
  }
  static __device__ __forceinline__ v4u put(const float* f) {
    v4u u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(f[i]);
    return u;
  }
};

// e^x of a difference to a running maximum.  The difference is formed before the factor
// log2(e): scaling the scores themselves would put that factor's rounding, times a
// score of 50, into the weights.
__device__ __forceinline__ float exp_diff(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
// unit e^x with the product's rounding and log2(e)'s made good, for the weights of fp32
// caches, whose outputs show them: e^-10 is off by 5e-7 without.  (Rescales and joins do
// without: what they are off by is no more than the rounding of a score as large.)
__device__ __forceinline__ float exp_diff_exact(float x, float unit) {
  x = x < -200.f ? -200.f : x;   // 0 either way; a NaN stays
  const float t = x * kLog2e, r = fmaf(x, kLog2e, -t) + x * 1.925963033500e-8f;
  return __builtin_amdgcn_exp2f(t) * fmaf(r, 0.6931471806f * unit, unit);
}

// The largest bf16 below a positive x, as the bits of a float; 0 of 0.  What is left, x minus
// it, is positive again, never 0 (at the least one step of x).
__device__ __forceinline__ uint32_t bf16_below(float x) {
  return __builtin_elementwise_sub_sat(__float_as_uint(x), 1u) & 0xffff0000u;
}

// Bounds keep a NaN.
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ int min_i(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int max_i(int a, int b) { return a > b ? a : b; }

// --------------------------------------------------------------------------- append
// New row r = off[i] + j of sequence i (m_i of them) is entry lengths[i] - m_i + j of
// the sequence.  With pos its rotary position and x < d / 2,
//   y[x]         = k[x] cos a - k[x + d/2] sin a
//   y[x + d/2]   = k[x + d/2] cos a + k[x] sin a,   a = pos theta^(-2x/d).
// The angle is a fraction of a turn in 32 bits, the upper half of pos times theta^(-2x/d)
// / (2 pi) in 64 fixed-point bits: whole turns drop out exactly (fp32 would leave a position
// of 10^6 four digits).  The frequency comes from doubles, 53 bits, so the angle is off by
// 2^-24 of a turn at a position of 2^31 and in proportion less below, then by its rounding to
// fp32 for sine and cosine, at most 2^-26 of a turn.
// Three kinds of workgroups: keys of all new rows of a page for some KV heads, whose
// bounds so take them in a fixed order without atomics; values of 16 entries; queries
// of up to 8 rows.  The first loads go out before the angles are formed.
// Bound: memory (each value read once, written once); 17928 rows, 32 / 8 heads of 128:
// 92 us (4.8 TB/s), a copy of as many bytes 89; 12 fp32 heads of 64: 72 us (4.6).  A step's
// rows (64 sequences): the latency of one pass, 6 us.
constexpr int kAppendThreads = 256, kAppendRows = 16, kAppendQueryRows = 8;

// cosine and sine of channel pair x at position pos
__device__ __forceinline__ float2 turn(const AppendArgs& a, int pos, int x) {
  if (!a.rotate) return make_float2(1.f, 0.f);
  const uint32_t lo = (uint32_t)a.freq[x], hi = (uint32_t)(a.freq[x] >> 32);
  uint32_t t = __umulhi((uint32_t)pos, lo) + (uint32_t)pos * hi;   // bits 32 .. 63 of the product
  if (pos < 0) t -= lo;                                            // pos = (uint32_t)pos - 2^32
  float s, c;
  sincospif((float)(int32_t)t * 0x1p-31f, &s, &c);
  return make_float2(c, s);
}

// A pair of 16-byte pieces, x .. and x + d/2 .., rotated.
template <typename T, int HALF>
struct Pair {
  v4u lo, hi;
  __device__ __forceinline__ void load(const T* src) {
    lo = *(const v4u*)src;
    hi = *(const v4u*)(src + HALF);
  }
  __device__ __forceinline__ void rotate(const float2* cs) {
    constexpr int VE = Pack<T>::N;
    float a[VE], b[VE], y[VE], z[VE];
    Pack<T>::get(lo, a);
    Pack<T>::get(hi, b);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const float2 c = cs[e];
      y[e] = a[e] * c.x - b[e] * c.y;
      z[e] = b[e] * c.x + a[e] * c.y;
    }
    lo = Pack<T>::put(y);
    hi = Pack<T>::put(z);
  }
  __device__ __forceinline__ void store(T* dst) const {
    *(v4u*)dst = lo;
    *(v4u*)(dst + HALF) = hi;
  }
};

// The entries that a call writes to the j-th page that it may write to of sequence s.
struct NewEntries {
  int page, in_page, n, row, entry;   // n entries from in_page on, from row `row` and entry `entry` on
  // block: a page block of the call (see launch_append)
  __device__ __forceinline__ NewEntries(const PagedView& cache, const PagedTable& tab, const AppendArgs& a,
                                        const SeqTable& st, int block) {
    n = 0;
    int s = block, j = 0, row0 = block, m = 1;
    if (!a.one_row) {
      int lo = 0, hi = st.n - 1;
      while (lo < hi) {   // the sequence whose page blocks hold this one
        const int mid = (lo + hi + 1) >> 1;
        if (a.block0[mid] <= block) lo = mid; else hi = mid - 1;
      }
      s = lo;
      j = block - a.block0[s];
      row0 = st.off[s];
      m = st.off[s + 1] - row0;
    }
    const int len = tab.lengths[s], first = (int)((uint32_t)len - (uint32_t)m);   // entries first .. len - 1
    const int p = (max_i(first, 0) >> cache.page_shift) + j;
    if (p >= tab.max_pages) return;
    const int e0 = max_i(max_i(first, 0), p << cache.page_shift), e1 = min_i(len, (p + 1) << cache.page_shift);
    if (e0 >= e1) return;
    page = tab.pages[(int64_t)s * tab.stride + p];
    if (page < 0 || page >= cache.n_pages) return;
    n = e1 - e0;
    in_page = e0 & ((1 << cache.page_shift) - 1);
    row = row0 + (e0 - first);
    entry = e0;
  }
};

template <typename T, int DH>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(PagedView cache, PagedTable tab, AppendArgs a,
                                                                SeqTable st) {
  constexpr int VE = Pack<T>::N, HALF = DH / 2, UPH = HALF / VE, NT = kAppendThreads, U = 4;
  __shared__ float2 cs[kAppendRows][HALF];
  const int tid = threadIdx.x, G = cache.n_kv, ps = 1 << cache.page_shift;
  int block = blockIdx.x;
  if (block >= a.key_blocks + a.value_blocks) {
    // ---- queries
    const int r0 = (block - a.key_blocks - a.value_blocks) * a.q_rows, n = min_i(a.q_rows, a.n_rows - r0);
    const int per_row = a.n_heads * UPH, total = n * per_row;
    Pair<T, HALF> raw[U];
    const auto at = [&](int i, int64_t stride) {
      const int rr = i / per_row, u = i - rr * per_row;
      return (int64_t)(r0 + rr) * stride + (u / UPH) * DH + (u % UPH) * VE;
    };
    const auto load = [&](int i0) {
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u].load((const T*)a.q + at(min_i(i0 + u * NT, total - 1), a.q_rs));
    };
    load(tid);
    for (int i = tid; i < n * HALF; i += NT) {
      const int r = r0 + i / HALF;
      int pos;
      if (a.positions) {
        pos = a.positions[r];
      } else if (a.one_row) {
        pos = (int)((uint32_t)tab.lengths[r] - 1u);
      } else {
        const int s = seq_of_row(st, r);
        pos = (int)((uint32_t)tab.lengths[s] - (uint32_t)(st.off[s + 1] - r));
      }
      cs[i / HALF][i % HALF] = turn(a, pos, i % HALF);
    }
    __syncthreads();
    for (int i0 = tid; i0 - tid < total; i0 += U * NT) {
      Pair<T, HALF> cur[U];
#pragma unroll
      for (int u = 0; u < U; ++u) cur[u] = raw[u];
      // in place: every piece is read by the thread that writes it, before it does
      if (i0 - tid + U * NT < total) load(i0 + U * NT);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * NT;
        if (i < total) {
          cur[u].rotate(&cs[i / per_row][i % UPH * VE]);
          cur[u].store((T*)a.q_out + at(i, a.qo_rs));
        }
      }
    }
    return;
  }
  if (block >= a.key_blocks) {
    // ---- values of up to 16 entries
    block -= a.key_blocks;
    const int subs = a.one_row ? 1 : ps / kAppendRows;
    const NewEntries w(cache, tab, a, st, block / subs);
    if (w.n == 0) return;
    int e0 = w.in_page, e1 = w.in_page + w.n;   // within the page
    if (subs > 1) {
      e0 = max_i(e0, block % subs * kAppendRows);
      e1 = min_i(e1, (block % subs + 1) * kAppendRows);
    }
    constexpr int CPH = DH / VE;
    const int per_row = G * CPH, total = (e1 - e0) * per_row;
    for (int i0 = tid; i0 < total; i0 += U * NT) {
      v4u raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = min_i(i0 + u * NT, total - 1), rr = i / per_row, c = i - rr * per_row;
        raw[u] = *(const v4u*)((const T*)a.v + (int64_t)(w.row + e0 - w.in_page + rr) * a.v_rs +
                               (int64_t)(c / CPH) * a.v_hs + c % CPH * VE);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * NT, rr = i / per_row, c = i - rr * per_row;
        if (i < total)
          *(v4u*)((T*)cache.v + (((int64_t)w.page * G + c / CPH) * ps + e0 + rr) * DH + c % CPH * VE) = raw[u];
      }
    }
    return;
  }
  // ---- keys of one page, `heads` KV heads from h0 on; a thread keeps its head and channels
  const NewEntries w(cache, tab, a, st, block / a.head_blocks);
  const int h0 = block % a.head_blocks * a.heads, heads = min_i(a.heads, G - h0);
  if (w.n == 0 || heads <= 0) return;
  __shared__ float red[NT][2 * VE];
  const int units = heads * UPH, RP = NT / units, rp = tid / units, u = tid - rp * units;   // RP >= 4 rows at a time
  const int h = h0 + u / UPH, x = u % UPH * VE;
  T* kc = (T*)cache.k + (((int64_t)w.page * G + h) * ps + w.in_page) * DH + x;
  const T* src = (const T*)a.k + (int64_t)w.row * a.k_rs + (int64_t)h * a.k_hs + x;
  float bl[2 * VE], bh[2 * VE];
#pragma unroll
  for (int e = 0; e < 2 * VE; ++e) { bl[e] = INFINITY; bh[e] = -INFINITY; }
  for (int b = 0; b < w.n; b += kAppendRows) {
    const int nb = min_i(kAppendRows, w.n - b);
    Pair<T, HALF> raw[U];
    if (rp < RP) {
#pragma unroll
      for (int q = 0; q < U; ++q) raw[q].load(src + (int64_t)(b + min_i(rp + q * RP, nb - 1)) * a.k_rs);
    }
    __syncthreads();   // the last rows' angles are done with
    for (int i = tid; i < nb * HALF; i += NT) {
      const int rr = b + i / HALF;
      cs[i / HALF][i % HALF] = turn(a, a.positions ? a.positions[w.row + rr] : w.entry + rr, i % HALF);
    }
    __syncthreads();
    if (rp < RP) {
#pragma unroll
      for (int q = 0; q < U; ++q) {
        const int rr = rp + q * RP;
        if (rr < nb) {
          raw[q].rotate(&cs[rr][x]);
          raw[q].store(kc + (int64_t)(b + rr) * DH);
          if (cache.bounds) {   // of the keys as stored
            float y[2 * VE];
            Pack<T>::get(raw[q].lo, y);
            Pack<T>::get(raw[q].hi, y + VE);
#pragma unroll
            for (int e = 0; e < 2 * VE; ++e) {
              bl[e] = least(bl[e], y[e]);
              bh[e] = largest(bh[e], y[e]);
            }
          }
        }
      }
    }
  }
  if (!cache.bounds) return;
  T* bp = (T*)cache.bounds + ((int64_t)w.page * G + h) * 2 * DH + x;
  const int rows_used = min_i(RP, w.n);
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2 * VE; ++e) red[tid][e] = side ? bh[e] : bl[e];
    __syncthreads();
    if (rp == 0) {
      float y[2 * VE];
      if (w.in_page == 0) {   // the page starts here
#pragma unroll
        for (int e = 0; e < 2 * VE; ++e) y[e] = red[tid][e];
      } else {
        Pack<T>::get(*(const v4u*)(bp + side * DH), y);
        Pack<T>::get(*(const v4u*)(bp + side * DH + HALF), y + VE);
#pragma unroll
        for (int e = 0; e < 2 * VE; ++e) y[e] = side ? largest(y[e], red[tid][e]) : least(y[e], red[tid][e]);
      }
      for (int q = 1; q < rows_used; ++q)
#pragma unroll
        for (int e = 0; e < 2 * VE; ++e) {
          const float z = red[tid + q * units][e];
          y[e] = side ? largest(y[e], z) : least(y[e], z);
        }
      *(v4u*)(bp + side * DH) = Pack<T>::put(y);
      *(v4u*)(bp + side * DH + HALF) = Pack<T>::put(y + VE);
    }
  }
}

// Dispatch on the cache's element type and head size.
#define RK_PAGED_DISPATCH(bf16, dh, CALL)                                 \
  do {                                                                    \
    if (bf16) {                                                           \
      if (dh == 64) { CALL(bf16_t, 64); } else { CALL(bf16_t, 128); }     \
    } else {                                                              \
      if (dh == 32) { CALL(float, 32); }                                  \
      else if (dh == 64) { CALL(float, 64); }                             \
      else { CALL(float, 128); }                                          \
    }                                                                     \
  } while (0)

// Page blocks: the pages that the new rows of a sequence may touch, one sequence after the other.
int64_t append_plan(const PagedView& cache, const PagedTable& tab, const SeqTable& st, AppendArgs* a) {
  const int ps = 1 << cache.page_shift, G = cache.n_kv;
  int pages = 0;
  if (a->one_row) {
    pages = tab.n_seqs;
  } else {
    for (int i = 0; i < st.n; ++i) {   // m rows touch at most (m + ps - 2) / ps + 1 pages
      a->block0[i] = pages;
      const int m = st.off[i + 1] - st.off[i];
      if (m > 0) pages += (int)(((int64_t)m + ps - 2) / ps) + 1;
    }
  }
  if (pages == 0) return 0;
  // KV heads of a key block: at most a quarter of its threads wide (four rows at a time),
  // and few enough for 512 blocks (2048 rows in pages of 128, 8 heads: 59 us with whole
  // pages, 25 with single heads)
  const int widest = 64 / (cache.head_dim / 2 / (cache.bf16 ? 8 : 4));
  a->head_blocks = std::max((G + widest - 1) / widest, std::min(G, (512 + pages - 1) / pages));
  a->heads = (G + a->head_blocks - 1) / a->head_blocks;
  const int64_t key_blocks = (int64_t)pages * a->head_blocks;
  const int64_t value_blocks = (int64_t)pages * (a->one_row ? 1 : ps / kAppendRows);
  a->q_rows = std::max(1, std::min(kAppendQueryRows, a->n_rows / 1024));
  const int64_t q_blocks = a->q ? ((int64_t)a->n_rows + a->q_rows - 1) / a->q_rows : 0;
  a->key_blocks = (int)key_blocks;
  a->value_blocks = (int)value_blocks;
  return key_blocks + value_blocks + q_blocks;
}

hipError_t launch_append(const PagedView& cache, const PagedTable& tab, const AppendArgs& a, const SeqTable& st,
                         int64_t workgroups, hipStream_t s) {
  if (workgroups <= 0) return hipSuccess;
  const uint32_t blocks = (uint32_t)workgroups;
#define RK_APPEND(T, DH) append_kernel<T, DH><<<blocks, kAppendThreads, 0, s>>>(cache, tab, a, st)
  RK_PAGED_DISPATCH(cache.bf16, cache.head_dim, RK_APPEND);
#undef RK_APPEND
  return hipGetLastError();
}

// --------------------------------------------------------------------------- page selection
// Score of a page for one KV head: sum over the query heads h that share it of
// sum_x max(q_hx lo_x, q_hx hi_x), an upper bound of the summed products with any key
// of the page.  The heads can be summed first: sum_x hi_x Q+_x + lo_x Q-_x with
// Q+ = sum_h max(q_h, 0), Q- = sum_h min(q_h, 0).  In double precision throughout, so
// the choice does not hang on the order of a sum.  Bound: memory, the bounds of every
// page read once, and below a few megabytes latency: 4 rows of 512 pages, 8 KV heads of
// 128, 7 MB: 7 us.
//
// A score becomes a whole number that orders the same way: larger for a larger score;
// the largest of all for pages that are always kept, 0 for pages that hold nothing (a
// NaN score counts as -inf).
__device__ __forceinline__ uint64_t score_key(double x) {
  if (x != x) x = -INFINITY;
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);   // -0 and 0 are one score
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

__device__ __forceinline__ int table_length(const PagedTable& tab, int row, int page_shift) {
  return max_i(0, (int)min((int64_t)tab.lengths[row], (int64_t)tab.max_pages << page_shift));
}

constexpr int kSelectThreads = 256;
constexpr int kWavePages = 1024;    // pages whose keys one wave holds in registers

// Q-, Q+ of a KV head, by the first DH threads
template <typename T, int DH>
__device__ __forceinline__ void sum_queries(const SelectArgs& a, int seq, int hk, int grp, double (*qs)[DH]) {
  const int x = threadIdx.x;
  if (x >= DH) return;
  double lo = 0.0, hi = 0.0;
  const T* qp = (const T*)a.q + (int64_t)seq * a.q_rs + (int64_t)hk * grp * DH + x;
  for (int h = 0; h < grp; ++h) {
    const double v = (double)Act<T>::load(qp + (int64_t)h * DH);
    lo += v < 0.0 ? v : 0.0;
    hi += v < 0.0 ? 0.0 : v;
  }
  qs[0][x] = lo;
  qs[1][x] = hi;
}

// The workgroup: keys of pages first .. last - 1 of a sequence's `count`.  A group of LPP
// lanes takes a page (its lower bounds, then its upper ones), four pages in flight, the
// first of them before the queries are summed.  put(p, key).
template <typename T, int DH, typename Put>
__device__ __forceinline__ void score_pages(const PagedView& cache, const PagedTable& tab, const SelectArgs& a, int seq,
                                            int hk, int count, int first, int last, double (*qs)[DH], Put put) {
  constexpr int VE = Pack<T>::N, LPP = 2 * DH / VE, PER = kSelectThreads / LPP, U = 4;
  const int group = threadIdx.x / LPP, sub = threadIdx.x % LPP, x0 = (sub * VE) % DH, side = sub * VE / DH;
  const int32_t* pages = tab.pages + (int64_t)seq * tab.stride;
  v4u raw[U];
  bool ok[U];
  const auto load = [&](int p0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int page = pages[min_i(p0 + group + u * PER, last - 1)];
      ok[u] = page >= 0 && page < cache.n_pages;
      raw[u] = *(const v4u*)((const T*)cache.bounds + ((int64_t)(ok[u] ? page : 0) * cache.n_kv + hk) * 2 * DH + sub * VE);
    }
  };
  if (first < last) load(first);
  sum_queries<T, DH>(a, seq, hk, a.n_heads / cache.n_kv, qs);
  __syncthreads();
  double q[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) q[e] = qs[side][x0 + e];
  for (int p0 = first; p0 < last; p0 += PER * U) {
    if (p0 > first) load(p0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = p0 + group + u * PER;
      float f[VE];
      Pack<T>::get(raw[u], f);
      double s = 0.0;
#pragma unroll
      for (int e = 0; e < VE; ++e) s += q[e] * (q[e] != 0.0 ? (double)f[e] : 0.0);   // an infinite bound of 0 counts 0
#pragma unroll
      for (int d = LPP / 2; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
      if (sub == 0 && p < last)
        put(p, !ok[u] ? 0ull : p < a.keep_first || p >= count - a.keep_last ? ~0ull : score_key(s));
    }
  }
}

struct SelectShared {
  uint64_t range[kSelectThreads / 64][2];
  int hist[256], scan[kSelectThreads / 64], found[3], has_last;
};

// One wave: the n_select largest keys of `count` <= kWavePages pages, ties to the lower
// page, by halving an interval of keys until exactly that many reach its lower end (a
// dozen steps on scores that differ; 64 and a tie at most).  Every step is counting in
// registers, no barrier: 512 pages 2 us less than by digits in a workgroup.
// key(p): 0 for a page that holds nothing, never taken.  put(i, p, page): the i-th is page
// p of the sequence.  Returns the entries of the chosen pages: whole pages, but for the
// sequence's last one, which comes last.
template <typename Key, typename Put>
__device__ __forceinline__ int take_pages_wave(const int32_t* pages, int n, int len, int count, int page_shift, Key key,
                                               Put put) {
  constexpr int HELD = kWavePages / 64;
  const int lane = threadIdx.x & 63;
  const uint64_t lower = (1ull << lane) - 1;
  uint64_t k[HELD];
  int page[HELD];
  int real = 0, forced = 0;
  uint32_t top = 0, bottom = 0;   // of the upper halves of the keys in between: the largest, the complement of the least
  // whole runs of loads, no branch between them
#pragma unroll
  for (int i0 = 0; i0 < HELD; i0 += 4) {
    if (i0 * 64 < count) {
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) {
        k[i] = key(min_i(i * 64 + lane, count - 1));
        page[i] = pages[min_i(i * 64 + lane, count - 1)];
      }
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) k[i] = i * 64 + lane < count ? k[i] : 0ull;
    } else {
#pragma unroll
      for (int i = i0; i < i0 + 4; ++i) k[i] = 0;
    }
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (i * 64 >= count) break;
    real += __popcll(__ballot(k[i] != 0));
    forced += __popcll(__ballot(k[i] == ~0ull));
    if (k[i] != 0 && k[i] != ~0ull) {
      top = max(top, (uint32_t)(k[i] >> 32));
      bottom = max(bottom, ~(uint32_t)(k[i] >> 32));
    }
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    top = max(top, (uint32_t)__shfl_xor((int)top, d, 64));
    bottom = max(bottom, (uint32_t)__shfl_xor((int)bottom, d, 64));
  }
  // first by the upper halves, in which scores that differ by a millionth differ
  uint32_t lo32 = ~(uint32_t)__builtin_amdgcn_readfirstlane((int)bottom);
  uint32_t hi32 = (uint32_t)__builtin_amdgcn_readfirstlane((int)top);
  bool exact = real <= n || forced == n;
  const bool given = exact;
  while (!exact && lo32 < hi32) {
    const uint32_t mid = lo32 + (hi32 - lo32) / 2 + 1;
    int c = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (i * 64 < count) c += __popcll(__ballot((uint32_t)(k[i] >> 32) >= mid));
    if (c >= n) lo32 = mid; else hi32 = mid - 1;
    exact = c == n;
  }
  uint64_t lo = given ? (real <= n ? 1ull : ~0ull) : (uint64_t)lo32 << 32;
  uint64_t hi = (uint64_t)lo32 << 32 | 0xffffffffu;
  while (!exact && lo < hi) {
    const uint64_t mid = lo + (hi - lo) / 2 + 1;
    int c = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (i * 64 < count) c += __popcll(__ballot(k[i] >= mid));
    if (c >= n) lo = mid; else hi = mid - 1;
    exact = c == n;
  }
  int want = n;   // of the keys equal to lo
  if (!exact) {
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (i * 64 < count) want -= __popcll(__ballot(k[i] > lo));
  }
  int taken = 0;
  bool last = false;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (i * 64 >= count) break;
    bool take = k[i] > lo || (exact && k[i] == lo);
    if (!exact) {
      const uint64_t e = __ballot(k[i] == lo);
      if (k[i] == lo && __popcll(e & lower) < want) take = true;
      want -= __popcll(e);
    }
    const uint64_t b = __ballot(take);
    if (take) put(taken + __popcll(b & lower), i * 64 + lane, page[i]);
    taken += __popcll(b);
    if ((count - 1) / 64 == i) last = b >> ((count - 1) & 63) & 1;
  }
  for (int i = taken + lane; i < n; i += 64) put(i, -1, -1);
  return (taken << page_shift) - (last ? (count << page_shift) - len : 0);
}

// The workgroup: the same for any number of pages, by the digits of the key, 8 bits a step
// from the highest bit in which any two differ; the search ends as soon as the pages at
// or above the digits found are exactly those wanted.  The list goes to the workspace.
template <typename Key>
__device__ __forceinline__ void take_pages(const PagedView& cache, const PagedTable& tab, const SelectArgs& a, int seq,
                                           int sh_row, int len, int count, SelectShared& sh, Key key) {
  constexpr int NT = kSelectThreads, NW = NT / 64;
  static_assert(NT == 256, "a thread per digit");
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, ps = 1 << cache.page_shift;
  const int32_t* pages = tab.pages + (int64_t)seq * tab.stride;
  const auto put = [&](int i, int p, int page) {
    a.list[(int64_t)sh_row * a.n_select + i] = page;
    if (a.selected) a.selected[(int64_t)sh_row * a.n_select + i] = p;
  };
  // keys that agree with prefix above `shift` bits: `want` of them are still to be chosen
  uint64_t prefix = 1;
  int want = a.n_select, shift = 64;
  bool exact = count <= a.n_select;   // every key from prefix up is taken
  if (tid == 0) sh.has_last = 0;
  if (!exact) {
    uint64_t lo = ~0ull, hi = 0;
    for (int p = tid; p < count; p += NT) {
      const uint64_t k = key(p);
      lo = k < lo ? k : lo;
      hi = k > hi ? k : hi;
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
      const uint64_t l = __shfl_xor((unsigned long long)lo, d, 64), h = __shfl_xor((unsigned long long)hi, d, 64);
      lo = l < lo ? l : lo;
      hi = h > hi ? h : hi;
    }
    if (lane == 0) { sh.range[w][0] = lo; sh.range[w][1] = hi; }
    __syncthreads();
    for (int i = 0; i < NW; ++i) {
      lo = sh.range[i][0] < lo ? sh.range[i][0] : lo;
      hi = sh.range[i][1] > hi ? sh.range[i][1] : hi;
    }
    shift = lo == hi ? 0 : 64 - __builtin_clzll(lo ^ hi);   // bits that are not the same in all keys
    prefix = shift == 64 ? 0 : hi >> shift << shift;
  }
  while (!exact && shift > 0) {
    const int width = min_i(shift, 8), above = shift;
    shift -= width;
    sh.hist[tid] = 0;
    __syncthreads();
    for (int p = tid; p < count; p += NT) {
      const uint64_t k = key(p);
      if (above == 64 || (k >> above) == (prefix >> above)) atomicAdd(&sh.hist[(k >> shift) & ((1 << width) - 1)], 1);
    }
    __syncthreads();
    // thread t holds digit 255 - t: the digit at which the counts from the top reach `want`
    const int c = sh.hist[255 - tid];
    int sum = c;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d, 64);
      if (lane >= d) sum += o;
    }
    if (lane == 63) sh.scan[w] = sum;
    __syncthreads();
    for (int i = 0; i < w; ++i) sum += sh.scan[i];
    if (sum >= want && sum - c < want) {
      sh.found[0] = 255 - tid;
      sh.found[1] = sum - c;
      sh.found[2] = c;
    }
    __syncthreads();
    prefix |= (uint64_t)sh.found[0] << shift;
    want -= sh.found[1];
    exact = sh.found[2] == want;
  }
  // keys above the prefix, and of those equal to it (all digits used) the first `want`
  int taken = 0, equal = 0;
  for (int p0 = 0; p0 < count; p0 += NT) {
    const int p = p0 + tid;
    const uint64_t k = p < count ? key(p) : 0ull;
    bool take = k != 0 && (exact ? k >= prefix : k > prefix);
    const bool eq = !exact && k != 0 && k == prefix;
    if (!exact) {   // rank among the equal keys, in page order
      const uint64_t b = __ballot(eq);
      __syncthreads();
      if (lane == 0) sh.scan[w] = __popcll(b);
      __syncthreads();
      int before = equal;
      for (int i = 0; i < NW; ++i) {
        before += i < w ? sh.scan[i] : 0;
        equal += sh.scan[i];
      }
      if (eq && before + __popcll(b & ((1ull << lane) - 1)) < want) take = true;
    }
    const uint64_t b = __ballot(take);
    __syncthreads();
    if (lane == 0) sh.scan[w] = __popcll(b);
    __syncthreads();
    int at = taken + __popcll(b & ((1ull << lane) - 1));
    for (int i = 0; i < NW; ++i) {
      at += i < w ? sh.scan[i] : 0;
      taken += sh.scan[i];
    }
    if (take) {
      put(at, p, pages[p]);
      if (p == count - 1) sh.has_last = 1;
    }
  }
  for (int i = taken + tid; i < a.n_select; i += NT) put(i, -1, -1);
  __syncthreads();
  if (tid == 0) a.list_len[sh_row] = taken * ps - (sh.has_last ? count * ps - len : 0);
}

// Keys of a run of pages per workgroup.
template <typename T, int DH>
__global__ __launch_bounds__(kSelectThreads) void page_scores_kernel(PagedView cache, PagedTable tab, SelectArgs a,
                                                                     int chunks) {
  __shared__ double qs[2][DH];
  const int G = cache.n_kv, chunk = blockIdx.x % chunks, row = blockIdx.x / chunks, seq = row / G, hk = row % G;
  const int len = table_length(tab, seq, cache.page_shift);
  const int count = (len + (1 << cache.page_shift) - 1) >> cache.page_shift;
  const int per = (tab.max_pages + chunks - 1) / chunks, first = chunk * per, last = min_i(count, first + per);
  if (first >= last) return;
  score_pages<T, DH>(cache, tab, a, seq, hk, count, first, last, qs,
                     [&](int p, uint64_t k) { a.keys[(int64_t)row * tab.max_pages + p] = k; });
}

// More pages than a wave holds: the choice by itself, for the attention to read.
__global__ __launch_bounds__(kSelectThreads) void page_select_kernel(PagedView cache, PagedTable tab, SelectArgs a) {
  __shared__ SelectShared sh;
  const int row = blockIdx.x, seq = row / cache.n_kv;
  const int len = table_length(tab, seq, cache.page_shift);
  const int count = (len + (1 << cache.page_shift) - 1) >> cache.page_shift;
  const uint64_t* keys = a.keys + (int64_t)row * tab.max_pages;
  take_pages(cache, tab, a, seq, row, len, count, sh, [&](int p) { return keys[p]; });
}

// --------------------------------------------------------------------------- attention of one new token
// o_h = sum_u softmax_u(scale q_h . k_u) v_u over the entries u < length of the
// sequence; query head h reads KV head h / (H / H_kv).  One pass over the cache with a
// running maximum m, sum l and output o per wave.  A workgroup = 4 waves serves one
// (sequence, KV head, part of the length) and up to 16 of the query heads that share
// the KV head; its waves take the part's 32-entry tiles in turn and are joined through
// LDS, the parts by a second kernel.
//   scores  S^T[entry, head] = K Q^T: the cache's rows are the A operand as they lie
//           in memory, so K goes from memory to the matrix unit's registers directly;
//   output  O^T[d, head] = V^T P^T: a lane's scores are already the B operand of that
//           product (entries 4 g + i of its 16-lane group g), and V^T comes out of a
//           row-major LDS tile with transposing reads (bf16) or from memory with d
//           spread over the product's rows (fp32).
// bf16: a weight p is the sum of three bf16 numbers, all of its 24 bits: the matrix unit has
// the time (a tile's 16 KB take longer to arrive than 32 MFMAs), and the output then carries
// only its own rounding.  All three are positive, so that an infinite value stays one (a part
// of the other sign, or of 0, would make it NaN).
// Entries on pages outside the cache and entries past the length weigh nothing; their
// scores are replaced by -inf and their values by 0, whatever memory holds there.
// Bound: memory.  8 KV heads of 128, 32 query heads, with the join: 64 sequences of 4096
// 191 us (5.6 TB/s, a plain read of as much 6), 32 of 100 .. 8192 112 us (5.3), 2 of up to
// 32768 50 us (5.1: the join and the first tile's way, lengths to pages to keys, are 9 of
// them).  8 waves a workgroup, three workgroups per CU, equal runs of tiles for every
// workgroup whatever the sequences' lengths: all slower or the same.
constexpr int kDecodeWaves = 4, kTile = 32;

template <typename T, int DH> struct DecodeTile;

template <int DH> struct DecodeTile<bf16_t, DH> {
  static constexpr int CH = DH / 8;          // 16-byte pieces of a row
  static constexpr int NC = DH / 32;         // k-steps of the scores
  static constexpr int NV = kTile * CH / 64; // 16-byte loads of V per lane
  static constexpr int ND = DH / 16;         // 16-row blocks of O^T
  static constexpr int LDS = kTile * DH * 2; // bytes per wave
  bf16x8_t q[NC];
  v4u k[2][NC], v[NV];

  // the 32-byte pair of pieces that ds_read_b64_tr_b16 takes from a row, placed so
  // that eight consecutive rows use all 64 banks
  static __device__ __forceinline__ int swz(int row) { return DH == 128 ? (row & 7) << 1 : ((row >> 1) & 3) << 1; }

  __device__ __forceinline__ void load_q(const bf16_t* qp, int lane) {   // row of this lane's head
#pragma unroll
    for (int c = 0; c < NC; ++c)
      q[c] = __builtin_bit_cast(bf16x8_t, *(const v4u*)(qp + c * 32 + (lane >> 4) * 8));
  }
  // rows of the tile's two 16-entry halves
  __device__ __forceinline__ void load_k(const bf16_t* k0, const bf16_t* k1, int lane) {
    const uint32_t at = (lane & 15) * DH + (lane >> 4) * 8;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      k[0][c] = *(const v4u*)(k0 + at + c * 32);
      k[1][c] = *(const v4u*)(k1 + at + c * 32);
    }
  }
  __device__ __forceinline__ void load_v(const bf16_t* v0, const bf16_t* v1, int lane) {
    // a load covers 64 / CH rows, all of one half
    const uint32_t at = lane * 8;
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = *(const v4u*)((i < NV / 2 ? v0 : v1) + at + i % (NV / 2) * 512);
  }
  __device__ __forceinline__ void clear_values(uint32_t seen, int lane) {   // bit r: row r counts
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (!(seen >> ((i * 64 + lane) / CH) & 1)) v[i] = v4u{0, 0, 0, 0};
  }
  __device__ __forceinline__ void scores(f32x4_t s[2]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c)
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[t][c]), q[c], s[t], 0, 0, 0);
    }
  }
  // the values' registers are free after stage_v
  __device__ __forceinline__ void stage_v(char* lds, int lane) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int slot = i * 64 + lane, row = slot / CH, ch = slot % CH;
      *(v4u*)(lds + (row * CH + (ch ^ swz(row))) * 16) = v[i];
    }
    wave_sync();
  }
  static constexpr bool kStaged = true;
  __device__ __forceinline__ void values(const f32x4_t p[2], f32x4_t* o, char* lds, int lane) const {
    v4u part[3];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float x = p[e >> 2][e & 3], y = p[e >> 2][(e & 3) + 1];
      const uint32_t x0 = bf16_below(x), y0 = bf16_below(y);
      const float x1 = x - __uint_as_float(x0), y1 = y - __uint_as_float(y0);
      const uint32_t x2 = bf16_below(x1), y2 = bf16_below(y1);
      part[0][e / 2] = __builtin_amdgcn_perm(y0, x0, 0x07060302u);   // the upper halves
      part[1][e / 2] = __builtin_amdgcn_perm(y2, x2, 0x07060302u);
      part[2][e / 2] = (uint32_t)f2bf(x1 - __uint_as_float(x2)) | ((uint32_t)f2bf(y1 - __uint_as_float(y2)) << 16);
    }
    const int g = lane >> 4, jj = lane & 15, r = 4 * g + (jj >> 2);
#pragma unroll
    for (int b = 0; b < ND; ++b) {
      const int ch = 2 * b + ((jj & 3) >> 1);
      const char* at = lds + (r * CH + (ch ^ swz(r))) * 16 + (jj & 1) * 8;   // swz(r + 16) = swz(r)
      const s16x4_t a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      const s16x4_t a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 16 * CH * 16));
      const v4u a = {__builtin_bit_cast(v2u, a0)[0], __builtin_bit_cast(v2u, a0)[1], __builtin_bit_cast(v2u, a1)[0],
                     __builtin_bit_cast(v2u, a1)[1]};
#pragma unroll
      for (int i = 0; i < 3; ++i)
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                       __builtin_bit_cast(bf16x8_t, part[i]), o[b], 0, 0, 0);
    }
    wave_sync();
  }
  // channel of element i of output block b in 16-lane group g
  static __device__ __forceinline__ int channel(int b, int g, int i) { return b * 16 + 4 * g + i; }
};

template <int DH> struct DecodeTile<float, DH> {
  static constexpr int NC = DH / 16;
  static constexpr int VEC = DH >= 64 ? 4 : 2;   // channels per lane and load of V
  static constexpr int NP = DH / (16 * VEC);     // loads per entry
  static constexpr int ND = DH / 16;
  static constexpr int LDS = 0;
  typedef float vecf __attribute__((ext_vector_type(VEC)));
  f32x4_t q[NC], k[2][NC];
  vecf v[2][4][NP];

  __device__ __forceinline__ void load_q(const float* qp, int lane) {
#pragma unroll
    for (int c = 0; c < NC; ++c) q[c] = *(const f32x4_t*)(qp + c * 16 + (lane >> 4) * 4);
  }
  __device__ __forceinline__ void load_k(const float* k0, const float* k1, int lane) {
    const uint32_t at = (lane & 15) * DH + (lane >> 4) * 4;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      k[0][c] = *(const f32x4_t*)(k0 + at + c * 16);
      k[1][c] = *(const f32x4_t*)(k1 + at + c * 16);
    }
  }
  __device__ __forceinline__ void load_v(const float* v0, const float* v1, int lane) {
    const uint32_t at = (lane >> 4) * 4 * DH + (lane & 15) * VEC;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < NP; ++c) {
        v[0][i][c] = *(const vecf*)(v0 + at + i * DH + c * 16 * VEC);
        v[1][i][c] = *(const vecf*)(v1 + at + i * DH + c * 16 * VEC);
      }
  }
  static constexpr bool kStaged = false;
  __device__ __forceinline__ void stage_v(char*, int) const {}
  __device__ __forceinline__ void clear_values(uint32_t seen, int lane) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!(seen >> (t * 16 + 4 * (lane >> 4) + i) & 1))
#pragma unroll
          for (int c = 0; c < NP; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[t][i][c][e] = 0.f;
  }
  __device__ __forceinline__ void scores(f32x4_t s[2]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // four sums over a quarter of the channels each: shorter chains, and none waits for another
      f32x4_t a[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        a[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) a[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[t][c][e], q[c][e], a[e], 0, 0, 0);
      }
      s[t] = (a[0] + a[1]) + (a[2] + a[3]);
    }
  }
  __device__ __forceinline__ void values(const f32x4_t p[2], f32x4_t* o, char*, int) const {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < NP; ++c)
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            o[c * VEC + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[t][i][c][e], p[t][i], o[c * VEC + e], 0, 0, 0);
  }
  static __device__ __forceinline__ int channel(int b, int g, int i) {
    return (b / VEC) * 16 * VEC + VEC * (4 * g + i) + b % VEC;
  }
};

// Entries of one part of a length: whole tiles for every wave, at most n_parts parts.
__device__ __forceinline__ int part_entries(int len, int n_parts) {
  constexpr int unit = kTile * kDecodeWaves;
  const int per = (len + n_parts - 1) / n_parts;
  return max_i((per + unit - 1) / unit, 1) * unit;
}

// SEL: attention over selected pages.  kKeys: their keys are in the workspace; kScores:
// the workgroup forms them; either way its first wave then makes the choice, the same
// one in every part of a row (what that costs, a few microseconds, is less than a launch
// and the way through memory).
enum class Sel { kNone, kKeys, kScores };

template <typename T, int DH, Sel SEL>
__global__ __launch_bounds__(64 * kDecodeWaves) void decode_kernel(PagedView cache, PagedTable tab, DecodeArgs a,
                                                                   SelectArgs sel) {
  using Tile = DecodeTile<T, DH>;
  constexpr int NW = kDecodeWaves, SP = DH + 4;
  constexpr int AREA0 = Tile::LDS * NW > NW * 16 * SP * 4 ? Tile::LDS * NW : NW * 16 * SP * 4;
  constexpr int SCORES = SEL == Sel::kScores ? 2 * DH * 8 + kWavePages * 8 : 0;
  constexpr int AREA = AREA0 > SCORES ? AREA0 : SCORES;
  __shared__ __attribute__((aligned(16))) char area[AREA];
  __shared__ float sm[NW][16], sl[NW][16];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = cache.n_kv, grp = a.n_heads / G, tiles_h = (grp + 15) / 16;
  // block = ((sequence * G + KV head) * head tiles + head tile) * parts + part
  int b = blockIdx.x;
  const int part = b % a.n_parts; b /= a.n_parts;
  const int ht = b % tiles_h; b /= tiles_h;
  const int hk = b % G;
  int seq = b / G, row, len;
  if (a.longest_first) {   // lane i knows sequence i
    const int mine = lane < tab.n_seqs ? table_length(tab, lane, cache.page_shift) : -1;
    const int key = min_i(mine, 0x1ffffff) * 64 + 63 - lane;   // no two equal
    int before = 0;
    for (int j = 0; j < tab.n_seqs; ++j) before += __builtin_amdgcn_readlane(key, j) > key;
    seq = row = __builtin_ctzll(__ballot(before == seq && lane < tab.n_seqs));
    len = __builtin_amdgcn_readlane(mine, seq);
  } else {
    row = tab.per_head ? seq * G + hk : seq;
    len = table_length(tab, row, cache.page_shift);
  }
  const int32_t* pages = tab.pages + (int64_t)row * tab.stride;
  __shared__ int chosen[SEL == Sel::kNone ? 1 : kWavePages], chosen_len;
  if constexpr (SEL != Sel::kNone) {
    const int count = (len + (1 << cache.page_shift) - 1) >> cache.page_shift, list = seq * G + hk;
    const uint64_t* keys = sel.keys + (int64_t)list * tab.max_pages;
    if constexpr (SEL == Sel::kScores) {
      static_assert(kSelectThreads == 64 * NW, "score_pages");
      double (*qs)[DH] = reinterpret_cast<double (*)[DH]>(area);
      uint64_t* scored = reinterpret_cast<uint64_t*>(area + 2 * DH * 8);
      score_pages<T, DH>(cache, tab, sel, seq, hk, count, 0, count, qs, [&](int p, uint64_t k) { scored[p] = k; });
      keys = scored;
      __syncthreads();
    }
    if (w == 0) {
      const bool tell = part == 0 && ht == 0;
      const int n = take_pages_wave(pages, sel.n_select, len, count, cache.page_shift,
                                    [&](int p) { return keys[p]; },
                                    [&](int i, int p, int page) {
                                      chosen[i] = page;
                                      if (tell && sel.selected) sel.selected[(int64_t)list * sel.n_select + i] = p;
                                    });
      if (lane == 0) {
        chosen_len = n;
        if (tell) sel.list_len[list] = n;   // for the joining kernel
      }
    }
    __syncthreads();
    len = chosen_len;
  }
  const auto page_at = [&](int i) { return SEL == Sel::kNone ? pages[i] : chosen[i]; };
  const int per = part_entries(len, a.n_parts);
  const int start = part * per, end = min_i(len, start + per);
  if (part > 0 && start >= len) return;   // the joining kernel knows; part 0 of an empty sequence stays
  const int nh = min_i(16, grp - ht * 16), h0 = hk * grp + ht * 16;
  const int shift = cache.page_shift, in_mask = (1 << shift) - 1;
  const int64_t head_at = (int64_t)hk << shift, page_rows = (int64_t)G << shift;

  Tile tile;
  const int col = lane & 15, g = lane >> 4;
  tile.load_q((const T*)a.q + (int64_t)seq * a.q_rs + (int64_t)(h0 + min_i(col, nh - 1)) * DH, lane);
  f32x4_t o[Tile::ND];
#pragma unroll
  for (int i = 0; i < Tile::ND; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  // Weights count in units of a power of two above the part's entries: their sum stays below
  // 1, and that of weighted values below the largest, however large they are.
  const float unit = __uint_as_float((127u - (32u - __builtin_clz(max_i(end - start, 1)))) << 23);
  // Pages of the tile at entry k0 (at the part's last tile where k0 lies past its end) and
  // its rows.  A page that holds nothing is read as page 0 and not used.
  struct Pages {
    int k0, p0, p1;
  };
  struct Where {
    int64_t at0, at1;   // element offsets of the two halves
    uint32_t seen;      // entries that count
  };
  const int step = NW * kTile, first = start + w * kTile;
  const int last = first + (max_i(end - 1 - first, 0) / step) * step;
  const auto pages_of = [&](int k) {
    const int k0 = min_i(k, last);
    return Pages{k0, page_at(k0 >> shift), page_at(min_i(k0 + 16, end - 1) >> shift)};
  };
  const auto where = [&](Pages p) {
    const int p0 = __builtin_amdgcn_readfirstlane(p.p0), p1 = __builtin_amdgcn_readfirstlane(p.p1);
    const bool ok0 = p0 >= 0 && p0 < cache.n_pages, ok1 = p1 >= 0 && p1 < cache.n_pages;
    Where wh;
    wh.at0 = ((ok0 ? p0 : 0) * page_rows + head_at + (p.k0 & in_mask)) * DH;
    wh.at1 = ((ok1 ? p1 : 0) * page_rows + head_at + ((p.k0 + 16) & in_mask)) * DH;
    wh.seen = (ok0 ? 0xffffu : 0u) | (ok1 ? 0xffff0000u : 0u);
    if (end - p.k0 < 32) wh.seen &= (1u << (end - p.k0)) - 1u;
    return wh;
  };
  const T* kc = (const T*)cache.k;
  const T* vc = (const T*)cache.v;
  // The next tile's rows are asked for as soon as this one's leave their registers: its
  // keys after the scores, its values once they are in LDS; their pages a tile earlier.
  // After the last tile these loads repeat it, so that no wait depends on a branch.
  Where cur{}, nxt{};
  Pages ahead{};
  if (first < end) {
    cur = where(pages_of(first));
    tile.load_k(kc + cur.at0, kc + cur.at1, lane);
    tile.load_v(vc + cur.at0, vc + cur.at1, lane);
    nxt = where(pages_of(first + step));
    ahead = pages_of(first + 2 * step);
  }
  for (int k0 = first; k0 < end; k0 += step) {
    const uint32_t seen = cur.seen;
    f32x4_t s[2];
    tile.scores(s);
    tile.load_k(kc + nxt.at0, kc + nxt.at1, lane);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] *= a.scale;
    if (seen != 0xffffffffu) {
      tile.clear_values(seen, lane);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(seen >> (t * 16 + 4 * g + i) & 1)) s[t][i] = -INFINITY;
    }
    cur = nxt;
    if constexpr (Tile::kStaged) {
      tile.stage_v(area + w * Tile::LDS, lane);
      tile.load_v(vc + cur.at0, vc + cur.at1, lane);
    }
    nxt = where(ahead);
    ahead = pages_of(k0 + 3 * step);
    float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                     fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;
    const float corr = exp_diff(m - ref);
    m = m_new;
    l *= corr;
#pragma unroll
    for (int i = 0; i < Tile::ND; ++i) o[i] *= corr;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[t][i] = sizeof(T) == 4 ? exp_diff_exact(s[t][i] - ref, unit) : exp_diff(s[t][i] - ref) * unit;
        l += s[t][i];
      }
    tile.values(s, o, area + w * Tile::LDS, lane);
    if constexpr (!Tile::kStaged) tile.load_v(vc + cur.at0, vc + cur.at1, lane);
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  __syncthreads();   // the tiles are done with: their area takes the waves' outputs
  float* so = (float*)area;
  if (g == 0) { sm[w][col] = m; sl[w][col] = l; }
#pragma unroll
  for (int i = 0; i < Tile::ND; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) so[(w * 16 + col) * SP + Tile::channel(i, g, e)] = o[i][e];
  __syncthreads();
  for (int i = tid; i < nh * DH; i += 64 * NW) {
    const int h = i / DH, x = i % DH;
    float M = sm[0][h];
#pragma unroll
    for (int q = 1; q < NW; ++q) M = fmaxf(M, sm[q][h]);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f, v = 0.f;
#pragma unroll
    for (int q = 0; q < NW; ++q) {
      const float c = exp_diff(sm[q][h] - ref);
      L += sl[q][h] * c;
      v += so[(q * 16 + h) * SP + x] * c;
    }
    // nothing seen: 0, with a log-sum-exp of -inf (a NaN sum stays NaN)
    v = L == 0.f ? 0.f : v / L;
    const float lse = L == 0.f ? -INFINITY : ref + logf(L / unit);
    const int64_t at = (int64_t)seq * a.n_heads + h0 + h;
    if (a.n_parts == 1) {
      Act<T>::store((T*)a.out + (int64_t)seq * a.out_rs + (int64_t)(h0 + h) * DH + x, v);
      if (a.lse && x == 0) a.lse[at] = lse;
    } else {
      a.part_o[(at * a.n_parts + part) * DH + x] = v;
      if (x == 0) a.part_lse[at * a.n_parts + part] = lse;
    }
  }
}

// Joins the parts of one (sequence, query head): o = sum_s e^(lse_s - M) o_s / sum_s e^(lse_s - M).
// A workgroup of 256 threads: every wave forms the weights (the same sums in the same
// order), 256 / DH thread groups take the parts in turn, eight loads in flight each.
// Bound: latency; 64 parts of 128 channels, 64 rows: 5.4 us, with one group and a load
// at a time 19.5.
constexpr int kMaxDecodeParts = 256;

template <typename T, int DH>
__global__ __launch_bounds__(256) void decode_join_kernel(PagedTable tab, DecodeArgs a, int n_kv, int page_shift) {
  constexpr int NG = 256 / DH;
  __shared__ float wt[kMaxDecodeParts], red[NG][DH];
  const int tid = threadIdx.x, lane = tid & 63, x = tid % DH, g = tid / DH;
  const int seq = blockIdx.x / a.n_heads, h = blockIdx.x % a.n_heads;
  const int row = tab.per_head ? seq * n_kv + h / (a.n_heads / n_kv) : seq;
  const int len = table_length(tab, row, page_shift);
  const int per = part_entries(len, a.n_parts), n = max_i(1, (len + per - 1) / per);
  const int64_t at = (int64_t)blockIdx.x * a.n_parts;
  float M = -INFINITY, lse[kMaxDecodeParts / 64];
#pragma unroll
  for (int i = 0; i < kMaxDecodeParts / 64; ++i) {
    lse[i] = i * 64 + lane < n ? a.part_lse[at + i * 64 + lane] : -INFINITY;
    M = fmaxf(M, lse[i]);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d, 64));
  const float ref = M == -INFINITY ? 0.f : M;
  float L = 0.f;
#pragma unroll
  for (int i = 0; i < kMaxDecodeParts / 64; ++i) {
    lse[i] = exp_diff(lse[i] - ref) * (1.0f / kMaxDecodeParts);   // so that no sum of outputs overflows
    L += lse[i];
    if (tid < 64 && i * 64 < n) wt[i * 64 + lane] = lse[i];
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) L += __shfl_xor(L, d, 64);
  __syncthreads();
  const float* po = a.part_o + at * DH + x;
  float v = 0.f;
#pragma unroll 8
  for (int p = g; p < n; p += NG) v = fmaf(wt[p], po[(int64_t)p * DH], v);
  red[g][x] = v;
  __syncthreads();
  if (g != 0) return;
#pragma unroll
  for (int i = 1; i < NG; ++i) v += red[i][x];
  Act<T>::store((T*)a.out + (int64_t)seq * a.out_rs + (int64_t)h * DH + x, L == 0.f ? 0.f : v / L);
  if (a.lse && x == 0) a.lse[blockIdx.x] = L == 0.f ? -INFINITY : ref + logf(L * kMaxDecodeParts);
}

// Parts per row, a row being a (sequence, KV head, head tile), from the longest that a
// sequence may be; no part shorter than 256 entries.  A split costs its join (4 - 5 us) and
// gains where rows leave CUs idle or, being of unequal length, end at different times.  us
// for 8 KV heads of 128 in bf16, all of that length | lengths from 100 up to it:
//   up to 512 one part: a workgroup's 512 entries take as long as the join (1 row of 8 heads
//     9.0, two parts 9.9; 256 rows 14.5 | 12.0 and 19.6 | 17.0);
//   up to 1024 for 256 workgroups, but one part from 96 rows on (128 rows 15.2 | 14.7, two
//     parts 18.0 | 15.3; 32 rows 14.4 | 14.2, four 11.4 | 11.1);
//   below 4096 for 256, one to a CU (64 rows of 2048: 4 parts 18.0 | 14.6, 8 19.8 | 17.5;
//     256 rows: 1 part 49.4 | 35.0, 4 58.1 | 41.0), but two where one would leave some CUs two
//     rows and the others one (288 rows of 64 channels: 40.0 | 25.0, two parts 38.5 | 22.5);
//   from 4096 for 256, and four as long as that is no more than 1280 workgroups: unequal
//     lengths cost more than the join (8192, 256 rows: 1 part 188 | 120, 4 195 | 106, 512
//     rows 367 | 227, 2 parts 379 | 195; 32 rows: 8 parts 32.7 | 21.1, 32 36.0 | 26.3).
// The longest that a sequence may be is the width of its table: see the price of a table
// with room at launch_decode.
int decode_parts(int n_seqs, int n_heads, int n_kv, int64_t max_entries) {
  const int64_t rows = (int64_t)n_seqs * n_kv * ((n_heads / n_kv + 15) / 16);
  int64_t want = 256 / rows;
  if (max_entries <= 512 || (max_entries <= 1024 && rows >= 96)) want = 1;
  else if (max_entries >= 4096) want = std::max(want, std::min<int64_t>(4, 1280 / rows));
  else if (max_entries > 1024 && rows > 256 && rows < 512) want = 2;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, max_entries / 256), kMaxDecodeParts));
}

// The lengths lie on the device, so everything here goes by the table's width.  With 4 and 16
// times the width that the sequences need: 4 sequences of 300, 8 KV heads of 128: 7.9 us, then
// 9.5 and 10.4; 64 of 100 .. 300: 15.4, 15.3, 27.1; 16 of 1500 .. 2048, 12 heads of 64: 18.5,
// 22.1, 21.8; 2 of up to 32768: 48, 49, 47.  Selected pages: 8 of 2048, 26 pages of 16: 14.6,
// 16.3, 20.4; 4 of up to 32768, 64 pages of 64: 31, 38, 53 (the choice in a launch of its own).
hipError_t launch_decode(const PagedView& cache, const PagedTable& tab, DecodeArgs a, hipStream_t s) {
  const int64_t blocks =
      (int64_t)tab.n_seqs * cache.n_kv * ((a.n_heads / cache.n_kv + 15) / 16) * a.n_parts;
  // more workgroups than run at a time: the longest sequences' first, so that the last to
  // start are short (32 sequences of 100 .. 8192 entries, 8 KV heads: 118 -> 109 us; 64 equal
  // ones 188 -> 191; more than 64 are taken in their order, a wave has 64 lanes to know them)
  a.longest_first = blocks > 512 && tab.n_seqs <= 64 && !tab.per_head;
#define RK_DECODE(T, DH)                                                                                           \
  do {                                                                                                             \
    decode_kernel<T, DH, Sel::kNone><<<(uint32_t)blocks, 64 * kDecodeWaves, 0, s>>>(cache, tab, a, SelectArgs{});  \
    if (a.n_parts > 1)                                                                                             \
      decode_join_kernel<T, DH><<<tab.n_seqs * a.n_heads, 256, 0, s>>>(tab, a, cache.n_kv, cache.page_shift);      \
  } while (0)
  RK_PAGED_DISPATCH(cache.bf16, cache.head_dim, RK_DECODE);
#undef RK_DECODE
  return hipGetLastError();
}

// Bounds of a row up to which the attention's workgroups score the pages themselves: a CU
// reads them in less time than another launch takes.  8 sequences of 2048 in pages of 16,
// 12 heads of 64, 32 KB of bounds a row: 14.6 us, with the scores in a launch of their own
// 15.0; half as many pages 12.1 and 14.0; twice as many, 64 KB, 18.9 and 16.7.  Not where more
// than two parts of a row outnumber the places that 256 CUs have for them: 32 sequences of
// 16384 in pages of 256, 16 of them read, 8 KV heads of 128, 4 parts: 117 and 112.  Nor
// where more than 16 query heads share a KV head: they would be scored by several
// workgroups, one of which may have written its outputs over the queries that another
// still reads.
constexpr int64_t kScoreBytes = 1 << 15;

hipError_t launch_decode_selected(const PagedView& cache, const PagedTable& tab, const DecodeArgs& a,
                                  const SelectArgs& sel, hipStream_t s) {
  const int rows = tab.n_seqs * cache.n_kv, page_bytes = 2 * cache.head_dim * (cache.bf16 ? 2 : 4);
  PagedTable lists = tab;   // a row for each (sequence, KV head): its chosen pages
  lists.pages = sel.list; lists.lengths = sel.list_len; lists.stride = lists.max_pages = sel.n_select;
  lists.per_head = true;
  const bool held = tab.max_pages <= kWavePages && sel.n_select <= kWavePages;
  const int head_tiles = (a.n_heads / cache.n_kv + 15) / 16;
  const bool alone = held && head_tiles == 1 && (int64_t)tab.max_pages * page_bytes <= kScoreBytes &&
                     (a.n_parts <= 2 || (int64_t)rows * a.n_parts <= 512);
  if (!alone) {
    // a workgroup's threads four times over, split further while CUs are idle
    const int per_pass = kSelectThreads * 16 * 4 / page_bytes;
    const int chunks = std::max(1, std::min((tab.max_pages + per_pass - 1) / per_pass, std::max(1, 2048 / rows)));
#define RK_SCORES(T, DH) \
  page_scores_kernel<T, DH><<<(uint32_t)rows * chunks, kSelectThreads, 0, s>>>(cache, tab, sel, chunks)
    RK_PAGED_DISPATCH(cache.bf16, cache.head_dim, RK_SCORES);
#undef RK_SCORES
  }
  if (!held) {
    page_select_kernel<<<rows, kSelectThreads, 0, s>>>(cache, tab, sel);
    return launch_decode(cache, lists, a, s);
  }
  DecodeArgs d = a;
  d.longest_first = false;
  const uint32_t blocks = (uint32_t)((int64_t)rows * head_tiles * a.n_parts);
#define RK_DECODE(T, DH)                                                                                              \
  do {                                                                                                                \
    if (alone) decode_kernel<T, DH, Sel::kScores><<<blocks, 64 * kDecodeWaves, 0, s>>>(cache, tab, d, sel);           \
    else decode_kernel<T, DH, Sel::kKeys><<<blocks, 64 * kDecodeWaves, 0, s>>>(cache, tab, d, sel);                   \
    if (a.n_parts > 1)                                                                                                \
      decode_join_kernel<T, DH><<<tab.n_seqs * a.n_heads, 256, 0, s>>>(lists, d, cache.n_kv, cache.page_shift);       \
  } while (0)
  RK_PAGED_DISPATCH(cache.bf16, cache.head_dim, RK_DECODE);
#undef RK_DECODE
  return hipGetLastError();
}

}  // namespace rk
