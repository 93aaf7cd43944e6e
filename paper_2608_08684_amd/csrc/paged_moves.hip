// Entries out of the paged cache (read), to other places of their sequence (keep), and from
// sequence to sequence (reorder).  Copies: all are bound by memory, and below a few megabytes by
// the way from lengths to pages to entries.
#include <algorithm>
#include <type_traits>

#include "paged_tile.h"

namespace rk {
namespace {

// The cache's row of KV head 0 that entry e of sequence s is on, or -1; the rows of the other
// heads follow page_size apart.
__device__ __forceinline__ int64_t entry_row(const PagedView& cache, const PagedTable& tab, int s, int64_t e) {
  if (e < 0 || e >= (int64_t)tab.max_pages << cache.page_shift) return -1;
  const int page = tab.pages[(int64_t)s * tab.stride + (e >> cache.page_shift)];
  if (page < 0 || page >= cache.n_pages) return -1;
  return ((int64_t)page * cache.n_kv << cache.page_shift) + (e & ((1 << cache.page_shift) - 1));
}

// --------------------------------------------------------------------------- read
// A workgroup takes up to 16 rows, fewer while CUs are idle: where they lie, then their
// 16-byte pieces, keys first, U loads in flight a thread.  17928 8-bit rows of 8 heads of 128 to
// bf16: 25.7 us (110 MB, 4.3 TB/s); 64 rows 3.1 us, the way from lengths to pages to rows.  The same rows
// again and again, in part out of the cache: 22.2, bf16 ones 25.9 (147 MB), 12 heads of 64 in fp32 37.2
// (220 MB); 64 rows of either 2.8 and 3.0.
constexpr int kReadRows = 16, kMoveThreads = 256;

template <typename T, typename C, int DH>
__global__ __launch_bounds__(kMoveThreads) void read_kernel(PagedView cache, PagedTable tab, ReadArgs a, SeqTable st,
                                                            int rows_each) {
  constexpr int VE = 16 / sizeof(T), CPH = DH / VE, NT = kMoveThreads, U = 4;
  __shared__ int64_t at[kReadRows];
  const int tid = threadIdx.x, G = cache.n_kv;
  const int r0 = blockIdx.x * rows_each, n = min_i(rows_each, a.n_rows - r0);
  if (tid < n) {
    const int r = r0 + tid;
    const int s = a.one_row ? r : seq_of_row(st, r);
    const int64_t e = (int64_t)tab.lengths[s] - (a.one_row ? 1 : st.off[s + 1] - r);
    at[tid] = entry_row(cache, tab, s, e);
  }
  __syncthreads();
  const int per_row = G * CPH, each = n * per_row, total = each * ((a.k != nullptr) + (a.v != nullptr));
  constexpr bool kScaled = std::is_same<C, e4m3_t>::value;
  using Raw = std::conditional_t<kScaled, v2u, v4u>;
  for (int i0 = tid; i0 < total; i0 += U * NT) {
    Raw raw[U];
    uint32_t scale[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int i = min_i(i0 + u * NT, total - 1);
      const bool key = a.k && i < each;
      i -= i >= each ? each : 0;
      const int rr = i / per_row, c = i - rr * per_row;
      const int64_t row = at[rr] + ((int64_t)(c / CPH) << cache.page_shift);
      there[u] = at[rr] >= 0;
      const C* src = (const C*)(key ? cache.k : cache.v) + (there[u] ? row * DH : 0) + c % CPH * VE;
      raw[u] = *(const Raw*)src;
      if constexpr (kScaled) scale[u] = (key ? cache.k_scales : cache.v_scales)[there[u] ? row : 0];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int i = i0 + u * NT;
      if (i >= total) break;
      const bool key = a.k && i < each;
      i -= i >= each ? each : 0;
      const int rr = i / per_row, c = i - rr * per_row;
      v4u y;
      if constexpr (kScaled) y = e4m3_to_bf16(raw[u][0], raw[u][1], e4m3_scale(scale[u]));
      else y = raw[u];
      if (!there[u]) y = v4u{0, 0, 0, 0};
      T* dst = (T*)(key ? a.k : a.v) + (int64_t)(r0 + rr) * (key ? a.k_rs : a.v_rs) +
               (int64_t)(c / CPH) * (key ? a.k_hs : a.v_hs) + c % CPH * VE;
      *(v4u*)dst = y;
    }
  }
}

// --------------------------------------------------------------------------- keep
// A workgroup takes the path of one sequence and KV head, its keys or its values: all rows go
// to LDS before any is written, so a row's new place may be another's old one.  The keys'
// workgroup then forms the bounds of the pages, a channel a thread, in the order of the path.
// Bound: latency, lengths -> pages -> rows -> bounds: 4.7 us for 32 sequences of up to 26 drafts
// with bounds, 3.6 for 8 of 64 fp32 rows of 64 channels without.  A thread's loads hang on where its rows
// go, so each is waited for before the next: 8 x 63 fp32 rows of 128 channels, 8 loads a thread, 6.1 us.
template <typename T, typename C, int DH>
__global__ __launch_bounds__(kMoveThreads) void keep_kernel(PagedView cache, PagedTable tab, SeqTable st,
                                                            const int32_t* kept, int64_t kept_stride, int n_kept) {
  constexpr int CP = DH * sizeof(C) / 16, NT = kMoveThreads;
  constexpr bool kScaled = std::is_same<C, e4m3_t>::value;
  __shared__ v4u rows[RK_MAX_DRAFTS * CP];
  __shared__ uint8_t scales[RK_MAX_DRAFTS];
  __shared__ int64_t from[RK_MAX_DRAFTS], to[RK_MAX_DRAFTS];   // rows of the cache; to = -1: not moved
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63, G = cache.n_kv;
  const bool keys = blockIdx.x & 1;
  const int hk = (blockIdx.x >> 1) % G, seq = (blockIdx.x >> 1) / G;
  const int m = st.off[seq + 1] - st.off[seq];
  const int64_t base = (int64_t)tab.lengths[seq] - m;
  if (tid < 64) {
    const int t = lane < n_kept ? kept[(int64_t)seq * kept_stride + lane] : -1;
    const int prev = __shfl_up(t, 1, 64);
    const bool on = t >= 0 && t < m && (lane == 0 || t > prev);
    const uint64_t off = ~__ballot(on);
    const int n = off ? __builtin_ctzll(off) : 64;
    if (lane < n) {
      const int64_t f = entry_row(cache, tab, seq, base + t), d = entry_row(cache, tab, seq, base + lane);
      from[lane] = f + ((int64_t)hk << cache.page_shift);
      to[lane] = f < 0 || d < 0 ? -1 : d + ((int64_t)hk << cache.page_shift);
    }
    if (lane == 0) count = n;
  }
  __syncthreads();
  const int n = count;
  C* data = (C*)(keys ? cache.k : cache.v);
  uint8_t* scale = keys ? cache.k_scales : cache.v_scales;
#pragma unroll 4
  for (int i = tid; i < n * CP; i += NT)
    if (to[i / CP] >= 0) rows[i] = *(const v4u*)(data + from[i / CP] * DH + i % CP * (16 / sizeof(C)));
  if (kScaled && tid < n && to[tid] >= 0) scales[tid] = scale[from[tid]];
  __syncthreads();
  for (int i = tid; i < n * CP; i += NT)
    if (to[i / CP] >= 0 && to[i / CP] != from[i / CP]) *(v4u*)(data + to[i / CP] * DH + i % CP * (16 / sizeof(C))) = rows[i];
  if (kScaled && tid < n && to[tid] >= 0) scale[to[tid]] = scales[tid];
  if (!keys || !cache.bounds || tid >= DH) return;
  const int mask = (1 << cache.page_shift) - 1;
  float lo = INFINITY, hi = -INFINITY;
  bool fresh = false;
  int64_t row = -1;          // of the page: one that has been moved
  for (int j = 0; j < n; ++j) {
    const int64_t e = base + j;
    if (to[j] >= 0) {
      float x;
      if constexpr (kScaled)
        x = __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t*)rows)[j * DH + tid], 0) * e4m3_scale(scales[j]);
      else
        x = Act<T>::load((const T*)rows + j * DH + tid);
      lo = least(lo, x);
      hi = largest(hi, x);
      fresh |= (e & mask) == 0;
      row = to[j];
    }
    if ((e & mask) != mask && j + 1 < n) continue;   // the page goes on
    if (row >= 0) {
      T* b = (T*)cache.bounds + (row >> cache.page_shift) * 2 * DH + tid;
      if (!fresh) {
        lo = least(lo, Act<T>::load(b));
        hi = largest(hi, Act<T>::load(b + DH));
      }
      Act<T>::store(b, lo);
      Act<T>::store(b + DH, hi);
    }
    lo = INFINITY; hi = -INFINITY;
    fresh = false;
    row = -1;
  }
}

// --------------------------------------------------------------------------- reorder
// A thread takes one 16-byte place of the page in progress (keys, values, scales, bounds) and
// reads it from the pages of all of a group's parents before it writes any: the beams'
// pages may be each other's sources.  The table's workgroups do the same with its columns.
// Both read the table of before, so they share a launch unless the table is changed in place.
// 16 groups of 8 beams, 52 entries of 8 KV heads of 128 in the page: up to 54 MB, 14.8 us; 4 beams,
// 12 heads of 64: 3.7.  Bound: a thread's loads hang on there being a copy, and for up to 8 beams each is
// waited for before the next (beyond, they go out together); 5 .. 8 beams take 240 registers, two
// waves to a SIMD.
template <typename T, typename C, int DH, int NB>
__global__ __launch_bounds__(kMoveThreads) void reorder_kernel(PagedView cache, PagedTable tab, ReorderArgs a,
                                                               int chunks, int table_chunks) {
  constexpr int CP = DH * sizeof(C) / 16, BP = 2 * DH * sizeof(T) / 16;
  constexpr bool kScaled = std::is_same<C, e4m3_t>::value;
  __shared__ int from[NB], src[NB], dst[NB];
  const int tid = threadIdx.x, G = cache.n_kv, nb = a.n_beams, shift = cache.page_shift;
  const int each = G * chunks + table_chunks, group = blockIdx.x / each, block = blockIdx.x - group * each;
  const int seq0 = group * nb;
  const int64_t entries = max_i(0, (int)min((int64_t)tab.lengths[seq0], (int64_t)tab.max_pages << shift));
  const int full = (int)(entries >> shift), rest = (int)(entries & ((1 << shift) - 1));
  if (tid < nb) {
    const int p = a.parents[seq0 + tid], f = p >= 0 && p < nb ? p : tid;
    from[tid] = f;
    int s = -1, d = -1;
    if (rest && f != tid) {
      s = tab.pages[(int64_t)(seq0 + f) * tab.stride + full];
      d = tab.pages[(int64_t)(seq0 + tid) * tab.stride + full];
    }
    const bool there = s >= 0 && s < cache.n_pages && d >= 0 && d < cache.n_pages;
    src[tid] = there ? s : -1;
    dst[tid] = there ? d : -1;
  }
  __syncthreads();
  if (block >= G * chunks) {
    const int x = (block - G * chunks) * kMoveThreads + tid;
    if (x >= tab.max_pages) return;
    int32_t page[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
      if (b < nb) page[b] = tab.pages[(int64_t)(seq0 + (x < full ? from[b] : b)) * tab.stride + x];
#pragma unroll
    for (int b = 0; b < NB; ++b)
      if (b < nb) a.pages_out[(int64_t)(seq0 + b) * a.out_stride + x] = page[b];
    return;
  }
  if (rest == 0) return;
  const int hk = block / chunks;
  int i = (block - hk * chunks) * kMoveThreads + tid;
  // keys, values, their scales, the bounds, one after the other
  const int scale_pieces = kScaled ? (rest + 15) / 16 : 0;
  char* data = (char*)cache.k;
  int64_t head_bytes = (int64_t)(DH * sizeof(C)) << shift;
  if (i >= rest * CP) {
    i -= rest * CP;
    data = (char*)cache.v;
    if (i >= rest * CP) {
      i -= rest * CP;
      data = (char*)cache.k_scales;
      head_bytes = (int64_t)1 << shift;
      if (i >= scale_pieces) {
        i -= scale_pieces;
        data = (char*)cache.v_scales;
        if (i >= scale_pieces) {
          i -= scale_pieces;
          data = (char*)cache.bounds;
          head_bytes = 2 * DH * sizeof(T);
          if (!data || i >= BP) return;
        }
      }
    }
  }
  data += hk * head_bytes + (int64_t)i * 16;
  const int64_t page_bytes = G * head_bytes;
  v4u piece[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b)
    if (b < nb && src[b] >= 0) piece[b] = *(const v4u*)(data + src[b] * page_bytes);
#pragma unroll
  for (int b = 0; b < NB; ++b)
    if (b < nb && src[b] >= 0) *(v4u*)(data + dst[b] * page_bytes) = piece[b];
}

}  // namespace

int64_t read_blocks(int n_rows) {
  const int rows_each = std::max(1, std::min(kReadRows, n_rows / 512));
  return ((int64_t)n_rows + rows_each - 1) / rows_each;
}

hipError_t launch_read(const PagedView& cache, const PagedTable& tab, const ReadArgs& a, const SeqTable& st,
                       hipStream_t s) {
  if (a.n_rows <= 0 || (!a.k && !a.v)) return hipSuccess;
  const int rows_each = std::max(1, std::min(kReadRows, a.n_rows / 512));
  const uint32_t blocks = (uint32_t)read_blocks(a.n_rows);
#define RK_READ(T, C, DH) read_kernel<T, C, DH><<<blocks, kMoveThreads, 0, s>>>(cache, tab, a, st, rows_each)
  RK_PAGED_DISPATCH(cache, RK_READ);
#undef RK_READ
  return hipGetLastError();
}

hipError_t launch_keep(const PagedView& cache, const PagedTable& tab, const SeqTable& st, const int32_t* kept,
                       int64_t kept_stride, int n_kept, hipStream_t s) {
  const uint32_t blocks = (uint32_t)st.n * cache.n_kv * 2;
#define RK_KEEP(T, C, DH) \
  keep_kernel<T, C, DH><<<blocks, kMoveThreads, 0, s>>>(cache, tab, st, kept, kept_stride, n_kept)
  RK_PAGED_DISPATCH(cache, RK_KEEP);
#undef RK_KEEP
  return hipGetLastError();
}

// Workgroups of a group: of its entries and of its table.
static void reorder_chunks(const PagedView& cache, int max_pages, int* chunks, int* table_chunks) {
  const int ps = 1 << cache.page_shift, es = cache.e4m3 ? 1 : cache.bf16 ? 2 : 4;
  // the page in progress has at least one free entry
  const int pieces = 2 * (ps - 1) * cache.head_dim * es / 16 + (cache.e4m3 ? 2 * ((ps + 14) / 16) : 0) +
                     (cache.bounds ? 2 * cache.head_dim * (cache.bf16 ? 2 : 4) / 16 : 0);
  *chunks = (pieces + kMoveThreads - 1) / kMoveThreads;
  *table_chunks = (max_pages + kMoveThreads - 1) / kMoveThreads;
}

int64_t reorder_blocks(const PagedView& cache, int n_seqs, int n_beams, int max_pages) {
  int chunks, table_chunks;
  reorder_chunks(cache, max_pages, &chunks, &table_chunks);
  return (int64_t)(n_seqs / n_beams) * ((int64_t)cache.n_kv * chunks + table_chunks);
}

hipError_t launch_reorder(const PagedView& cache, const PagedTable& tab, const ReorderArgs& a, hipStream_t s) {
  int chunks, table_chunks;
  reorder_chunks(cache, tab.max_pages, &chunks, &table_chunks);
  const int groups = tab.n_seqs / a.n_beams;
  const bool in_place = a.pages_out == tab.pages;
#define RK_REORDER_AS(T, C, DH, NB)                                                                                   \
  do {                                                                                                                \
    const int with = a.pages_out && !in_place ? table_chunks : 0;                                                     \
    reorder_kernel<T, C, DH, NB><<<(uint32_t)groups * (cache.n_kv * chunks + with), kMoveThreads, 0, s>>>(            \
        cache, tab, a, chunks, with);                                                                                 \
    if (in_place)                                                                                                     \
      reorder_kernel<T, C, DH, NB><<<(uint32_t)groups * table_chunks, kMoveThreads, 0, s>>>(cache, tab, a, 0, table_chunks); \
  } while (0)
#define RK_REORDER(T, C, DH)                              \
  do {                                                    \
    if (a.n_beams <= 4) RK_REORDER_AS(T, C, DH, 4);       \
    else if (a.n_beams <= 8) RK_REORDER_AS(T, C, DH, 8);  \
    else if (a.n_beams <= 16) RK_REORDER_AS(T, C, DH, 16); \
    else RK_REORDER_AS(T, C, DH, RK_MAX_BEAMS);           \
  } while (0)
  RK_PAGED_DISPATCH(cache, RK_REORDER);
#undef RK_REORDER
#undef RK_REORDER_AS
  return hipGetLastError();
}

}  // namespace rk
