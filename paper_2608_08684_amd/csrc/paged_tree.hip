// Attention of a tree of drafted tokens of each sequence over its paged cache.
#include <algorithm>
#include <type_traits>

#include "paged_tile.h"

namespace rk {

// Sequence i's m drafts are its last m entries, b .. b + m - 1, and draft j of query head h
//   o_j,h = sum_u softmax_u(scale q_j,h . k_u) v_u,  u < b, or u = b + t with bit t of mask_j.
// The m x H / H_kv query rows of a KV head are the columns of one pass over its cache: a
// workgroup of 4 waves takes 16 N of them and a part of the length, its waves the part's
// 32-entry tiles in turn, so that keys and values go from memory to registers once for all
// of the columns (N = 1, 2 or 4 by how many there are).  Column blocks of one part follow each
// other on the same XCD: the second finds the cache in its L2.
// A column keeps a reference R, the sum l of its weights e^(s - R) and its output.  R is
// moved only when a score has passed it by kRaise: the output's rescale, a multiplication of
// every accumulator, is then rare, and the accumulators stay where the matrix unit has them.
// bf16 and 8-bit caches: R is held times log2(e) and the weight's exponent is one fma of the
// score; what its rounding puts into a weight, 2^-24 of a score, is far below the output's
// bf16.  R also holds the power of two above the part's entries (the weights' sum stays below
// 1, and no weighted sum overflows).  Weights enter the second product as two bf16 numbers, 16
// bits and more, where a tile has several column blocks: the third of paged_attention's would
// cost as much again in the matrix unit and changes the output by 2^-17 of itself.
// A value that is infinite or NaN must not reach the columns whose mask leaves its draft out,
// but 0 times it would: in the tiles that hold drafts such values are taken out of the
// product, and added to the columns that see them by products of their own.
constexpr float kRaise = 8.f;            // of a score, natural units
constexpr float kUnset = -3.0e38f;       // R of a column that has seen nothing

template <typename T, typename C, int DH, int N>
__global__ __launch_bounds__(64 * kDecodeWaves) void tree_kernel(PagedView cache, PagedTable tab, SeqTable st,
                                                                 TreeArgs a) {
  using Tile = CacheTile<C, DH>;
  constexpr int NW = kDecodeWaves, SP = DH + 4, PIECES = N == 1 ? 3 : 2;
  constexpr bool kFp32 = std::is_same<T, float>::value;
  constexpr int AREA = Tile::LDS * NW > NW * 16 * SP * 4 ? Tile::LDS * NW : NW * 16 * SP * 4;
  __shared__ __attribute__((aligned(16))) char area[AREA];
  __shared__ float sm[NW][16], sl[NW][16];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = cache.n_kv, grp = a.n_heads / G;
  // an XCD's workgroups: the column blocks of one item, then those of the next.  item =
  // (rank of the sequence by falling length * G + KV head) * parts + part
  const int y = blockIdx.x >> 3, cb = y % a.col_blocks;
  int item = (y / a.col_blocks) * 8 + (blockIdx.x & 7);
  if (item >= st.n * G * a.n_parts) return;
  const int part = item % a.n_parts; item /= a.n_parts;
  const int hk = item % G, rank = item / G;
  const int mine = lane < st.n ? table_length(tab, lane, cache.page_shift) : -1;
  int before = 0;
  for (int j = 0; j < st.n; ++j) {
    const int other = __builtin_amdgcn_readlane(mine, j);
    before += other > mine || (other == mine && j < lane);
  }
  const int seq = __builtin_ctzll(__ballot(before == rank && lane < st.n));
  const int len = __builtin_amdgcn_readlane(mine, seq);
  const int row0 = st.off[seq], m = st.off[seq + 1] - row0, cols = m * grp, c0 = cb * 16 * N;
  if (c0 >= cols) return;
  const int base = (int)((uint32_t)tab.lengths[seq] - (uint32_t)m);
  const int per = part_entries(len, a.n_parts);
  const int start = part * per, end = min_i(len, start + per);
  if (part > 0 && start >= len) return;   // the joining kernel knows; part 0 of an empty sequence stays
  const int32_t* pages = tab.pages + (int64_t)seq * tab.stride;
  const int shift = cache.page_shift, in_mask = (1 << shift) - 1;
  const int64_t head_at = (int64_t)hk << shift, page_rows = (int64_t)G << shift;

  Tile tile;
  typename Tile::Query query[N];
  uint64_t word[N];
  const int col = lane & 15, g = lane >> 4;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int c = min_i(c0 + n * 16 + col, cols - 1), j = c / grp;
    Tile::load_q(query[n], (const T*)a.q + (int64_t)(row0 + j) * a.q_rs + (int64_t)(hk * grp + c - j * grp) * DH, lane);
    word[n] = a.masks ? a.masks[row0 + j] : (2ull << j) - 1;
  }
  f32x4_t o[N][Tile::ND];
  float R[N], l[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    R[n] = kUnset;
    l[n] = 0.f;
#pragma unroll
    for (int i = 0; i < Tile::ND; ++i) o[n][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  // the weights' unit: a power of two above the part's entries and e^kRaise
  const int bits = 32 - __builtin_clz(max_i(end - start, 1)) + 12;
  const float unit = __uint_as_float((uint32_t)(127 - bits) << 23);
  const float c2 = a.scale * kLog2e;
  struct Pages {
    int k0, p0, p1;
  };
  struct Where {
    int64_t r0, r1;     // rows of the cache at which the two halves begin
    uint32_t seen;      // entries that count
  };
  const int step = NW * kTile, first = start + w * kTile;
  const int last = first + (max_i(end - 1 - first, 0) / step) * step;
  const auto pages_of = [&](int k) {
    const int k0 = min_i(k, last);
    return Pages{k0, pages[k0 >> shift], pages[min_i(k0 + 16, end - 1) >> shift]};
  };
  const auto where = [&](Pages p) {
    const int p0 = __builtin_amdgcn_readfirstlane(p.p0), p1 = __builtin_amdgcn_readfirstlane(p.p1);
    const bool ok0 = p0 >= 0 && p0 < cache.n_pages, ok1 = p1 >= 0 && p1 < cache.n_pages;
    Where wh;
    wh.r0 = (ok0 ? p0 : 0) * page_rows + head_at + (p.k0 & in_mask);
    wh.r1 = (ok1 ? p1 : 0) * page_rows + head_at + ((p.k0 + 16) & in_mask);
    wh.seen = (ok0 ? 0xffffu : 0u) | (ok1 ? 0xffff0000u : 0u);
    if (end - p.k0 < 32) wh.seen &= (1u << (end - p.k0)) - 1u;
    return wh;
  };
  // loads run a tile ahead, their pages two, as in the attention of one token
  Where cur{}, nxt{};
  Pages ahead{};
  if (first < end) {
    cur = where(pages_of(first));
    tile.load_k(cache, cur.r0, cur.r1, lane);
    tile.load_v(cache, cur.r0, cur.r1, lane);
    nxt = where(pages_of(first + step));
    ahead = pages_of(first + 2 * step);
  }
  for (int k0 = first; k0 < end; k0 += step) {
    const Where was = cur;
    f32x4_t s[N][2];
    tile.template scores<N>(query, s);
    tile.load_k(cache, nxt.r0, nxt.r1, lane);
    if constexpr (kFp32) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t) s[n][t] *= a.scale;
    }
    bool poison = false;
    if (was.seen != 0xffffffffu) {
      tile.clear_values(was.seen, lane);
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(was.seen >> (t * 16 + 4 * g + i) & 1)) s[n][t][i] = -INFINITY;
    }
    if (k0 + 32 > base) {   // drafts among the entries
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int at = k0 + t * 16 + 4 * g - base;   // draft of the lane's first entry of this half
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d = at + i;
            if (d >= 0 && !(word[n] >> (d & 63) & 1)) s[n][t][i] = -INFINITY;
          }
      }
      poison = __ballot(tile.take_out(0)) != 0;
    }
    cur = nxt;
    if constexpr (Tile::kStaged) {
      tile.stage_v(area + w * Tile::LDS, lane);
      tile.load_v(cache, cur.r0, cur.r1, lane);
    }
    nxt = where(ahead);
    ahead = pages_of(k0 + 3 * step);
    // weights
    bool above = false;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float mx = s[n][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[n][i >> 2][i & 3]);
      above |= kFp32 ? mx > R[n] + kRaise : fmaf(mx, c2, -R[n]) > kRaise * kLog2e - (float)bits;
    }
    if (__ballot(above)) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float mx = s[n][0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[n][i >> 2][i & 3]);
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float to = fmaxf(R[n], kFp32 ? mx : fmaf(mx, c2, (float)bits));
        const float corr = kFp32 ? exp_diff(R[n] - to) : __builtin_amdgcn_exp2f(R[n] - to);
        R[n] = to;
        l[n] *= corr;
#pragma unroll
        for (int i = 0; i < Tile::ND; ++i) o[n][i] *= corr;
      }
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[n][t][i] = kFp32 ? exp_diff_exact(s[n][t][i] - R[n], unit)
                             : __builtin_amdgcn_exp2f(fmaf(s[n][t][i], c2, -R[n]));
          l[n] += s[n][t][i];
        }
    tile.template values<N, PIECES>(s, o, area + w * Tile::LDS, lane);
    if (poison) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[n][t][i] = s[n][t][i] > 0.f ? 3.3e38f : 0.f;   // times 2: an infinity
      for (int sign = 1; sign >= -1; sign -= 2) {
        Tile x;
        x.load_v(cache, was.r0, was.r1, lane);
        if (was.seen != 0xffffffffu) x.clear_values(was.seen, lane);
        x.take_out(sign);
        if constexpr (Tile::kStaged) x.stage_v(area + w * Tile::LDS, lane);
#pragma unroll
        for (int n = 0; n < N; ++n) {   // sums of their own: an infinity in o would swallow the other one
          f32x4_t add[1][Tile::ND];
#pragma unroll
          for (int i = 0; i < Tile::ND; ++i) add[0][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          x.template values<1, PIECES>(s + n, add, area + w * Tile::LDS, lane);
#pragma unroll
          for (int i = 0; i < Tile::ND; ++i) o[n][i] += add[0][i];
        }
      }
    }
    if constexpr (!Tile::kStaged) tile.load_v(cache, cur.r0, cur.r1, lane);
  }
  float* so = (float*)area;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (c0 + n * 16 >= cols) return;
    l[n] += __shfl_xor(l[n], 16, 64);
    l[n] += __shfl_xor(l[n], 32, 64);
    __syncthreads();   // the tiles, or the last columns' outputs, are done with
    if (g == 0) { sm[w][col] = R[n]; sl[w][col] = l[n]; }
#pragma unroll
    for (int i = 0; i < Tile::ND; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) so[(w * 16 + col) * SP + Tile::channel(i, g, e)] = o[n][i][e];
    __syncthreads();
    for (int i = tid; i < 16 * DH; i += 64 * NW) {
      const int cc = i / DH, x = i % DH, c = c0 + n * 16 + cc;
      if (c >= cols) break;
      float M = sm[0][cc];
#pragma unroll
      for (int q = 1; q < NW; ++q) M = fmaxf(M, sm[q][cc]);
      float L = 0.f, v = 0.f;
#pragma unroll
      for (int q = 0; q < NW; ++q) {
        const float f = kFp32 ? exp_diff(sm[q][cc] - M) : __builtin_amdgcn_exp2f(sm[q][cc] - M);
        L += sl[q][cc] * f;
        v += so[(q * 16 + cc) * SP + x] * f;
      }
      // nothing seen: 0, with a log-sum-exp of -inf (a NaN sum stays NaN)
      v = L == 0.f ? 0.f : v / L;
      const float lse = L == 0.f ? -INFINITY : kFp32 ? M + logf(L / unit) : fmaf(M, 0.6931471805599453f, logf(L));
      const int j = c / grp, h = hk * grp + c - j * grp;
      const int64_t at = (int64_t)(row0 + j) * a.n_heads + h;
      if (a.n_parts == 1) {
        Act<T>::store((T*)a.out + (int64_t)(row0 + j) * a.out_rs + (int64_t)h * DH + x, v);
        if (a.lse && x == 0) a.lse[at] = lse;
      } else {
        a.part_o[(at * a.n_parts + part) * DH + x] = v;
        if (x == 0) a.part_lse[at * a.n_parts + part] = lse;
      }
    }
  }
}

// Joins the parts of each (draft, query head): o = sum_p e^(lse_p - M) o_p / sum_p e^(lse_p - M).
// A group of DH / 4 threads for each, four channels a thread.
template <typename T, int DH>
__global__ __launch_bounds__(256) void tree_join_kernel(PagedTable tab, SeqTable st, TreeArgs a, int page_shift) {
  constexpr int W = DH / 4, NG = 256 / W;
  const int64_t at = (int64_t)blockIdx.x * NG + threadIdx.x / W;   // row * heads + head
  const int x = threadIdx.x % W * 4;
  if (at >= (int64_t)st.rows * a.n_heads) return;
  const int row = (int)(at / a.n_heads), h = (int)(at - (int64_t)row * a.n_heads);
  const int len = table_length(tab, seq_of_row(st, row), page_shift);
  const int per = part_entries(len, a.n_parts), n = max_i(1, (len + per - 1) / per);
  const float* lse = a.part_lse + at * a.n_parts;
  const float* po = a.part_o + at * a.n_parts * DH + x;
  float M = -INFINITY;
  for (int p = 0; p < n; ++p) M = fmaxf(M, lse[p]);
  const float ref = M == -INFINITY ? 0.f : M;
  float L = 0.f;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < n; ++p) {
    const float f = exp_diff(lse[p] - ref) * (1.0f / kMaxTreeParts);   // so that no sum of outputs overflows
    const f32x4_t u = *(const f32x4_t*)(po + (int64_t)p * DH);
    L += f;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(f, u[e], v[e]);
  }
  T* out = (T*)a.out + (int64_t)row * a.out_rs + (int64_t)h * DH + x;
#pragma unroll
  for (int e = 0; e < 4; ++e) Act<T>::store(out + e, L == 0.f ? 0.f : v[e] / L);
  if (a.lse && x == 0) a.lse[at] = L == 0.f ? -INFINITY : ref + logf(L * kMaxTreeParts);
}

// Column blocks of 16 of a workgroup, for the widest tree of a call.
int tree_width(const PagedView& cache, int max_drafts, int n_heads) {
  const int cols = max_drafts * (n_heads / cache.n_kv);
  return cols <= 16 ? 1 : cols <= 32 || !cache.bf16 ? 2 : 4;
}

// Parts of a length: enough for the CUs, none shorter than 512 entries.
int tree_parts(const PagedView& cache, int n_seqs, int max_drafts, int n_heads, int64_t max_entries) {
  const int width = 16 * tree_width(cache, max_drafts, n_heads), cols = max_drafts * (n_heads / cache.n_kv);
  const int64_t rows = (int64_t)n_seqs * cache.n_kv * ((cols + width - 1) / width);
  const int64_t want = 512 / std::max<int64_t>(rows, 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min(want, max_entries / 512), kMaxTreeParts));
}

int64_t tree_blocks(const PagedView& cache, const SeqTable& st, const TreeArgs& a) {
  const int64_t cols = (int64_t)st.max_len * (a.n_heads / cache.n_kv), width = 16 * tree_width(cache, st.max_len, a.n_heads);
  const int64_t items = (int64_t)st.n * cache.n_kv * a.n_parts;
  return (items + 7) / 8 * 8 * ((cols + width - 1) / width);
}

hipError_t launch_tree(const PagedView& cache, const PagedTable& tab, const SeqTable& st, TreeArgs a, hipStream_t s) {
  const int cols = st.max_len * (a.n_heads / cache.n_kv), N = tree_width(cache, st.max_len, a.n_heads);
  a.col_blocks = (cols + 16 * N - 1) / (16 * N);
  const uint32_t blocks = (uint32_t)tree_blocks(cache, st, a);
  const int64_t outs = (int64_t)st.rows * a.n_heads;
#define RK_TREE(T, C, DH)                                                                                     \
  do {                                                                                                        \
    constexpr int kWide = std::is_same<T, float>::value ? 2 : 4;                                              \
    if (N == 1) tree_kernel<T, C, DH, 1><<<blocks, 64 * kDecodeWaves, 0, s>>>(cache, tab, st, a);             \
    else if (N == 2) tree_kernel<T, C, DH, 2><<<blocks, 64 * kDecodeWaves, 0, s>>>(cache, tab, st, a);        \
    else tree_kernel<T, C, DH, kWide><<<blocks, 64 * kDecodeWaves, 0, s>>>(cache, tab, st, a);                \
    if (a.n_parts > 1) {                                                                                      \
      const int groups = 256 / (DH / 4);                                                                      \
      tree_join_kernel<T, DH><<<(uint32_t)((outs + groups - 1) / groups), 256, 0, s>>>(tab, st, a, cache.page_shift); \
    }                                                                                                         \
  } while (0)
  RK_PAGED_DISPATCH(cache, RK_TREE);
#undef RK_TREE
  return hipGetLastError();
}

}  // namespace rk
