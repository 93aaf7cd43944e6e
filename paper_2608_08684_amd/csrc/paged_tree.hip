// Attention of a tree of drafted tokens of each sequence over its paged cache.
//
// Sequence i's m drafts are its last m entries, b .. b + m - 1, and draft j of query head h
//   o_j,h = sum_u softmax_u(scale q_j,h . k_u) v_u,  u < b, or u = b + t with bit t of mask_j.
// The m x H / H_kv query rows of a KV head are the columns of one pass over its cache, so that
// an entry is read once for 16 .. 128 of them.  Two kernels (width_of chooses):
//   16 columns a workgroup: its waves take the tiles of its part of the length in turn, as in
//     the attention of one token (tree_narrow_kernel);
//   up to 128: all waves go through the same tiles, which LDS holds for them, each with columns
//     of its own (tree_wide_kernel).
//
// A column keeps a reference R, the sum l of its weights e^(s - R) and its output.  R is
// moved only when a score has passed it by kRaise: the output's rescale, a multiplication of
// every accumulator, is then rare.  The other columns of the wave go through it with a factor of
// 1, so that no bit of a row hangs on what other rows see.  bf16 and 8-bit caches: R is held times
// log2(e) and a weight's exponent is one fma of the score; what its rounding puts into a weight,
// 2^-24 of a score, is far below the output's bf16.  R also holds the power of two above the part's
// entries (the weights' sum stays below 1, and no weighted sum overflows).
//
// A value that is infinite or NaN must not reach the columns whose mask leaves its draft out,
// but 0 times it would: in the tiles that hold drafts such values are taken out of the
// product, and added afterwards to the columns that see them, by products of their own.
#include <algorithm>
#include <type_traits>

#include "paged_tile.h"

namespace rk {
namespace {

constexpr float kRaise = 8.f;            // of a score, natural units
constexpr float kUnset = -3.0e38f;       // R of a column that has seen nothing
constexpr float kHuge = 3.3e38f;         // the weight that makes an infinity of 2
constexpr uint32_t kHugeBits = 0x7f78u;  // and in bf16

// A workgroup's share: item = (rank of the sequence by falling length * parts + part) * G + KV
// head, and a column block of it.  The column blocks of an item follow each other on the same
// XCD, so that the second finds the cache in its L2; the longest sequences come first, so that
// the last to start are short; and neighbours are heads, which have the same to do, not parts,
// of which short sequences have fewer (they would leave every other XCD idle).
struct Share {
  int seq, hk, part, parts, cb, len, row0, m, base, start, end;   // parts: of this sequence
  bool none;
  __device__ __forceinline__ Share(const PagedView& cache, const PagedTable& tab, const SeqTable& st, const TreeArgs& a,
                                   int lane, int width) {
    const int G = cache.n_kv, y = blockIdx.x >> 3;
    cb = y % a.col_blocks;
    int item = (y / a.col_blocks) * 8 + (blockIdx.x & 7);
    none = item >= st.n * G * a.n_parts;
    if (none) return;
    hk = item % G; item /= G;
    part = item % a.n_parts;
    const int rank = item / a.n_parts;
    const int mine = lane < st.n ? table_length(tab, lane, cache.page_shift) : -1;
    int before = 0;
    for (int j = 0; j < st.n; ++j) {
      const int other = __builtin_amdgcn_readlane(mine, j);
      before += other > mine || (other == mine && j < lane);
    }
    seq = __builtin_ctzll(__ballot(before == rank && lane < st.n));
    len = __builtin_amdgcn_readlane(mine, seq);
    row0 = st.off[seq];
    m = st.off[seq + 1] - row0;
    base = (int)((uint32_t)tab.lengths[seq] - (uint32_t)m);
    const int per = part_entries(len, a.n_parts);
    start = part * per;
    end = min_i(len, start + per);
    parts = max_i(1, (len + per - 1) / per);
    // without columns; or a part past the end, which the joining kernel knows of (part 0 of an
    // empty sequence stays)
    none = cb * width >= m * (a.n_heads / G) || (part > 0 && start >= len);
  }
};

// A bit for each of 32 entries that a column sees: the text's, then by its mask.  first: the first one's
// number among the drafts (negative: text).
__device__ __forceinline__ uint32_t sees(uint64_t word, int first) {
  if (first >= 0) return (uint32_t)(word >> (first & 63));
  return first <= -32 ? ~0u : (uint32_t)word << -first | ((1u << -first) - 1u);
}

// --------------------------------------------------------------------------- few columns
// As the attention of one token, with a draft's mask for each column.  Weights in three bf16 pieces.
// Bound: memory where entries are many (2 sequences of 8192, 16 columns of 128: 23.6 us), else the
// latency of lengths -> pages -> tiles -> join through LDS (one fp32 sequence of 257, 5 drafts, three
// rounds of tiles: 9.7 us).
template <typename T, typename C, int DH>
__global__ __launch_bounds__(64 * kDecodeWaves) void tree_narrow_kernel(PagedView cache, PagedTable tab, SeqTable st,
                                                                        TreeArgs a) {
  using Tile = CacheTile<C, DH>;
  constexpr int NW = kDecodeWaves, SP = DH + 4;
  constexpr bool kFp32 = std::is_same<T, float>::value;
  constexpr int AREA = Tile::LDS * NW > NW * 16 * SP * 4 ? Tile::LDS * NW : NW * 16 * SP * 4;
  __shared__ __attribute__((aligned(16))) char area[AREA];
  __shared__ float sm[NW][16], sl[NW][16];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Share sh(cache, tab, st, a, lane, 16);
  if (sh.none) return;
  const int G = cache.n_kv, grp = a.n_heads / G, cols = sh.m * grp, c0 = sh.cb * 16;
  const int start = sh.start, end = sh.end, base = sh.base;
  const int32_t* pages = tab.pages + (int64_t)sh.seq * tab.stride;
  const int shift = cache.page_shift, in_mask = (1 << shift) - 1;
  const int64_t head_at = (int64_t)sh.hk << shift, page_rows = (int64_t)G << shift;

  Tile tile;
  typename Tile::Query query;
  const int col = lane & 15, g = lane >> 4;
  const int mine = min_i(c0 + col, cols - 1), row = mine / grp;   // this lane's column and draft
  Tile::load_q(query, (const T*)a.q + (int64_t)(sh.row0 + row) * a.q_rs + (int64_t)(sh.hk * grp + mine - row * grp) * DH,
               lane);
  const uint64_t word = a.masks ? a.masks[sh.row0 + row] : (2ull << row) - 1;
  f32x4_t o[Tile::ND];
#pragma unroll
  for (int i = 0; i < Tile::ND; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float R = kUnset, l = 0.f;
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
  // scores of what is not seen, or by the mask not seen by the column, are -inf
  const auto hide = [&](f32x4_t* s, int k0, uint32_t seen) {
    const uint32_t on = (seen & sees(word, k0 - base)) >> 4 * g;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = on >> (t * 16 + i) & 1 ? s[t][i] : -INFINITY;
  };
  const auto weight = [&](float s) {
    return kFp32 ? exp_diff_exact(s * a.scale - R, unit) : __builtin_amdgcn_exp2f(fmaf(s, c2, -R));
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
  bool poison = false;
  for (int k0 = first; k0 < end; k0 += step) {
    const uint32_t seen = cur.seen;
    f32x4_t s[2];
    tile.scores(query, s);
    tile.load_k(cache, nxt.r0, nxt.r1, lane);
    if (seen != 0xffffffffu) tile.clear_values(seen, lane);
    if (seen != 0xffffffffu || k0 + 32 > base) hide(s, k0, seen);
    if (k0 + 32 > base) poison |= tile.take_out_values(0);   // drafts among the entries
    cur = nxt;
    if constexpr (Tile::kStaged) {
      tile.stage_v(area + w * Tile::LDS, lane);
      tile.load_v(cache, cur.r0, cur.r1, lane);
    }
    nxt = where(ahead);
    ahead = pages_of(k0 + 3 * step);
    float mx = s[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i >> 2][i & 3]);
    const auto above = [&](float x) {
      return kFp32 ? x * a.scale > R + kRaise : fmaf(x, c2, -R) > kRaise * kLog2e - (float)bits;
    };
    if (__ballot(above(mx))) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float to = above(mx) ? (kFp32 ? mx * a.scale : fmaf(mx, c2, (float)bits)) : R;
      const float corr = kFp32 ? exp_diff(R - to) : __builtin_amdgcn_exp2f(R - to);
      R = to;
      l *= corr;
#pragma unroll
      for (int i = 0; i < Tile::ND; ++i) o[i] *= corr;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[t][i] = weight(s[t][i]);
        l += s[t][i];
      }
    tile.values(s, o, area + w * Tile::LDS, lane);
    if constexpr (!Tile::kStaged) tile.load_v(cache, cur.r0, cur.r1, lane);
  }
  if (__ballot(poison)) {
    for (int k0 = first; k0 < end; k0 += step) {
      if (k0 + 32 <= base) continue;
      const Where wh = where(pages_of(k0));
      tile.load_k(cache, wh.r0, wh.r1, lane);
      f32x4_t s[2];
      tile.scores(query, s);
      hide(s, k0, wh.seen);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][i] = weight(s[t][i]) > 0.f ? kHuge : 0.f;
#pragma unroll 1
      for (int sign = 1; sign >= -1; sign -= 2) {
        tile.load_v(cache, wh.r0, wh.r1, lane);
        tile.clear_values(wh.seen, lane);
        tile.take_out_values(sign);
        if constexpr (Tile::kStaged) tile.stage_v(area + w * Tile::LDS, lane);
        f32x4_t sum[Tile::ND];   // of their own: an infinity in o would swallow the other one
#pragma unroll
        for (int i = 0; i < Tile::ND; ++i) sum[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        tile.values(s, sum, area + w * Tile::LDS, lane);
#pragma unroll
        for (int i = 0; i < Tile::ND; ++i) o[i] += sum[i];
      }
    }
  }
  float* so = (float*)area;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  __syncthreads();   // the tiles are done with: their area takes the waves' outputs
  if (g == 0) { sm[w][col] = R; sl[w][col] = l; }
#pragma unroll
  for (int i = 0; i < Tile::ND; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) so[(w * 16 + col) * SP + Tile::channel(i, g, e)] = o[i][e];
  __syncthreads();
  for (int i = tid; i < 16 * DH; i += 64 * NW) {
    const int cc = i / DH, x = i % DH, c = c0 + cc;
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
    const int j = c / grp, h = sh.hk * grp + c - j * grp;
    const int64_t at = (int64_t)(sh.row0 + j) * a.n_heads + h;
    if (sh.parts == 1) {
      Act<T>::store((T*)a.out + (int64_t)(sh.row0 + j) * a.out_rs + (int64_t)h * DH + x, v);
      if (a.lse && x == 0) a.lse[at] = lse;
    } else {
      a.part_o[(at * a.n_parts + sh.part) * DH + x] = v;
      if (x == 0) a.part_lse[at * a.n_parts + sh.part] = lse;
    }
  }
}

// --------------------------------------------------------------------------- many columns
// A workgroup's tile of 64 entries in LDS as bf16, K and V, 8-bit rows widened on the way.  Each
// thread brings the same pieces of every tile; the 16 entries of a granule lie on one page, and a
// wave's i-th piece lies in one granule.
template <typename C, int DH> struct WideTile {
  static constexpr int ROWS = 64, NT = 64 * kDecodeWaves;
  static constexpr int CH = DH / 8;                         // 16-byte pieces of a row in LDS
  static constexpr int PB = DH * (int)sizeof(C) / 16;       // and of the cache
  static constexpr int NP = ROWS * PB / NT;                 // pieces of a thread
  static constexpr int BYTES = ROWS * DH * 2;               // of K, and of V
  static constexpr bool kScaled = std::is_same<C, e4m3_t>::value;
  v4u k[NP], v[NP];
  uint32_t ks[kScaled ? NP : 1], vs[kScaled ? NP : 1];

  static __device__ __forceinline__ int row_of(int i, int tid) { return (i * NT + tid) / PB; }
  static __device__ __forceinline__ int granule(int i, int w) { return (i * NT + w * 64) / PB / 16; }
  static __device__ __forceinline__ int k_swz(int row) { return DH == 128 ? row & 15 : (row >> 1) & 7; }

  // at[i]: the cache's row at which granule(i, w) begins
  __device__ __forceinline__ void load(const PagedView& cache, const int64_t* at, int tid) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int in = row_of(i, tid) & 15, piece = tid % PB;
      const uint32_t off = (uint32_t)(in * PB + piece) * 16;
      k[i] = *(const v4u*)((const char*)cache.k + at[i] * (PB * 16) + off);
      v[i] = *(const v4u*)((const char*)cache.v + at[i] * (PB * 16) + off);
      if constexpr (kScaled) {
        ks[i] = (cache.k_scales + at[i])[in];
        vs[i] = (cache.v_scales + at[i])[in];
      }
    }
  }
  __device__ __forceinline__ void clear_values(uint64_t seen, int tid) {
#pragma unroll
    for (int i = 0; i < NP; ++i)
      if (!(seen >> row_of(i, tid) & 1)) {
        v[i] = v4u{0, 0, 0, 0};
        if constexpr (kScaled) vs[i] = 127;
      }
  }
  __device__ __forceinline__ bool take_out_values(int sign) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if constexpr (kScaled) {
        any |= take_out<C>(v[i], sign, vs[i]);
        if (sign != 0) vs[i] = 127;
      } else {
        any |= take_out<C>(v[i], sign);
      }
    }
    return any;
  }
  __device__ __forceinline__ void store(char* lds, int tid) const {
    char *lk = lds, *lv = lds + BYTES;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int row = row_of(i, tid), piece = tid % PB;
      const int kx = k_swz(row), vx = StagedValues<DH>::swz(row);
      if constexpr (kScaled) {
        const float sk = e4m3_scale(ks[i]), sv = e4m3_scale(vs[i]);
        *(v4u*)(lk + (row * CH + ((2 * piece) ^ kx)) * 16) = e4m3_to_bf16(k[i][0], k[i][1], sk);
        *(v4u*)(lk + (row * CH + ((2 * piece + 1) ^ kx)) * 16) = e4m3_to_bf16(k[i][2], k[i][3], sk);
        *(v4u*)(lv + (row * CH + ((2 * piece) ^ vx)) * 16) = e4m3_to_bf16(v[i][0], v[i][1], sv);
        *(v4u*)(lv + (row * CH + ((2 * piece + 1) ^ vx)) * 16) = e4m3_to_bf16(v[i][2], v[i][3], sv);
      } else {
        *(v4u*)(lk + (row * CH + (piece ^ kx)) * 16) = k[i];
        *(v4u*)(lv + (row * CH + (piece ^ vx)) * 16) = v[i];
      }
    }
  }
};

// A wave has 16 N columns.  For each 32 entries it forms the weights of the scores (vector unit)
// and then multiplies them with the values, and the next 32 entries' keys with its queries
// (matrix unit).  The waves read all of K and V from LDS; 32 columns a wave keep that below what
// the products take.
// Weights enter the product in two bf16 pieces: what is left out, at most 2^-16 of a weight, is
// 2^-8 of the output's own rounding.  One piece (2^-8 of a weight) took 117 us where two took 135,
// with outputs off by up to 1.4 times as much.
// Bound: issue.  The vector unit is busy 54% of the cycles (a fifth of that are the matrix
// instructions' own) and the matrix unit 40%, and they go together badly: a wave's 32 matrix
// instructions beside another's 128 fmas take 0.67 of the sum of both, two waves that do both in turn
// 0.8 - 0.86.  256 registers leave two waves to a SIMD.  16 sequences of 100 .. 8192 in e4m3, 64
// drafts of 32 query heads of 128 over 8 KV heads: 110 us and 13.7 of the join (0.53 PFLOP/s of the
// formula's products in 124); 8 of 500 .. 4096 in bf16, up to 26 drafts: 28.5 and 5.9.  (Of calls one
// after the other; the first twenty after a pause take 134 and 31.)  Trials, with what stood then
// beside them: the waves' priority in the matrix part 167 -> 154.  Not taken: 8 waves in two groups
// that alternate between the units (157 where 150 stood), vector and matrix instructions mixed by
// the schedule (154 -> 280, registers spill), one block of 16 columns a wave for all (179), keys half
// a tile ahead of the values for one barrier a tile instead of two (147 -> 152), another priority for
// every second wave (146 -> 153 .. 158).
template <typename C, int DH, int N>
__global__ __launch_bounds__(64 * kDecodeWaves, 2) void tree_wide_kernel(PagedView cache, PagedTable tab, SeqTable st,
                                                                         TreeArgs a) {
  using Tile = WideTile<C, DH>;
  using Values = StagedValues<DH>;
  constexpr int NW = kDecodeWaves, ND = DH / 16, NC = DH / 32, CH = DH / 8, ROWS = Tile::ROWS;
  __shared__ __attribute__((aligned(16))) char area[2][2 * Tile::BYTES];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Share sh(cache, tab, st, a, lane, 16 * N * NW);
  if (sh.none) return;
  const int G = cache.n_kv, grp = a.n_heads / G, cols = sh.m * grp, c0 = (sh.cb * NW + w) * 16 * N;
  const int start = sh.start, end = sh.end, base = sh.base;
  const int32_t* pages = tab.pages + (int64_t)sh.seq * tab.stride;
  const int shift = cache.page_shift, in_mask = (1 << shift) - 1;
  const int64_t head_at = (int64_t)sh.hk << shift, page_rows = (int64_t)G << shift;
  const bool busy = c0 < cols;   // the other waves only bring their pieces
  const int col = lane & 15, g = lane >> 4;

  v4u query[N][NC];
  uint64_t word[N];
  f32x4_t o[N][ND];
  float R[N], l[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int c = min_i(c0 + n * 16 + col, cols - 1), j = c / grp;
    const bf16_t* q = (const bf16_t*)a.q + (int64_t)(sh.row0 + j) * a.q_rs + (int64_t)(sh.hk * grp + c - j * grp) * DH;
#pragma unroll
    for (int x = 0; x < NC; ++x) query[n][x] = *(const v4u*)(q + x * 32 + g * 8);
    word[n] = a.masks ? a.masks[sh.row0 + j] : (2ull << j) - 1;
    R[n] = kUnset;
    l[n] = 0.f;
#pragma unroll
    for (int i = 0; i < ND; ++i) o[n][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int bits = 32 - __builtin_clz(max_i(end - start, 1)) + 12;
  const float c2 = a.scale * kLog2e;
  // the pages of a tile's granules, one in each of lanes 0 .. 3 (past the end: the last one's)
  const auto pages_of = [&](int k0) { return pages[min_i(k0 + 16 * (lane & 3), end - 1) >> shift]; };
  const auto seen_of = [&](int page, int k0) {
    const uint64_t b = __ballot(page >= 0 && page < cache.n_pages);
    uint64_t seen = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) seen |= (b >> j & 1 ? 0xffffull : 0ull) << (16 * j);
    return end - k0 < 64 ? seen & ((1ull << (end - k0)) - 1) : seen;
  };
  const auto rows_of = [&](int page, int k0, int64_t* at) {
#pragma unroll
    for (int i = 0; i < Tile::NP; ++i) {
      const int gr = Tile::granule(i, w), p = __builtin_amdgcn_readlane(page, gr);
      at[i] = (p >= 0 && p < cache.n_pages ? p : 0) * page_rows + head_at + ((k0 + 16 * gr) & in_mask);
    }
  };
  // scores of 32 entries, rows `first` .. of the tile in LDS
  const auto scores = [&](f32x4_t (*s)[2], const char* lds, int first) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = first + t * 16 + col;
#pragma unroll
      for (int n = 0; n < N; ++n) s[n][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < NC; ++x) {
        const v4u key = *(const v4u*)(lds + (row * CH + ((x * 4 + g) ^ Tile::k_swz(row))) * 16);
#pragma unroll
        for (int n = 0; n < N; ++n)
          s[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, key),
                                                            __builtin_bit_cast(bf16x8_t, query[n][x]), s[n][t], 0, 0, 0);
      }
    }
  };
  // .. of entries k0 .. of which `seen` count
  const auto hide = [&](f32x4_t (*s)[2], int k0, uint32_t seen) {
    if (seen == 0xffffffffu && k0 + 32 <= base) return;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint32_t on = (seen & sees(word[n], k0 - base)) >> 4 * g;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][t][i] = on >> (t * 16 + i) & 1 ? s[n][t][i] : -INFINITY;
    }
  };
  const auto raise = [&](const f32x4_t (*s)[2]) {
    const auto above = [&](float x, int n) { return fmaf(x, c2, -R[n]) > kRaise * kLog2e - (float)bits; };
    float mx[N];
    bool any = false;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      mx[n] = s[n][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx[n] = fmaxf(mx[n], s[n][i >> 2][i & 3]);
      any |= above(mx[n], n);
    }
    if (!__ballot(any)) return;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float x = fmaxf(mx[n], __shfl_xor(mx[n], 16, 64));
      x = fmaxf(x, __shfl_xor(x, 32, 64));
      const float to = above(x, n) ? fmaf(x, c2, (float)bits) : R[n];
      const float corr = __builtin_amdgcn_exp2f(R[n] - to);
      R[n] = to;
      l[n] *= corr;
#pragma unroll
      for (int i = 0; i < ND; ++i) o[n][i] *= corr;
    }
  };
  const auto weights = [&](f32x4_t (*s)[2], v4u (*part)[2]) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[n][t][i] = __builtin_amdgcn_exp2f(fmaf(s[n][t][i], c2, -R[n]));
          l[n] += s[n][t][i];
        }
#pragma unroll
    for (int n = 0; n < N; ++n) Values::template pieces<2>(s[n], part[n]);
  };
  Tile tile;
  bool poison = false;
  const auto bring = [&](char* lds, int k0, uint64_t seen, int sign) {   // the tile's registers to LDS
    if (seen != ~0ull) tile.clear_values(seen, tid);
    if (k0 + ROWS > base) poison |= tile.take_out_values(sign);
    tile.store(lds, tid);
  };
  int64_t at[Tile::NP];
  uint64_t seen = 0, seen_next = 0;
  int ahead = 0;
  if (start < end) {
    const int page = pages_of(start);
    seen = seen_of(page, start);
    rows_of(page, start, at);
    tile.load(cache, at, tid);
    ahead = pages_of(start + ROWS);
    bring(area[0], start, seen, 0);
  }
  // the queries have arrived: left to the loop, the wait for them would be one for the next
  // tile's loads, in every turn
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int x = 0; x < NC; ++x) asm volatile("" : "+v"(query[n][x]));
  __syncthreads();
  f32x4_t s[N][2];      // scores of 32 entries
  v4u part[N][2];       // their weights
  if (busy && start < end) scores(s, area[0], 0);
  int buf = 0;
  // half 0 or 1 of the tile in area[buf]
  const auto weigh = [&](int k0, int half) {
    hide(s, k0 + 32 * half, (uint32_t)(seen >> 32 * half));
    raise(s);
    weights(s, part);
  };
  const auto load_next = [&](int k0) {    // the tile at k0 to registers, if there is one
    if (k0 >= end) return;
    seen_next = seen_of(ahead, k0);
    rows_of(ahead, k0, at);
    tile.load(cache, at, tid);
    ahead = pages_of(k0 + ROWS);
  };
  load_next(start + ROWS);
  for (int k0 = start; k0 < end; k0 += ROWS, buf ^= 1) {
    const bool more = k0 + ROWS < end;
    const char* values = area[buf] + Tile::BYTES;
    if (busy) {
      weigh(k0, 0);
      __builtin_amdgcn_s_setprio(1);
      scores(s, area[buf], 32);
      Values::template add<N, 2>(part, o, values, lane);
      __builtin_amdgcn_s_setprio(0);
    }
    const uint64_t then = seen_next;
    if (more) bring(area[buf ^ 1], k0 + ROWS, then, 0);
    load_next(k0 + 2 * ROWS);
    __syncthreads();
    if (busy) {
      weigh(k0, 1);
      __builtin_amdgcn_s_setprio(1);
      if (more) scores(s, area[buf ^ 1], 0);
      Values::template add<N, 2>(part, o, values + Tile::BYTES / 2, lane);
      __builtin_amdgcn_s_setprio(0);
    }
    seen = then;
    __syncthreads();   // the tile is done with
  }
  if (__syncthreads_or(poison)) {
    for (int k0 = start; k0 < end; k0 += ROWS) {
      if (k0 + ROWS <= base) continue;
      const int page = pages_of(k0);
      seen = seen_of(page, k0);
      rows_of(page, k0, at);
#pragma unroll 1
      for (int sign = 1; sign >= -1; sign -= 2) {
        tile.load(cache, at, tid);
        bring(area[0], k0, seen, sign);
        __syncthreads();
        if (busy) {
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            scores(s, area[0], 32 * half);
            hide(s, k0 + 32 * half, (uint32_t)(seen >> 32 * half));
#pragma unroll
            for (int n = 0; n < N; ++n) {   // sums of their own: an infinity in o would swallow the other one
              v4u huge[1][1];
              f32x4_t sum[1][ND];
#pragma unroll
              for (int e = 0; e < 8; e += 2) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[n][e >> 2][e & 3], c2, -R[n]));
                const float y = __builtin_amdgcn_exp2f(fmaf(s[n][e >> 2][(e & 3) + 1], c2, -R[n]));
                huge[0][0][e / 2] = (x > 0.f ? kHugeBits : 0u) | (y > 0.f ? kHugeBits << 16 : 0u);
              }
#pragma unroll
              for (int i = 0; i < ND; ++i) sum[0][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
              Values::template add<1, 1>(huge, sum, area[0] + Tile::BYTES + half * (Tile::BYTES / 2), lane);
#pragma unroll
              for (int i = 0; i < ND; ++i) o[n][i] += sum[0][i];
            }
          }
        }
        __syncthreads();
      }
    }
  }
  if (!busy) return;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    l[n] += __shfl_xor(l[n], 16, 64);
    l[n] += __shfl_xor(l[n], 32, 64);
    const int c = c0 + n * 16 + col;
    if (c >= cols) continue;
    const float L = l[n], inv = L == 0.f ? 0.f : 1.f / (L * kTwoPieces);   // nothing seen: 0, with a log-sum-exp of -inf
    const float lse = L == 0.f ? -INFINITY : fmaf(R[n], 0.6931471805599453f, logf(L));
    const int j = c / grp, h = sh.hk * grp + c - j * grp;
    const int64_t row = (int64_t)(sh.row0 + j) * a.n_heads + h;
    if (sh.parts == 1) {
      bf16_t* out = (bf16_t*)a.out + (int64_t)(sh.row0 + j) * a.out_rs + (int64_t)h * DH + 4 * g;
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        v2u u;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          u[e] = (uint32_t)f2bf(o[n][i][2 * e] * inv) | ((uint32_t)f2bf(o[n][i][2 * e + 1] * inv) << 16);
        *(v2u*)(out + 16 * i) = u;
      }
      if (a.lse && g == 0) a.lse[row] = lse;
    } else {
      float* out = a.part_o + (row * a.n_parts + sh.part) * DH + 4 * g;
#pragma unroll
      for (int i = 0; i < ND; ++i) *(f32x4_t*)(out + 16 * i) = o[n][i] * inv;
      if (g == 0) a.part_lse[row * a.n_parts + sh.part] = lse;
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
  const int per = part_entries(len, a.n_parts), n = (len + per - 1) / per;
  if (n <= 1) return;   // the one part has written the output
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

// Columns of a workgroup, for the widest tree of a call, and whether its waves share their tiles.
// Sharing pays where entries are many or workgroups are: a tile takes a workgroup 2.6 us by
// itself, and a shared one starts 3 us later.  bf16, 8 KV heads of 128, us not shared | shared: 1
// sequence of 360, 148 columns 11.4 | 21.8; 4 of 1000, 104: 19.0 | 27.2; 1 of 1500, 256: 18.9 | 27.4; 1 of
// 4096, 64: 17.8 | 19.4; 8 of 2048, 32: 26.2 | 24.5; 2 of 8192, 64: 34.7 | 27.9; 60 of 300, 64: 63.7 | 25.2.
// 12 KV heads of 64: 2 of 900, 30 columns 11.1 | 14.6; 4 of 2048, 32: 16.8 | 16.3.  fp32 has no shared
// kernel: its products take eight times as long as its loads.
// The lengths lie on the device, so the choice, and that of the parts below, goes by the table's width.  A
// call with its join under a table as wide as its longest sequence needs | 4 | 16 times as wide:
// 1 of 360, 148 columns of 128: 10.6 | 12.9 | 16.0 (shared); 4 of 1000, 104: 17.6 | 22.5 | 22.6 (shared
// from 4 on); 32 of 300, 32: 22.5 | 22.4 | 28.3; 8 of 500 .. 4096, 104: 34.6 | 36.7 | 36.7; 16 of 100 ..
// 8192 in e4m3, 256: 125 | 127 | 126; 2 of 900, 30 of 64: 10.4 | 11.3 | 11.4 (shared); one fp32 sequence
// of 257: 9.8 | 11.0 | 9.9.
struct Width {
  int columns;
  bool shared;
};
Width width_of(const PagedView& cache, int n_seqs, int max_drafts, int n_heads, int64_t max_entries) {
  const int64_t cols = (int64_t)max_drafts * (n_heads / cache.n_kv);
  const int64_t narrow = (int64_t)n_seqs * cache.n_kv * ((cols + 15) / 16);
  const bool few = narrow <= 256 && (max_entries <= 1024 || narrow * max_entries <= 1600 * cache.head_dim);
  if (cols <= 16 || !cache.bf16 || few) return {16, false};
  return {cols <= 64 ? 64 : 128, true};
}

}  // namespace

// Parts of a length: two workgroups to a CU, in parts of 256 entries or more (of a workgroup whose
// waves share their tiles, or up to 24 of 128; 512 otherwise, as in the attention of one token); and
// twice as many of 1024 or more (512 of 64 channels), so that unequal lengths level out: what a part
// costs, its fp32 outputs written and read again, has to be little beside its entries.
//   2 x 8192 entries, 64 columns of 128: 16 parts of 512 29.0, 32 of 256 28.5; 16 columns: 23.6 and 32.1;
//   1 x 3000, 256 columns: 11 parts of 256 28.2, 23 of 128 25.5; 2 x 4096, 104: 16 of 256 26.8, 32 28.4;
//   4 x 1000, 104 columns, shared: 1 part 54.5, 3 30.1; 16 x 4096, 64 columns: 4 parts 72, 8 84;
//   16 x 100 .. 8192, 256 columns: 2 parts 190, 4 150, 8 180 (all of 4096: 146, 157, 185);
//   16 x 100 .. 2048, 32 columns of 64: 2 parts 29.2, 4 22.2.
int tree_parts(const PagedView& cache, int n_seqs, int max_drafts, int n_heads, int64_t max_entries) {
  const Width width = width_of(cache, n_seqs, max_drafts, n_heads, max_entries);
  const int64_t cols = (int64_t)max_drafts * (n_heads / cache.n_kv);
  const int64_t rows = (int64_t)n_seqs * cache.n_kv * ((cols + width.columns - 1) / width.columns);
  const int64_t least = std::max(512, 8 * cache.head_dim);
  const int64_t fill = std::min(512 / rows, width.shared ? std::max(max_entries / 256, std::min<int64_t>(max_entries / 128, 24))
                                                         : max_entries / 512);
  const int64_t level = std::min(1024 / rows, max_entries / least);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::max(fill, level), kMaxTreeParts));
}

// As many of them as the longest sequence has when each has whole tiles for every wave
// (part_entries); workgroups for more would end at once, and leave some CUs less to do than others (2 x
// 4096, 104 columns, 24 parts that are 16: 26.8 us, 28.5 with the empty ones).
int tree_full_parts(int n_parts, int64_t max_entries) {
  constexpr int64_t unit = kTile * kDecodeWaves;
  const int64_t each = ((max_entries + n_parts - 1) / n_parts + unit - 1) / unit * unit;
  return (int)((max_entries + each - 1) / each);
}

int64_t tree_blocks(const PagedView& cache, const PagedTable& tab, const SeqTable& st, const TreeArgs& a) {
  const int64_t cols = (int64_t)st.max_len * (a.n_heads / cache.n_kv);
  const int64_t width = width_of(cache, st.n, st.max_len, a.n_heads, (int64_t)tab.max_pages << cache.page_shift).columns;
  const int64_t items = (int64_t)st.n * cache.n_kv * a.n_parts;
  return (items + 7) / 8 * 8 * ((cols + width - 1) / width);
}

hipError_t launch_tree(const PagedView& cache, const PagedTable& tab, const SeqTable& st, TreeArgs a, hipStream_t s) {
  const Width width = width_of(cache, st.n, st.max_len, a.n_heads, (int64_t)tab.max_pages << cache.page_shift);
  a.col_blocks = (int)(((int64_t)st.max_len * (a.n_heads / cache.n_kv) + width.columns - 1) / width.columns);
  const uint32_t blocks = (uint32_t)tree_blocks(cache, tab, st, a);
  const int64_t outs = (int64_t)st.rows * a.n_heads;
#define RK_TREE(T, C, DH)                                                                                          \
  do {                                                                                                             \
    if constexpr (std::is_same<T, float>::value) {                                                                 \
      Timed timed("paged_tree_narrow", s);                                                                         \
      tree_narrow_kernel<T, C, DH><<<blocks, 64 * kDecodeWaves, 0, s>>>(cache, tab, st, a);                        \
    } else {                                                                                                       \
      Timed timed(!width.shared ? "paged_tree_narrow" : "paged_tree_shared", s);                                   \
      if (!width.shared) tree_narrow_kernel<T, C, DH><<<blocks, 64 * kDecodeWaves, 0, s>>>(cache, tab, st, a);     \
      else if (width.columns == 64) tree_wide_kernel<C, DH, 1><<<blocks, 256, 0, s>>>(cache, tab, st, a);          \
      else tree_wide_kernel<C, DH, 2><<<blocks, 256, 0, s>>>(cache, tab, st, a);                                   \
    }                                                                                                              \
    if (a.n_parts > 1) {                                                                                           \
      const int groups = 256 / (DH / 4);                                                                           \
      tree_join_kernel<T, DH><<<(uint32_t)((outs + groups - 1) / groups), 256, 0, s>>>(tab, st, a, cache.page_shift); \
    }                                                                                                              \
  } while (0)
  RK_PAGED_DISPATCH(cache, RK_TREE);
#undef RK_TREE
  return hipGetLastError();
}

}  // namespace rk
