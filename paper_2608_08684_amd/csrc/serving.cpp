// C ABI of the paged cache (append, read, attention of one new token, the same over selected
// pages, trees of drafts, beams) and of the token log probabilities: checks of arguments,
// workspace plans, launches.
#include <math.h>

#include <algorithm>

#include "rk_internal.h"

namespace rk {
namespace {

const int64_t kMaxGrid = 0x7fffffff;
const int32_t kMaxSeqs = 1 << 23;
const int64_t kMaxEntries = 1 << 30;   // of one sequence: part bounds stay within 32 bits

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

rk_status bad(rk_status e, const char* msg) {
  set_error("%s", msg);
  return e;
}

rk_status hip_status(const char* what, hipError_t e) {
  if (e == hipSuccess) return RK_OK;
  set_error("HIP error in %s: %s", what, hipGetErrorString(e));
  return RK_ERR_HIP;
}

// A stream of another device would run the kernels there.
rk_status check_stream(hipStream_t s) {
  if (!s) return RK_OK;
  int dev = 0, sdev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipStreamGetDevice(s, &sdev);
  if (e == hipSuccess && dev != sdev) e = hipErrorInvalidDevice;
  return hip_status("the stream's device", e);
}

// Sizes of a cache alone (workspace queries take no buffers).
rk_status check_cache(const rk_paged_cache* c, PagedView* v) {
  if (!c) return bad(RK_ERR_ARG, "null cache");
  if (c->dtype != RK_F32 && c->dtype != RK_BF16 && c->dtype != RK_E4M3) return bad(RK_ERR_ARG, "unknown cache dtype");
  const bool e4m3 = c->dtype == RK_E4M3, bf16 = c->dtype == RK_BF16 || e4m3;
  if (c->n_pages < 1 || c->n_pages > kMaxGrid || c->n_kv_heads < 1 || c->n_kv_heads > 65536)
    return bad(RK_ERR_ARG, "n_pages must be in [1, 2^31) and n_kv_heads in [1, 65536]");
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
    return bad(RK_ERR_UNSUPPORTED, "page_size must be a power of two in [16, 256]");
  if (bf16 ? (c->head_dim != 64 && c->head_dim != 128) : (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128))
    return bad(RK_ERR_UNSUPPORTED, "head_dim must be 64 or 128 (bf16, e4m3) or 32, 64 or 128 (fp32)");
  v->k = c->k; v->v = c->v; v->bounds = c->key_bounds;
  v->k_scales = e4m3 ? c->k_scales : nullptr; v->v_scales = e4m3 ? c->v_scales : nullptr;
  v->n_pages = c->n_pages;
  v->page_shift = __builtin_ctz((unsigned)c->page_size);
  v->n_kv = c->n_kv_heads; v->head_dim = c->head_dim; v->bf16 = bf16; v->e4m3 = e4m3;
  return RK_OK;
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

rk_status check_buffers(const PagedView& v) {
  if (!v.k || !v.v) return bad(RK_ERR_ARG, "null cache buffer");
  if (misaligned(v.k) || misaligned(v.v) || misaligned(v.bounds)) return bad(RK_ERR_ARG, "cache buffers must be 16-byte aligned");
  if (v.e4m3 && (!v.k_scales || !v.v_scales || misaligned(v.k_scales) || misaligned(v.v_scales)))
    return bad(RK_ERR_ARG, "an e4m3 cache needs k_scales and v_scales, 16-byte aligned");
  return RK_OK;
}

rk_status check_seqs(const rk_paged_seqs* q, const PagedView& v, PagedTable* t) {
  if (!q || !q->pages || !q->lengths) return bad(RK_ERR_ARG, "null sequences, pages or lengths");
  if (q->n_seqs < 1 || q->max_pages < 1) return bad(RK_ERR_ARG, "n_seqs and max_pages must be positive");
  if (q->n_seqs > kMaxSeqs) return bad(RK_ERR_SHAPE, "n_seqs must be at most 2^23");
  if (q->page_stride < q->max_pages) return bad(RK_ERR_ARG, "page_stride below max_pages");
  if (((int64_t)q->max_pages << v.page_shift) > kMaxEntries) return bad(RK_ERR_SHAPE, "max_pages * page_size must be at most 2^30");
  t->pages = q->pages; t->lengths = q->lengths; t->stride = q->page_stride;
  t->n_seqs = q->n_seqs; t->max_pages = q->max_pages; t->per_head = false;
  return RK_OK;
}

// rows of heads of `width` elements in all, read or written in 16-byte pieces
rk_status check_rows(const void* p, int64_t stride, int64_t width, bool bf16, const char* what) {
  if (misaligned(p) || stride % (bf16 ? 8 : 4)) { set_error("%s: rows must be 16-byte aligned", what); return RK_ERR_ARG; }
  if (stride < width) { set_error("%s: row stride below %lld", what, (long long)width); return RK_ERR_ARG; }
  return RK_OK;
}

// Rows of the sequences by host offsets.
rk_status check_offsets(const int64_t* offsets, int n_seqs, int64_t most_each, SeqTable* st) {
  if (n_seqs > RK_MAX_BATCH_SEQS) { set_error("at most %d sequences with row offsets", RK_MAX_BATCH_SEQS); return RK_ERR_SHAPE; }
  if (offsets[0] != 0) return bad(RK_ERR_SHAPE, "row offsets must start at 0");
  st->max_len = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (offsets[i + 1] < offsets[i] || offsets[i + 1] > (1 << 30))
      return bad(RK_ERR_SHAPE, "row offsets must not decrease and must stay at or below 2^30");
    if (offsets[i + 1] - offsets[i] > most_each) { set_error("at most %lld rows of a sequence", (long long)most_each); return RK_ERR_SHAPE; }
    st->max_len = std::max(st->max_len, (int32_t)(offsets[i + 1] - offsets[i]));
  }
  st->n = n_seqs;
  for (int i = 0; i <= n_seqs; ++i) st->off[i] = (int32_t)offsets[i];
  st->rows = st->off[n_seqs];
  return RK_OK;
}

// rows of n_rows x n_kv heads of d elements, in 16-byte pieces
rk_status check_strided(const void* p, int64_t rs, int64_t hs, int64_t n_rows, const PagedView& v, const char* what) {
  const int64_t d = v.head_dim, es8 = v.bf16 ? 8 : 4;
  if (misaligned(p) || rs % es8 || hs % es8 || rs < 0 || hs < 0) {
    set_error("%s must be 16-byte aligned, its strides whole 16-byte pieces and not negative", what);
    return RK_ERR_ARG;
  }
  if ((n_rows > 1 && rs < d) || (v.n_kv > 1 && hs < d)) { set_error("%s: stride below head_dim", what); return RK_ERR_ARG; }
  return RK_OK;
}

// Workspace of the attention calls: the parts' outputs and log-sum-exps, and for the
// selection the pages' keys and each (sequence, KV head)'s chosen pages.
struct PagedPlan {
  size_t part_o, part_lse, keys, list, list_len, total;
  int n_parts;
};

PagedPlan paged_plan(const PagedView& v, int n_seqs, int max_pages, int n_heads, int n_select) {
  PagedPlan p;
  const int64_t pages = n_select > 0 ? std::min(n_select, max_pages) : max_pages;
  p.n_parts = decode_parts(n_seqs, n_heads, v.n_kv, pages << v.page_shift);
  const size_t parts = p.n_parts > 1 ? (size_t)n_seqs * n_heads * p.n_parts : 0;
  size_t o = 0;
  p.part_o = o;   o += align256(parts * v.head_dim * 4);
  p.part_lse = o; o += align256(parts * 4);
  p.keys = o;
  if (n_select > 0) o += align256((size_t)n_seqs * v.n_kv * max_pages * 8);
  p.list = o;
  if (n_select > 0) o += align256((size_t)n_seqs * v.n_kv * n_select * 4);
  p.list_len = o;
  if (n_select > 0) o += align256((size_t)n_seqs * v.n_kv * 4);
  p.total = std::max<size_t>(o, 256);
  // a workspace for a selection serves the attention over every page too
  if (n_select > 0) p.total = std::max(p.total, paged_plan(v, n_seqs, max_pages, n_heads, 0).total);
  return p;
}

rk_status check_heads(const PagedView& v, int n_seqs, int n_heads) {
  if (n_heads < 1 || n_heads % v.n_kv) return bad(RK_ERR_ARG, "n_heads must be a positive multiple of n_kv_heads");
  if ((int64_t)n_seqs * n_heads > kMaxGrid / 256) return bad(RK_ERR_SHAPE, "n_seqs * n_heads must be below 2^23");
  return RK_OK;
}

rk_status attention(const rk_paged_cache* cache, const rk_paged_seqs* seqs, const rk_page_selection* sel,
                    const void* q, int64_t q_row_stride, int32_t n_heads, float scale, void* out,
                    int64_t out_row_stride, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  PagedView v;
  PagedTable t;
  rk_status e;
  if ((e = check_cache(cache, &v)) != RK_OK || (e = check_buffers(v)) != RK_OK) return e;
  if ((e = check_seqs(seqs, v, &t)) != RK_OK || (e = check_heads(v, t.n_seqs, n_heads)) != RK_OK) return e;
  if (!q || !out || !workspace) return bad(RK_ERR_ARG, "null q, out or workspace");
  if (misaligned(workspace)) return bad(RK_ERR_ARG, "the workspace must be 16-byte aligned");
  const int64_t width = (int64_t)n_heads * v.head_dim;
  if ((e = check_rows(q, q_row_stride, width, v.bf16, "q")) != RK_OK) return e;
  if ((e = check_rows(out, out_row_stride, width, v.bf16, "out")) != RK_OK) return e;
  if (q == out && t.n_seqs > 1 && q_row_stride != out_row_stride)
    return bad(RK_ERR_ARG, "outputs over the queries need one row stride");
  if (!isfinite(scale) || scale < 0.f) return bad(RK_ERR_ARG, "scale must be finite and >= 0 (0: 1 / sqrt(head_dim))");
  if (sel) {
    if (!v.bounds) return bad(RK_ERR_ARG, "the selection needs key_bounds");
    if (sel->n_select < 1 || sel->keep_first < 0 || sel->keep_last < 0 ||
        (int64_t)sel->keep_first + sel->keep_last > sel->n_select)
      return bad(RK_ERR_ARG, "n_select must be positive, keep_first and keep_last >= 0 and together at most n_select");
    if (((int64_t)sel->n_select << v.page_shift) > kMaxEntries) return bad(RK_ERR_SHAPE, "n_select * page_size must be at most 2^30");
  }
  const PagedPlan p = paged_plan(v, t.n_seqs, t.max_pages, n_heads, sel ? sel->n_select : 0);
  if (ws_bytes < p.total) { set_error("workspace too small (%zu < %zu)", ws_bytes, p.total); return RK_ERR_WORKSPACE; }
  hipStream_t s = (hipStream_t)stream;
  if ((e = check_stream(s)) != RK_OK) return e;
  char* ws = (char*)workspace;
  DecodeArgs a{};
  a.q = q; a.out = out; a.lse = lse; a.q_rs = q_row_stride; a.out_rs = out_row_stride;
  a.n_heads = n_heads; a.n_parts = p.n_parts;
  a.scale = scale > 0.f ? scale : (float)(1.0 / sqrt((double)v.head_dim));
  a.part_o = (float*)(ws + p.part_o); a.part_lse = (float*)(ws + p.part_lse);
  Timed timed("paged_attention", s);
  if (!sel) return hip_status("paged attention", launch_decode(v, t, a, s));
  SelectArgs c{};
  c.q = q; c.q_rs = q_row_stride;
  c.n_heads = n_heads; c.n_select = sel->n_select; c.keep_first = sel->keep_first; c.keep_last = sel->keep_last;
  c.keys = (uint64_t*)(ws + p.keys); c.list = (int32_t*)(ws + p.list); c.list_len = (int32_t*)(ws + p.list_len);
  c.selected = sel->selected;
  return hip_status("attention over selected pages", launch_decode_selected(v, t, a, c, s));
}

// Workspace of the trees' attention: the parts' outputs and log-sum-exps.
struct TreePlan {
  int n_parts;
  size_t part_lse, total;
};

TreePlan tree_plan(const PagedView& v, int n_seqs, int max_drafts, int64_t rows, int max_pages, int n_heads) {
  TreePlan p;
  p.n_parts = tree_parts(v, n_seqs, max_drafts, n_heads, (int64_t)max_pages << v.page_shift);
  const size_t parts = p.n_parts > 1 ? (size_t)rows * n_heads * p.n_parts : 0;
  p.part_lse = align256(parts * v.head_dim * 4);
  p.total = std::max<size_t>(256, p.part_lse + align256(parts * 4));
  return p;
}

}  // namespace
}  // namespace rk

using namespace rk;

extern "C" {

rk_status rk_paged_append(const rk_paged_cache* cache, const rk_paged_seqs* seqs, const rk_paged_rows* rows,
                          void* stream) {
  PagedView v;
  PagedTable t;
  rk_status e;
  if ((e = check_cache(cache, &v)) != RK_OK || (e = check_buffers(v)) != RK_OK) return e;
  if ((e = check_seqs(seqs, v, &t)) != RK_OK) return e;
  if (!rows || !rows->k || !rows->v) return bad(RK_ERR_ARG, "null rows, k or v");
  AppendArgs a{};
  SeqTable st{};
  a.one_row = rows->offsets == nullptr;
  if (a.one_row) {
    a.n_rows = t.n_seqs;
  } else {
    if ((e = check_offsets(rows->offsets, t.n_seqs, 1 << 30, &st)) != RK_OK) return e;
    a.n_rows = st.rows;
  }
  const int64_t d = v.head_dim;
  if ((e = check_strided(rows->k, rows->k_row_stride, rows->k_head_stride, a.n_rows, v, "k")) != RK_OK) return e;
  if ((e = check_strided(rows->v, rows->v_row_stride, rows->v_head_stride, a.n_rows, v, "v")) != RK_OK) return e;
  if (!(rows->rope_theta == 0.f || rows->rope_theta > 1.f) || !isfinite(rows->rope_theta))
    return bad(RK_ERR_ARG, "rope_theta must be 0 (no rotation) or > 1");
  if ((rows->q != nullptr) != (rows->q_out != nullptr)) return bad(RK_ERR_ARG, "q and q_out go together");
  if (rows->q) {
    if ((e = check_heads(v, 1, rows->n_heads)) != RK_OK) return e;
    if ((e = check_rows(rows->q, rows->q_row_stride, rows->n_heads * d, v.bf16, "q")) != RK_OK) return e;
    if ((e = check_rows(rows->q_out, rows->q_out_row_stride, rows->n_heads * d, v.bf16, "q_out")) != RK_OK) return e;
    if (rows->q == rows->q_out && rows->q_row_stride != rows->q_out_row_stride)
      return bad(RK_ERR_ARG, "q rotated in place needs one row stride");
    a.n_heads = rows->n_heads;
  }
  a.k = rows->k; a.v = rows->v; a.q = rows->q; a.q_out = rows->q_out;
  a.k_rs = rows->k_row_stride; a.k_hs = rows->k_head_stride;
  a.v_rs = rows->v_row_stride; a.v_hs = rows->v_head_stride;
  a.q_rs = rows->q_row_stride; a.qo_rs = rows->q_out_row_stride;
  a.positions = rows->positions;
  a.rotate = rows->rope_theta != 0.f;
  if (a.rotate) {   // theta^(-2x/d) / (2 pi): each power of two of x once, the others products of those
    double freq[64];
    freq[0] = 0.15915494309189533577;
    for (int b = 1; b < v.head_dim / 2; b *= 2) {
      const double f = pow((double)rows->rope_theta, -2.0 * b / v.head_dim);
      for (int x = b; x < 2 * b; ++x) freq[x] = freq[x - b] * f;
    }
    for (int x = 0; x < v.head_dim / 2; ++x) a.freq[x] = (uint64_t)(freq[x] * 0x1p64);   // below 2^62
  }
  const int64_t blocks = append_plan(v, t, st, &a);
  if (blocks > kMaxWorkgroups) {
    set_error("%lld workgroups: more than the %lld of a launch", (long long)blocks, (long long)kMaxWorkgroups);
    return RK_ERR_SHAPE;
  }
  hipStream_t s = (hipStream_t)stream;
  if ((e = check_stream(s)) != RK_OK) return e;
  Timed timed("paged_append", s);
  return hip_status("paged append", launch_append(v, t, a, st, blocks, s));
}

size_t rk_paged_workspace_size(const rk_paged_cache* cache, int32_t n_seqs, int32_t max_pages, int32_t n_heads,
                               int32_t n_select) {
  PagedView v;
  if (check_cache(cache, &v) != RK_OK || n_seqs < 1 || max_pages < 1 || n_select < 0) return 0;
  if (((int64_t)std::max(max_pages, n_select) << v.page_shift) > kMaxEntries || check_heads(v, n_seqs, n_heads) != RK_OK) return 0;
  // fewer rows may be split into more parts; from 2048 rows on none is (decode_parts)
  size_t most = paged_plan(v, n_seqs, max_pages, n_heads, n_select).total;
  for (int n = std::min(n_seqs, 2048); n >= 1; --n) most = std::max(most, paged_plan(v, n, max_pages, n_heads, n_select).total);
  return most;
}

rk_status rk_paged_attention(const rk_paged_cache* cache, const rk_paged_seqs* seqs, const void* q,
                             int64_t q_row_stride, int32_t n_heads, float scale, void* out, int64_t out_row_stride,
                             float* lse, void* workspace, size_t ws_bytes, void* stream) {
  return attention(cache, seqs, nullptr, q, q_row_stride, n_heads, scale, out, out_row_stride, lse, workspace, ws_bytes,
                   stream);
}

rk_status rk_paged_attention_selected(const rk_paged_cache* cache, const rk_paged_seqs* seqs,
                                      const rk_page_selection* selection, const void* q, int64_t q_row_stride,
                                      int32_t n_heads, float scale, void* out, int64_t out_row_stride, float* lse,
                                      void* workspace, size_t ws_bytes, void* stream) {
  if (!selection) return bad(RK_ERR_ARG, "null selection");
  return attention(cache, seqs, selection, q, q_row_stride, n_heads, scale, out, out_row_stride, lse, workspace,
                   ws_bytes, stream);
}

rk_status rk_paged_read(const rk_paged_cache* cache, const rk_paged_seqs* seqs, const int64_t* offsets, void* k_out,
                        int64_t k_row_stride, int64_t k_head_stride, void* v_out, int64_t v_row_stride,
                        int64_t v_head_stride, void* stream) {
  PagedView v;
  PagedTable t;
  ReadArgs a{};
  SeqTable st{};
  rk_status e;
  if ((e = check_cache(cache, &v)) != RK_OK || (e = check_buffers(v)) != RK_OK) return e;
  if ((e = check_seqs(seqs, v, &t)) != RK_OK) return e;
  if (!k_out && !v_out) return bad(RK_ERR_ARG, "no output");
  a.one_row = offsets == nullptr;
  if (!a.one_row && (e = check_offsets(offsets, t.n_seqs, 1 << 30, &st)) != RK_OK) return e;
  a.n_rows = a.one_row ? t.n_seqs : st.rows;
  if (k_out && (e = check_strided(k_out, k_row_stride, k_head_stride, a.n_rows, v, "k_out")) != RK_OK) return e;
  if (v_out && (e = check_strided(v_out, v_row_stride, v_head_stride, a.n_rows, v, "v_out")) != RK_OK) return e;
  if (read_blocks(a.n_rows) > kMaxWorkgroups) return bad(RK_ERR_SHAPE, "more rows than a launch takes (2^28)");
  a.k = k_out; a.v = v_out;
  a.k_rs = k_row_stride; a.k_hs = k_head_stride; a.v_rs = v_row_stride; a.v_hs = v_head_stride;
  hipStream_t s = (hipStream_t)stream;
  if ((e = check_stream(s)) != RK_OK) return e;
  Timed timed("paged_read", s);
  return hip_status("paged read", launch_read(v, t, a, st, s));
}

size_t rk_paged_tree_workspace_size(const rk_paged_cache* cache, int32_t n_seqs, int64_t n_rows, int32_t max_pages,
                                    int32_t n_heads) {
  PagedView v;
  if (check_cache(cache, &v) != RK_OK || n_seqs < 1 || n_seqs > RK_MAX_BATCH_SEQS || max_pages < 1 || n_rows < 0) return 0;
  if (n_rows > (int64_t)n_seqs * RK_MAX_DRAFTS || ((int64_t)max_pages << v.page_shift) > kMaxEntries) return 0;
  if (check_heads(v, (int)std::max<int64_t>(n_rows, 1), n_heads) != RK_OK) return 0;
  // fewer sequences, or narrower trees, may be split into more parts
  size_t most = 256;
  for (int n = 1; n <= n_seqs; ++n)
    for (int m = 1; m <= RK_MAX_DRAFTS && m <= n_rows; ++m)
      most = std::max(most, tree_plan(v, n, m, std::min(n_rows, (int64_t)n * m), max_pages, n_heads).total);
  return most;
}

rk_status rk_paged_attention_tree(const rk_paged_cache* cache, const rk_paged_seqs* seqs, const int64_t* offsets,
                                  const uint64_t* masks, const void* q, int64_t q_row_stride, int32_t n_heads,
                                  float scale, void* out, int64_t out_row_stride, float* lse, void* workspace,
                                  size_t ws_bytes, void* stream) {
  PagedView v;
  PagedTable t;
  SeqTable st{};
  rk_status e;
  if ((e = check_cache(cache, &v)) != RK_OK || (e = check_buffers(v)) != RK_OK) return e;
  if ((e = check_seqs(seqs, v, &t)) != RK_OK) return e;
  if (!offsets) return bad(RK_ERR_ARG, "null row offsets");
  if ((e = check_offsets(offsets, t.n_seqs, RK_MAX_DRAFTS, &st)) != RK_OK) return e;
  if ((e = check_heads(v, std::max(st.rows, 1), n_heads)) != RK_OK) return e;
  if (!isfinite(scale) || scale < 0.f) return bad(RK_ERR_ARG, "scale must be finite and >= 0 (0: 1 / sqrt(head_dim))");
  if (st.rows == 0) return RK_OK;   // the buffers of no rows may be NULL
  if (!q || !out || !workspace) return bad(RK_ERR_ARG, "null q, out or workspace");
  if (misaligned(workspace) || ((uintptr_t)masks & 7)) return bad(RK_ERR_ARG, "the workspace must be 16-byte aligned, masks 8");
  const int64_t width = (int64_t)n_heads * v.head_dim;
  if ((e = check_rows(q, q_row_stride, width, v.bf16, "q")) != RK_OK) return e;
  if ((e = check_rows(out, out_row_stride, width, v.bf16, "out")) != RK_OK) return e;
  if (q == out && st.rows > 1 && q_row_stride != out_row_stride)
    return bad(RK_ERR_ARG, "outputs over the queries need one row stride");
  const TreePlan p = tree_plan(v, st.n, st.max_len, st.rows, t.max_pages, n_heads);
  if (ws_bytes < p.total) { set_error("workspace too small (%zu < %zu)", ws_bytes, p.total); return RK_ERR_WORKSPACE; }
  TreeArgs a{};
  a.q = q; a.out = out; a.lse = lse; a.masks = masks; a.q_rs = q_row_stride; a.out_rs = out_row_stride;
  a.n_heads = n_heads;
  a.n_parts = tree_full_parts(p.n_parts, (int64_t)t.max_pages << v.page_shift);
  a.scale = scale > 0.f ? scale : (float)(1.0 / sqrt((double)v.head_dim));
  a.part_o = (float*)workspace; a.part_lse = (float*)((char*)workspace + p.part_lse);
  if (tree_blocks(v, t, st, a) > kMaxWorkgroups) return bad(RK_ERR_SHAPE, "more heads and drafts than a launch takes");
  hipStream_t s = (hipStream_t)stream;
  if ((e = check_stream(s)) != RK_OK) return e;
  Timed timed("paged_tree", s);
  return hip_status("attention of drafts", launch_tree(v, t, st, a, s));
}

rk_status rk_paged_keep(const rk_paged_cache* cache, const rk_paged_seqs* seqs, const int64_t* offsets,
                        const int32_t* kept, int64_t kept_stride, int32_t n_kept, void* stream) {
  PagedView v;
  PagedTable t;
  SeqTable st{};
  rk_status e;
  if ((e = check_cache(cache, &v)) != RK_OK || (e = check_buffers(v)) != RK_OK) return e;
  if ((e = check_seqs(seqs, v, &t)) != RK_OK) return e;
  if (!offsets || !kept) return bad(RK_ERR_ARG, "null row offsets or kept");
  if ((e = check_offsets(offsets, t.n_seqs, RK_MAX_DRAFTS, &st)) != RK_OK) return e;
  if (n_kept < 1 || n_kept > RK_MAX_DRAFTS || kept_stride < n_kept) {
    set_error("n_kept must be in [1, %d] and kept_stride not below it", RK_MAX_DRAFTS);
    return RK_ERR_ARG;
  }
  if (st.rows == 0) return RK_OK;
  hipStream_t s = (hipStream_t)stream;
  if ((e = check_stream(s)) != RK_OK) return e;
  Timed timed("paged_keep", s);
  return hip_status("paged keep", launch_keep(v, t, st, kept, kept_stride, n_kept, s));
}

rk_status rk_paged_reorder(const rk_paged_cache* cache, const rk_paged_seqs* seqs, int32_t n_beams,
                           const int32_t* parents, int32_t* pages_out, int64_t pages_out_stride, void* stream) {
  PagedView v;
  PagedTable t;
  rk_status e;
  if ((e = check_cache(cache, &v)) != RK_OK || (e = check_buffers(v)) != RK_OK) return e;
  if ((e = check_seqs(seqs, v, &t)) != RK_OK) return e;
  if (!parents) return bad(RK_ERR_ARG, "null parents");
  if (n_beams < 1 || n_beams > RK_MAX_BEAMS || t.n_seqs % n_beams) {
    set_error("n_beams must be in [1, %d] and n_seqs a multiple of it", RK_MAX_BEAMS);
    return RK_ERR_ARG;
  }
  if (pages_out && pages_out_stride < t.max_pages) return bad(RK_ERR_ARG, "pages_out_stride below max_pages");
  if (pages_out == t.pages && t.n_seqs > 1 && pages_out_stride != t.stride)
    return bad(RK_ERR_ARG, "a table changed in place needs one row stride");
  if (reorder_blocks(v, t.n_seqs, n_beams, t.max_pages) > kMaxWorkgroups)
    return bad(RK_ERR_SHAPE, "more sequences, heads and pages than a launch takes");
  ReorderArgs a{};
  a.parents = parents; a.pages_out = pages_out; a.out_stride = pages_out_stride; a.n_beams = n_beams;
  hipStream_t s = (hipStream_t)stream;
  if ((e = check_stream(s)) != RK_OK) return e;
  Timed timed("paged_reorder", s);
  return hip_status("paged reorder", launch_reorder(v, t, a, s));
}

// Workspace: the parts' sums and best logits, where rows are split; 0 for invalid sizes.
struct LogprobPlan {
  int parts, part_logits;
  size_t top, total;
};

static LogprobPlan logprob_plan(int64_t n_rows, int32_t vocab, rk_dtype dtype, int32_t n_top) {
  LogprobPlan p{};
  if (n_rows < 0 || n_rows > kMaxWorkgroups || vocab < 1 || vocab > kMaxVocab) return p;
  if (n_top < 0 || n_top > RK_MAX_TOP || n_top > vocab || (dtype != RK_F32 && dtype != RK_BF16)) return p;
  logprob_parts(n_rows, vocab, dtype == RK_BF16, &p.parts, &p.part_logits);
  if (n_rows * p.parts > kMaxWorkgroups) return p;
  const size_t parts = p.parts > 1 ? (size_t)n_rows * p.parts : 0;
  p.top = align256(parts * sizeof(float4));
  p.total = std::max<size_t>(256, p.top + align256(parts * n_top * 8));
  return p;
}

size_t rk_token_logprobs_workspace_size(int64_t n_rows, int32_t vocab, rk_dtype dtype, int32_t n_top) {
  // fewer rows may be split into more parts; beyond 256 the number of rows changes nothing there
  size_t most = logprob_plan(n_rows, vocab, dtype, n_top).total;
  for (int64_t n = std::min<int64_t>(n_rows, 256); n >= 1 && most; --n) most = std::max(most, logprob_plan(n, vocab, dtype, n_top).total);
  return most;
}

rk_status rk_token_logprobs(const void *logits, rk_dtype dtype, int64_t n_rows, int32_t vocab, int64_t row_stride,
                            const int32_t* tokens, int32_t n_top, float* logprob, int32_t* rank, float* entropy,
                            int32_t* top_ids, float* top_logprobs, void* workspace, size_t ws_bytes, void* stream) {
  LogprobArgs a{};
  if (dtype != RK_F32 && dtype != RK_BF16) return bad(RK_ERR_ARG, "unknown dtype");
  const LogprobPlan p = logprob_plan(n_rows, vocab, dtype, n_top);
  if (p.total == 0) {
    set_error("n_rows (times the parts of a long row) must be in [0, 2^24), vocab in [1, 2^22], n_top in [0, min(vocab, %d)]",
              RK_MAX_TOP);
    return RK_ERR_ARG;
  }
  if (row_stride < vocab) return bad(RK_ERR_ARG, "row_stride below vocab");
  if (n_rows == 0) return RK_OK;   // the buffers of no rows may be NULL
  if (!tokens && (logprob || rank)) return bad(RK_ERR_ARG, "logprob and rank need tokens");
  if ((n_top > 0) != (top_ids || top_logprobs)) return bad(RK_ERR_ARG, "top_ids or top_logprobs go with n_top > 0");
  if (!logprob && !rank && !entropy && !n_top) return bad(RK_ERR_ARG, "no output");
  if (!logits || !workspace) return bad(RK_ERR_ARG, "null logits or workspace");
  if (((uintptr_t)logits & (dtype == RK_BF16 ? 1 : 3)) || misaligned(workspace))
    return bad(RK_ERR_ARG, "logits must be aligned to their type and the workspace to 16 bytes");
  if (ws_bytes < p.total) { set_error("workspace too small (%zu < %zu)", ws_bytes, p.total); return RK_ERR_WORKSPACE; }
  hipStream_t s = (hipStream_t)stream;
  rk_status e;
  if ((e = check_stream(s)) != RK_OK) return e;
  a.logits = logits; a.row_stride = row_stride; a.n_rows = n_rows; a.vocab = vocab; a.n_top = n_top;
  a.tokens = tokens; a.logprob = logprob; a.rank = rank; a.entropy = entropy;
  a.top_ids = top_ids; a.top_logprobs = top_logprobs;
  a.parts = p.parts; a.part_logits = p.part_logits;
  a.part = (float4*)workspace; a.part_top = (uint64_t*)((char*)workspace + p.top);
  Timed timed("token_logprobs", s);
  return hip_status("token log probabilities", launch_logprobs(a, dtype == RK_BF16, s));
}

// Workspace of the selection over beams: every row's sums and best logits (those of its parts).
static LogprobPlan beam_plan(int32_t n_groups, int32_t n_beams, int32_t vocab, rk_dtype dtype, int32_t n_out) {
  LogprobPlan p{};
  if (n_groups < 0 || n_beams < 1 || n_beams > RK_MAX_BEAMS || n_out < 1 || n_out > RK_MAX_TOP || vocab < 1) return p;
  const int64_t rows = (int64_t)n_groups * n_beams;
  const int n = std::min(n_out, vocab);
  p = logprob_plan(rows, vocab, dtype, n);
  if (!p.total) return p;
  beam_parts(rows, vocab, dtype == RK_BF16, &p.parts, &p.part_logits);
  p.top = align256((size_t)rows * p.parts * sizeof(float4));
  p.total = std::max<size_t>(256, p.top + align256((size_t)rows * p.parts * n * 8));
  return p;
}

size_t rk_beam_select_workspace_size(int32_t n_groups, int32_t n_beams, int32_t vocab, rk_dtype dtype, int32_t n_out) {
  // fewer rows may be split into more parts; beyond 256 the number of rows changes nothing there
  size_t most = beam_plan(n_groups, n_beams, vocab, dtype, n_out).total;
  for (int n = std::min(n_groups, 256); n >= 1 && most; --n)
    most = std::max(most, beam_plan(n, n_beams, vocab, dtype, n_out).total);
  return most;
}

rk_status rk_beam_select(const void* logits, rk_dtype dtype, int32_t n_groups, int32_t n_beams, int32_t vocab,
                         int64_t row_stride, const float* scores, const uint8_t* ended, int32_t end_token,
                         int32_t n_out, int32_t* parents, int32_t* tokens, float* scores_out, void* workspace,
                         size_t ws_bytes, void* stream) {
  if (dtype != RK_F32 && dtype != RK_BF16) return bad(RK_ERR_ARG, "unknown dtype");
  const LogprobPlan p = beam_plan(n_groups, n_beams, vocab, dtype, n_out);
  if (p.total == 0) {
    set_error("n_beams must be in [1, %d], n_out in [1, %d], vocab in [1, 2^22], rows (times the parts of a long row) in [0, 2^24)",
              RK_MAX_BEAMS, RK_MAX_TOP);
    return RK_ERR_ARG;
  }
  if (row_stride < vocab) return bad(RK_ERR_ARG, "row_stride below vocab");
  if (n_groups == 0) return RK_OK;   // the buffers of no rows may be NULL
  if (!logits || !scores || !parents || !tokens || !scores_out || !workspace)
    return bad(RK_ERR_ARG, "null logits, scores, output or workspace");
  if (((uintptr_t)logits & (dtype == RK_BF16 ? 1 : 3)) || misaligned(workspace))
    return bad(RK_ERR_ARG, "logits must be aligned to their type and the workspace to 16 bytes");
  if (scores_out == scores && n_out != n_beams) return bad(RK_ERR_ARG, "scores changed in place need n_out = n_beams");
  if (ws_bytes < p.total) { set_error("workspace too small (%zu < %zu)", ws_bytes, p.total); return RK_ERR_WORKSPACE; }
  hipStream_t s = (hipStream_t)stream;
  rk_status e;
  if ((e = check_stream(s)) != RK_OK) return e;
  LogprobArgs a{};
  a.logits = logits; a.row_stride = row_stride; a.n_rows = (int64_t)n_groups * n_beams; a.vocab = vocab;
  a.n_top = std::min(n_out, vocab);
  a.parts = p.parts; a.part_logits = p.part_logits;
  a.part = (float4*)workspace; a.part_top = (uint64_t*)((char*)workspace + p.top);
  BeamArgs b{};
  b.scores = scores; b.ended = ended; b.n_beams = n_beams; b.n_out = n_out; b.end_token = end_token;
  b.parents = parents; b.tokens = tokens; b.scores_out = scores_out;
  Timed timed("beam_select", s);
  return hip_status("beam selection", launch_beam_select(a, b, dtype == RK_BF16, s));
}

}  // extern "C"
