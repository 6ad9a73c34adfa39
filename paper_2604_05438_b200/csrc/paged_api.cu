// Entry points of the paged cache: argument validation, workspace layout, launches.
#include "host.cuh"
#include "paged.cuh"

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

using namespace tkphi;

namespace {

struct PagedShape {
  int page_shift, group, total_q;
  int64_t max_kv, max_q;
  int64_t max_pages_seq;                     // pages of the longest sequence that takes part
};

// Positive strides of the dims with more than one index, from the smallest up: each must step over all before it.
bool disjoint(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t inner) {
  int64_t n[3] = {n0, n1, n2}, s[3] = {s0, s1, s2};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (s[j] < s[i]) { std::swap(s[i], s[j]); std::swap(n[i], n[j]); }
  int64_t extent = inner;
  for (int i = 0; i < 3; ++i) {
    if (n[i] < 2) continue;
    if (s[i] < extent) return false;
    extent += s[i] * (n[i] - 1);
  }
  return true;
}

tkphi_status validate_paged(const tkphi_paged_desc* kv, PagedShape* sh, bool need_data, bool full_context) {
  if (!kv) return fail(TKPHI_ERR_INVALID_ARG, "kv descriptor is NULL");
  if (kv->batch < 1 || kv->batch > kMaxBatch)
    return fail(TKPHI_ERR_INVALID_ARG, "batch must be in [1, %d], got %d", kMaxBatch, kv->batch);
  if (kv->head_dim != 64 && kv->head_dim != 128)
    return fail(TKPHI_ERR_UNSUPPORTED, "head_dim must be 64 or 128, got %d", kv->head_dim);
  if (kv->dtype != TKPHI_DTYPE_BF16 && kv->dtype != TKPHI_DTYPE_FP16)
    return fail(TKPHI_ERR_UNSUPPORTED, "dtype must be TKPHI_DTYPE_BF16 or TKPHI_DTYPE_FP16, got %d", kv->dtype);
  if (kv->n_kv_heads < 1 || kv->n_q_heads < 1 || kv->n_q_heads % kv->n_kv_heads != 0)
    return fail(TKPHI_ERR_INVALID_ARG, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)",
                kv->n_q_heads, kv->n_kv_heads);
  sh->group = kv->n_q_heads / kv->n_kv_heads;
  if (sh->group > kMaxGroup) return fail(TKPHI_ERR_UNSUPPORTED, "group size %d > %d", sh->group, kMaxGroup);
  if (kv->n_kv_heads > 4096) return fail(TKPHI_ERR_UNSUPPORTED, "n_kv_heads = %d > 4096", kv->n_kv_heads);
  sh->page_shift = 0;
  for (int s = 4; s <= 7; ++s)
    if (kv->page_size == 1 << s) sh->page_shift = s;
  if (!sh->page_shift) return fail(TKPHI_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128, got %d", kv->page_size);
  if (kv->n_pages < 1 || kv->n_pages > (1 << 30) || kv->max_pages < 1 || kv->max_pages > (1 << 30))
    return fail(TKPHI_ERR_INVALID_ARG, "n_pages (%d) and max_pages (%d) must be in [1, 2^30]", kv->n_pages, kv->max_pages);
  if (!kv->kv_lens_host || !kv->cu_q_host) return fail(TKPHI_ERR_INVALID_ARG, "kv_lens_host or cu_q_host is NULL");
  const int64_t* cu = kv->cu_q_host;
  if (cu[0] != 0) return fail(TKPHI_ERR_INVALID_ARG, "cu_q[0] must be 0");
  const int64_t room = std::min<int64_t>((int64_t)kv->max_pages * kv->page_size, kMaxKvLen);
  sh->max_kv = 0; sh->max_q = 0;
  for (int b = 0; b < kv->batch; ++b) {
    // no overflow: both checked against small bounds before they are subtracted
    if (cu[b + 1] < cu[b] || cu[b + 1] > (int64_t)INT_MAX / 2)
      return fail(TKPHI_ERR_INVALID_ARG, "cu_q must be non-decreasing and below 2^30 (sequence %d)", b);
    const int64_t q = cu[b + 1] - cu[b], len = kv->kv_lens_host[b];
    if (len < 0 || len > room)
      return fail(TKPHI_ERR_INVALID_ARG, "kv_lens[%d] = %lld outside [0, %lld]", b, (long long)len, (long long)room);
    if (!full_context && len < q)
      return fail(TKPHI_ERR_INVALID_ARG, "sequence %d: %lld new tokens in a cache of %lld rows", b, (long long)q, (long long)len);
    if (q > 0) { sh->max_kv = std::max(sh->max_kv, len); sh->max_q = std::max(sh->max_q, q); }
  }
  sh->total_q = (int)cu[kv->batch];
  sh->max_pages_seq = (sh->max_kv + kv->page_size - 1) / kv->page_size;
  if ((int64_t)sh->total_q * kv->n_q_heads > (int64_t)INT_MAX / 2)
    return fail(TKPHI_ERR_UNSUPPORTED, "%d tokens of %d heads are too many for one call", sh->total_q, kv->n_q_heads);
  if (need_data) {
    if (!kv->k || !kv->v || !aligned16(kv->k) || !aligned16(kv->v))
      return fail(TKPHI_ERR_INVALID_ARG, "k or v is NULL or not 16-byte aligned");
    if (!kv->page_table || !kv->kv_lens_dev || !kv->cu_q_dev || !kv->status)
      return fail(TKPHI_ERR_INVALID_ARG, "page_table, kv_lens_dev, cu_q_dev or status is NULL");
    if ((reinterpret_cast<uintptr_t>(kv->page_table) | reinterpret_cast<uintptr_t>(kv->status)) & 3u ||
        (reinterpret_cast<uintptr_t>(kv->kv_lens_dev) | reinterpret_cast<uintptr_t>(kv->cu_q_dev)) & 7u)
      return fail(TKPHI_ERR_INVALID_ARG, "page_table, kv_lens_dev, cu_q_dev or status is not aligned to its type");
    if (kv->key_bounds && !aligned16(kv->key_bounds))
      return fail(TKPHI_ERR_INVALID_ARG, "key_bounds must be 16-byte aligned");
    const int64_t st[3] = {kv->stride_page, kv->stride_head, kv->stride_token};
    for (int64_t s : st)
      if (s < 0 || s % 8 != 0 || s >= (1ll << 38))
        return fail(TKPHI_ERR_INVALID_ARG, "cache strides must be non-negative multiples of 8 elements below 2^38, got %lld", (long long)s);
    if (!disjoint(kv->n_pages, kv->stride_page, kv->n_kv_heads, kv->stride_head, kv->page_size, kv->stride_token, kv->head_dim))
      return fail(TKPHI_ERR_INVALID_ARG, "the cache strides (page %lld, head %lld, token %lld) let elements share memory",
                  (long long)st[0], (long long)st[1], (long long)st[2]);
  }
  return TKPHI_OK;
}

// 4-D view [page][head][slot][dim] of k or v; box = 64 dims x min(page_size, 64) slots of one head, 128-byte swizzle.
tkphi_status make_page_map(const tkphi_paged_desc* kv, const void* base, CUtensorMap* tm) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return fail(TKPHI_ERR_CUDA, "cuTensorMapEncodeTiled is not available from this driver");
  const cuuint64_t dims[4] = {(cuuint64_t)kv->head_dim, (cuuint64_t)kv->page_size, (cuuint64_t)kv->n_kv_heads,
                              (cuuint64_t)kv->n_pages};
  // (a dim of one index: any legal stride will do, the caller's may be 0)
  const cuuint64_t st[3] = {(cuuint64_t)kv->stride_token * 2,
                            kv->n_kv_heads > 1 ? (cuuint64_t)kv->stride_head * 2 : (cuuint64_t)kv->head_dim * 2,
                            kv->n_pages > 1 ? (cuuint64_t)kv->stride_page * 2 : (cuuint64_t)kv->head_dim * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)std::min(kv->page_size, 64), 1, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  const CUresult r = fn(tm, kv->dtype == TKPHI_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                        4, const_cast<void*>(base), dims, st, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(TKPHI_ERR_CUDA, "cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
  return TKPHI_OK;
}

// 4-D view [token][KV head][query head of the group][dim] of the step's queries; box = 64 dims x the group x the tokens of
// an MMA tile of one KV head: a tile's rows as they lie in shared memory.
tkphi_status make_query_map(const tkphi_paged_desc* kv, const PagedShape& sh, const void* q, CUtensorMap* tm) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return fail(TKPHI_ERR_CUDA, "cuTensorMapEncodeTiled is not available from this driver");
  const cuuint64_t row = (cuuint64_t)kv->head_dim * 2;
  const cuuint64_t dims[4] = {(cuuint64_t)kv->head_dim, (cuuint64_t)sh.group, (cuuint64_t)kv->n_kv_heads, (cuuint64_t)sh.total_q};
  const cuuint64_t st[3] = {row, row * sh.group, row * kv->n_q_heads};
  const cuuint32_t box[4] = {64, (cuuint32_t)sh.group, 1, (cuuint32_t)(128 / sh.group)};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  const CUresult r = fn(tm, kv->dtype == TKPHI_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                        4, const_cast<void*>(q), dims, st, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(TKPHI_ERR_CUDA, "cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
  return TKPHI_OK;
}

// What a call launches and where its pieces of the workspace lie; a function of the host lengths and the device's
// multiprocessor count only, so that the size query and the call agree.
struct AttendPlan {
  int max_rows;                  // rows of the widest sequence of the row kernel
  int64_t row_tiles;             // tiles of the row kernel
  int row_ctas, row_split, row_grid;   // row_split > 0: clusters of that many CTAs per unit, nothing to join
  bool any_rows, any_tiles;
  int chunk, max_chunks, tile_grid;
  size_t row_part, row_stat, tile_part, tile_stat, total;
};

// Sequences with at most this many rows per KV head go to the row kernel: one tile of its matrix instruction.
constexpr int kRowsLimit = 16;

// Keys per CTA of the tile kernel: the whole context if the row tiles alone fill the SMs evenly, otherwise a part of it.
// The estimate of a choice, in key tiles of one CTA: the larger of the waves' sum and the balanced share plus half of
// the longest CTA; a CTA costs about four tiles of set-up and, if its output is partial, a thirtieth of a tile of the
// device's time for writing and joining it.
int choose_chunk(const tkphi_paged_desc* kv, const PagedShape& sh, int64_t longest, int n_sm) {
  int best = 0;
  double best_cost = 0;
  for (int parts = 1; parts <= 64; ++parts) {
    const int64_t per = (longest + parts - 1) / parts;
    if (parts > 1 && per < 4) break;
    double ctas = 0, work = 0;
    for (int b = 0; b < kv->batch; ++b) {
      const int64_t q = kv->cu_q_host[b + 1] - kv->cu_q_host[b], len = kv->kv_lens_host[b];
      if (q * sh.group <= kRowsLimit) continue;
      const int pair = 2 * tile_rows(sh.group);
      const double rt = (double)((q * sh.group + pair - 1) / pair) * kv->n_kv_heads;
      const double seen = std::max<double>(1., ((double)len - 0.5 * (double)std::min(q, len)) / kTileKeys);   // of an average row tile
      ctas += rt * std::max(1., seen / (double)per + (seen > (double)per ? 0.5 : 0.));
      work += rt * seen;
    }
    const double mean = work / ctas + 4, joined = parts > 1 ? ctas / 30 : 0;
    const double waves = std::ceil(ctas / n_sm) * mean, shared = (work + 4 * ctas) / n_sm + 0.5 * ((double)per + 4);
    const double cost = std::max(waves, shared) + joined;
    if (!best || cost < best_cost * 0.98) { best = (int)per; best_cost = cost; }
  }
  return best * kTileKeys;
}

// CTAs per unit of the row kernel's cluster form, or 0 for the line: units of at most `tiles` tiles.
int split_rows(int64_t units, int64_t tiles, int n_sm) {
  int split = 1;
  while (split < 8 && tiles > 2 * split && units * split * 2 <= n_sm) split *= 2;
  return tiles <= 16 * split ? split : 0;
}

tkphi_status plan_attend(const tkphi_paged_desc* kv, const PagedShape& sh, AttendPlan* pl) {
  const int n_sm = sm_count_current_device();
  *pl = AttendPlan{};
  int64_t longest_row = 0, longest = 0;
  for (int b = 0; b < kv->batch; ++b) {
    const int64_t q = kv->cu_q_host[b + 1] - kv->cu_q_host[b];
    if (q == 0) continue;
    const int64_t rows = q * sh.group, len = kv->kv_lens_host[b];
    if (rows > kRowsLimit) {
      pl->any_tiles = true;
      longest = std::max<int64_t>(longest, len > 0 ? (len + kTileKeys - 1) / kTileKeys : 1);
      continue;
    }
    const int64_t tiles = len > 0 ? (len + kRowKeys - 1) / kRowKeys : 1;
    pl->any_rows = true;
    pl->max_rows = (int)std::max<int64_t>(pl->max_rows, rows);
    pl->row_tiles += tiles * kv->n_kv_heads * ((rows + kRowTile - 1) / kRowTile);
    longest_row = std::max(longest_row, tiles);
  }
  if (pl->row_tiles > INT_MAX / 2) return fail(TKPHI_ERR_UNSUPPORTED, "too many key tiles for one call");
  const int units = kv->batch * kv->n_kv_heads;
  pl->row_split = split_rows(units, longest_row, n_sm);
  pl->row_ctas = pl->row_split ? 0 : (int)std::min<int64_t>(2 * n_sm, pl->row_tiles);
  pl->row_grid = pl->row_split ? units * pl->row_split : pl->row_ctas;
  if (pl->any_tiles) {
    pl->chunk = choose_chunk(kv, sh, longest, n_sm);
    const int pair = 2 * tile_rows(sh.group);
    int64_t grid = 0;
    for (int b = 0; b < kv->batch; ++b) {
      const int64_t rows = (kv->cu_q_host[b + 1] - kv->cu_q_host[b]) * sh.group, len = kv->kv_lens_host[b];
      if (rows <= kRowsLimit) continue;
      const int64_t chunks = len > pl->chunk ? (len + pl->chunk - 1) / pl->chunk : 1;
      pl->max_chunks = (int)std::max<int64_t>(pl->max_chunks, chunks);
      grid += (rows + pair - 1) / pair * chunks * kv->n_kv_heads;
    }
    if (grid > INT_MAX / 2) return fail(TKPHI_ERR_UNSUPPORTED, "too many query rows for one call");
    pl->tile_grid = (int)grid;
  }
  size_t o = 0;
  pl->row_part = o; o = align_up(o + sizeof(float) * 2 * pl->row_ctas * kRowTile * kv->head_dim, 256);
  pl->row_stat = o; o = align_up(o + sizeof(float) * 2 * pl->row_ctas * kRowTile * 2, 256);
  const size_t parts = pl->max_chunks > 1 ? (size_t)pl->tile_grid * kTileRows : 0;
  pl->tile_part = o; o = align_up(o + sizeof(float) * parts * kv->head_dim, 256);
  pl->tile_stat = o; o = align_up(o + sizeof(float) * parts * 2, 256);
  pl->total = std::max<size_t>(o, 256);
  return TKPHI_OK;
}

struct BlockPlan {
  int n_split, n_keep, key_stride, row_tiles, mag_parts;
  bool cluster;                  // the CTAs of a unit are a cluster and join their pieces themselves
  size_t scores, keys, mags, list, part, stat, total;
};

tkphi_status plan_block(const tkphi_paged_desc* kv, const PagedShape& sh, const tkphi_page_selection* sel, BlockPlan* pl) {
  if (!sel) return fail(TKPHI_ERR_INVALID_ARG, "selection is NULL");
  if (sel->n_sink_pages < 0 || sel->n_tail_pages < 1 || sel->topk_pages < 0)
    return fail(TKPHI_ERR_INVALID_ARG, "n_sink_pages (%d) and topk_pages (%d) must be >= 0, n_tail_pages (%d) >= 1",
                sel->n_sink_pages, sel->topk_pages, sel->n_tail_pages);
  const int64_t keep = (int64_t)sel->n_sink_pages + sel->n_tail_pages + sel->topk_pages;
  if (keep > (1 << 20)) return fail(TKPHI_ERR_UNSUPPORTED, "%lld selected pages > 2^20", (long long)keep);
  pl->n_keep = (int)keep;
  const int64_t units = (int64_t)sh.total_q * kv->n_kv_heads;
  const int64_t middle = sh.max_pages_seq - sel->n_sink_pages - sel->n_tail_pages;
  if (sh.max_pages_seq > kMaxSelectPages)
    return fail(TKPHI_ERR_UNSUPPORTED, "%lld pages in a sequence > %d", (long long)sh.max_pages_seq, kMaxSelectPages);
  pl->key_stride = (int)((std::max<int64_t>(middle > sel->topk_pages ? middle : 0, 1) + 3) & ~(int64_t)3);
  const int64_t tiles = ((std::min<int64_t>(keep, std::max<int64_t>(sh.max_pages_seq, 1)) << sh.page_shift) + kRowKeys - 1) / kRowKeys;
  const int n_sm = sm_count_current_device();
  pl->n_split = split_rows(units, tiles, n_sm);
  pl->cluster = pl->n_split > 0;
  if (!pl->cluster) pl->n_split = (int)std::max<int64_t>(1, std::min<int64_t>((tiles + 1) / 2, units > 0 ? 2 * n_sm / units : 1));
  size_t o = 0;
  // score row tiles: tokens of one sequence, 16 rows at a time
  const int tpt = kRowTile / padded_group(sh.group);
  int64_t row_tiles = 0;
  for (int b = 0; b < kv->batch; ++b) row_tiles += (kv->cu_q_host[b + 1] - kv->cu_q_host[b] + tpt - 1) / tpt;
  pl->row_tiles = (int)row_tiles;
  pl->mag_parts = paged_score_parts(pl->row_tiles, kv->n_kv_heads, pl->key_stride);
  pl->scores = o; o = align_up(o + sizeof(float) * units * pl->key_stride, 256);
  pl->keys = o; o = align_up(o + sizeof(unsigned long long) * units * pl->key_stride, 256);
  pl->mags = o; o = align_up(o + 16 * units * pl->mag_parts, 256);
  pl->list = o; o = align_up(o + sizeof(int) * units * pl->n_keep, 256);
  const size_t parts = pl->n_split > 1 && !pl->cluster ? (size_t)units * pl->n_split : 0;
  pl->part = o; o = align_up(o + sizeof(float) * parts * kRowTile * kv->head_dim, 256);
  pl->stat = o; o = align_up(o + sizeof(float) * parts * kRowTile * 2, 256);
  pl->total = std::max<size_t>(o, 256);
  return TKPHI_OK;
}

PagedProblem problem_of(const tkphi_paged_desc* kv, const PagedShape& sh, const void* q, void* y, float* lse, float scale) {
  PagedProblem p{};
  p.batch = kv->batch; p.hq = kv->n_q_heads; p.hkv = kv->n_kv_heads; p.group = sh.group;
  p.page_shift = sh.page_shift; p.n_pages = kv->n_pages; p.max_pages = kv->max_pages;
  p.table = kv->page_table;
  p.kv_lens = reinterpret_cast<const long long*>(kv->kv_lens_dev);
  p.cu_q = reinterpret_cast<const long long*>(kv->cu_q_dev);
  p.max_kv = (int)sh.max_kv; p.total_q = sh.total_q;
  p.q = q; p.y = y; p.lse = lse;
  p.scale_log2 = (scale == 0.f ? 1.0f / sqrtf((float)kv->head_dim) : scale) * kLog2e;
  p.causal = 1;
  p.status = kv->status;
  p.bounds = kv->key_bounds;
  return p;
}

tkphi_status check_io(const void* q, const void* y, const float* lse, float scale) {
  if (!q || !aligned16(q)) return fail(TKPHI_ERR_INVALID_ARG, "q is NULL or not 16-byte aligned");
  if (!y || !aligned16(y)) return fail(TKPHI_ERR_INVALID_ARG, "y_out is NULL or not 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(lse) & 3u) return fail(TKPHI_ERR_INVALID_ARG, "lse_out must be 4-byte aligned");
  if (!std::isfinite(scale) || scale < 0.f) return fail(TKPHI_ERR_INVALID_ARG, "scale must be finite and positive (0: 1/sqrt(head_dim))");
  return TKPHI_OK;
}

}  // namespace

extern "C" {

size_t tkphi_paged_workspace_bytes(const tkphi_paged_desc* kv, const tkphi_page_selection* selection, int which) {
  clear_error();
  PagedShape sh{};
  if (which == TKPHI_WS_PAGED_ATTENTION) {
    AttendPlan pl{};
    // the size does not depend on the mask, so that the looser rule of the lengths is enough
    if (validate_paged(kv, &sh, false, true) != TKPHI_OK || plan_attend(kv, sh, &pl) != TKPHI_OK) return 0;
    return pl.total;
  }
  if (which == TKPHI_WS_PAGED_BLOCK_ATTENTION) {
    BlockPlan pl{};
    if (validate_paged(kv, &sh, false, false) != TKPHI_OK || plan_block(kv, sh, selection, &pl) != TKPHI_OK) return 0;
    return pl.total;
  }
  fail(TKPHI_ERR_INVALID_ARG, "unknown workspace kind %d", which);
  return 0;
}

tkphi_status tkphi_paged_append(const tkphi_paged_desc* kv, const tkphi_append_desc* step, void* cuda_stream) {
  clear_error();
  PagedShape sh{};
  tkphi_status st = validate_paged(kv, &sh, true, false);
  if (st != TKPHI_OK) return st;
  if (!step) return fail(TKPHI_ERR_INVALID_ARG, "step descriptor is NULL");
  if (sh.total_q == 0) return TKPHI_OK;
  if (!step->k_new || !step->v_new || !aligned16(step->k_new) || !aligned16(step->v_new))
    return fail(TKPHI_ERR_INVALID_ARG, "k_new or v_new is NULL or not 16-byte aligned");
  if ((step->q == nullptr) != (step->q_out == nullptr))
    return fail(TKPHI_ERR_INVALID_ARG, "q and q_out must both be NULL or both be given");
  if (!aligned16(step->q) || !aligned16(step->q_out)) return fail(TKPHI_ERR_INVALID_ARG, "q and q_out must be 16-byte aligned");
  if (step->rot_dim < 0 || step->rot_dim > kv->head_dim || step->rot_dim % 16 != 0)
    return fail(TKPHI_ERR_UNSUPPORTED, "rot_dim must be a multiple of 16 in [0, head_dim], got %d", step->rot_dim);
  if (step->rot_dim > 0 && (!step->inv_freq || (reinterpret_cast<uintptr_t>(step->inv_freq) & 3u)))
    return fail(TKPHI_ERR_INVALID_ARG, "inv_freq is NULL or not 4-byte aligned");
  if (reinterpret_cast<uintptr_t>(step->positions) & 7u) return fail(TKPHI_ERR_INVALID_ARG, "positions must be 8-byte aligned");
  if (step->pairs != 0 && step->pairs != 1) return fail(TKPHI_ERR_INVALID_ARG, "pairs must be 0 or 1, got %d", step->pairs);
  const int64_t strides[8] = {step->k_stride_token, step->k_stride_head, step->v_stride_token, step->v_stride_head,
                              step->q ? step->q_stride_token : 0, step->q ? step->q_stride_head : 0,
                              step->q ? step->o_stride_token : 0, step->q ? step->o_stride_head : 0};
  for (int64_t s : strides)
    if (s < 0 || s % 8 != 0 || s >= (1ll << 38))
      return fail(TKPHI_ERR_INVALID_ARG, "strides of the new tokens must be non-negative multiples of 8 elements below 2^38, got %lld", (long long)s);
  if (step->q && !disjoint(sh.total_q, step->o_stride_token, kv->n_q_heads, step->o_stride_head, 1, 0, kv->head_dim))
    return fail(TKPHI_ERR_INVALID_ARG, "the strides of q_out let elements share memory");
  if (step->q && step->q == step->q_out &&
      (step->q_stride_token != step->o_stride_token || step->q_stride_head != step->o_stride_head))
    return fail(TKPHI_ERR_INVALID_ARG, "q_out is q with other strides");
  int64_t items = 0;
  const int64_t span = std::max(kv->page_size, 64);          // positions of a CTA
  for (int b = 0; b < kv->batch; ++b) {
    const int64_t q = kv->cu_q_host[b + 1] - kv->cu_q_host[b];
    if (q > 0) items += ((q + span - 2) / span) + 1;
  }
  AppendProblem p{};
  p.batch = kv->batch; p.hq = kv->n_q_heads; p.hkv = kv->n_kv_heads; p.group = sh.group; p.d = kv->head_dim;
  p.page_shift = sh.page_shift; p.n_pages = kv->n_pages; p.max_pages = kv->max_pages;
  p.table = kv->page_table;
  p.kv_lens = reinterpret_cast<const long long*>(kv->kv_lens_dev);
  p.cu_q = reinterpret_cast<const long long*>(kv->cu_q_dev);
  p.max_kv = sh.max_kv;
  p.k = kv->k; p.v = kv->v;
  p.stride_page = kv->stride_page; p.stride_head = kv->stride_head; p.stride_token = kv->stride_token;
  p.k_new = step->k_new; p.k_new_token = step->k_stride_token; p.k_new_head = step->k_stride_head;
  p.v_new = step->v_new; p.v_new_token = step->v_stride_token; p.v_new_head = step->v_stride_head;
  p.q = step->q; p.q_token = step->q_stride_token; p.q_head = step->q_stride_head;
  p.q_out = step->q_out; p.q_out_token = step->o_stride_token; p.q_out_head = step->o_stride_head;
  p.inv_freq = step->inv_freq; p.rot = step->rot_dim; p.pairs = step->pairs;
  p.positions = reinterpret_cast<const long long*>(step->positions);
  p.bounds = kv->key_bounds;
  p.status = kv->status;
  p.items = (int)items;
  p.total_q = sh.total_q;
  cudaStream_t cs = reinterpret_cast<cudaStream_t>(cuda_stream);
  ScopedSpan sp(cs, TKPHI_KERNEL_PAGED_APPEND);
  const cudaError_t e = launch_paged_append(p, kv->dtype == TKPHI_DTYPE_BF16, cs);
  return e == cudaSuccess ? TKPHI_OK : cuda_fail(e, "paged append launch");
}

tkphi_status tkphi_paged_attention(const tkphi_paged_desc* kv, const void* q, void* y_out, float* lse_out, float scale,
                                   uint32_t flags, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  clear_error();
  if (flags & ~(uint32_t)TKPHI_FLAG_FULL_CONTEXT) return fail(TKPHI_ERR_INVALID_ARG, "unknown flag bits 0x%x", flags);
  PagedShape sh{};
  tkphi_status st = validate_paged(kv, &sh, true, (flags & TKPHI_FLAG_FULL_CONTEXT) != 0);
  if (st != TKPHI_OK) return st;
  if (sh.total_q == 0) return TKPHI_OK;
  st = check_io(q, y_out, lse_out, scale);
  if (st != TKPHI_OK) return st;
  AttendPlan pl{};
  st = plan_attend(kv, sh, &pl);
  if (st != TKPHI_OK) return st;
  st = check_ws(workspace, workspace_bytes, pl.total);
  if (st != TKPHI_OK) return st;
  CUtensorMap tk, tv;
  st = make_page_map(kv, kv->k, &tk);
  if (st != TKPHI_OK) return st;
  st = make_page_map(kv, kv->v, &tv);
  if (st != TKPHI_OK) return st;
  PagedProblem p = problem_of(kv, sh, q, y_out, lse_out, scale);
  p.causal = (flags & TKPHI_FLAG_FULL_CONTEXT) ? 0 : 1;
  char* w = static_cast<char*>(workspace);
  p.rows_limit = kRowsLimit;
  p.row_ctas = pl.row_ctas;
  p.n_split = pl.row_split;
  p.beside = pl.any_tiles ? 1 : 0;
  p.row_part = reinterpret_cast<float*>(w + pl.row_part);
  p.row_stat = reinterpret_cast<float*>(w + pl.row_stat);
  p.chunk = pl.chunk;
  p.tile_part = reinterpret_cast<float*>(w + pl.tile_part);
  p.tile_stat = reinterpret_cast<float*>(w + pl.tile_stat);
  const bool bf16 = kv->dtype == TKPHI_DTYPE_BF16;
  cudaStream_t cs = reinterpret_cast<cudaStream_t>(cuda_stream);
  // tiles, rows (may start beside the tiles' last CTAs), then the joins
  cudaError_t e = cudaSuccess;
  if (pl.any_tiles) {
    CUtensorMap tq;
    st = make_query_map(kv, sh, q, &tq);
    if (st != TKPHI_OK) return st;
    ScopedSpan sp(cs, TKPHI_KERNEL_PAGED_TILES);
    e = launch_paged_tiles(p, tk, tv, tq, kv->head_dim, bf16, pl.tile_grid, cs);
  }
  if (e == cudaSuccess && pl.any_rows) {
    ScopedSpan sp(cs, TKPHI_KERNEL_PAGED_ROWS);
    e = launch_paged_rows(p, tk, tv, kv->head_dim, bf16, false, pl.row_split > 0, pl.row_grid, cs);
  }
  if (e == cudaSuccess && pl.max_chunks > 1) {
    ScopedSpan sp(cs, TKPHI_KERNEL_PAGED_TILES);
    e = launch_paged_tiles_merge(p, kv->head_dim, bf16, cs);
  }
  if (e == cudaSuccess && pl.any_rows && !pl.row_split) {
    ScopedSpan sp(cs, TKPHI_KERNEL_PAGED_ROWS);
    e = launch_paged_rows_merge(p, kv->head_dim, bf16, false, kv->batch * kv->n_kv_heads, pl.max_rows, cs);
  }
  return e == cudaSuccess ? TKPHI_OK : cuda_fail(e, "paged attention launch");
}

tkphi_status tkphi_paged_block_attention(const tkphi_paged_desc* kv, const tkphi_page_selection* selection,
                                         const void* q, void* y_out, float* lse_out, int32_t* page_idx_out, float scale,
                                         void* workspace, size_t workspace_bytes, void* cuda_stream) {
  clear_error();
  PagedShape sh{};
  tkphi_status st = validate_paged(kv, &sh, true, false);
  if (st != TKPHI_OK) return st;
  if (!kv->key_bounds) return fail(TKPHI_ERR_INVALID_ARG, "key_bounds is NULL");
  if (sh.total_q == 0) return TKPHI_OK;
  st = check_io(q, y_out, lse_out, scale);
  if (st != TKPHI_OK) return st;
  BlockPlan pl{};
  st = plan_block(kv, sh, selection, &pl);
  if (st != TKPHI_OK) return st;
  st = check_ws(workspace, workspace_bytes, pl.total);
  if (st != TKPHI_OK) return st;
  if (reinterpret_cast<uintptr_t>(page_idx_out) & 3u) return fail(TKPHI_ERR_INVALID_ARG, "page_idx_out must be 4-byte aligned");
  CUtensorMap tk, tv;
  st = make_page_map(kv, kv->k, &tk);
  if (st != TKPHI_OK) return st;
  st = make_page_map(kv, kv->v, &tv);
  if (st != TKPHI_OK) return st;
  PagedProblem p = problem_of(kv, sh, q, y_out, lse_out, scale);
  char* w = static_cast<char*>(workspace);
  p.n_split = pl.n_split; p.n_keep = pl.n_keep;
  p.n_sink = selection->n_sink_pages; p.n_tail = selection->n_tail_pages; p.topk = selection->topk_pages;
  p.page_scores = reinterpret_cast<float*>(w + pl.scores);
  p.page_keys = reinterpret_cast<unsigned long long*>(w + pl.keys); p.key_stride = pl.key_stride;
  p.page_mags = reinterpret_cast<uint4*>(w + pl.mags); p.mag_parts = pl.mag_parts;
  p.page_list = reinterpret_cast<int*>(w + pl.list);
  p.page_out = page_idx_out;
  p.row_part = reinterpret_cast<float*>(w + pl.part);
  p.row_stat = reinterpret_cast<float*>(w + pl.stat);
  const bool bf16 = kv->dtype == TKPHI_DTYPE_BF16;
  const int units = sh.total_q * kv->n_kv_heads;
  cudaStream_t cs = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  {
    ScopedSpan sp(cs, TKPHI_KERNEL_PAGED_SELECT);
    e = launch_paged_select(p, kv->head_dim, bf16, (int)sh.max_pages_seq, pl.row_tiles, cs);
  }
  if (e != cudaSuccess) return cuda_fail(e, "page selection launch");
  {
    ScopedSpan sp(cs, TKPHI_KERNEL_PAGED_ROWS);
    e = launch_paged_rows(p, tk, tv, kv->head_dim, bf16, true, pl.cluster, units * pl.n_split, cs);
    if (e == cudaSuccess && pl.n_split > 1 && !pl.cluster) e = launch_paged_rows_merge(p, kv->head_dim, bf16, true, units, sh.group, cs);
  }
  if (e != cudaSuccess) return cuda_fail(e, "paged block attention launch");
  return TKPHI_OK;
}

}  // extern "C"
