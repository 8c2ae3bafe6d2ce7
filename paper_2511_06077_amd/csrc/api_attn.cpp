// C ABI of the stand-alone attention and of the paged history cache.  Every
// launch decision depends on the arguments alone: shapes, the batch and its
// host offsets where given.
#include <algorithm>
#include <cmath>

#include "api_common.h"
#include "attn_ops.h"

using namespace stca;
using namespace stca::api;
using namespace stca::ops;

namespace {

constexpr int64_t kMaxRows = 0x7fff0000;  // rows of one call: indices a few blocks past the end stay int32
constexpr int kNoHostChunks = 16;         // chunks per request where the host knows no lengths
constexpr int kMostChunks = 512;          // of a request, in a backward of several passes
constexpr int kMaxPagesOfChunk = 1024;    // a chunk's pages are listed in LDS

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int es_of(int dtype) { return dtype == STCA_BF16 ? 2 : 4; }

stca_status_t check_attn(const stca_attn_t* a) {
  if (!a || a->n_heads < 1 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads != 0 || a->d_head < 1 ||
      (a->dtype != STCA_F32 && a->dtype != STCA_BF16) || !std::isfinite(a->scale) || !std::isfinite(a->softcap) ||
      a->softcap < 0.f || a->n_buckets < 0 || a->n_buckets > kMaxBuckets)
    return STCA_ERR_INVALID_ARG;
  // (the factors that the kernels multiply scores by, see attn_fwd.h)
  const float most = std::fmax(std::fabs(a->scale), a->softcap) * kLog2e, in = std::fabs(a->scale) / a->softcap;
  if (!std::isfinite(most) || (a->softcap > 0.f && a->scale != 0.f && !std::isnormal(in))) return STCA_ERR_INVALID_ARG;
  if (a->n_buckets > 1) {
    if (!a->edges_host || a->edges_host[0] < 1) return STCA_ERR_INVALID_ARG;
    for (int i = 1; i < a->n_buckets - 1; ++i)
      if (a->edges_host[i] <= a->edges_host[i - 1]) return STCA_ERR_INVALID_ARG;
    if (a->edges_host[a->n_buckets - 2] == INT32_MAX) return STCA_ERR_INVALID_ARG;
  }
  if ((a->d_head != 32 && a->d_head != 64 && a->d_head != 128) || a->n_heads / a->n_kv_heads > kMaxGroup ||
      static_cast<int64_t>(a->n_heads) * a->d_head > 65536)
    return STCA_ERR_UNSUPPORTED;
  return STCA_OK;
}

stca_status_t check_rows_of(const stca_batch_t* b) {
  if (!b || b->n_requests < 1 || b->n_hist < 0 || b->n_tgt < 0 || !b->hist_off || !b->tgt_off ||
      (b->hist_off_host == nullptr) != (b->tgt_off_host == nullptr))
    return STCA_ERR_INVALID_ARG;
  if (b->n_hist > kMaxRows || b->n_tgt > kMaxRows) return STCA_ERR_UNSUPPORTED;
  if (b->hist_off_host) {
    const int32_t *h = b->hist_off_host, *t = b->tgt_off_host;
    if (h[0] != 0 || t[0] != 0 || h[b->n_requests] != b->n_hist || t[b->n_requests] != b->n_tgt)
      return STCA_ERR_INVALID_ARG;
    for (int r = 0; r < b->n_requests; ++r)
      if (h[r + 1] < h[r] || t[r + 1] < t[r]) return STCA_ERR_INVALID_ARG;
  }
  return STCA_OK;
}

stca_status_t check_cache(const stca_cache_t* c, bool pages) {
  if (!c || c->n_pages < 1 || c->n_kv_heads < 1 || c->d_head < 1 || c->page_size < 1 ||
      (c->format != STCA_CACHE_BF16 && c->format != STCA_CACHE_INT8))
    return STCA_ERR_INVALID_ARG;
  if ((c->d_head != 32 && c->d_head != 64 && c->d_head != 128) || c->page_size < 16 || c->page_size > 256 ||
      (c->page_size & (c->page_size - 1)) != 0 || static_cast<int64_t>(c->n_kv_heads) * c->d_head > 65536)
    return STCA_ERR_UNSUPPORTED;
  if (pages) {
    if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v) || !aligned4(c->pos)) return STCA_ERR_INVALID_ARG;
    if (c->format == STCA_CACHE_INT8 && (!c->k_exp || !c->v_exp || !aligned16(c->k_exp) || !aligned16(c->v_exp)))
      return STCA_ERR_INVALID_ARG;
  }
  return STCA_OK;
}

int shift_of(int page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}

// Row stride: 0 = dense; else at least the row and a multiple of 16 bytes.
bool stride(int64_t given, int64_t dense, int es, int64_t* out) {
  *out = given == 0 ? dense : given;
  return *out >= dense && *out * es % 16 == 0 && *out * es < (int64_t(1) << 24);
}

void fill_edges(const stca_attn_t* a, Buckets* b) {
  b->n = a->n_buckets;
  b->multi = 0;
  const int n = std::max(0, a->n_buckets - 1);
  for (int i = 0; i < n; ++i) b->edges[i] = a->edges_host[i];
  for (int i = n; i < kMaxBuckets; ++i) b->edges[i] = INT32_MAX;
  // an entry of the lookup holds one edge: which lowest x has not passed, but
  // the cell's other ones may
  for (int c = 0, k = 0; c < kHiddenCell; ++c) {
    const int64_t low = cell_low(c), last = cell_low(c + 1) - 1;
    while (k < n && b->edges[k] < low) ++k;
    b->cell[c] = static_cast<uint8_t>(k);
    if (k + 1 < n && b->edges[k + 1] < last) b->multi = 1;
  }
  b->cell[kHiddenCell] = 0;
}

struct Plan {
  int chunk, max_chunks, units, tiles, zgroups, btiles, passes, hw, part_tgt, max_tgt;
  size_t hdr, part_o, part_ml, part_dq, part_db, acc_kv, rows, total;
};

// Chunk length that gives about `per_cu` workgroups per CU, each of which is to
// have `rows` history rows times `per_row` workgroups to itself: a workgroup
// costs its start, the join of its waves and a partial to merge, and the last
// ones to run leave CUs idle, the less the more there are (window of 256
// requests, 16 targets, 2048 rows, d_h = 32, no bias: 4 a CU 139 us forward, 504
// backward, 8 128 and 291, 16 136 and 302).  Pages, whose chunks are whole runs of
// 256 rows, take 4: 128 requests of 10240 8-bit rows, 32 targets: 2 246 us, 4 246, 6
// 284, 8 255, one target 199, 199, 216, 185; 24 requests of 1 to 10240 bf16 rows of
// 128 features 160, 110, 153, 109, all of 10240 182, 190, 201, 214.
constexpr int kPackedPerCu = 8, kPagedPerCu = 4;
// ... and the fewest rows a wave is to have of it: shorter chunks are mostly
// start and join, longer ones leave CUs idle (64 requests of 1024 rows, 4 heads of
// 32, mask and 32 buckets: 64 rows 28.8 us forward, 128 25.0, 256 29.5; 32 rows 59.8
// backward, 64 54.8, 128 56.8).
constexpr int kWaveRows = 128, kWaveRowsBack = 64;
int chunk_for(int64_t rows, int64_t per_row, int per_cu, int step) {
  const int64_t want = static_cast<int64_t>(per_cu) * device_cus();
  const int64_t c = round_up(std::max<int64_t>(1, ceil_div(rows * per_row, want)), step);
  return static_cast<int>(std::min<int64_t>(c, kMaxRows / step * step));
}

// kv heads a workgroup takes: 32 features of bf16 are half a cache line, and a
// line whose other half another workgroup reads later comes from memory twice
// (window of 256 requests of 2048 rows, 8 heads of 32, no bias: 4 heads a workgroup
// 128 us forward, two 133, one 179; two 291 us backward, one 500).  In the backward
// two at most (registers fetch, and LDS holds, the rows of as many), and one where
// each holds four tiles; only where a wave to a head then has 256 history rows on every SIMD of
// the card, since fewer heads a workgroup are shorter chunks for as many waves;
// and no more than the LDS holds the tables of (`lds` of a workgroup of hw heads),
// forward of two workgroups, which is what the registers leave room for (32
// requests of 4096 rows, 4 x 32 heads of 128 features, 128 buckets: one of 4 heads
// a CU 342 us, two of 2 heads 151; 64 x 4096, 4 x 64 of 32: 840 and 406).
template <typename Lds>
int heads_of(int Hk, int64_t n_hist, bool backward, int tiles, Lds lds) {
  const int most = !backward ? 4 : tiles < 4 ? 2 : 1;
  int hw = most % 4 == 0 && Hk % 4 == 0 ? 4 : most % 2 == 0 && Hk % 2 == 0 ? 2 : 1;
  if (n_hist * Hk < 256 * 4 * static_cast<int64_t>(device_cus())) hw = 1;
  while (hw > 1 && lds(hw) > (backward ? kMaxLds : kMaxLds / 2)) hw /= 2;
  return hw;
}

// Rows of partials of chunks of that many rows (a row is a target's heads), and
// which of the two layouts (see part_row) has fewer.
int64_t part_rows_of(const stca_batch_t* b, int64_t max_m, int64_t max_l, int64_t chunk, int* part_tgt) {
  const int64_t chunks = ceil_div(max_l, chunk), flat = chunks * b->n_tgt, units = (b->n_hist / chunk + b->n_requests) * max_m;
  *part_tgt = chunks > 1 && units < flat ? static_cast<int>(max_m) : 0;
  return chunks > 1 ? std::min(flat, units) : 0;
}

// Partials that are always taken, and how many times what the batch's chunks and
// targets add up to, request by request: beyond both chunks become longer (one
// history of 32768 rows and 512 targets among 2047 of 256 rows and 16).
constexpr int64_t kFreePartials = 64 << 20;
constexpr int kSparePartials = 2;

bool ragged_plan(const stca_attn_t* a, const stca_batch_t* b, bool backward, Plan* p) {
  const int H = a->n_heads, Hk = a->n_kv_heads, G = H / Hk, dh = a->d_head;
  int64_t max_m = b->n_tgt, max_l = b->n_hist;
  if (b->hist_off_host) {
    max_m = max_l = 0;
    for (int r = 0; r < b->n_requests; ++r) {
      max_m = std::max<int64_t>(max_m, b->tgt_off_host[r + 1] - b->tgt_off_host[r]);
      max_l = std::max<int64_t>(max_l, b->hist_off_host[r + 1] - b->hist_off_host[r]);
    }
  }
  p->tiles = forward_tiles(a->dtype, dh, static_cast<int>(std::min<int64_t>(max_m * G, 1 << 20)), false);
  p->zgroups = static_cast<int>(std::min<int64_t>(std::max<int64_t>(1, ceil_div(max_m * G, 16 * p->tiles)),
                                                  b->hist_off_host ? 1024 : 8));
  const int64_t need = ceil_div(max_m, 16);
  p->btiles = backward_tiles(a->dtype, dh, static_cast<int>(std::min<int64_t>(need, 1 << 20)), G);
  p->passes = static_cast<int>(std::max<int64_t>(1, ceil_div(need, p->btiles) * G));
  auto lds = [&](int hw) {
    return backward ? backward_lds(a->dtype, dh, p->btiles, p->passes > 1 ? 2 : 1, hw, G, a->n_buckets)
                    : forward_lds(dh, hw, G, a->n_buckets, 0);
  };
  p->hw = backward && p->passes > 1 ? 1 : heads_of(Hk, b->n_hist, backward, p->btiles, lds);
  if (lds(p->hw) > kMaxLds) return false;
  const int parts = 4 / p->hw;
  if (backward && p->passes > 1) {
    // one step a wave, unless that makes more chunks than dq's partials are worth
    p->chunk = static_cast<int>(std::max<int64_t>(16 * parts, round_up(ceil_div(max_l, kMostChunks), 16 * parts)));
  } else {
    p->chunk = chunk_for(b->n_hist, static_cast<int64_t>(Hk / p->hw) * (backward ? 1 : p->zgroups), kPackedPerCu, 16 * parts);
    p->chunk = std::max(p->chunk, (backward ? kWaveRowsBack : kWaveRows) * parts);
  }
  if (!b->hist_off_host)
    p->chunk = static_cast<int>(std::max<int64_t>(p->chunk, round_up(ceil_div(b->n_hist, kNoHostChunks), 64)));
  p->chunk = static_cast<int>(std::min<int64_t>(p->chunk, std::max<int64_t>(64, round_up(max_l, 64))));
  int64_t parts_rows = part_rows_of(b, max_m, max_l, p->chunk, &p->part_tgt);
  if (b->hist_off_host && parts_rows * H * dh * 4 > kFreePartials) {
    int64_t own = 0;
    for (int r = 0; r < b->n_requests; ++r)
      own += std::max<int64_t>(1, ceil_div(b->hist_off_host[r + 1] - b->hist_off_host[r], p->chunk)) *
             (b->tgt_off_host[r + 1] - b->tgt_off_host[r]);
    const int64_t most = std::max(kSparePartials * own, kFreePartials / (static_cast<int64_t>(H) * dh * 4));
    while (parts_rows > most) {  // (two chunks are always few enough, so a chunk stays below 2^31 rows)
      p->chunk *= 2;
      parts_rows = part_rows_of(b, max_m, max_l, p->chunk, &p->part_tgt);
    }
  }
  p->max_chunks = static_cast<int>(std::max<int64_t>(1, ceil_div(max_l, p->chunk)));
  // (the layout by units has room for that many)
  p->max_tgt = p->part_tgt ? p->part_tgt : backward && p->passes == 1 ? 16 * p->btiles : INT32_MAX;
  const int64_t units = b->n_hist / p->chunk + b->n_requests;
  if (units * Hk * p->zgroups > 0x7f000000) return false;
  p->units = static_cast<int>(units);
  Bump m;
  p->hdr = m.take(sizeof(WsHeader));
  const size_t rows = static_cast<size_t>(b->n_tgt) * H, split = static_cast<size_t>(parts_rows) * H;
  if (!backward) {
    p->part_o = m.take(4 * split * dh);
    p->part_ml = m.take(8 * split);
  } else {
    p->rows = m.take(16 * rows);
    p->part_dq = m.take(4 * split * dh);
    p->part_db = m.take(4 * static_cast<size_t>(p->units) * H * a->n_buckets);
    p->acc_kv = m.take(p->passes > 1 && p->chunk > 16 * parts ? 8 * static_cast<size_t>(b->n_hist) * Hk * dh : 0);
  }
  p->total = m.off;
  return true;
}

void fill_attn(const stca_attn_t* a, AttnArgs* g) {
  g->H = a->n_heads;
  g->Hk = a->n_kv_heads;
  g->G = a->n_heads / a->n_kv_heads;
  g->masked = a->masked != 0;
  g->placed = a->masked != 0 || a->n_buckets > 0;
  g->scale = a->scale;
  g->cap = a->softcap;
  fill_edges(a, &g->b);
}

stca_status_t fill_ragged(const stca_attn_t* a, const stca_batch_t* b, const stca_attn_in_t* in, AttnArgs* g) {
  const int es = es_of(a->dtype);
  if (!in || (b->n_tgt > 0 && !in->q) || (b->n_hist > 0 && (!in->k || !in->v)) || !aligned16(in->q) ||
      !aligned16(in->k) || !aligned16(in->v) || !aligned4(in->tgt_pos) || !aligned4(in->hist_pos) ||
      !aligned4(in->bias))
    return STCA_ERR_INVALID_ARG;
  fill_attn(a, g);
  if ((g->placed && b->n_tgt > 0 && !in->tgt_pos) || (a->n_buckets > 0 && !in->bias)) return STCA_ERR_INVALID_ARG;
  if (!stride(in->ldq, static_cast<int64_t>(g->H) * a->d_head, es, &g->ldq) ||
      !stride(in->ldk, static_cast<int64_t>(g->Hk) * a->d_head, es, &g->ldk) ||
      !stride(in->ldv, static_cast<int64_t>(g->Hk) * a->d_head, es, &g->ldv))
    return STCA_ERR_INVALID_ARG;
  g->q = in->q;
  g->k = in->k;
  g->v = in->v;
  g->hist_off = b->hist_off;
  g->tgt_off = b->tgt_off;
  g->tgt_pos = in->tgt_pos;
  g->hist_pos = g->placed ? in->hist_pos : nullptr;
  g->bias = in->bias;
  g->R = b->n_requests;
  g->n_hist = b->n_hist;
  g->n_tgt = b->n_tgt;
  return STCA_OK;
}

bool saved_layout(const stca_attn_t* a, const stca_batch_t* b, stca_attn_saved_layout_t* s) {
  if (check_attn(a) != STCA_OK || check_rows_of(b) != STCA_OK) return false;
  const size_t rows = static_cast<size_t>(b->n_tgt) * a->n_heads;
  Bump m;
  s->a = m.take(4 * rows * a->d_head);
  s->max = m.take(4 * rows);
  s->sum = m.take(4 * rows);
  s->total = m.off;
  return true;
}

stca_status_t checked(const stca_attn_t* a, const stca_batch_t* b) {
  const stca_status_t s = check_attn(a);
  return s != STCA_OK ? s : check_rows_of(b);
}

bool paged_plan(const stca_attn_t* a, const stca_cache_t* c, const stca_cache_batch_t* b, Plan* p) {
  const int H = a->n_heads, Hk = a->n_kv_heads, G = H / Hk, dh = a->d_head;
  int64_t max_m = b->n_tgt;
  if (b->tgt_off_host) {
    max_m = 0;
    for (int r = 0; r < b->n_requests; ++r)
      max_m = std::max<int64_t>(max_m, b->tgt_off_host[r + 1] - b->tgt_off_host[r]);
  }
  p->tiles = forward_tiles(STCA_BF16, dh, static_cast<int>(std::min<int64_t>(max_m * G, 1 << 20)), true);
  p->zgroups = static_cast<int>(std::min<int64_t>(std::max<int64_t>(1, ceil_div(max_m * G, 16 * p->tiles)),
                                                  b->tgt_off_host ? 1024 : 8));
  p->chunk = chunk_for(static_cast<int64_t>(b->n_requests) * b->max_len, static_cast<int64_t>(Hk) * p->zgroups, kPagedPerCu, kPageStep);
  p->chunk = std::min(p->chunk, kMaxPagesOfChunk * c->page_size);
  p->chunk = static_cast<int>(std::min<int64_t>(p->chunk, std::max<int64_t>(kPageStep, round_up(b->max_len, kPageStep))));
  p->max_chunks = static_cast<int>(std::max<int64_t>(1, ceil_div(b->max_len, p->chunk)));
  const int64_t units = static_cast<int64_t>(b->n_requests) * p->max_chunks;
  if (units * Hk * p->zgroups > 0x7f000000) return false;
  p->units = static_cast<int>(units);
  p->hw = 1;  // (a head's pages are contiguous)
  if (forward_lds(dh, 1, G, a->n_buckets, p->chunk / c->page_size + 1) > kMaxLds) return false;
  Bump m;
  p->hdr = m.take(sizeof(WsHeader));
  const size_t rows = static_cast<size_t>(b->n_tgt) * H, split = p->max_chunks > 1 ? p->max_chunks : 0;
  p->part_o = m.take(4 * split * rows * dh);
  p->part_ml = m.take(8 * split * rows);
  p->total = m.off;
  return true;
}

stca_status_t check_paged(const stca_attn_t* a, const stca_cache_t* c, const stca_cache_batch_t* b, bool pages) {
  stca_status_t s = check_attn(a);
  if (s != STCA_OK) return s;
  s = check_cache(c, pages);
  if (s != STCA_OK) return s;
  if (!b || b->n_requests < 1 || b->n_tgt < 0 || b->max_len < 0 || b->table_ld < 0 || !b->tgt_off || !b->lens ||
      (b->max_len > 0 && !b->table) || static_cast<int64_t>(b->table_ld) * c->page_size < b->max_len ||
      a->n_kv_heads != c->n_kv_heads || a->d_head != c->d_head)
    return STCA_ERR_INVALID_ARG;
  if (a->dtype != STCA_BF16 || b->n_tgt > kMaxRows || b->max_len > kMaxRows) return STCA_ERR_UNSUPPORTED;
  if (b->tgt_off_host) {
    const int32_t* t = b->tgt_off_host;
    if (t[0] != 0 || t[b->n_requests] != b->n_tgt) return STCA_ERR_INVALID_ARG;
    for (int r = 0; r < b->n_requests; ++r)
      if (t[r + 1] < t[r]) return STCA_ERR_INVALID_ARG;
  }
  return STCA_OK;
}

stca_status_t move_rows(const stca_cache_t* c, const stca_cache_rows_t* rows, int32_t dtype, const void* k,
                        const void* v, int64_t ldk, int64_t ldv, const int32_t* pos, void* ws, bool write,
                        hipStream_t stream) {
  const stca_status_t s = check_cache(c, true);
  if (s != STCA_OK) return s;
  if (dtype != STCA_F32 && dtype != STCA_BF16) return STCA_ERR_INVALID_ARG;
  if (!rows || rows->n_requests < 1 || rows->n_rows < 0 || rows->table_ld < 0 || !rows->row_off || !rows->start ||
      (rows->n_rows > 0 && (!rows->table || !k || !v)) || !aligned16(k) || !aligned16(v) || !aligned4(pos) ||
      !aligned16(ws))
    return STCA_ERR_INVALID_ARG;
  if (rows->n_rows > kMaxRows) return STCA_ERR_UNSUPPORTED;
  CacheArgs a{};
  const int64_t dense = static_cast<int64_t>(c->n_kv_heads) * c->d_head;
  if (!stride(ldk, dense, es_of(dtype), &a.ldk) || !stride(ldv, dense, es_of(dtype), &a.ldv))
    return STCA_ERR_INVALID_ARG;
  a.k = c->k;
  a.v = c->v;
  a.ke = c->k_exp;
  a.ve = c->v_exp;
  a.pos = c->pos;
  a.xk = k;
  a.xv = v;
  a.xpos = pos;
  a.row_off = rows->row_off;
  a.start = rows->start;
  a.table = rows->table;
  a.table_ld = rows->table_ld;
  a.page_shift = shift_of(c->page_size);
  a.n_pages = c->n_pages;
  a.R = rows->n_requests;
  a.Hk = c->n_kv_heads;
  a.n_rows = rows->n_rows;
  a.hdr = static_cast<WsHeader*>(ws);
  if ((a.n_rows / 64 + 2 * static_cast<int64_t>(a.R)) * a.Hk > 0x7f000000) return STCA_ERR_UNSUPPORTED;
  HIPCHK(write ? cache_write(a, dtype, c->format == STCA_CACHE_INT8, c->d_head, stream)
               : cache_read(a, dtype, c->format == STCA_CACHE_INT8, c->d_head, stream));
  return STCA_OK;
}

}  // namespace

extern "C" {

size_t stca_attn_workspace_size(const stca_attn_t* attn, const stca_batch_t* batch, int with_backward) {
  Plan f, b;
  if (checked(attn, batch) != STCA_OK || !ragged_plan(attn, batch, false, &f)) return 0;
  if (!with_backward) return f.total;
  if (!ragged_plan(attn, batch, true, &b)) return 0;
  return std::max(f.total, b.total);
}

size_t stca_attn_saved_size(const stca_attn_t* attn, const stca_batch_t* batch) {
  stca_attn_saved_layout_t s;
  return saved_layout(attn, batch, &s) ? s.total : 0;
}

stca_status_t stca_attn_saved_layout(const stca_attn_t* attn, const stca_batch_t* batch,
                                     stca_attn_saved_layout_t* layout) {
  const stca_status_t s = checked(attn, batch);
  if (s != STCA_OK) return s;
  if (!layout) return STCA_ERR_INVALID_ARG;
  saved_layout(attn, batch, layout);
  return STCA_OK;
}

stca_status_t stca_attn_forward(const stca_attn_t* attn, const stca_batch_t* batch, const stca_attn_in_t* in,
                                void* out, void* saved, void* ws, size_t ws_bytes, hipStream_t stream) {
  stca_status_t s = checked(attn, batch);
  if (s != STCA_OK) return s;
  AttnArgs a{};
  s = fill_ragged(attn, batch, in, &a);
  if (s != STCA_OK) return s;
  if (!ws || !aligned16(ws) || !aligned16(saved) || !aligned16(out) || (batch->n_tgt > 0 && !out))
    return STCA_ERR_INVALID_ARG;
  Plan p;
  if (!ragged_plan(attn, batch, false, &p)) return STCA_ERR_UNSUPPORTED;
  if (ws_bytes < p.total) return STCA_ERR_WORKSPACE;
  a.chunk = p.chunk;
  a.max_chunks = p.max_chunks;
  a.units = p.units;
  a.hw = p.hw;
  a.zgroups = p.zgroups;
  a.max_tgt = p.max_tgt;
  a.part_tgt = p.part_tgt;
  a.out = out;
  if (saved) {
    stca_attn_saved_layout_t l;
    saved_layout(attn, batch, &l);
    a.sa = at<float>(saved, l.a);
    a.sm = at<float>(saved, l.max);
    a.sl = at<float>(saved, l.sum);
  }
  a.part_o = at<float>(ws, p.part_o);
  a.part_ml = at<float>(ws, p.part_ml);
  a.hdr = at<WsHeader>(ws, p.hdr);
  HIPCHK(attn_forward(a, attn->dtype, attn->d_head, p.tiles, stream));
  if (p.max_chunks > 1 && batch->n_tgt > 0) HIPCHK(attn_merge(a, attn->dtype == STCA_BF16, false, attn->d_head, stream));
  return STCA_OK;
}

stca_status_t stca_attn_backward(const stca_attn_t* attn, const stca_batch_t* batch, const stca_attn_in_t* in,
                                 const void* saved, const void* dout, const stca_attn_grads_t* grads, void* ws,
                                 size_t ws_bytes, hipStream_t stream) {
  stca_status_t s = checked(attn, batch);
  if (s != STCA_OK) return s;
  AttnArgs a{};
  s = fill_ragged(attn, batch, in, &a);
  if (s != STCA_OK) return s;
  const int es = es_of(attn->dtype);
  if (!ws || !aligned16(ws) || !saved || !aligned16(saved) || !aligned16(dout) || (batch->n_tgt > 0 && !dout) ||
      !grads || !aligned16(grads->dq) || !aligned16(grads->dk) || !aligned16(grads->dv) || !aligned4(grads->dbias) ||
      (batch->n_tgt > 0 && !grads->dq) || (batch->n_hist > 0 && (!grads->dk || !grads->dv)) ||
      (attn->n_buckets > 0 && !grads->dbias) ||
      !stride(grads->lddq, static_cast<int64_t>(a.H) * attn->d_head, es, &a.lddq) ||
      !stride(grads->lddk, static_cast<int64_t>(a.Hk) * attn->d_head, es, &a.lddk) ||
      !stride(grads->lddv, static_cast<int64_t>(a.Hk) * attn->d_head, es, &a.lddv))
    return STCA_ERR_INVALID_ARG;
  Plan p;
  if (!ragged_plan(attn, batch, true, &p)) return STCA_ERR_UNSUPPORTED;
  if (ws_bytes < p.total) return STCA_ERR_WORKSPACE;
  stca_attn_saved_layout_t l;
  saved_layout(attn, batch, &l);
  a.fa = at<float>(saved, l.a);
  a.fm = at<float>(saved, l.max);
  a.fl = at<float>(saved, l.sum);
  a.dout = dout;
  a.dq = grads->dq;
  a.dk = grads->dk;
  a.dv = grads->dv;
  a.dbias = grads->dbias;
  a.chunk = p.chunk;
  a.max_chunks = p.max_chunks;
  a.units = p.units;
  a.bufs = p.passes > 1 ? 2 : 1;
  a.hw = p.hw;
  a.zgroups = 1;
  a.max_tgt = p.max_tgt;
  a.part_tgt = p.part_tgt;
  a.part_dq = at<float>(ws, p.part_dq);
  a.part_db = at<float>(ws, p.part_db);
  a.acc_kv = at<float>(ws, p.acc_kv);
  a.rows = at<float>(ws, p.rows);
  a.hdr = at<WsHeader>(ws, p.hdr);
  HIPCHK(attn_backward(a, attn->dtype, attn->d_head, p.btiles, stream));
  return STCA_OK;
}

stca_status_t stca_bias_edges(int32_t n_buckets, int32_t n_exact, int32_t max_distance, int32_t* edges) {
  if (n_buckets < 2 || n_buckets > kMaxBuckets || n_exact < 1 || n_exact >= n_buckets || max_distance < n_buckets ||
      max_distance == INT32_MAX || !edges)
    return STCA_ERR_INVALID_ARG;
  const int n = n_buckets - 1;
  for (int i = 0; i < n; ++i) {
    int64_t e = i + 1;
    if (i >= n_exact)
      e = std::llround(n_exact * std::pow(static_cast<double>(max_distance) / n_exact,
                                          static_cast<double>(i - n_exact + 1) / (n - n_exact)));
    if (i > 0) e = std::max<int64_t>(e, edges[i - 1] + int64_t(1));
    edges[i] = static_cast<int32_t>(std::min<int64_t>(e, static_cast<int64_t>(max_distance) - (n - 1 - i)));
  }
  return STCA_OK;
}

stca_status_t stca_cache_write(const stca_cache_t* cache, const stca_cache_rows_t* rows, int32_t dtype,
                               const void* k, const void* v, int64_t ldk, int64_t ldv, const int32_t* pos,
                               void* ws, hipStream_t stream) {
  return move_rows(cache, rows, dtype, k, v, ldk, ldv, pos, ws, true, stream);
}

stca_status_t stca_cache_read(const stca_cache_t* cache, const stca_cache_rows_t* rows, int32_t dtype, void* k,
                              void* v, int64_t ldk, int64_t ldv, int32_t* pos, void* ws, hipStream_t stream) {
  return move_rows(cache, rows, dtype, k, v, ldk, ldv, pos, ws, false, stream);
}

size_t stca_cache_attn_workspace_size(const stca_attn_t* attn, const stca_cache_t* cache,
                                      const stca_cache_batch_t* batch) {
  Plan p;
  if (check_paged(attn, cache, batch, false) != STCA_OK || !paged_plan(attn, cache, batch, &p)) return 0;
  return p.total;
}

stca_status_t stca_cache_attn(const stca_attn_t* attn, const stca_cache_t* cache, const stca_cache_batch_t* batch,
                              const void* q, int64_t ldq, const int32_t* tgt_pos, const float* bias, void* out,
                              void* ws, size_t ws_bytes, hipStream_t stream) {
  const stca_status_t s = check_paged(attn, cache, batch, true);
  if (s != STCA_OK) return s;
  AttnArgs a{};
  fill_attn(attn, &a);
  if (!ws || !aligned16(ws) || !aligned16(q) || !aligned16(out) || !aligned4(tgt_pos) || !aligned4(bias) ||
      (batch->n_tgt > 0 && (!q || !out || (a.placed && !tgt_pos))) || (attn->n_buckets > 0 && !bias) ||
      !stride(ldq, static_cast<int64_t>(a.H) * attn->d_head, 2, &a.ldq))
    return STCA_ERR_INVALID_ARG;
  Plan p;
  if (!paged_plan(attn, cache, batch, &p)) return STCA_ERR_UNSUPPORTED;
  if (ws_bytes < p.total) return STCA_ERR_WORKSPACE;
  a.q = q;
  a.k = cache->k;
  a.v = cache->v;
  a.ke = cache->k_exp;
  a.ve = cache->v_exp;
  a.tgt_off = batch->tgt_off;
  a.tgt_pos = tgt_pos;
  a.hist_pos = a.placed ? cache->pos : nullptr;
  a.bias = bias;
  a.table = batch->table;
  a.table_ld = batch->table_ld;
  a.lens = batch->lens;
  a.max_len = batch->max_len;
  a.page_shift = shift_of(cache->page_size);
  a.n_pages = cache->n_pages;
  a.R = batch->n_requests;
  a.n_tgt = batch->n_tgt;
  a.chunk = p.chunk;
  a.max_chunks = p.max_chunks;
  a.units = p.units;
  a.hw = p.hw;
  a.zgroups = p.zgroups;
  a.max_tgt = INT32_MAX;
  a.out = out;
  a.part_o = at<float>(ws, p.part_o);
  a.part_ml = at<float>(ws, p.part_ml);
  a.hdr = at<WsHeader>(ws, p.hdr);
  HIPCHK(cache_attend(a, cache->format == STCA_CACHE_INT8, attn->d_head, p.tiles, stream));
  if (p.max_chunks > 1 && batch->n_tgt > 0) HIPCHK(attn_merge(a, true, true, attn->d_head, stream));
  return STCA_OK;
}

}  // extern "C"
