// C ABI of the operators between ids, rows and gradients: embedding rows and
// their tables' gradients, norms around a block, the norm of all gradients.
#include <algorithm>
#include <cmath>
#include <vector>

#include "api_common.h"
#include "layer_ops.h"

using namespace stca;
using namespace stca::api;
using namespace stca::layers;

namespace {

constexpr int64_t kMaxRows = 0x7fff0000;  // rows, tokens or ids of one call

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool is_dtype(int t) { return t == STCA_F32 || t == STCA_BF16; }
int es_of(int dtype) { return dtype == STCA_BF16 ? 2 : 4; }

// Row stride: 0 = dense; else at least the row and a multiple of 16 bytes.
bool stride(int64_t given, int64_t d, int es, int64_t* out) {
  *out = given == 0 ? d : given;
  return *out >= d && *out * es % 16 == 0 && *out * es < (int64_t(1) << 24);
}

stca_status_t check_width(int32_t d, int32_t most) {
  if (d < 1) return STCA_ERR_INVALID_ARG;
  return d % 8 != 0 || d > most ? STCA_ERR_UNSUPPORTED : STCA_OK;
}

constexpr int kMaxEmbed = 8192, kMaxNorm = 4096;

// ---- embedding

stca_status_t check_grad(const stca_embed_grad_t* g, int64_t n) {
  if (!g || !is_dtype(g->dtype) || !std::isfinite(g->scale) || g->n_rows < 1 || n < 0) return STCA_ERR_INVALID_ARG;
  if (g->n_rows > kMaxRows || n > kMaxRows) return STCA_ERR_UNSUPPORTED;
  return check_width(g->d, kMaxEmbed);
}

struct GradLayout {
  size_t hdr, counts, bad, pairs[2], tokens, head_sum, slot[2], slot_val[2], total;
};

GradLayout grad_layout(const stca_embed_grad_t* g, int64_t n) {
  const EmbedGradPlan p = embed_grad_plan(n, static_cast<uint32_t>(g->n_rows), g->d, g->dtype);
  GradLayout l{};
  Bump m;
  l.hdr = m.take(sizeof(WsHeader));
  if (n > 0) {
    if (!p.small) {
      l.counts = m.take(4 * 256 * 256);
      l.bad = m.take(4 * static_cast<size_t>(p.blocks));
    }
    for (int i = 0; i < 2; ++i) l.pairs[i] = m.take(!p.small && i < p.passes ? 8 * static_cast<size_t>(n) : 0);
    l.tokens = m.take(8 * static_cast<size_t>(n));
    l.head_sum = m.take(p.small ? 0 : 4 * 256);
    const int64_t groups[2] = {p.groups > 1 ? p.groups : 0, p.groups > 1 && p.next_groups > 1 ? p.next_groups : 0};
    for (int i = 0; i < 2; ++i) {
      l.slot[i] = m.take(16 * static_cast<size_t>(groups[i]));
      l.slot_val[i] = m.take(8 * static_cast<size_t>(groups[i]) * g->d);
    }
  }
  l.total = m.off;
  return l;
}

stca_status_t embed_grad_call(const stca_embed_grad_t* g, const stca_embed_part_t* parts, int32_t n_parts,
                              EmbedGradArgs* a, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!g || n_parts < 1 || n_parts > kMaxParts || !parts || !ws || !aligned16(ws)) return STCA_ERR_INVALID_ARG;
  int64_t n = 0;
  for (int i = 0; i < n_parts; ++i) {
    const stca_embed_part_t& p = parts[i];
    if (p.n < 0 || (p.n > 0 && (!p.ids || !p.dout)) || !aligned4(p.ids) || !aligned16(p.dout)) return STCA_ERR_INVALID_ARG;
    if (p.n > kMaxRows) return STCA_ERR_UNSUPPORTED;
    n += p.n;
  }
  const stca_status_t s = check_grad(g, n);
  if (s != STCA_OK) return s;
  for (int i = 0; i < n_parts; ++i) {
    a->ids[i] = parts[i].ids;
    a->dout[i] = parts[i].dout;
    if (!stride(parts[i].ld, g->d, es_of(g->dtype), &a->ld[i])) return STCA_ERR_INVALID_ARG;
    a->end[i] = (i ? a->end[i - 1] : 0) + parts[i].n;
  }
  for (int i = n_parts; i < kMaxParts; ++i) a->end[i] = n;
  const GradLayout l = grad_layout(g, n);
  if (ws_bytes < l.total) return STCA_ERR_WORKSPACE;
  a->n = n;
  a->d = g->d;
  a->n_rows = static_cast<uint32_t>(g->n_rows);
  a->scale = g->scale;
  a->hdr = at<WsHeader>(ws, l.hdr);
  a->counts = at<int32_t>(ws, l.counts);
  a->bad = at<int32_t>(ws, l.bad);
  a->tokens = at<int2>(ws, l.tokens);
  a->head_sum = at<int32_t>(ws, l.head_sum);
  for (int i = 0; i < 2; ++i) {
    a->pairs[i] = at<uint64_t>(ws, l.pairs[i]);
    a->slot[i] = at<int2>(ws, l.slot[i]);
    a->slot_val[i] = at<float>(ws, l.slot_val[i]);
  }
  HIPCHK(embed_grad(*a, g->dtype, stream));
  return STCA_OK;
}

// ---- norms

stca_status_t check_norm(const stca_norm_t* m, int64_t n) {
  if (!m || !is_dtype(m->dtype) || (m->kind != STCA_NORM_RMS && m->kind != STCA_NORM_LAYER) || m->gate < STCA_GATE_NONE ||
      m->gate > STCA_GATE_SILU || !std::isfinite(m->scale) || !(m->eps >= 1e-20f) || !std::isfinite(m->eps) || n < 0)
    return STCA_ERR_INVALID_ARG;
  if (n > kMaxRows) return STCA_ERR_UNSUPPORTED;
  return check_width(m->d, kMaxNorm);
}

stca_status_t norm_call(const stca_norm_t* m, const stca_norm_in_t* in, int64_t n, NormArgs* a) {
  const stca_status_t s = check_norm(m, n);
  if (s != STCA_OK) return s;
  const int es = es_of(m->dtype);
  if (!in || (n > 0 && !in->x) || !aligned16(in->x) || !aligned16(in->block) || !aligned16(in->gate) ||
      !aligned4(in->pre_w) || !aligned4(in->pre_b) || !aligned4(in->post_w) || !aligned4(in->post_b) ||
      !aligned4(in->layer_scale) || !stride(in->ldx, m->d, es, &a->ldx) || !stride(in->ldblock, m->d, es, &a->ldb) ||
      !stride(in->ldgate, m->d, es, &a->ldg))
    return STCA_ERR_INVALID_ARG;
  // what belongs to the block is given with a block (of no rows: whatever the pointer)
  if (!in->block && n > 0 && (m->post || m->gate != STCA_GATE_NONE || in->layer_scale || !m->pre)) return STCA_ERR_INVALID_ARG;
  if ((m->gate != STCA_GATE_NONE && n > 0 && !in->gate) || (m->gate == STCA_GATE_NONE && in->gate) ||
      (!m->pre && (in->pre_w || in->pre_b)) || (!m->post && (in->post_w || in->post_b)))
    return STCA_ERR_INVALID_ARG;
  a->x = in->x;
  a->block = in->block;
  a->gate = in->gate;
  a->pre_w = in->pre_w;
  a->pre_b = in->pre_b;
  a->post_w = in->post_w;
  a->post_b = in->post_b;
  a->ls = in->layer_scale;
  a->n = n;
  a->d = m->d;
  a->layer = m->kind == STCA_NORM_LAYER;
  a->act = m->gate;
  a->post = m->post != 0;
  a->pre = m->pre != 0;
  a->scale = m->scale;
  a->eps = m->eps;
  return STCA_OK;
}

// ---- norm of all gradients

int64_t pieces_of(const stca_grad_t& g) { return ceil_div(g.n, kGradPiece); }

stca_status_t check_grads(const stca_grad_t* list, int32_t n) {
  if (n < 0 || (n > 0 && !list)) return STCA_ERR_INVALID_ARG;
  struct Span {
    uintptr_t at, end;
    bool out;
    int i;
  };
  std::vector<Span> spans;
  spans.reserve(2 * static_cast<size_t>(n));
  for (int i = 0; i < n; ++i) {
    const stca_grad_t& g = list[i];
    if (!is_dtype(g.dtype) || !is_dtype(g.out_dtype) || g.n < 0 || g.n > (int64_t(1) << 40) || (g.n > 0 && !g.g) ||
        (g.count && (g.row < 1 || g.n % g.row != 0 || !aligned4(g.count))))
      return STCA_ERR_INVALID_ARG;
    const uintptr_t p = reinterpret_cast<uintptr_t>(g.g), o = reinterpret_cast<uintptr_t>(g.out);
    if (p % es_of(g.dtype) != 0 || (g.out && o % es_of(g.out_dtype) != 0)) return STCA_ERR_INVALID_ARG;
    if (g.n == 0) continue;
    spans.push_back({p, p + static_cast<uintptr_t>(g.n) * es_of(g.dtype), false, i});
    if (!g.out) continue;
    if (o == p && g.dtype != g.out_dtype) return STCA_ERR_INVALID_ARG;
    spans.push_back({o, o + static_cast<uintptr_t>(g.n) * es_of(g.out_dtype), true, i});
  }
  // a result may lie exactly where its own gradient lies, and on nothing else
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.at != b.at ? a.at < b.at : a.out > b.out; });
  uintptr_t end_out = 0, end_in = 0;  // of the results (which are disjoint) and of the gradients so far
  int last_out = -1;
  for (const Span& s : spans) {
    if (s.out) {
      if (s.at < end_out || s.at < end_in) return STCA_ERR_INVALID_ARG;
      end_out = s.end;
      last_out = s.i;
    } else {
      if (s.at < end_out && (last_out != s.i || list[s.i].out != list[s.i].g)) return STCA_ERR_INVALID_ARG;
      end_in = std::max(end_in, s.end);
    }
  }
  return STCA_OK;
}

int launches_of(int32_t n) { return std::max(1, static_cast<int>(ceil_div(n, kGradsPerLaunch))); }

}  // namespace

extern "C" {

stca_status_t stca_embed_forward(const stca_embed_t* embed, const stca_embed_field_t* fields, int32_t n_fields, int64_t n,
                                 void* out, int64_t ldo, void* ws, hipStream_t stream) {
  if (!embed || !is_dtype(embed->table_dtype) || !is_dtype(embed->out_dtype) || !std::isfinite(embed->scale) ||
      n_fields < 1 || !fields || n < 0 || (n > 0 && !out) || !aligned16(out) || !aligned16(ws))
    return STCA_ERR_INVALID_ARG;
  const stca_status_t s = check_width(embed->d, kMaxEmbed);
  if (s != STCA_OK) return s;
  if (n_fields > kMaxFields || n > kMaxRows) return STCA_ERR_UNSUPPORTED;
  EmbedArgs a{};
  for (int f = 0; f < n_fields; ++f) {
    const stca_embed_field_t& t = fields[f];
    if (!t.table || !aligned16(t.table) || t.n_rows < 1 || (n > 0 && !t.ids) || !aligned4(t.ids) ||
        !stride(t.ld, embed->d, es_of(embed->table_dtype), &a.ld[f]))
      return STCA_ERR_INVALID_ARG;
    if (t.n_rows > kMaxRows) return STCA_ERR_UNSUPPORTED;
    a.table[f] = t.table;
    a.ids[f] = t.ids;
    a.n_rows[f] = static_cast<uint32_t>(t.n_rows);
  }
  if (!stride(ldo, embed->d, es_of(embed->out_dtype), &a.ldo)) return STCA_ERR_INVALID_ARG;
  a.n_fields = n_fields;
  a.d = embed->d;
  a.n = n;
  a.scale = embed->scale;
  a.out = out;
  a.hdr = static_cast<WsHeader*>(ws);
  HIPCHK(embed_forward(a, embed->table_dtype, embed->out_dtype, device_cus(), stream));
  return STCA_OK;
}

size_t stca_embed_grad_workspace_size(const stca_embed_grad_t* grad, int64_t n) {
  if (check_grad(grad, n) != STCA_OK) return 0;
  // (few ids are divided finer and may need more than many: a workspace for n serves fewer as well)
  return std::max(grad_layout(grad, n).total, grad_layout(grad, std::min<int64_t>(n, kEmbedSmall)).total);
}

stca_status_t stca_embed_grad_dense(const stca_embed_grad_t* grad, const stca_embed_part_t* parts, int32_t n_parts,
                                    float* dtable, int64_t ld, int accumulate, void* ws, size_t ws_bytes,
                                    hipStream_t stream) {
  EmbedGradArgs a{};
  if (!grad || !dtable || !aligned16(dtable)) return STCA_ERR_INVALID_ARG;
  if (!stride(ld, grad->d, 4, &a.ldt)) return STCA_ERR_INVALID_ARG;
  a.dtable = dtable;
  a.accumulate = accumulate != 0;
  return embed_grad_call(grad, parts, n_parts, &a, ws, ws_bytes, stream);
}

stca_status_t stca_embed_grad_sparse(const stca_embed_grad_t* grad, const stca_embed_part_t* parts, int32_t n_parts,
                                     int32_t* rows, float* grads, int32_t* count, void* ws, size_t ws_bytes,
                                     hipStream_t stream) {
  EmbedGradArgs a{};
  if (!rows || !aligned4(rows) || !grads || !aligned16(grads) || !count || !aligned4(count)) return STCA_ERR_INVALID_ARG;
  a.rows = rows;
  a.grads = grads;
  a.count = count;
  return embed_grad_call(grad, parts, n_parts, &a, ws, ws_bytes, stream);
}

stca_status_t stca_norm_forward(const stca_norm_t* norm, const stca_norm_in_t* in, int64_t n, void* h, int64_t ldh,
                                void* y, int64_t ldy, hipStream_t stream) {
  NormArgs a{};
  const stca_status_t s = norm_call(norm, in, n, &a);
  if (s != STCA_OK) return s;
  const int es = es_of(norm->dtype);
  if (!aligned16(h) || !aligned16(y) || (n > 0 && (in->block != nullptr) != (h != nullptr)) ||
      (n > 0 && a.pre != (y != nullptr)) || !stride(ldh, a.d, es, &a.ldh) || !stride(ldy, a.d, es, &a.ldy))
    return STCA_ERR_INVALID_ARG;
  a.h = h;
  a.y = y;
  HIPCHK(norm_forward(a, norm->dtype, device_cus(), stream));
  return STCA_OK;
}

size_t stca_norm_workspace_size(const stca_norm_t* norm, int64_t n) {
  if (check_norm(norm, n) != STCA_OK) return 0;
  Bump m;
  m.take(4 * static_cast<size_t>(std::max(1, norm_partials(n, norm->d, device_cus()))) * 5 * norm->d);
  return m.off;
}

stca_status_t stca_norm_backward(const stca_norm_t* norm, const stca_norm_in_t* in, int64_t n, const void* dh,
                                 int64_t lddh, const void* dy, int64_t lddy, const stca_norm_grads_t* grads, void* ws,
                                 size_t ws_bytes, hipStream_t stream) {
  NormArgs a{};
  const stca_status_t s = norm_call(norm, in, n, &a);
  if (s != STCA_OK) return s;
  const int es = es_of(norm->dtype);
  if (!grads || !aligned16(dh) || !aligned16(dy) || (n > 0 && a.pre != (dy != nullptr)) || (n > 0 && !a.pre && !dh) ||
      !stride(lddh, a.d, es, &a.lddh) || !stride(lddy, a.d, es, &a.lddy) || !aligned16(grads->dx) ||
      !aligned16(grads->dblock) || !aligned16(grads->dgate) || !stride(grads->lddx, a.d, es, &a.lddx) ||
      !stride(grads->lddblock, a.d, es, &a.lddb) || !stride(grads->lddgate, a.d, es, &a.lddg) ||
      !aligned4(grads->dpre_w) || !aligned4(grads->dpre_b) || !aligned4(grads->dpost_w) || !aligned4(grads->dpost_b) ||
      !aligned4(grads->dlayer_scale) || (n > 0 && ((grads->dblock && !a.block) || (grads->dgate && !a.act))) ||
      (!a.pre && (grads->dpre_w || grads->dpre_b)) || (!a.post && (grads->dpost_w || grads->dpost_b)) || !ws ||
      !aligned16(ws))
    return STCA_ERR_INVALID_ARG;
  if (ws_bytes < stca_norm_workspace_size(norm, n)) return STCA_ERR_WORKSPACE;
  a.dh = dh;
  a.dy = dy;
  a.dx = grads->dx;
  a.dblock = grads->dblock;
  a.dgate = grads->dgate;
  float* const sums[5] = {grads->dpre_w, grads->dpre_b, grads->dpost_w, grads->dpost_b, grads->dlayer_scale};
  for (int i = 0; i < 5; ++i) a.sums[i] = sums[i];
  a.part = static_cast<float*>(ws);
  HIPCHK(norm_backward(a, norm->dtype, device_cus(), stream));
  return STCA_OK;
}

size_t stca_clip_workspace_size(int32_t n_grads) {
  if (n_grads < 0) return 0;
  return 8 * static_cast<size_t>(launches_of(n_grads)) * kGradGroups;
}

stca_status_t stca_clip(const stca_grad_t* grads, int32_t n_grads, double max_norm, float* norm, void* ws,
                        size_t ws_bytes, hipStream_t stream) {
  if (!(max_norm > 0.) || !ws || !aligned16(ws) || !aligned4(norm)) return STCA_ERR_INVALID_ARG;
  stca_status_t s;
  try {
    s = check_grads(grads, n_grads);
  } catch (...) {  // (host memory for the list's intervals)
    s = STCA_ERR_UNSUPPORTED;
  }
  if (s != STCA_OK) return s;
  if (ws_bytes < stca_clip_workspace_size(n_grads)) return STCA_ERR_WORKSPACE;
  const int launches = launches_of(n_grads);
  int n_part = 0;
  for (int pass = 0; pass < 2; ++pass)
    for (int l = 0; l < launches; ++l) {
      ClipArgs a{};
      const int first = l * kGradsPerLaunch;
      a.n_t = std::min(n_grads - first, kGradsPerLaunch);
      bool writes = pass == 0;
      for (int i = 0; i < a.n_t; ++i) {
        const stca_grad_t& g = grads[first + i];
        a.t[i] = {g.g, g.out, g.count, g.n, g.row, (g.dtype == STCA_BF16 ? 1 : 0) | (g.out_dtype == STCA_BF16 ? 2 : 0), a.pieces};
        a.pieces += pieces_of(g);
        writes |= g.out != nullptr;
      }
      const int grid = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(a.pieces, kGradGroups)));
      a.max_norm = max_norm;
      if (pass == 0) {
        a.part = static_cast<double*>(ws) + n_part;
        n_part += grid;
        HIPCHK(clip_sum(a, grid, stream));
      } else {
        a.part = static_cast<double*>(ws);
        a.n_part = n_part;
        a.norm = l == 0 ? norm : nullptr;
        if (!writes) {
          if (!a.norm) continue;
          a.pieces = 0;
        }
        HIPCHK(clip_scale(a, a.pieces > 0 ? grid : 1, stream));
      }
    }
  return STCA_OK;
}

}  // extern "C"
