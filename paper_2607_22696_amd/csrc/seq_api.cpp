// C-ABI entry points of the packed-sequence and paged attention: argument validation and dispatch.
// The operations and the conventions are described in include/dsa3d_seq.h.
#include "dsa3d_seq.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "api_util.h"
#include "seq_internal.h"

namespace {

using dsa3d::api::aligned;
using dsa3d::api::overlaps;
using dsa3d::api::Span;
using dsa3d::api::span_of;

constexpr int64_t kIndexLimit = 1ll << 31;
constexpr float kLog2e = 1.4426950408889634f;

// A row stride in elements: 0 selects the row itself.  Returns false for one below a row, not a
// multiple of 16 bytes, or of 16 MiB and more (offsets within a tile are 32 bits).
bool check_stride(int64_t given, int64_t row, int item, int64_t* stride) {
  *stride = given == 0 ? row : given;
  return *stride >= row && *stride < (1 << 24) / item && *stride * item % 16 == 0;
}

dsa3d_status check_heads(int32_t heads, int32_t kv_heads, int32_t head_dim, float scale,
                         dsa3d_dtype dtype) {
  if (heads < 1 || kv_heads < 1 || head_dim < 1 || heads % kv_heads != 0)
    return DSA3D_ERR_INVALID_SHAPE;
  if (!std::isfinite(scale) || scale < 0.0f) return DSA3D_ERR_INVALID_SHAPE;
  if (dtype != DSA3D_BF16 && dtype != DSA3D_F32) return DSA3D_ERR_UNSUPPORTED;
  if (head_dim != 64 && head_dim != 128) return DSA3D_ERR_UNSUPPORTED;
  return DSA3D_OK;
}

dsa3d_status check_bias(int32_t rel_min, int32_t rel_span, int32_t rel_buckets) {
  if (rel_buckets < 0) return DSA3D_ERR_INVALID_SHAPE;
  if (rel_buckets == 0) return DSA3D_OK;
  if (rel_span < 1 || rel_min < -(1 << 24) || rel_min > (1 << 24)) return DSA3D_ERR_INVALID_SHAPE;
  if (rel_span > DSA3D_SEQ_MAX_SPAN || rel_buckets > DSA3D_SEQ_MAX_BUCKETS)
    return DSA3D_ERR_UNSUPPORTED;
  return DSA3D_OK;
}

uint64_t strided_bytes(int64_t rows, int64_t stride, int64_t row, int item) {
  return rows > 0 ? (uint64_t)((rows - 1) * stride + row) * item : 0;
}

// Every output against every input and every other output.
dsa3d_status check_alias(const Span* in, int nin, const Span* outs, int nout) {
  for (int a = 0; a < nout; ++a) {
    if (outs[a].lo == outs[a].hi) continue;
    for (int b = 0; b < nin; ++b)
      if (in[b].lo != in[b].hi && overlaps(outs[a], in[b])) return DSA3D_ERR_ALIAS;
    for (int b = a + 1; b < nout; ++b)
      if (outs[b].lo != outs[b].hi && overlaps(outs[a], outs[b])) return DSA3D_ERR_ALIAS;
  }
  return DSA3D_OK;
}

struct SeqSizes {
  int item;
  uint64_t q, k, v, out, kv, lse, table, map, cu;  // bytes
};

dsa3d_status check_seq(const dsa3d_seq_desc* d, bool own_keys, dsa3d::SeqGeometry* g,
                       SeqSizes* s) {
  if (d == nullptr) return DSA3D_ERR_NULL_POINTER;
  if (d->batch < 1 || d->batch >= (1 << 24) || d->total_q < 0 || d->total_k < 0 ||
      (d->causal != 0 && d->causal != 1))
    return DSA3D_ERR_INVALID_SHAPE;
  dsa3d_status st = check_heads(d->heads, d->kv_heads, d->head_dim, d->scale, d->dtype);
  if (st == DSA3D_OK) st = check_bias(d->rel_min, d->rel_span, d->rel_buckets);
  if (st != DSA3D_OK) return st;
  if (own_keys && d->total_k != d->total_q) return DSA3D_ERR_INVALID_SHAPE;
  if ((int64_t)d->total_q * d->heads >= kIndexLimit ||
      (int64_t)d->total_k * d->kv_heads >= kIndexLimit)
    return DSA3D_ERR_INVALID_SHAPE;
  s->item = d->dtype == DSA3D_BF16 ? 2 : 4;
  const int64_t qrow = (int64_t)d->heads * d->head_dim, krow = (int64_t)d->kv_heads * d->head_dim;
  if (!check_stride(d->q_stride, qrow, s->item, &g->qs) ||
      !check_stride(d->k_stride, krow, s->item, &g->ks) ||
      !check_stride(d->v_stride, krow, s->item, &g->vs))
    return DSA3D_ERR_INVALID_SHAPE;
  g->B = d->batch;
  g->nq = d->total_q;
  g->nk = d->total_k;
  g->H = d->heads;
  g->KH = d->kv_heads;
  g->group = d->heads / d->kv_heads;
  g->D = d->head_dim;
  g->causal = d->causal;
  g->nb = d->rel_buckets;
  g->rel_min = d->rel_buckets > 0 ? d->rel_min : 0;
  g->span = d->rel_buckets > 0 ? d->rel_span : 1;
  g->scale = d->scale != 0.0f ? d->scale : 1.0f / std::sqrt((float)d->head_dim);
  g->scale_log2 = g->scale * kLog2e;
  g->q_tiles = dsa3d::seq_spread(g->KH, g->nq / dsa3d::kSeqTile + g->B + 1);
  g->k_tiles = dsa3d::seq_spread(g->KH, g->nk / dsa3d::kSeqTile + g->B + 1);
  g->parts = dsa3d::seq_backward_parts(*g, d->dtype == DSA3D_BF16);
  if (dsa3d::seq_blocks(g->q_tiles, g->group) > dsa3d::kMostBlocks ||
      dsa3d::seq_blocks(g->k_tiles, g->parts) > dsa3d::kMostBlocks)
    return DSA3D_ERR_INVALID_SHAPE;
  s->q = strided_bytes(d->total_q, g->qs, qrow, s->item);
  s->k = strided_bytes(d->total_k, g->ks, krow, s->item);
  s->v = strided_bytes(d->total_k, g->vs, krow, s->item);
  s->out = (uint64_t)d->total_q * qrow * s->item;
  s->kv = (uint64_t)d->total_k * krow * s->item;
  s->lse = (uint64_t)d->total_q * d->heads * 4;
  s->table = (uint64_t)d->rel_buckets * d->heads * 4;
  s->map = d->rel_buckets > 0 ? (uint64_t)d->rel_span * 4 : 0;
  s->cu = ((uint64_t)d->batch + 1) * 4;
  return DSA3D_OK;
}

bool missing(const void* p, uint64_t bytes) { return p == nullptr && bytes > 0; }

}  // namespace

extern "C" {

dsa3d_status dsa3d_seq_forward(const dsa3d_seq_desc* desc, const void* q, const void* k,
                               const void* v, const int32_t* cu_q, const int32_t* cu_k,
                               const float* bias_table, const int32_t* bias_map, void* out,
                               void* out_res, float* lse, hipStream_t stream) {
  dsa3d::SeqGeometry g;
  SeqSizes s;
  const dsa3d_status st = check_seq(desc, cu_k == nullptr, &g, &s);
  if (st != DSA3D_OK) return st;
  const bool bf16 = desc->dtype == DSA3D_BF16;
  if (out_res != nullptr && !bf16) return DSA3D_ERR_UNSUPPORTED;
  if (!cu_q || missing(q, s.q) || missing(k, s.k) || missing(v, s.v) || missing(out, s.out) ||
      missing(bias_table, s.table) || missing(bias_map, s.map))
    return DSA3D_ERR_NULL_POINTER;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) ||
      !aligned(out_res, 16) || !aligned(lse, 4) || !aligned(cu_q, 4) || !aligned(cu_k, 4) ||
      !aligned(bias_table, 4) || !aligned(bias_map, 4))
    return DSA3D_ERR_MISALIGNED;
  const Span in[] = {span_of(q, s.q),       span_of(k, s.k),
                     span_of(v, s.v),       span_of(cu_q, s.cu),
                     span_of(cu_k, cu_k ? s.cu : 0), span_of(bias_table, s.table),
                     span_of(bias_map, s.map)};
  const Span outs[] = {span_of(out, s.out), span_of(out_res, out_res ? s.out : 0),
                       span_of(lse, lse ? s.lse : 0)};
  const dsa3d_status al = check_alias(in, 7, outs, 3);
  if (al != DSA3D_OK) return al;
  const dsa3d::SeqTensors t = {q, k, v, cu_q, cu_k ? cu_k : cu_q, bias_table, bias_map};
  const hipError_t e = dsa3d::launch_seq_forward(g, bf16, t, out, out_res, lse, stream);
  return e == hipSuccess ? DSA3D_OK : DSA3D_ERR_DEVICE;
}

size_t dsa3d_seq_backward_workspace_size(const dsa3d_seq_desc* desc) {
  dsa3d::SeqGeometry g;
  SeqSizes s;
  if (check_seq(desc, false, &g, &s) != DSA3D_OK) return 0;
  return dsa3d::seq_backward_workspace(g, g.nb > 0);
}

dsa3d_status dsa3d_seq_backward(const dsa3d_seq_desc* desc, const void* q, const void* k,
                                const void* v, const int32_t* cu_q, const int32_t* cu_k,
                                const float* bias_table, const int32_t* bias_map, const void* out,
                                const void* out_res, const float* lse, const void* dout, void* dq,
                                void* dk, void* dv, float* d_table, void* workspace,
                                size_t workspace_bytes, hipStream_t stream) {
  dsa3d::SeqGeometry g;
  SeqSizes s;
  const dsa3d_status st = check_seq(desc, cu_k == nullptr, &g, &s);
  if (st != DSA3D_OK) return st;
  const bool bf16 = desc->dtype == DSA3D_BF16;
  if (out_res != nullptr && !bf16) return DSA3D_ERR_UNSUPPORTED;
  if (d_table != nullptr && g.nb == 0) return DSA3D_ERR_INVALID_SHAPE;
  if (!cu_q || missing(q, s.q) || missing(k, s.k) || missing(v, s.v) || missing(out, s.out) ||
      missing(lse, s.lse) || missing(dout, s.out) || missing(dq, s.out) || missing(dk, s.kv) ||
      missing(dv, s.kv) || missing(bias_table, s.table) || missing(bias_map, s.map))
    return DSA3D_ERR_NULL_POINTER;
  const uint64_t need = dsa3d::seq_backward_workspace(g, d_table != nullptr);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return DSA3D_ERR_WORKSPACE;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) ||
      !aligned(out_res, 16) || !aligned(dout, 16) || !aligned(dq, 16) || !aligned(dk, 16) ||
      !aligned(dv, 16) || !aligned(lse, 4) || !aligned(cu_q, 4) || !aligned(cu_k, 4) ||
      !aligned(bias_table, 4) || !aligned(bias_map, 4) || !aligned(d_table, 4) ||
      !aligned(workspace, 256))
    return DSA3D_ERR_MISALIGNED;
  const Span in[] = {span_of(q, s.q),
                     span_of(k, s.k),
                     span_of(v, s.v),
                     span_of(cu_q, s.cu),
                     span_of(cu_k, cu_k ? s.cu : 0),
                     span_of(bias_table, s.table),
                     span_of(bias_map, s.map),
                     span_of(out, s.out),
                     span_of(out_res, out_res ? s.out : 0),
                     span_of(lse, s.lse),
                     span_of(dout, s.out)};
  const Span outs[] = {span_of(dq, s.out), span_of(dk, s.kv), span_of(dv, s.kv),
                       span_of(d_table, d_table ? s.table : 0), span_of(workspace, need)};
  const dsa3d_status al = check_alias(in, 11, outs, 5);
  if (al != DSA3D_OK) return al;
  const dsa3d::SeqTensors t = {q, k, v, cu_q, cu_k ? cu_k : cu_q, bias_table, bias_map};
  const hipError_t e = dsa3d::launch_seq_backward(g, bf16, t, out, out_res, lse, dout, dq, dk, dv,
                                                  d_table, workspace, stream);
  return e == hipSuccess ? DSA3D_OK : DSA3D_ERR_DEVICE;
}

dsa3d_status dsa3d_relative_buckets(int32_t buckets, int32_t max_distance, int32_t both,
                                    int32_t* map, int32_t* rel_min, int32_t* rel_span) {
  if (!rel_min || !rel_span) return DSA3D_ERR_NULL_POINTER;
  if (buckets < 1 || max_distance < 1 || (both && buckets % 2 != 0))
    return DSA3D_ERR_INVALID_SHAPE;
  const int side = both ? buckets / 2 : buckets, exact_to = side / 2, wide = side - exact_to;
  if (side < 2 || max_distance <= exact_to) return DSA3D_ERR_INVALID_SHAPE;
  const int64_t span = (int64_t)max_distance * (both ? 2 : 1) + 1;
  if (span > DSA3D_SEQ_MAX_SPAN || buckets > DSA3D_SEQ_MAX_BUCKETS) return DSA3D_ERR_UNSUPPORTED;
  *rel_min = -max_distance;
  *rel_span = (int32_t)span;
  if (map == nullptr) return DSA3D_OK;
  // floor(wide log(n / e) / log(max / e)): the quotient is a whole number exactly where n stands
  // on a border, and 64-bit logarithms then miss it by less than 1e-9, so that anything so close
  // below a whole number is that number.
  const auto bucket = [&](int n) {
    if (n < exact_to) return n;
    const double x = wide * (std::log((double)n) - std::log((double)exact_to)) /
                     (std::log((double)max_distance) - std::log((double)exact_to));
    return exact_to + std::min(wide - 1, (int)std::floor(x + 1e-9));
  };
  for (int64_t i = 0; i < span; ++i) {
    const int d = (int)i - max_distance;  // key minus query
    map[i] = d <= 0 ? bucket(-d) : side + bucket(d);
  }
  return DSA3D_OK;
}

}  // extern "C"

// ---------------------------------------------------------------------------- paged

namespace {

struct PagedSizes {
  int item;
  uint64_t q, out, pages, cache, cu, lens, lse, table, map;
};

// x / d as (x * mul) >> shift, exact for 0 <= x < 2^31: with 2^(s-1) < d <= 2^s and
// mul = floor(2^(31+s) / d) + 1, the product exceeds x 2^(31+s) / d by at most x < 2^31 <=
// 2^(31+s) / d, less than the step to the next whole quotient.
void divisor(int d, uint32_t* mul, uint32_t* shift) {
  int s = 0;
  while ((1ll << s) < d) ++s;
  *mul = d == 1 ? 1u : (uint32_t)((1ull << (31 + s)) / d + 1);
  *shift = d == 1 ? 0 : 31 + s;
}

dsa3d_status check_paged(const dsa3d_paged_desc* d, bool append, dsa3d::PagedGeometry* g,
                         PagedSizes* s) {
  if (d == nullptr) return DSA3D_ERR_NULL_POINTER;
  if (d->batch < 1 || d->batch >= (1 << 24) || d->total_q < 0 || d->num_pages < 0 ||
      d->page_size < 1 || d->max_pages < 0 || d->max_kv < 0 ||
      (d->causal != 0 && d->causal != 1))
    return DSA3D_ERR_INVALID_SHAPE;
  const int32_t heads = append ? d->kv_heads : d->heads;
  dsa3d_status st = check_heads(heads, d->kv_heads, d->head_dim, d->scale, d->dtype);
  if (st == DSA3D_OK && !append) st = check_bias(d->rel_min, d->rel_span, d->rel_buckets);
  if (st != DSA3D_OK) return st;
  if ((int64_t)d->num_pages * d->page_size >= kIndexLimit ||
      (int64_t)d->total_q * heads >= kIndexLimit)
    return DSA3D_ERR_INVALID_SHAPE;
  s->item = d->dtype == DSA3D_BF16 ? 2 : 4;
  const int64_t qrow = (int64_t)heads * d->head_dim, krow = (int64_t)d->kv_heads * d->head_dim;
  if (append) {
    g->qs = 0;
    if (!check_stride(d->k_stride, krow, s->item, &g->ks) ||
        !check_stride(d->v_stride, krow, s->item, &g->vs))
      return DSA3D_ERR_INVALID_SHAPE;
  } else {
    if (!check_stride(d->q_stride, qrow, s->item, &g->qs)) return DSA3D_ERR_INVALID_SHAPE;
    g->ks = g->vs = krow;
  }
  const int64_t held = (int64_t)d->max_pages * d->page_size;
  const int64_t most = d->num_pages == 0 ? 0  // no cache: no tokens
                       : d->max_kv > 0   ? std::min<int64_t>(d->max_kv, held)
                                         : held;
  if (!append && most > (1 << 30)) return DSA3D_ERR_INVALID_SHAPE;
  g->B = d->batch;
  g->nq = d->total_q;
  g->H = heads;
  g->KH = d->kv_heads;
  g->group = heads / d->kv_heads;
  g->D = d->head_dim;
  g->num_pages = d->num_pages;
  g->page_size = d->page_size;
  g->max_pages = d->max_pages;
  g->max_kv = (int)std::min<int64_t>(most, 1 << 30);
  divisor(g->page_size, &g->page_mul, &g->page_shift);
  divisor(g->group, &g->group_mul, &g->group_shift);
  g->causal = d->causal;
  g->nb = append ? 0 : d->rel_buckets;
  g->rel_min = g->nb > 0 ? d->rel_min : 0;
  g->span = g->nb > 0 ? d->rel_span : 1;
  if (g->nb > 0 && (int64_t)g->group * g->span > DSA3D_PAGED_MAX_BIAS)
    return DSA3D_ERR_UNSUPPORTED;
  g->scale = d->scale != 0.0f ? d->scale : 1.0f / std::sqrt((float)d->head_dim);
  g->scale_log2 = g->scale * kLog2e;
  dsa3d::set_plan(*g);
  if (!append && dsa3d::seq_blocks(g->tiles, g->splits) > dsa3d::kMostBlocks)
    return DSA3D_ERR_INVALID_SHAPE;
  s->q = strided_bytes(d->total_q, g->qs, qrow, s->item);
  s->out = (uint64_t)d->total_q * qrow * s->item;
  s->pages = (uint64_t)d->batch * d->max_pages * 4;
  s->cache = (uint64_t)d->num_pages * d->page_size * krow * s->item;
  s->cu = ((uint64_t)d->batch + 1) * 4;
  s->lens = (uint64_t)d->batch * 4;
  s->lse = (uint64_t)d->total_q * heads * 4;
  s->table = (uint64_t)g->nb * heads * 4;
  s->map = g->nb > 0 ? (uint64_t)g->span * 4 : 0;
  return DSA3D_OK;
}

}  // namespace

extern "C" {

dsa3d_status dsa3d_paged_append(const dsa3d_paged_desc* desc, const void* k, const void* v,
                                const int32_t* cu_q, const int32_t* kv_lens, const int32_t* pages,
                                void* k_pages, void* v_pages, hipStream_t stream) {
  dsa3d::PagedGeometry g;
  PagedSizes s;
  const dsa3d_status st = check_paged(desc, true, &g, &s);
  if (st != DSA3D_OK) return st;
  const int64_t row = (int64_t)g.KH * g.D;
  const uint64_t kb = strided_bytes(g.nq, g.ks, row, s.item),
                 vb = strided_bytes(g.nq, g.vs, row, s.item);
  if (!cu_q || !kv_lens || missing(k, kb) || missing(v, vb) || missing(pages, s.pages) ||
      missing(k_pages, s.cache) || missing(v_pages, s.cache))
    return DSA3D_ERR_NULL_POINTER;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) ||
      !aligned(cu_q, 4) || !aligned(kv_lens, 4) || !aligned(pages, 4))
    return DSA3D_ERR_MISALIGNED;
  const Span in[] = {span_of(k, kb), span_of(v, vb), span_of(cu_q, s.cu),
                     span_of(kv_lens, s.lens), span_of(pages, s.pages)};
  const Span outs[] = {span_of(k_pages, s.cache), span_of(v_pages, s.cache)};
  const dsa3d_status al = check_alias(in, 5, outs, 2);
  if (al != DSA3D_OK) return al;
  const hipError_t e =
      dsa3d::launch_paged_append(g, desc->dtype == DSA3D_BF16, k, v, cu_q, kv_lens, pages, k_pages,
                                 v_pages, stream);
  return e == hipSuccess ? DSA3D_OK : DSA3D_ERR_DEVICE;
}

size_t dsa3d_paged_forward_workspace_size(const dsa3d_paged_desc* desc) {
  dsa3d::PagedGeometry g;
  PagedSizes s;
  if (check_paged(desc, false, &g, &s) != DSA3D_OK) return 0;
  return dsa3d::paged_workspace(g);
}

dsa3d_status dsa3d_paged_forward(const dsa3d_paged_desc* desc, const void* q, const void* k_pages,
                                 const void* v_pages, const int32_t* pages,
                                 const int32_t* kv_lens, const int32_t* cu_q,
                                 const float* bias_table, const int32_t* bias_map, void* out,
                                 float* lse, void* workspace, size_t workspace_bytes,
                                 hipStream_t stream) {
  dsa3d::PagedGeometry g;
  PagedSizes s;
  const dsa3d_status st = check_paged(desc, false, &g, &s);
  if (st != DSA3D_OK) return st;
  if (!cu_q || !kv_lens || missing(q, s.q) || missing(out, s.out) || missing(pages, s.pages) ||
      missing(k_pages, s.cache) || missing(v_pages, s.cache) || missing(bias_table, s.table) ||
      missing(bias_map, s.map))
    return DSA3D_ERR_NULL_POINTER;
  const uint64_t need = dsa3d::paged_workspace(g);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return DSA3D_ERR_WORKSPACE;
  if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(out, 16) ||
      !aligned(lse, 4) || !aligned(cu_q, 4) || !aligned(kv_lens, 4) || !aligned(pages, 4) ||
      !aligned(bias_table, 4) || !aligned(bias_map, 4) || !aligned(workspace, 256))
    return DSA3D_ERR_MISALIGNED;
  const Span in[] = {span_of(q, s.q),
                     span_of(k_pages, s.cache),
                     span_of(v_pages, s.cache),
                     span_of(pages, s.pages),
                     span_of(kv_lens, s.lens),
                     span_of(cu_q, s.cu),
                     span_of(bias_table, s.table),
                     span_of(bias_map, s.map)};
  const Span outs[] = {span_of(out, s.out), span_of(lse, lse ? s.lse : 0),
                       span_of(workspace, need)};
  const dsa3d_status al = check_alias(in, 8, outs, 3);
  if (al != DSA3D_OK) return al;
  const hipError_t e = dsa3d::launch_paged_forward(
      g, desc->dtype == DSA3D_BF16, q, k_pages, v_pages, pages, kv_lens, cu_q, bias_table,
      bias_map, out, lse, workspace, stream);
  return e == hipSuccess ? DSA3D_OK : DSA3D_ERR_DEVICE;
}

}  // extern "C"
