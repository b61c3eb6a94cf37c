// Device code shared by the paged attention kernels (paged.hip, paged_mx.hip): which rows and keys a
// workgroup has, the running softmax, the bias.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_rules.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace dsa3d {
namespace paged {

using namespace seq;

constexpr int kThreads = 256;

__device__ inline int div_by(uint32_t x, uint32_t mul, uint32_t shift) {
  return (int)(((uint64_t)x * mul) >> shift);
}

// One workgroup's rows and keys.
struct Span1 {
  int b, begin;      // request and its first new token
  int n, m, off;     // new tokens, held tokens (also those not attended to), position of token 0
  int r0, rows;      // first row of the tile, rows of the request
  int k_lo, k_hi;    // keys of this part that any of its rows sees
  bool only;         // this part has all of them: no join
  int seen;          // keys below this exist for the call
};

template <int TILE>
__device__ inline bool locate(const PagedGeometry& g, const int32_t* cu_q, const int32_t* kv_lens,
                              int slot, int split, Span1& s) {
  const Slot sq = find_slot<TILE>(cu_q, g.B, g.nq, g.group, slot);
  s.b = sq.b;
  s.begin = sq.begin;
  s.n = sq.end - sq.begin;
  s.rows = s.n * g.group;
  s.r0 = sq.tile * TILE;
  if (s.r0 >= s.rows) return false;
  s.m = sq.b < g.B ? max(__builtin_amdgcn_readfirstlane(kv_lens[sq.b]), 0) : 0;
  s.off = s.m - s.n;
  s.seen = sq.b < g.B ? min(s.m, g.max_kv) : 0;
  int hi = s.seen;
  if (g.causal) {
    const int i_last = div_by(min(s.r0 + TILE, s.rows) - 1, g.group_mul, g.group_shift);
    hi = min(hi, s.off + i_last + 1);
  }
  // The keys that the tile sees, in at most g.splits parts of at least g.part.
  constexpr int kStep = kFewKeys;  // parts begin at tiles
  const int even = (max(hi, 0) + g.splits - 1) / g.splits;
  const int part = max(g.part, (even + kStep - 1) / kStep * kStep);
  s.k_lo = min(split * (int64_t)part, (int64_t)max(hi, 0));
  s.k_hi = min((int64_t)hi, (int64_t)s.k_lo + part);
  s.only = hi <= part;
  return !(s.only && split > 0);
}

struct Row {
  int i, head;    // token of the request, head
  bool ok;
  int64_t q_at, out_at;
};
__device__ inline Row row_of(const PagedGeometry& g, const Span1& s, int u, int r) {
  Row x;
  x.ok = r < s.rows;
  const int rr = x.ok ? r : 0;
  x.i = div_by(rr, g.group_mul, g.group_shift);
  x.head = u * g.group + rr - x.i * g.group;
  const int64_t tok = s.begin + x.i;
  x.q_at = tok * g.qs + (int64_t)x.head * g.D;
  x.out_at = tok * g.H + x.head;
  return x;
}

// Running softmax of one query over 32-key blocks (lanes l and l ^ 32 keep identical maxima and
// a sum each over their half of the keys).  The logits are `scale` times the values given (base 2).
struct Softmax {
  float top = -INFINITY, base = 0.0f, l = 0.0f;

  template <int DB>
  __device__ inline void raise_to(const float (&s)[16], float scale, f32x16_t (&o)[DB]) {
    float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
    for (int i = 3; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = pair_max(mx) * scale;  // scale > 0
    const bool raise = mx > top + kSlack;
    if (__any(raise)) {
      const float corr = raise ? __builtin_amdgcn_exp2f(top - mx) : 1.0f;
      if (raise) top = base = mx;
      l *= corr;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= corr;
    }
  }
  __device__ inline void weigh(float (&s)[16], float scale) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale, -base));
      l += s[i];
    }
  }
};

// The bias of the group's heads by distance: [group][span].
__device__ inline void fill_bias(float* tab, const PagedGeometry& g, const float* table,
                                 const int32_t* map, int u) {
  for (int i = threadIdx.x; i < g.group * g.span; i += kThreads) {
    const int h = i / g.span;
    tab[i] = bias_of(table, map, g.H, g.nb, u * g.group + h, i - h * g.span);
  }
}

// The logits in base-2 units where there is a bias (their scale is 1 then): element i is key
// kb + c_row(i), the row's token stands at position pos.
__device__ inline void add_bias(float (&s)[16], const PagedGeometry& g, const float* tab,
                                int head_in_group, int kb, int pos) {
  const int hh = (threadIdx.x & 63) >> 5;
  const float* t = tab + head_in_group * g.span;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    s[i] = fmaf(s[i], g.scale_log2,
                t[min(max(kb + c_row(i, hh) - pos - g.rel_min, 0), g.span - 1)]);
}

}  // namespace paged
}  // namespace dsa3d
