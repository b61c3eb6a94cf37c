// Attention of new tokens over keys and values kept in pages, and the write of new tokens into
// the pages (include/dsa3d_seq.h), gfx950 kernels.
//
// The heads of a group read the same keys, so a workgroup's rows are (token, head of the group)
// pairs of one request and key head: keys and values come from memory once for all of them.  Two
// forms: where requests have few rows (a token or a few each) a workgroup holds 32 rows and its
// four waves share out the keys of each tile, whose reading is the time; where they have many, it
// holds 128 rows, 32 per wave, and every wave takes every key.  Either way the keys of a long
// cache are dealt out in parts to several workgroups and a second kernel joins their results.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "seq_device.h"
#include "seq_internal.h"

namespace dsa3d {
namespace {

using namespace seq;

constexpr int kThreads = 256;
constexpr int kFewRows = 32, kManyRows = 128;
constexpr int kFewKeys = 128;  // keys per tile of the form with few rows: 32 per wave
constexpr int kRing = 4;       // row tables of tiles in flight

__device__ inline int div_by(uint32_t x, uint32_t mul, uint32_t shift) {
  return (int)(((uint64_t)x * mul) >> shift);
}

// One workgroup's rows and keys.
struct Span1 {
  int b, begin;      // request and its first new token
  int n, m, off;     // new tokens, held tokens (also those not attended to), position of token 0
  int r0, rows;      // first row of the tile, rows of the request
  int k_lo, k_hi;    // keys of this part that any of its rows sees
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
  s.k_lo = split * g.part;
  s.k_hi = min(hi, s.k_lo + g.part);
  return true;
}

// Cache rows (page * page_size + row) of keys base .. base + KT - 1 into tab; -1 where there is
// none (past the keys of this part, or a page number outside the tensors).  bad[wave]: whether one
// of the wave's 64 keys has none.  Called by the first KT threads' waves.
template <int KT>
__device__ inline void fill_rows(int* tab, int* bad, const PagedGeometry& g, const int32_t* pages,
                                 const Span1& s, int base) {
  if (threadIdx.x < KT) {
    const int j = base + (int)threadIdx.x;
    int row = -1;
    if (j < s.k_hi) {
      const int page = div_by(j, g.page_mul, g.page_shift);
      const int p = pages[(int64_t)s.b * g.max_pages + page];
      if (p >= 0 && p < g.num_pages) row = p * g.page_size + (j - page * g.page_size);
    }
    tab[threadIdx.x] = row;
    const int none = __any(row < 0) ? 1 : 0;
    if ((threadIdx.x & 63) == 0) bad[threadIdx.x >> 6] = none;
  }
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
// a sum each over their half of the keys).
struct Softmax {
  float top = -INFINITY, base = 0.0f, l = 0.0f;

  template <int DB>
  __device__ inline void step(float (&s)[16], f32x16_t (&o)[DB]) {
    float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
    for (int i = 3; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = pair_max(mx);
    const bool raise = mx > top + kSlack;
    if (__any(raise)) {
      const float corr = raise ? __builtin_amdgcn_exp2f(top - mx) : 1.0f;
      if (raise) top = base = mx;
      l *= corr;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= corr;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - base);
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

// Logits in base-2 units with bias and mask: element i is key kb + c_row(i), a row's token stands
// at position pos.  rows: the block's cache rows (-1: no key).
template <bool BIAS>
__device__ inline void finish_logits(float (&s)[16], const PagedGeometry& g, const float* tab,
                                     int head_in_group, int kb, int pos, int last, bool masked,
                                     const int* rows) {
  const int hh = (threadIdx.x & 63) >> 5;
  if constexpr (BIAS) {
    const float* t = tab + head_in_group * g.span;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      s[i] = fmaf(s[i], g.scale_log2,
                  t[min(max(kb + c_row(i, hh) - pos - g.rel_min, 0), g.span - 1)]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= g.scale_log2;
  }
  if (masked) {
    asm volatile("");  // a branch: blocks that every row sees do not pay for it
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (kb + c_row(i, hh) > last || rows[c_row(i, hh)] < 0) s[i] = -INFINITY;
  }
}

// ------------------------------------------------------------------------- many rows

template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2)))
void paged_rows_kernel(PagedGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                       const T* __restrict__ v, const int32_t* __restrict__ pages,
                       const int32_t* __restrict__ kv_lens, const int32_t* __restrict__ cu_q,
                       const float* __restrict__ table, const int32_t* __restrict__ map,
                       T* __restrict__ out, float* __restrict__ lse, float* __restrict__ part_o,
                       float* __restrict__ part_l) {
  constexpr int KT = Type<T>::kKeyTile;
  using Tl = Tile<T, D, KT>;
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = KT / 32;
  __shared__ __attribute__((aligned(16))) T Ks[2][Tl::kElems];
  __shared__ __attribute__((aligned(16))) T Vs[2][Tl::kElems];
  __shared__ int tab[kRing][KT];
  __shared__ int bad[kRing];
  extern __shared__ float bias[];

  Work w;
  if (!work_of(g.tiles, g.splits, w)) return;
  const int split = w.head - w.u * g.splits;
  Span1 s;
  if (!locate<kManyRows>(g, cu_q, kv_lens, w.slot, split, s)) return;
  const int ntiles = s.k_hi > s.k_lo ? (s.k_hi - s.k_lo + KT - 1) / KT : 0;
  for (int i = 0; i < 3 && i < ntiles; ++i)
    fill_rows<KT>(tab[i], &bad[i], g, pages, s, s.k_lo + i * KT);
  if constexpr (BIAS) fill_bias(bias, g, table, map, w.u);

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const int rw = s.r0 + wave * 32;
  const Row x = row_of(g, s, w.u, rw + (lane & 31));
  Frag qf[KS];
  load_frag<T, D>(qf, q + x.q_at, x.ok);
  const int pos = s.off + x.i;
  const int last = g.causal ? min(s.seen - 1, pos) : s.seen - 1;
  int wave_last = -1, all_see = s.seen - 1;
  if (rw < s.rows) {
    wave_last = s.seen - 1;
    if (g.causal) {
      all_see = min(all_see, s.off + div_by(rw, g.group_mul, g.group_shift));
      wave_last = min(wave_last, s.off + div_by(min(rw + 31, s.rows - 1), g.group_mul,
                                                g.group_shift));
    }
  }

  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16_t{};
  Softmax sm;
  const T *kp = k + w.u * D, *vp = v + w.u * D;
  uint4 kr[Tl::NL], vr[Tl::NL];
  __syncthreads();
  if (ntiles > 0) {
    Tl::load(kr, kp, g.ks, tab[0]);
    Tl::load(vr, vp, g.vs, tab[0]);
    Tl::store(Ks[0], kr);
    Tl::store(Vs[0], vr);
    if (ntiles > 1) {
      Tl::load(kr, kp, g.ks, tab[1]);
      Tl::load(vr, vp, g.vs, tab[1]);
    }
  }
  __syncthreads();
  for (int kt = 0; kt < ntiles; ++kt) {
    const T *kc = Ks[kt & 1], *vc = Vs[kt & 1];
    if (kt + 1 < ntiles) {
      Tl::store(Ks[(kt + 1) & 1], kr);
      Tl::store(Vs[(kt + 1) & 1], vr);
    }
    if (kt + 2 < ntiles) {
      Tl::load(kr, kp, g.ks, tab[(kt + 2) % kRing]);
      Tl::load(vr, vp, g.vs, tab[(kt + 2) % kRing]);
    }
    if (kt + 3 < ntiles)
      fill_rows<KT>(tab[(kt + 3) % kRing], &bad[(kt + 3) % kRing], g, pages, s,
                    s.k_lo + (kt + 3) * KT);
    const int kbase = s.k_lo + kt * KT;
    const int nb = wave_last < kbase ? 0 : min(NB, (wave_last - kbase) / 32 + 1);
    const bool some_bad = bad[kt % kRing] != 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (b >= nb) break;
      Frag a[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) a[ks] = Tl::a_rows(kc, b * 32, ks);
      f32x16_t acc = f32x16_t{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) acc = mfma(a[ks], qf[ks], acc);
      Frag av[DB][2];
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int p = 0; p < 2; ++p) av[db][p] = Tl::a_cols(vc, db * 32, b, p);
      float t[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) t[i] = acc[i];
      const int kb = kbase + b * 32;
      finish_logits<BIAS>(t, g, bias, x.head - w.u * g.group, kb, pos, last,
                          some_bad || kb + 31 > all_see, tab[kt % kRing] + b * 32);
      sm.step(t, o);
      Frag pf[2];
      to_frags(t, pf);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int p = 0; p < 2; ++p) o[db] = mfma(av[db][p], pf[p], o[db]);
    }
    __syncthreads();
  }
  const float ltot = pair_sum(sm.l);
  const float inv = ltot > 0.0f ? 1.0f / ltot : ltot;
  const float l2 = ltot == 0.0f ? -INFINITY : sm.base + __builtin_amdgcn_logf(ltot);
  if (!x.ok) return;
  if (g.splits == 1) {
#pragma unroll
    for (int db = 0; db < DB; ++db) store_block(out + x.out_at * D, db, o[db], inv);
    if (hh == 0 && lse != nullptr) lse[x.out_at] = l2 * kLn2;
  } else {
    const int64_t at = (int64_t)split * g.nq * g.H + x.out_at;
    if (ltot != 0.0f) {  // the join skips the parts of a row without keys
#pragma unroll
      for (int db = 0; db < DB; ++db) store_block(part_o + at * D, db, o[db], inv);
    }
    if (hh == 0) part_l[at] = l2;
  }
}

// ------------------------------------------------------------------------- few rows

template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2)))
void paged_keys_kernel(PagedGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                       const T* __restrict__ v, const int32_t* __restrict__ pages,
                       const int32_t* __restrict__ kv_lens, const int32_t* __restrict__ cu_q,
                       const float* __restrict__ table, const int32_t* __restrict__ map,
                       T* __restrict__ out, float* __restrict__ lse, float* __restrict__ part_o,
                       float* __restrict__ part_l) {
  constexpr int KT = kFewKeys;
  using Tl = Tile<T, D, KT>;
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32;
  // a tile of keys and one of values; at the end the four waves' results in float32
  __shared__ __attribute__((aligned(16))) T KV[2 * Tl::kElems];
  static_assert(sizeof(T) * 2 * Tl::kElems >= 4u * kFewRows * D * 4, "room for the results");
  __shared__ int tab[kRing][KT];
  __shared__ int bad[kRing][KT / 64];
  __shared__ float tops[4][kFewRows], totals[4][kFewRows];
  extern __shared__ float bias[];

  Work w;
  if (!work_of(g.tiles, g.splits, w)) return;
  const int split = w.head - w.u * g.splits;
  Span1 s;
  if (!locate<kFewRows>(g, cu_q, kv_lens, w.slot, split, s)) return;
  const int ntiles = s.k_hi > s.k_lo ? (s.k_hi - s.k_lo + KT - 1) / KT : 0;
  for (int i = 0; i < 3 && i < ntiles; ++i)
    fill_rows<KT>(tab[i], bad[i], g, pages, s, s.k_lo + i * KT);
  if constexpr (BIAS) fill_bias(bias, g, table, map, w.u);

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const Row x = row_of(g, s, w.u, s.r0 + (lane & 31));
  Frag qf[KS];
  load_frag<T, D>(qf, q + x.q_at, x.ok);
  const int pos = s.off + x.i;
  const int last = g.causal ? min(s.seen - 1, pos) : s.seen - 1;
  const int all_see = g.causal ? min(s.seen - 1, s.off + div_by(s.r0, g.group_mul, g.group_shift))
                               : s.seen - 1;

  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16_t{};
  Softmax sm;
  T *Ks = KV, *Vs = KV + Tl::kElems;
  const T *kp = k + w.u * D, *vp = v + w.u * D;
  uint4 kr[Tl::NL], vr[Tl::NL];
  __syncthreads();
  if (ntiles > 0) {
    Tl::load(kr, kp, g.ks, tab[0]);
    Tl::load(vr, vp, g.vs, tab[0]);
  }
  for (int kt = 0; kt < ntiles; ++kt) {
    Tl::store(Ks, kr);
    Tl::store(Vs, vr);
    if (kt + 1 < ntiles) {  // in flight while this tile is worked on
      Tl::load(kr, kp, g.ks, tab[(kt + 1) % kRing]);
      Tl::load(vr, vp, g.vs, tab[(kt + 1) % kRing]);
    }
    if (kt + 3 < ntiles)
      fill_rows<KT>(tab[(kt + 3) % kRing], bad[(kt + 3) % kRing], g, pages, s,
                    s.k_lo + (kt + 3) * KT);
    __syncthreads();
    const int kb = s.k_lo + kt * KT + wave * 32;
    if (kb < s.k_hi) {
      Frag a[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) a[ks] = Tl::a_rows(Ks, wave * 32, ks);
      f32x16_t acc = f32x16_t{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) acc = mfma(a[ks], qf[ks], acc);
      float t[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) t[i] = acc[i];
      finish_logits<BIAS>(t, g, bias, x.head - w.u * g.group, kb, pos, last,
                          bad[kt % kRing][wave / 2] != 0 || kb + 31 > all_see,
                          tab[kt % kRing] + wave * 32);
      sm.step(t, o);
      Frag pf[2];
      to_frags(t, pf);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int p = 0; p < 2; ++p) o[db] = mfma(Tl::a_cols(Vs, db * 32, wave, p), pf[p], o[db]);
    }
    __syncthreads();
  }

  // The four waves' sums join over a common maximum.
  const float lw = pair_sum(sm.l);
  if (hh == 0) {
    tops[wave][lane] = sm.top;
    totals[wave][lane] = lw;
  }
  __syncthreads();
  const int c = lane & 31;
  const float top = fmaxf(fmaxf(tops[0][c], tops[1][c]), fmaxf(tops[2][c], tops[3][c]));
  const float mine = sm.top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm.top - top);
  float* sums = reinterpret_cast<float*>(KV) + wave * kFewRows * D;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) {
      const int chunk = db * 8 + 2 * blk + hh;  // four channels; permuted against bank conflicts
      *reinterpret_cast<float4*>(sums + c * D + ((chunk ^ (c & 15)) << 2)) =
          make_float4(o[db][4 * blk] * mine, o[db][4 * blk + 1] * mine, o[db][4 * blk + 2] * mine,
                      o[db][4 * blk + 3] * mine);
    }
  __syncthreads();
  const int count = min(s.rows - s.r0, kFewRows);
  for (int e = threadIdx.x; e < count * (D / 4); e += kThreads) {
    const int r = e / (D / 4), chunk = e % (D / 4);
    const float tr = fmaxf(fmaxf(tops[0][r], tops[1][r]), fmaxf(tops[2][r], tops[3][r]));
    float total = 0.0f;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = tops[i][r] == -INFINITY ? totals[i][r]
                                              : totals[i][r] * __builtin_amdgcn_exp2f(tops[i][r] - tr);
      total += f;
      const float4 y = *reinterpret_cast<const float4*>(
          reinterpret_cast<const float*>(KV) + (i * kFewRows + r) * D + ((chunk ^ (r & 15)) << 2));
      sum.x += y.x;
      sum.y += y.y;
      sum.z += y.z;
      sum.w += y.w;
    }
    const float inv = total > 0.0f ? 1.0f / total : total;
    const float l2 = total == 0.0f ? -INFINITY
                                   : (tr == -INFINITY ? 0.0f : tr) + __builtin_amdgcn_logf(total);
    const float4 y = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
    const Row z = row_of(g, s, w.u, s.r0 + r);
    if (g.splits == 1) {
      T* to = out + z.out_at * D + chunk * 4;
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(to) = y;
      } else {
        const uint16_t h[4] = {to_bf16(y.x), to_bf16(y.y), to_bf16(y.z), to_bf16(y.w)};
        *reinterpret_cast<uint2*>(to) = __builtin_bit_cast(uint2, h);
      }
      if (chunk == 0 && lse != nullptr) lse[z.out_at] = l2 * kLn2;
    } else {
      const int64_t at = (int64_t)split * g.nq * g.H + z.out_at;
      if (total != 0.0f) *reinterpret_cast<float4*>(part_o + at * D + chunk * 4) = y;
      if (chunk == 0) part_l[at] = l2;
    }
  }
}

// Joins the parts of each row: weights 2^(l - max l), one wave per row.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(int64_t rows, int splits,
                                                              const float* __restrict__ part_o,
                                                              const float* __restrict__ part_l,
                                                              T* __restrict__ out,
                                                              float* __restrict__ lse) {
  constexpr int PER = D / 64;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (row >= rows) return;
  // lane s holds part s's log-sum-exp (at most 64 parts)
  const float mine = lane < splits ? part_l[lane * rows + row] : -INFINITY;
  float top = mine;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float weight = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - top);
  float total = weight;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
  float sum[PER] = {};
  for (int s = 0; s < splits; ++s) {
    const float ws = __shfl(weight, s);
    if (__shfl(mine, s) == -INFINITY) continue;  // nothing was written for this part
#pragma unroll
    for (int j = 0; j < PER; ++j)
      sum[j] = fmaf(ws, part_o[(s * rows + row) * D + lane * PER + j], sum[j]);
  }
  const float inv = total > 0.0f ? 1.0f / total : total;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const float y = sum[j] * inv;
    if constexpr (sizeof(T) == 4) out[row * D + lane * PER + j] = y;
    else out[row * D + lane * PER + j] = to_bf16(y);
  }
  if (lane == 0 && lse != nullptr)
    lse[row] = total == 0.0f ? -INFINITY
                             : ((top == -INFINITY ? 0.0f : top) + __builtin_amdgcn_logf(total)) * kLn2;
}

// ------------------------------------------------------------------------- append

// One wave per new token: finds its request and place, copies its row of k and v.
__global__ __launch_bounds__(kThreads) void paged_append_kernel(
    PagedGeometry g, int chunks, const uint4* __restrict__ k, const uint4* __restrict__ v,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ kv_lens,
    const int32_t* __restrict__ pages, uint4* __restrict__ k_pages, uint4* __restrict__ v_pages) {
  const int tok = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (tok >= g.nq) return;
  const int b = search(g.B, tok, [&](int i) { return cu_at(cu_q, i, g.nq); });
  if (b >= g.B) return;
  const int begin = cu_at(cu_q, b, g.nq), n = max(cu_at(cu_q, b + 1, g.nq), begin) - begin;
  const int64_t at = (int64_t)kv_lens[b] - n + (tok - begin);
  if (tok < begin || tok - begin >= n || at < 0 || at >= (int64_t)g.max_pages * g.page_size) return;
  const int page = div_by((uint32_t)at, g.page_mul, g.page_shift);
  const int p = pages[(int64_t)b * g.max_pages + page];
  if (p < 0 || p >= g.num_pages) return;
  const int64_t to = ((int64_t)p * g.page_size + (at - (int64_t)page * g.page_size)) * chunks;
  const uint4 *ks = k + tok * g.ks, *vs = v + tok * g.vs;  // strides in 16-byte chunks here
  for (int c = lane; c < chunks; c += 64) {
    const uint4 a = ks[c], e = vs[c];
    k_pages[to + c] = a;
    v_pages[to + c] = e;
  }
}

template <typename... A>
hipError_t launch(const void* fn, dim3 grid, size_t lds, hipStream_t s, A... args) {
  void* a[] = {(void*)&args...};
  return hipLaunchKernel(fn, grid, dim3(kThreads), a, lds, s);
}

size_t round_256(size_t x) { return (x + 255) & ~size_t(255); }

template <typename T, int D>
hipError_t forward_d(const PagedGeometry& g, const T* q, const T* k, const T* v,
                     const int32_t* pages, const int32_t* kv_lens, const int32_t* cu_q,
                     const float* table, const int32_t* map, T* out, float* lse, void* ws,
                     hipStream_t s) {
  const bool bias = g.nb > 0;
  const int64_t rows = (int64_t)g.nq * g.H;
  float* part_l = g.splits > 1 ? (float*)ws : nullptr;
  float* part_o = g.splits > 1 ? (float*)((char*)ws + round_256((size_t)g.splits * rows * 4))
                               : nullptr;
  const void* fn =
      g.tile == kFewRows
          ? (bias ? (const void*)&paged_keys_kernel<T, D, true>
                  : (const void*)&paged_keys_kernel<T, D, false>)
          : (bias ? (const void*)&paged_rows_kernel<T, D, true>
                  : (const void*)&paged_rows_kernel<T, D, false>);
  hipError_t e = launch(fn, dim3((unsigned)seq_blocks(g.tiles, g.splits)),
                        bias ? (size_t)g.group * g.span * 4 : 0, s, g, q, k, v, pages, kv_lens,
                        cu_q, table, map, out, lse, part_o, part_l);
  if (e == hipSuccess && g.splits > 1) {
    constexpr int per = kThreads / 64;
    e = launch((const void*)&paged_join_kernel<T, D>, dim3((unsigned)((rows + per - 1) / per)), 0,
               s, rows, g.splits, (const float*)part_o, (const float*)part_l, out, lse);
  }
  return e;
}

}  // namespace

// Rows per workgroup and parts of the keys.  32 rows where the requests have no more on average.
// Parts: enough that the key heads, tiles and parts make about kTarget workgroups (eight per
// compute unit, so that requests of different lengths even out), but none below kLeast keys, for
// which the float32 results a part writes and the join reads would weigh against its keys.
void paged_plan(PagedGeometry& g, bool) {
  constexpr int kTarget = 2048, kLeast = 512, kMost = 64;
  const int64_t rows = (int64_t)g.nq * g.group;
  g.tile = rows <= (int64_t)kFewRows * g.B ? kFewRows : kManyRows;
  const int64_t tiles = std::max<int64_t>((rows + g.tile - 1) / g.tile, std::min(g.B, g.nq));
  const int64_t want = kTarget / std::max<int64_t>(1, tiles * g.KH);
  const int most = std::min(kMost, std::max(1, g.max_kv / kLeast));
  g.splits = (int)std::min<int64_t>(std::max<int64_t>(want, 1), most);
  const int step = kFewKeys;  // parts begin at tiles
  g.part = (int)(((int64_t)g.max_kv + g.splits - 1) / g.splits + step - 1) / step * step;
  g.part = std::max(g.part, step);
  g.splits = std::max(1, (int)(((int64_t)g.max_kv + g.part - 1) / g.part));
  g.tiles = seq_spread(g.KH, (int)(rows / g.tile) + g.B + 1);
}

size_t paged_workspace(const PagedGeometry& g) {
  if (g.splits == 1) return 0;
  const size_t rows = (size_t)g.splits * g.nq * g.H;
  return round_256(rows * 4) + round_256(rows * g.D * 4);
}

hipError_t launch_paged_forward(const PagedGeometry& g, bool bf16, const void* q,
                                const void* k, const void* v, const int32_t* pages,
                                const int32_t* kv_lens, const int32_t* cu_q, const float* table,
                                const int32_t* map, void* out, float* lse, void* ws,
                                hipStream_t s) {
  if (g.nq == 0) return hipSuccess;
  typedef uint16_t B;
  typedef float F;
  if (bf16)
    return g.D == 64 ? forward_d<B, 64>(g, (const B*)q, (const B*)k, (const B*)v, pages, kv_lens,
                                        cu_q, table, map, (B*)out, lse, ws, s)
                     : forward_d<B, 128>(g, (const B*)q, (const B*)k, (const B*)v, pages, kv_lens,
                                         cu_q, table, map, (B*)out, lse, ws, s);
  return g.D == 64 ? forward_d<F, 64>(g, (const F*)q, (const F*)k, (const F*)v, pages, kv_lens,
                                      cu_q, table, map, (F*)out, lse, ws, s)
                   : forward_d<F, 128>(g, (const F*)q, (const F*)k, (const F*)v, pages, kv_lens,
                                       cu_q, table, map, (F*)out, lse, ws, s);
}

hipError_t launch_paged_append(const PagedGeometry& g0, bool bf16, const void* k, const void* v,
                               const int32_t* cu_q, const int32_t* kv_lens, const int32_t* pages,
                               void* k_pages, void* v_pages, hipStream_t s) {
  if (g0.nq == 0) return hipSuccess;
  PagedGeometry g = g0;
  const int per16 = bf16 ? 8 : 4;
  g.ks /= per16;
  g.vs /= per16;
  constexpr int per = kThreads / 64;
  return launch((const void*)&paged_append_kernel, dim3((unsigned)((g.nq + per - 1) / per)), 0, s,
                g, g.KH * g.D / per16, (const uint4*)k, (const uint4*)v, cu_q, kv_lens, pages,
                (uint4*)k_pages, (uint4*)v_pages);
}

}  // namespace dsa3d
