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

#include "paged_device.h"

namespace dsa3d {
namespace {

using namespace paged;

constexpr int kRing = 4;       // row tables of tiles in flight

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

// What the join reads of a part: its log-sum-exp (base 2); kDone as the first part's where the
// row needs no join.
constexpr float kDone = INFINITY;
__device__ inline float part_lse(float l2) { return l2 == INFINITY ? NAN : l2; }

// ------------------------------------------------------------------------- many rows

// Where the cache rows of the 64 keys from `base` on lie, in bytes, by the first wave.  A key
// without a place (past the part's keys, or a page number outside the tensors) gets the row of one
// that has one, so that what is copied is what some query sees, and is left out of the mask; a tile
// with none has mask 0 and rows that are never read.
template <typename T>
__device__ inline void fill_tile(int64_t* tab, uint64_t* mask, const PagedGeometry& g,
                                 const int32_t* pages, const Span1& s, int base, int keys) {
  if (threadIdx.x < 64) {
    const int j = base + (int)threadIdx.x;
    int row = -1;
    if ((int)threadIdx.x < keys && j < s.k_hi) {
      const int page = div_by(j, g.page_mul, g.page_shift);
      const int p = pages[(int64_t)s.b * g.max_pages + page];
      if (p >= 0 && p < g.num_pages) row = p * g.page_size + (j - page * g.page_size);
    }
    const uint64_t there = __ballot(row >= 0);
    const int some = there != 0 ? __shfl(row, __ffsll((unsigned long long)there) - 1) : 0;
    if ((int)threadIdx.x < keys)
      tab[threadIdx.x] = (row >= 0 ? row : some) * (g.ks * (int)sizeof(T));
    if (threadIdx.x == 0) *mask = there;
  }
}

// As the forward of seqattn.hip (tiles copied straight to LDS, a tile's second block multiplied
// beside the first one's softmax), through the page table.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2)))
void paged_rows_kernel(PagedGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                       const T* __restrict__ v, const int32_t* __restrict__ pages,
                       const int32_t* __restrict__ kv_lens, const int32_t* __restrict__ cu_q,
                       const float* __restrict__ table, const int32_t* __restrict__ map,
                       T* __restrict__ out, float* __restrict__ lse, float* __restrict__ part_o,
                       float* __restrict__ part_l) {
  constexpr int KT = kKeyTile<T, D>;
  using Tl = Tile<T, D, KT>;
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = KT / 32, E = Tl::kElems;
  __shared__ __attribute__((aligned(16))) T lds[Tl::kTwo];  // keys and values
  __shared__ int64_t tab[kRing][KT];
  __shared__ uint64_t there[kRing];
  extern __shared__ float bias[];

  Work w;
  if (!work_of(g.tiles, g.splits, w)) return;
  const int split = w.head - w.u * g.splits;
  Span1 s;
  if (!locate<kManyRows>(g, cu_q, kv_lens, w.slot, split, s)) return;
  const int ntiles = s.k_hi > s.k_lo ? (s.k_hi - s.k_lo + KT - 1) / KT : 0;
  for (int i = 0; i < 3 && i < ntiles; ++i)
    fill_tile<T>(tab[i], &there[i], g, pages, s, s.k_lo + i * KT, KT);
  if constexpr (BIAS) fill_bias(bias, g, table, map, w.u);

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const int rw = s.r0 + wave * 32;
  const bool live = rw < s.rows;
  const Row x = row_of(g, s, w.u, rw + (lane & 31));
  Frag qf[KS];
  load_frag<T, D>(qf, q + x.q_at, x.ok);
  const int pos = s.off + x.i;
  const int last = g.causal ? min(s.seen - 1, pos) : s.seen - 1;
  int wave_last = live ? s.seen - 1 : -1, all_see = s.seen - 1;
  if (live && g.causal) {
    all_see = min(all_see, s.off + div_by(rw, g.group_mul, g.group_shift));
    wave_last = min(wave_last, s.off + div_by(min(rw + 31, s.rows - 1), g.group_mul,
                                              g.group_shift));
  }

  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16_t{};
  Softmax sm;
  const T *kp = k + w.u * D, *vp = v + w.u * D;
  auto fetch = [&](int kt, int buf) {
    Tl::copy(lds + Tl::kPlace * buf, kp, lds + Tl::kPlace * buf + E, vp, tab[kt % kRing]);
  };
  auto products = [&](const uint16_t* kc, int b) {
    Frag a[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) a[ks] = Tl::a_rows(kc, b * 32, ks);
    f32x16_t acc = f32x16_t{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) acc = mfma(a[ks], qf[ks], acc);
    return acc;
  };
  const float scale = BIAS ? 1.0f : g.scale_log2;
  auto accumulate = [&](const uint16_t* vc, int b, const float (&t)[16]) {
    Frag pf[2];
    to_frags(t, pf);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        o[db] = mfma(Tl::a_cols(vc, db * 32, b, p), pf[p], o[db]);
  };
  auto advance = [&](int kt, int buf) {
    if (kt + 1 < ntiles) fetch(kt + 1, 1 - buf);
    if (kt + 3 < ntiles)
      fill_tile<T>(tab[(kt + 3) % kRing], &there[(kt + 3) % kRing], g, pages, s,
                s.k_lo + (kt + 3) * KT, KT);
  };
  auto mask_of = [&](int kt) {
    const uint64_t m = there[kt % kRing];
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(m >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
  };
  constexpr uint64_t kFull = ~0ull >> (64 - KT);

  __syncthreads();
  if (ntiles > 0) fetch(0, 0);
  wait_copies();
  __syncthreads();
  // Tiles that all of the workgroup's rows see whole, as in seqattn.hip's forward
  const int first_sees = g.causal ? s.off + div_by(s.r0, g.group_mul, g.group_shift) : s.seen - 1;
  const int whole = BIAS ? 0 : max(min(s.k_hi, first_sees + 1) - s.k_lo, 0) / KT;
  int kt = 0;
  while (kt < ntiles) {
    if constexpr (sizeof(T) == 2) {
      if ((kt & 1) == 0 && kt < whole && mask_of(kt) == kFull) {
        f32x16_t next = f32x16_t{};
        if (live) next = products(lds, 0);
        auto tile = [&](int t, int buf) {
          const T *kc = lds + 2 * E * buf, *kn = lds + 2 * E * (1 - buf);
          advance(t, buf);
  #pragma unroll
          for (int b = 0; b < NB; ++b) {
            float y[16];
            if (live) {
  #pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = next[i];
              sm.raise_to(y, scale, o);
            }
            if (b == NB - 1) {  // the next tile is in LDS
              wait_copies();
              __syncthreads();
            }
            if (live) {
              next = b + 1 < NB ? products(kc, b + 1) : products(kn, 0);
              sm.weigh(y, scale);
              accumulate(kc + E, b, y);
            }
          }
          __syncthreads();
        };
        do {
          tile(kt++, 0);
          if (kt >= whole || mask_of(kt) != kFull) break;
          tile(kt++, 1);
        } while (kt < whole && mask_of(kt) == kFull);
        continue;
      }
    }
    const uint16_t *kc = Tl::operands(lds, kt & 1), *vc = kc + Tl::kSecond;
    advance(kt, kt & 1);
    const int kbase = s.k_lo + kt * KT;
    const uint64_t mask = mask_of(kt);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int kb = kbase + b * 32;
      const uint32_t bits = (uint32_t)(mask >> (b * 32));
      if (bits == 0 || wave_last < kb) continue;
      const f32x16_t x0 = products(kc, b);
      float y[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = x0[i];
      if constexpr (BIAS) add_bias(y, g, bias, x.head - w.u * g.group, kb, pos);
      if (bits != ~0u || kb + 31 > all_see) {
        asm volatile("");  // a branch: blocks that every row sees do not pay for it
        const int seen = last - kb - 4 * hh;
        const uint32_t mine = bits >> (4 * hh);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c_row(i, 0) > seen || (mine >> c_row(i, 0) & 1) == 0) y[i] = -INFINITY;
      }
      sm.raise_to(y, scale, o);
      sm.weigh(y, scale);
      accumulate(vc, b, y);
    }
    wait_copies();
    __syncthreads();
    ++kt;
  }
  const float ltot = pair_sum(sm.l);
  const float inv = ltot > 0.0f ? 1.0f / ltot : ltot;
  const float l2 = ltot == 0.0f ? -INFINITY : sm.base + __builtin_amdgcn_logf(ltot);
  if (!x.ok) return;
  if (s.only) {
#pragma unroll
    for (int db = 0; db < DB; ++db) store_block(out + x.out_at * D, db, o[db], inv);
    if (hh == 0 && lse != nullptr) lse[x.out_at] = l2 * kLn2;
    if (hh == 0 && g.splits > 1) part_l[x.out_at * g.splits] = kDone;
  } else {
    const int64_t at = x.out_at * g.splits + split;
    if (ltot != 0.0f) {  // the join skips the parts of a row without keys
#pragma unroll
      for (int db = 0; db < DB; ++db) store_block(part_o + at * D, db, o[db], inv);
    }
    if (hh == 0) part_l[at] = part_lse(l2);
  }
}

// ------------------------------------------------------------------------- few rows

template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2)))
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
      for (int ks = 0; ks < KS; ++ks) a[ks] = Tl::rows_of(Ks, wave * 32, ks);
      f32x16_t acc = f32x16_t{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) acc = mfma(a[ks], qf[ks], acc);
      float t[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) t[i] = acc[i];
      if constexpr (BIAS) add_bias(t, g, bias, x.head - w.u * g.group, kb, pos);
      if (bad[kt % kRing][wave / 2] != 0 || kb + 31 > all_see) {
        asm volatile("");  // a branch: blocks that every row sees do not pay for it
        const int* rows = tab[kt % kRing] + wave * 32;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (kb + c_row(i, hh) > last || rows[c_row(i, hh)] < 0) t[i] = -INFINITY;
      }
      const float scale = BIAS ? 1.0f : g.scale_log2;
      sm.raise_to(t, scale, o);
      sm.weigh(t, scale);
      Frag pf[2];
      to_frags(t, pf);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int p = 0; p < 2; ++p) o[db] = mfma(Tl::cols_of(Vs, db * 32, wave, p), pf[p], o[db]);
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
      float f = totals[i][r];
      if (tops[i][r] != -INFINITY) f *= __builtin_amdgcn_exp2f(tops[i][r] - tr);
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
    if (s.only) {
      T* to = out + z.out_at * D + chunk * 4;
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(to) = y;
      } else {
        const uint16_t h[4] = {to_bf16(y.x), to_bf16(y.y), to_bf16(y.z), to_bf16(y.w)};
        *reinterpret_cast<uint2*>(to) = __builtin_bit_cast(uint2, h);
      }
      if (chunk == 0 && lse != nullptr) lse[z.out_at] = l2 * kLn2;
      if (chunk == 0 && g.splits > 1) part_l[z.out_at * g.splits] = kDone;
    } else {
      const int64_t at = z.out_at * g.splits + split;
      if (total != 0.0f) *reinterpret_cast<float4*>(part_o + at * D + chunk * 4) = y;
      if (chunk == 0) part_l[at] = part_lse(l2);
    }
  }
}

// Joins the parts of each row: weights 2^(l - max l).  One wave per row, a quarter or half of it
// per part, four channels per lane; rows that one workgroup finished are left as they are.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(int64_t rows, int splits,
                                                              const float* __restrict__ part_o,
                                                              const float* __restrict__ part_l,
                                                              T* __restrict__ out,
                                                              float* __restrict__ lse) {
  constexpr int LANES = D / 4, SIDES = 64 / LANES;  // lanes per part, parts at a time
  const int64_t row = (int64_t)block_number() * (kThreads / 64) + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, side = lane / LANES, c = lane % LANES * 4;
  if (row >= rows) return;
  // lane s holds part s's log-sum-exp (at most 64 parts)
  const float mine = lane < splits ? part_l[row * splits + lane] : -INFINITY;
  if (__shfl(mine, 0) == kDone) return;
  float top = mine;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float weight = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - top);
  float total = weight;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int s = side; s < splits; s += SIDES) {
    const float ws = __shfl(weight, s), ls = __shfl(mine, s);
    if (ls != -INFINITY) {  // else nothing was written for this part
      const float4 x = *reinterpret_cast<const float4*>(part_o + (row * splits + s) * D + c);
      sum.x = fmaf(ws, x.x, sum.x);
      sum.y = fmaf(ws, x.y, sum.y);
      sum.z = fmaf(ws, x.z, sum.z);
      sum.w = fmaf(ws, x.w, sum.w);
    }
  }
#pragma unroll
  for (int d = 32; d >= LANES; d >>= 1) {
    sum.x += __shfl_xor(sum.x, d);
    sum.y += __shfl_xor(sum.y, d);
    sum.z += __shfl_xor(sum.z, d);
    sum.w += __shfl_xor(sum.w, d);
  }
  const float inv = total > 0.0f ? 1.0f / total : total;
  if (side == 0) {
    T* to = out + row * D + c;
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(to) =
          make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
    } else {
      const uint16_t h[4] = {to_bf16(sum.x * inv), to_bf16(sum.y * inv), to_bf16(sum.z * inv),
                             to_bf16(sum.w * inv)};
      *reinterpret_cast<uint2*>(to) = __builtin_bit_cast(uint2, h);
    }
  }
  if (lane == 0 && lse != nullptr) {
    const float base = top == -INFINITY ? 0.0f : top;
    lse[row] = total == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

// ------------------------------------------------------------------------- append

// One wave per new token: finds its request and place, copies its row of k and v.
__global__ __launch_bounds__(kThreads) void paged_append_kernel(
    PagedGeometry g, int chunks, const uint4* __restrict__ k, const uint4* __restrict__ v,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ kv_lens,
    const int32_t* __restrict__ pages, uint4* __restrict__ k_pages, uint4* __restrict__ v_pages) {
  const int64_t at_row = (int64_t)block_number() * (kThreads / 64) + (threadIdx.x >> 6);
  if (at_row >= g.nq) return;
  const int tok = (int)at_row, lane = threadIdx.x & 63;
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
  hipError_t e = seq_launch(fn, g.blocks, kThreads,
                            bias ? (size_t)g.group * g.span * 4 : 0, s, g, q, k, v, pages, kv_lens,
                            cu_q, table, map, out, lse, part_o, part_l);
  if (e == hipSuccess && g.splits > 1) {
    constexpr int per = kThreads / 64;
    e = seq_launch((const void*)&paged_join_kernel<T, D>, (rows + per - 1) / per, kThreads, 0,
                   s, rows, g.splits, (const float*)part_o, (const float*)part_l, out, lse);
  }
  return e;
}

}  // namespace

void set_plan(PagedGeometry& g) {
  const PagedPlan p = paged_plan(g.nq, g.group, g.KH, g.B, g.max_kv);
  g.tile = p.tile;
  g.splits = p.splits;
  g.part = p.part;
  g.tiles = seq_spread(g.KH, (int)((int64_t)g.nq * g.group / g.tile) + g.B + 1);
  g.blocks = seq_blocks(g.tiles, g.splits);
  g.target = 0;
  g.room = 0;
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
  const int64_t blocks = ((int64_t)g.nq + per - 1) / per;
  return seq_launch((const void*)&paged_append_kernel, blocks, kThreads, 0, s, g,
                    g.KH * g.D / per16, (const uint4*)k, (const uint4*)v, cu_q, kv_lens, pages,
                    (uint4*)k_pages, (uint4*)v_pages);
}

}  // namespace dsa3d
