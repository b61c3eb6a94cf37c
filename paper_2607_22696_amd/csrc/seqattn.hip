// Attention of packed sequences, forward and backward (include/dsa3d_seq.h), gfx950 kernels.
//
// Forward: one pass over the keys with a running maximum and sum.  A workgroup takes 128 or 256
// queries of one head (waves of 32) and streams the keys its mask leaves through LDS.  Bound by
// the matrix cores and the vector ALU together: per 32 x 32 block at 128 channels 16 products
// (512 cycles) beside 57 vector instructions, 16 of them exponentials, and 24 LDS reads.  What
// staging and reading cost was measured by leaving each out of a copy (8,192 tokens, 16 heads x
// 128, 596 us with tiles loaded to registers and stored to LDS): without the staging 474 us,
// without the operand reads 446, without the softmax 521.  Copies straight to LDS, LDS places that
// are constants and the next block's products beside this one's exponentials take 491 us
// (1.12 PFLOP/s; a 16384^3 matrix product reaches 1.37).
// Backward without atomics: a pass over query tiles (dq, Delta, the bias gradient) and one over
// key tiles (dk, dv), each recomputing alpha = exp(t - lse).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <numeric>

#include "seq_device.h"
#include "seq_internal.h"

namespace dsa3d {
namespace {

using namespace seq;

constexpr int kThreads = 256;

// What a wave needs to know of the bias: the table by distance in LDS and its two ends, which all
// farther distances share.
struct Bias {
  const float* tab;
  float behind, ahead;
};

// Fills tab (span floats) with the bias of `head`.  A barrier follows before its use.
template <int THREADS = kThreads>
__device__ inline void fill_bias(float* tab, const SeqGeometry& g, const float* table,
                                 const int32_t* map, int head) {
  for (int i = threadIdx.x; i < g.span; i += THREADS)
    tab[i] = bias_of(table, map, g.H, g.nb, head, i);
}

// t = s scale (+ bias) in base-2 units for a 32 x 32 block whose distances run from d_lo to d_hi;
// dist(i) is element i's.
template <typename Dist>
__device__ inline void add_bias(float (&s)[16], const SeqGeometry& g, const float* tab, int d_lo,
                                int d_hi, const Dist& dist) {
  const int last = g.span - 1;
  if (d_hi <= g.rel_min || d_lo >= g.rel_min + last) {  // all on one side: one value
    const float b = tab[d_hi <= g.rel_min ? 0 : last];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], g.scale_log2, b);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      s[i] = fmaf(s[i], g.scale_log2, tab[min(max(dist(i) - g.rel_min, 0), last)]);
  }
}

// ---------------------------------------------------------------------------- forward

// W waves of 32 queries each; KT keys per LDS tile, two tiles of keys and of values in LDS.
template <typename T, int D, int W, bool BIAS, bool RES>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2)))
void seq_fwd_kernel(SeqGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                    const T* __restrict__ v, const int32_t* __restrict__ cu_q,
                    const int32_t* __restrict__ cu_k, const float* __restrict__ table,
                    const int32_t* __restrict__ map, T* __restrict__ out,
                    T* __restrict__ out_res, float* __restrict__ lse) {
  constexpr int QT = W * 32, KT = W * (sizeof(T) == 2 ? 16 : 8);
  using Tl = Tile<T, D, KT, W * 64>;
  using Rows = Tile<T, D, QT, W * 64>;  // a tile of queries, or of results
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = KT / 32, E = Tl::kElems;
  constexpr bool kThroughLds = sizeof(T) == 2;  // queries and results fit a pair of tiles
  static_assert(!kThroughLds || Rows::kElems == 2 * E, "two tiles hold the queries");
  __shared__ __attribute__((aligned(16))) T lds[4 * E];  // keys, values of tile 0, of tile 1
  extern __shared__ float tab[];                         // the bias by distance

  Work w;
  if (!work_of(g.q_tiles, g.group, w)) return;
  const Slot sq = find_slot<QT>(cu_q, g.B, g.nq, 1, w.slot);
  const int q0 = sq.tile * QT, n = sq.end - sq.begin;
  if (q0 >= n) return;
  int k0, m;
  key_rows(cu_k, sq.b, g.B, g.nk, k0, m);
  const int off = m - n;  // position of query 0
  const int nkeys = g.causal ? min(m, min(q0 + QT, n) + off) : m;
  const int ntiles = nkeys > 0 ? (nkeys + KT - 1) / KT : 0;
  if constexpr (BIAS) fill_bias<W * 64>(tab, g, table, map, w.head);

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const int i0 = q0 + wave * 32, iq = i0 + (lane & 31);
  const bool qok = iq < n, live = i0 < n;
  const int64_t qrow = sq.begin + (qok ? iq : 0);

  // Tile i of keys and values is copied to LDS buffer i % 2.
  const T* kp = k + (int64_t)k0 * g.ks + w.u * D;
  const T* vp = v + (int64_t)k0 * g.vs + w.u * D;
  const uint32_t ksb = (uint32_t)g.ks * sizeof(T), vsb = (uint32_t)g.vs * sizeof(T);
  uint32_t ko[Tl::NC], vo[Tl::NC];
  Tl::copy_plan(ko, ksb);
  Tl::copy_plan(vo, vsb);
  auto fetch = [&](int kt, int buf) {
    const int64_t at = (int64_t)kt * KT;
    Tl::copy(lds + 2 * E * buf, kp + at * g.ks, ko, ksb, m - kt * KT);
    Tl::copy(lds + 2 * E * buf + E, vp + at * g.vs, vo, vsb, m - kt * KT);
  };
  Frag qf[KS];
  if constexpr (kThroughLds) {
    uint32_t qo[Rows::NC];
    const uint32_t qsb = (uint32_t)g.qs * sizeof(T);
    Rows::copy_plan(qo, qsb);
    Rows::copy(lds + 2 * E, q + (sq.begin + q0) * g.qs + w.head * D, qo, qsb, n - q0);
    if (ntiles > 0) fetch(0, 0);
    wait_copies();
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = Rows::a_rows(lds + 2 * E, wave * 32, ks);
  } else {
    if (ntiles > 0) fetch(0, 0);
    load_frag<T, D>(qf, q + qrow * g.qs + w.head * D, qok);
    wait_copies();
  }
  __syncthreads();

  // the last key this query sees, and the last one any of the wave's queries sees
  const int last = g.causal ? min(m - 1, iq + off) : m - 1;
  const int wave_last = !live ? -1 : g.causal ? min(m - 1, min(i0 + 31, n - 1) + off) : m - 1;
  const int all_see = g.causal ? min(m - 1, i0 + off) : m - 1;

  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16_t{};
  float mx_run = -INFINITY, l = 0.0f, base = 0.0f;  // base: mx_run, 0 while there is none

  auto logits = [&](const T* kb, int b) {
    Frag a[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) a[ks] = Tl::a_rows(kb, b * 32, ks);
    f32x16_t acc = f32x16_t{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) acc = mfma(a[ks], qf[ks], acc);
    return acc;
  };
  // The largest of a block's logits (base 2), and the running maximum raised where that exceeds
  // it by more than kSlack: alpha stays below 2^kSlack and the rescale of O is rare.  The result
  // does not depend on which maximum was used.
  auto raise_to = [&](const float (&s)[16]) {
    float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
    for (int i = 3; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = pair_max(mx);
    if constexpr (!BIAS) mx *= g.scale_log2;  // scale > 0
    const bool raise = mx > mx_run + kSlack;
    if (__any(raise)) {
      const float corr = raise ? __builtin_amdgcn_exp2f(mx_run - mx) : 1.0f;
      if (raise) mx_run = base = mx;
      l *= corr;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= corr;
    }
  };
  // alpha (unnormalised) in place of the logits, and its fragments
  auto weigh = [&](float (&s)[16], Frag (&ph)[2]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(BIAS ? s[i] - base : fmaf(s[i], g.scale_log2, -base));
      l += s[i];
    }
    to_frags(s, ph);
  };
  auto values = [&](const T* vc, int b, Frag (&av)[DB][2]) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int p = 0; p < 2; ++p) av[db][p] = Tl::a_cols(vc, db * 32, b, p);
  };
  auto accumulate = [&](const Frag (&av)[DB][2], const Frag (&ph)[2]) {
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = mfma(av[db][p], ph[p], o[db]);
  };

  // Tiles that every query of the workgroup sees whole, without a bias: the next block's logits
  // are on the matrix cores while this block's exponentials are on the vector ALU.  Two tiles per
  // turn, so that the LDS buffers' places are constants.
  int kt = 0;
  if constexpr (!BIAS && !RES) {
    const int whole = (g.causal ? min(m, q0 + off + 1) : m) / KT;
    f32x16_t next = f32x16_t{};
    if (whole > 0 && live) next = logits(lds, 0);
    auto tile = [&](int t, int buf) {
      const T *kc = lds + 2 * E * buf, *vc = kc + E, *kn = lds + 2 * E * (1 - buf);
      if (t + 1 < ntiles) fetch(t + 1, 1 - buf);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float s[16];
        if (live) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = next[i];
          raise_to(s);
        }
        if (b == NB - 1) {  // the next tile is in LDS
          wait_copies();
          __syncthreads();
        }
        if (live) {
          Frag av[DB][2], ph[2];
          next = b + 1 < NB ? logits(kc, b + 1) : logits(kn, 0);
          values(vc, b, av);
          weigh(s, ph);
          accumulate(av, ph);
        }
      }
      __syncthreads();
    };
    for (; kt + 1 < whole; kt += 2) {
      tile(kt, 0);
      tile(kt + 1, 1);
    }
    if (kt < whole) tile(kt++, 0);
  }
  for (; kt < ntiles; ++kt) {
    const T *kc = lds + 2 * E * (kt & 1), *vc = kc + E;
    if (kt + 1 < ntiles) fetch(kt + 1, (kt + 1) & 1);
    const int kbase = kt * KT;
    const int nb = wave_last < kbase ? 0 : min(NB, (wave_last - kbase) / 32 + 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (b >= nb) break;
      const f32x16_t cur = logits(kc, b);
      Frag av[DB][2], ph[2];
      values(vc, b, av);
      const int kb = kbase + b * 32;
      float s[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = cur[i];
      if constexpr (BIAS)
        add_bias(s, g, tab, kb - (i0 + 31 + off), kb + 31 - (i0 + off),
                 [&](int i) { return kb + c_row(i, hh) - iq - off; });
      if (kb + 31 > all_see) {
        asm volatile("");  // a branch: blocks that every query sees do not pay for it
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (kb + c_row(i, hh) > last) s[i] = -INFINITY;
      }
      raise_to(s);
      weigh(s, ph);
      accumulate(av, ph);
      if constexpr (RES) {
        Frag pl[2];
        to_low_frags(s, ph, pl);
        accumulate(av, pl);
      }
    }
    wait_copies();
    __syncthreads();
  }

  const float ltot = pair_sum(l);
  const float inv = ltot > 0.0f ? 1.0f / ltot : ltot;  // 0 for an empty row, NaN stays
  const int64_t row = qrow * g.H + w.head;
  if (qok && hh == 0 && lse != nullptr)
    lse[row] = ltot == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(ltot)) * kLn2;
  if (!live) return;
#pragma unroll
  for (int part = 0; part < (RES ? 2 : 1); ++part) {
    T* to = part == 0 ? out : out_res;
    if constexpr (kThroughLds) {
      // The wave's 32 rows through LDS (its own place, no other wave's), so that whole rows are
      // written, 16 bytes per lane.
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int blk = 0; blk < 4; ++blk) {
          __bf16 h[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = o[db][4 * blk + j] * inv;
            h[j] = (__bf16)(part == 0 ? x : x - (float)(__bf16)x);
          }
          *reinterpret_cast<uint2*>(
              lds + Rows::at(wave * 32 + (lane & 31), db * 32 + 8 * blk + 4 * hh)) =
              __builtin_bit_cast(uint2, h);
        }
      constexpr int PER = 64 / Rows::KCH;  // rows per instruction
#pragma unroll
      for (int i = 0; i < 32 / PER; ++i) {
        const int r = i * PER + lane / Rows::KCH, c = (lane % Rows::KCH) * 8;
        const uint4 u = *reinterpret_cast<const uint4*>(lds + Rows::at(wave * 32 + r, c));
        if (i0 + r < n)
          *reinterpret_cast<uint4*>(to + ((int64_t)(sq.begin + i0 + r) * g.H + w.head) * D + c) = u;
      }
    } else if (qok) {
#pragma unroll
      for (int db = 0; db < DB; ++db) store_block(to + row * D, db, o[db], inv);
    }
  }
}

// ---------------------------------------------------------------------------- backward

// dq pass: 128 queries of one head against the keys they see,
//   alpha = exp2(t - lse),  dP^T = V dout^T,  dS = alpha (dP - Delta),  dq^T += K^T dS^T,
// and Delta = <dout, out + out_res>, kept for the dk/dv pass.  The bias gradient sums dS by
// distance: distances inside the table in LDS, in an array of their own for each half of each
// wave, where one instruction's 32 lanes have 32 different distances (queries i .. i + 31 and one
// key), so that no two of its additions meet and the order of all is the program's; distances at
// and beyond the ends in a register per lane.  The workgroup's sums by bucket go to `partial`.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2)))
void seq_dq_kernel(SeqGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                   const T* __restrict__ v, const int32_t* __restrict__ cu_q,
                   const int32_t* __restrict__ cu_k, const float* __restrict__ table,
                   const int32_t* __restrict__ map, const T* __restrict__ out,
                   const T* __restrict__ out_res, const float* __restrict__ lse,
                   const T* __restrict__ dout, T* __restrict__ dq, float* __restrict__ delta,
                   float* __restrict__ partial) {
  constexpr int KT = Type<T>::kKeyTile;
  using Tl = Tile<T, D, KT>;
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = KT / 32;
  __shared__ __attribute__((aligned(16))) T Ks[2][Tl::kElems];
  __shared__ __attribute__((aligned(16))) T Vs[2][Tl::kElems];
  extern __shared__ float tab[];  // bias by distance; 8 arrays of sums by distance; 8 x 2 ends

  Work w;
  if (!work_of(g.q_tiles, g.group, w)) return;
  const Slot sq = find_slot<kSeqTile>(cu_q, g.B, g.nq, 1, w.slot);
  const int q0 = sq.tile * kSeqTile, n = sq.end - sq.begin;
  if (q0 >= n) {
    if (BIAS && partial != nullptr)
      for (int c = threadIdx.x; c < g.nb; c += kThreads)
        partial[((int64_t)w.slot * g.H + w.head) * g.nb + c] = 0.0f;
    return;
  }
  int k0, m;
  key_rows(cu_k, sq.b, g.B, g.nk, k0, m);
  const int off = m - n;
  const int nkeys = g.causal ? min(m, min(q0 + kSeqTile, n) + off) : m;
  const int ntiles = nkeys > 0 ? (nkeys + KT - 1) / KT : 0;

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const int i0 = q0 + wave * 32, iq = i0 + (lane & 31);
  const bool qok = iq < n;
  const int64_t qrow = sq.begin + (qok ? iq : 0), row = qrow * g.H + w.head;
  float* sums = tab + g.span + (wave * 2 + hh) * g.span;
  if constexpr (BIAS) {
    fill_bias(tab, g, table, map, w.head);
    if (partial != nullptr)
      for (int i = threadIdx.x; i < 8 * g.span; i += kThreads) tab[g.span + i] = 0.0f;
  }
  Frag qf[KS], gf[KS];
  load_frag<T, D>(qf, q + qrow * g.qs + w.head * D, qok);
  load_frag<T, D>(gf, dout + row * D, qok);
  float dl;
  {
    Frag of[KS];
    load_frag<T, D>(of, out + row * D, qok);
    float part = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int e = 0; e < 8; ++e) part = fmaf(frag_at(gf[ks], e), frag_at(of[ks], e), part);
    if (out_res != nullptr) {
      load_frag<T, D>(of, out_res + row * D, qok);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int e = 0; e < 8; ++e) part = fmaf(frag_at(gf[ks], e), frag_at(of[ks], e), part);
    }
    dl = pair_sum(part);
  }
  if (qok && hh == 0) delta[row] = dl;
  // an empty row (lse = -inf) gets alpha = exp2(-inf) = 0
  const float lse_row = qok ? lse[row] : -INFINITY;
  const float lse2 = lse_row == -INFINITY ? INFINITY : lse_row * kLog2e;
  const int last = g.causal ? min(m - 1, iq + off) : m - 1;
  const int wave_last = i0 >= n ? -1 : g.causal ? min(m - 1, min(i0 + 31, n - 1) + off) : m - 1;
  const int all_see = g.causal ? min(m - 1, i0 + off) : m - 1;

  f32x16_t acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x16_t{};
  float behind = 0.0f, ahead = 0.0f;

  const T* kp = Tl::first_chunk(k + (int64_t)k0 * g.ks + w.u * D, g.ks);
  const T* vp = Tl::first_chunk(v + (int64_t)k0 * g.vs + w.u * D, g.vs);
  uint4 kr[Tl::NL], vr[Tl::NL];
  if (ntiles > 0) {
    Tl::load(kr, kp, g.ks, m);
    Tl::load(vr, vp, g.vs, m);
    Tl::store(Ks[0], kr);
    Tl::store(Vs[0], vr);
    if (ntiles > 1) {
      Tl::load(kr, kp + KT * g.ks, g.ks, m - KT);
      Tl::load(vr, vp + KT * g.vs, g.vs, m - KT);
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
      const int at = (kt + 2) * KT;
      Tl::load(kr, kp + at * g.ks, g.ks, m - at);
      Tl::load(vr, vp + at * g.vs, g.vs, m - at);
    }
    const int kbase = kt * KT;
    const int nb = wave_last < kbase ? 0 : min(NB, (wave_last - kbase) / 32 + 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (b >= nb) break;
      f32x16_t sa = f32x16_t{}, pa = f32x16_t{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        sa = mfma(Tl::a_rows(kc, b * 32, ks), qf[ks], sa);
        pa = mfma(Tl::a_rows(vc, b * 32, ks), gf[ks], pa);
      }
      const int kb = kbase + b * 32;
      float s[16], ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = sa[i];
      const int d_lo = kb - (i0 + 31 + off), d_hi = kb + 31 - (i0 + off);
      if constexpr (BIAS)
        add_bias(s, g, tab, d_lo, d_hi, [&](int i) { return kb + c_row(i, hh) - iq - off; });
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(BIAS ? s[i] - lse2
                                                    : fmaf(s[i], g.scale_log2, -lse2));
        ds[i] = p * (pa[i] - dl);
      }
      if (kb + 31 > all_see || i0 + 31 >= n) {
        asm volatile("");
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (kb + c_row(i, hh) > last || !qok) ds[i] = 0.0f;
      }
      if (BIAS && partial != nullptr) {
        const int end = g.span - 1;
        if (d_hi <= g.rel_min || d_lo >= g.rel_min + end) {
          float sum = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) sum += ds[i];
          if (d_hi <= g.rel_min) behind += sum;
          else ahead += sum;
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int idx = kb + c_row(i, hh) - iq - off - g.rel_min;
            if (idx <= 0) {
              behind += ds[i];
            } else if (idx >= end) {
              ahead += ds[i];
            } else {
              __builtin_amdgcn_ds_atomic_fadd_f32((__attribute__((address_space(3))) float*)(sums + idx), ds[i]);
            }
          }
        }
      }
      Frag df[2];
      to_frags(ds, df);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int p = 0; p < 2; ++p)
          acc[db] = mfma(Tl::a_cols(kc, db * 32, b, p), df[p], acc[db]);
    }
    __syncthreads();
  }
  if (qok) {
#pragma unroll
    for (int db = 0; db < DB; ++db) store_block(dq + row * D, db, acc[db], g.scale);
  }
  if (BIAS && partial != nullptr) {
    // the lanes' ends join the wave's arrays lane by lane pairs in a fixed tree
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      behind += __shfl_xor(behind, d);
      ahead += __shfl_xor(ahead, d);
    }
    float* ends = tab + 9 * g.span;
    if (lane == 0) {
      ends[2 * wave] = behind;
      ends[2 * wave + 1] = ahead;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < g.span; i += kThreads) {
      float sum = 0.0f;
#pragma unroll
      for (int a = 0; a < 8; ++a) sum += tab[g.span * (1 + a) + i];
      if (i == 0) sum += (ends[0] + ends[2]) + (ends[4] + ends[6]);
      if (i == g.span - 1) sum += (ends[1] + ends[3]) + (ends[5] + ends[7]);
      tab[i] = sum;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < g.nb; c += kThreads) {
      float sum = 0.0f;
      for (int i = 0; i < g.span; ++i) sum += map[i] == c ? tab[i] : 0.0f;
      partial[((int64_t)w.slot * g.H + w.head) * g.nb + c] = sum;
    }
  }
}

// Sums the workgroups' bucket sums over the slots, in 64 bits and a fixed order: a workgroup per
// head, 256 / buckets' threads per bucket.
__global__ __launch_bounds__(256) void seq_table_kernel(int slots, int heads, int nb,
                                                        const float* __restrict__ partial,
                                                        float* __restrict__ d_table) {
  __shared__ double part[256];
  int width = 1;
  while (width < nb) width <<= 1;
  const int c = threadIdx.x % width, lanes = 256 / width, head = blockIdx.x;
  double sum = 0.0;
  if (c < nb)
    for (int s = threadIdx.x / width; s < slots; s += lanes)
      sum += (double)partial[((int64_t)s * heads + head) * nb + c];
  part[threadIdx.x] = sum;
  __syncthreads();
  if ((int)threadIdx.x < nb) {
    for (int j = 1; j < lanes; ++j) sum += part[threadIdx.x + j * width];
    d_table[(int64_t)threadIdx.x * heads + head] = (float)sum;
  }
}

// dk/dv pass: 128 keys of one key head (wave w owns keys 32 w .. +31, lanes l and l ^ 32 share
// key l % 32) against the queries that see them, head by head of the group:
//   S = Q K^T,  dP = dout V^T,  dv^T += dout^T alpha,  dk^T += Q^T dS.
template <typename T, int D, bool BIAS, bool DK, bool DV>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(
    sizeof(T) == 2 && !(DK && DV && D == 128) ? 2 : 1, 2)))
void seq_dkdv_kernel(SeqGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                     const T* __restrict__ v, const int32_t* __restrict__ cu_q,
                     const int32_t* __restrict__ cu_k, const float* __restrict__ table,
                     const int32_t* __restrict__ map, const float* __restrict__ lse,
                     const T* __restrict__ dout, const float* __restrict__ delta,
                     T* __restrict__ dk, T* __restrict__ dv) {
  constexpr int QT = Type<T>::kKeyTile;
  using Tl = Tile<T, D, QT>;
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = QT / 32;
  __shared__ __attribute__((aligned(16))) T Qs[2][Tl::kElems];
  __shared__ __attribute__((aligned(16))) T Gs[2][Tl::kElems];
  __shared__ __attribute__((aligned(16))) float Ls[2][QT];  // lse log2(e); +inf where none
  __shared__ __attribute__((aligned(16))) float Dl[2][QT];  // Delta
  extern __shared__ float tab[];

  Work w;
  if (!work_of(g.k_tiles, 1, w)) return;
  const Slot sk = find_slot<kSeqTile>(cu_k, g.B, g.nk, 1, w.slot);
  const int k0 = sk.tile * kSeqTile, m = sk.end - sk.begin;
  if (k0 >= m) return;
  int qbeg, n;
  key_rows(cu_q, sk.b, g.B, g.nq, qbeg, n);
  const int off = m - n;
  const int q_first = g.causal ? max(k0 - off, 0) / QT * QT : 0;  // first tile with a query that sees
  const int per_head = n > q_first ? (n - q_first + QT - 1) / QT : 0;
  const int ntiles = per_head * g.group;

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const int j0 = k0 + wave * 32, jk = j0 + (lane & 31);
  const bool kok = jk < m;
  const int64_t krow = sk.begin + (kok ? jk : 0);
  Frag kf[KS], vf[KS];
  load_frag<T, D>(kf, k + krow * g.ks + w.u * D, kok);
  if constexpr (DK) load_frag<T, D>(vf, v + krow * g.vs + w.u * D, kok);

  f32x16_t dka[DB], dva[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dka[db] = dva[db] = f32x16_t{};

  uint4 rq[Tl::NL], rg[Tl::NL];
  float ls = INFINITY, de = 0.0f;
  auto fetch = [&](int it) {
    const int head = w.u * g.group + it / per_head, at = q_first + it % per_head * QT;
    const int64_t row = qbeg + at, gs = (int64_t)g.H * D;
    Tl::load(rq, Tl::first_chunk(q + row * g.qs + head * D, g.qs), g.qs, n - at);
    Tl::load(rg, Tl::first_chunk(dout + row * gs + head * D, gs), gs, n - at);
    if (threadIdx.x < QT) {
      const bool ok = at + (int)threadIdx.x < n;
      const int64_t r = (row + (ok ? threadIdx.x : 0)) * g.H + head;
      const float x = ok ? lse[r] : -INFINITY;
      ls = x == -INFINITY ? INFINITY : x * kLog2e;
      de = ok && DK ? delta[r] : 0.0f;
    }
  };
  auto stage = [&](int buf) {
    Tl::store(Qs[buf], rq);
    Tl::store(Gs[buf], rg);
    if (threadIdx.x < QT) {
      Ls[buf][threadIdx.x] = ls;
      Dl[buf][threadIdx.x] = de;
    }
  };
  if (ntiles > 0) {
    fetch(0);
    stage(0);
    if (ntiles > 1) fetch(1);
  }
  for (int it = 0; it < ntiles; ++it) {
    if constexpr (BIAS) {
      if (it % per_head == 0) {
        __syncthreads();  // the previous head's table is no longer read
        fill_bias(tab, g, table, map, w.u * g.group + it / per_head);
      }
    }
    __syncthreads();
    const T *Qc = Qs[it & 1], *Gc = Gs[it & 1];
    const float *Lc = Ls[it & 1], *Dc = Dl[it & 1];
    if (it + 1 < ntiles) stage((it + 1) & 1);
    if (it + 2 < ntiles) fetch(it + 2);
    const int qbase = q_first + it % per_head * QT;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int qb = qbase + b * 32;
      if (qb >= n || j0 >= m || (g.causal && qb + 31 + off < j0)) continue;
      f32x16_t sa = f32x16_t{}, pa = f32x16_t{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        sa = mfma(Tl::a_rows(Qc, b * 32, ks), kf[ks], sa);
        if constexpr (DK) pa = mfma(Tl::a_rows(Gc, b * 32, ks), vf[ks], pa);
      }
      float s[16], ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = sa[i];
      if constexpr (BIAS)
        add_bias(s, g, tab, j0 - (qb + 31 + off), j0 + 31 - (qb + off),
                 [&](int i) { return jk - qb - c_row(i, hh) - off; });
#pragma unroll
      for (int blk = 0; blk < 4; ++blk) {
        const float4 l4 = *reinterpret_cast<const float4*>(Lc + b * 32 + 8 * blk + 4 * hh);
        const float4 d4 = *reinterpret_cast<const float4*>(Dc + b * 32 + 8 * blk + 4 * hh);
        const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = 4 * blk + j;
          s[i] = __builtin_amdgcn_exp2f(BIAS ? s[i] - lv[j] : fmaf(s[i], g.scale_log2, -lv[j]));
          if constexpr (DK) ds[i] = s[i] * (pa[i] - dl[j]);
        }
      }
      if (qb + 31 >= n || (g.causal && qb + off < j0 + 31)) {
        // queries before the key, and rows past the sequence's end
        asm volatile("");
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int iq = qb + c_row(i, hh);
          if (iq >= n || (g.causal && iq + off < jk)) {
            s[i] = 0.0f;
            if constexpr (DK) ds[i] = 0.0f;
          }
        }
      }
      if constexpr (DV) {
        Frag pf[2];
        to_frags(s, pf);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int p = 0; p < 2; ++p)
            dva[db] = mfma(Tl::a_cols(Gc, db * 32, b, p), pf[p], dva[db]);
      }
      if constexpr (DK) {
        Frag df[2];
        to_frags(ds, df);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int p = 0; p < 2; ++p)
            dka[db] = mfma(Tl::a_cols(Qc, db * 32, b, p), df[p], dka[db]);
      }
    }
  }
  if (!kok) return;
  const int64_t row = (krow * g.KH + w.u) * D;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    if constexpr (DK) store_block(dk + row, db, dka[db], g.scale);
    if constexpr (DV) store_block(dv + row, db, dva[db], 1.0f);
  }
}

// ---------------------------------------------------------------------------- launches

template <typename... A>
hipError_t launch(const void* fn, dim3 grid, int threads, size_t lds, hipStream_t s, A... args) {
  void* a[] = {(void*)&args...};
  return hipLaunchKernel(fn, grid, dim3(threads), a, lds, s);
}

template <typename T, int D, int W>
hipError_t forward_w(const SeqGeometry& g, const SeqTensors& t, T* out, T* res, float* lse,
                     hipStream_t s) {
  const bool bias = g.nb > 0;
  const void* fn;
  if constexpr (sizeof(T) == 2) {
    fn = bias ? (res ? (const void*)&seq_fwd_kernel<T, D, W, true, true>
                     : (const void*)&seq_fwd_kernel<T, D, W, true, false>)
              : (res ? (const void*)&seq_fwd_kernel<T, D, W, false, true>
                     : (const void*)&seq_fwd_kernel<T, D, W, false, false>);
  } else {
    fn = bias ? (const void*)&seq_fwd_kernel<T, D, W, true, false>
              : (const void*)&seq_fwd_kernel<T, D, W, false, false>;
  }
  SeqGeometry h = g;
  h.q_tiles = seq_spread(g.KH, g.nq / (W * 32) + g.B + 1);
  return launch(fn, dim3((unsigned)seq_blocks(h.q_tiles, g.group)), W * 64, bias ? g.span * 4 : 0,
                s, h, (const T*)t.q, (const T*)t.k, (const T*)t.v, t.cu_q, t.cu_k, t.table, t.map,
                out, res, lse);
}

template <typename T, int D>
hipError_t forward_d(const SeqGeometry& g, const SeqTensors& t, T* out, T* res, float* lse,
                     hipStream_t s) {
  // Eight waves halve the copies per product but leave half the workgroups: they pay where the
  // sequences are long and the workgroups many.  16 heads x 128, 4 / 8 waves: one causal sequence
  // of 16,384 tokens 1.025 / 1.001 ms, of 8,192 (all keys) 515 / 491 us; 32 sequences of 512
  // 77 / 81 us, four of 1,000 with 8 heads 27 / 31 us.
  const bool wide = g.nk >= 4096 * (int64_t)g.B && (int64_t)g.nq * g.H >= 256 * 512;
  if constexpr (sizeof(T) == 2) {
    if (wide) return forward_w<T, D, 8>(g, t, out, res, lse, s);
  }
  return forward_w<T, D, 4>(g, t, out, res, lse, s);
}

size_t round_256(size_t x) { return (x + 255) & ~size_t(255); }

template <typename T, int D>
hipError_t backward_d(const SeqGeometry& g, const SeqTensors& t, const T* out, const T* res,
                      const float* lse, const T* dout, T* dq, T* dk, T* dv, float* d_table,
                      void* workspace, hipStream_t s) {
  const bool bias = g.nb > 0;
  const T *q = (const T*)t.q, *k = (const T*)t.k, *v = (const T*)t.v;
  float* delta = (float*)workspace;
  float* partial = bias && d_table != nullptr
                       ? (float*)((char*)workspace + round_256((size_t)g.nq * g.H * 4))
                       : nullptr;
  hipError_t e = hipSuccess;
  if (g.nq > 0) {
    const void* fn = bias ? (const void*)&seq_dq_kernel<T, D, true>
                          : (const void*)&seq_dq_kernel<T, D, false>;
    const size_t lds = !bias ? 0 : partial ? (size_t)g.span * 36 + 64 : (size_t)g.span * 4;
    e = launch(fn, dim3((unsigned)seq_blocks(g.q_tiles, g.group)), kThreads, lds, s, g, q, k, v, t.cu_q,
               t.cu_k, t.table, t.map, out, res, lse, dout, dq, delta, partial);
  }
  if (e == hipSuccess && bias && d_table != nullptr)
    e = launch((const void*)&seq_table_kernel, dim3(g.H), kThreads, 0, s, g.nq > 0 ? g.q_tiles.slots : 0,
               g.H, g.nb, (const float*)partial, d_table);
  if (e == hipSuccess && g.nk > 0) {
    const dim3 grid((unsigned)seq_blocks(g.k_tiles, 1));
    const size_t lds = bias ? (size_t)g.span * 4 : 0;
    const float* cdelta = delta;
    const void* fn = bias ? (const void*)&seq_dkdv_kernel<T, D, true, true, true>
                          : (const void*)&seq_dkdv_kernel<T, D, false, true, true>;
    e = launch(fn, grid, kThreads, lds, s, g, q, k, v, t.cu_q, t.cu_k, t.table, t.map, lse, dout, cdelta,
               dk, dv);
  }
  return e;
}

}  // namespace

Spread seq_spread(int units, int slots) {
  Spread s;
  s.units = units;
  s.slots = slots;
  s.parts = 8 / std::gcd(8, units);
  s.local = units * s.parts / 8;
  s.ranks = (slots + s.parts - 1) / s.parts;
  return s;
}

hipError_t launch_seq_forward(const SeqGeometry& g, bool bf16, const SeqTensors& t, void* out,
                              void* res, float* lse, hipStream_t s) {
  if (g.nq == 0) return hipSuccess;
  if (bf16)
    return g.D == 64 ? forward_d<uint16_t, 64>(g, t, (uint16_t*)out, (uint16_t*)res, lse, s)
                     : forward_d<uint16_t, 128>(g, t, (uint16_t*)out, (uint16_t*)res, lse, s);
  return g.D == 64 ? forward_d<float, 64>(g, t, (float*)out, nullptr, lse, s)
                   : forward_d<float, 128>(g, t, (float*)out, nullptr, lse, s);
}

size_t seq_backward_workspace(const SeqGeometry& g, bool want_table) {
  size_t need = round_256((size_t)g.nq * g.H * 4);
  if (want_table) need += round_256((size_t)g.q_tiles.slots * g.H * g.nb * 4);
  return need;
}

hipError_t launch_seq_backward(const SeqGeometry& g, bool bf16, const SeqTensors& t,
                               const void* out, const void* res, const float* lse,
                               const void* dout, void* dq, void* dk, void* dv, float* d_table,
                               void* ws, hipStream_t s) {
  typedef uint16_t B;
  if (bf16)
    return g.D == 64 ? backward_d<B, 64>(g, t, (const B*)out, (const B*)res, lse, (const B*)dout,
                                         (B*)dq, (B*)dk, (B*)dv, d_table, ws, s)
                     : backward_d<B, 128>(g, t, (const B*)out, (const B*)res, lse,
                                          (const B*)dout, (B*)dq, (B*)dk, (B*)dv, d_table, ws, s);
  typedef float F;
  return g.D == 64 ? backward_d<F, 64>(g, t, (const F*)out, nullptr, lse, (const F*)dout, (F*)dq,
                                       (F*)dk, (F*)dv, d_table, ws, s)
                   : backward_d<F, 128>(g, t, (const F*)out, nullptr, lse, (const F*)dout, (F*)dq,
                                        (F*)dk, (F*)dv, d_table, ws, s);
}

}  // namespace dsa3d
