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

// The bias of one head in LDS: by distance, with kPad more entries at either end that repeat it, so
// that a 32 x 32 block whose distances reach into the table reads it without clamping; blocks
// beyond it share one value.
constexpr int kPad = 62;
__host__ __device__ inline int padded(int span) { return span + 2 * kPad; }
// A block's dS by diagonal: 63 rows of 32 keys, 36 floats apart, per wave.
constexpr int kSkew = 36, kSkewed = 63 * kSkew;

// A barrier follows before its use.
template <int THREADS = kThreads>
__device__ inline void fill_bias(float* tab, const SeqGeometry& g, const float* table,
                                 const int32_t* map, int head) {
  for (int i = threadIdx.x; i < padded(g.span); i += THREADS)
    tab[i] = bias_of(table, map, g.H, g.nb, head, min(max(i - kPad, 0), g.span - 1));
}

// What turns the values of a block into base-2 logits: mul x + add.
struct Affine {
  float mul, add;
};

// Whether no pair of a block, whose distances run from d_lo to d_hi = d_lo + 62, reaches into the
// table; the sums' and the reads' places are in range otherwise.
__device__ inline bool outside(const SeqGeometry& g, int d_lo) {
  return d_lo + 62 <= g.rel_min || d_lo >= g.rel_min + g.span - 1;
}

// Adds the bias to a block's values (or says what to add to all of them).  SIGN 1: element i is
// key c_row(i) of the block and this lane's query; -1: query c_row(i) and this lane's key.  d0 is
// the distance of element 0.
template <int SIGN>
__device__ inline Affine add_bias(float (&s)[16], const SeqGeometry& g, const float* tab, int d_lo,
                                  int d0) {
  if (outside(g, d_lo))
    return {g.scale_log2, tab[d_lo >= g.rel_min ? kPad + g.span - 1 : kPad]};
  const float* at = tab + kPad + d0 - g.rel_min;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], g.scale_log2, at[SIGN * c_row(i, 0)]);
  return {1.0f, 0.0f};
}

// ---------------------------------------------------------------------------- forward

// W waves of 32 queries each; KT keys per LDS tile, two tiles of keys and of values in LDS.
template <typename T, int D, int W, bool BIAS, bool RES>
__global__ __launch_bounds__(W * 64)
__attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 || D == 64 ? 2 : 1, 2)))
void seq_fwd_kernel(SeqGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                    const T* __restrict__ v, const int32_t* __restrict__ cu_q,
                    const int32_t* __restrict__ cu_k, const float* __restrict__ table,
                    const int32_t* __restrict__ map, T* __restrict__ out,
                    T* __restrict__ out_res, float* __restrict__ lse) {
  constexpr int QT = W * 32, KT = W / 4 * kKeyTile<T, D>;
  using Tl = Tile<T, D, KT, W * 64>;
  using Rows = Tile<T, D, QT, W * 64>;  // a tile of queries, or of results
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = KT / 32, E = Tl::kElems;
  constexpr bool kThroughLds = sizeof(T) == 2;  // queries and results fit a pair of tiles
  static_assert(!kThroughLds || Rows::kElems == 2 * E, "two tiles hold the queries");
  __shared__ __attribute__((aligned(16))) T lds[Tl::kTwo];  // keys and values
  extern __shared__ float tab[];                           // the bias by distance

  Work w;
  if (!work_of<false>(g.q_tiles, g.group, w)) return;
  const Place sq = place_of<QT, false>(cu_q, g.nq, cu_k, g.nk, g.B, g.causal, g.q_tiles.slots,
                                       w.slot);
  const int q0 = sq.tile * QT, n = sq.n, k0 = sq.other, m = sq.m;
  if (q0 >= n) return;
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
    Tl::copy(lds + Tl::kPlace * buf, kp + at * g.ks, ko, ksb, m - kt * KT);
    Tl::copy(lds + Tl::kPlace * buf + E, vp + at * g.vs, vo, vsb, m - kt * KT);
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

  auto logits = [&](const uint16_t* kb, int b) {
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
  auto raise_to = [&](const float (&s)[16], const Affine& f) {
    float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
    for (int i = 3; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = fmaf(pair_max(mx), f.mul, f.add);  // mul > 0
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
  auto weigh = [&](float (&s)[16], const Affine& f, Frag (&ph)[2]) {
    const float add = f.add - base;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], f.mul, add));
      l += s[i];
    }
    to_frags(s, ph);
  };
  auto biased = [&](float (&s)[16], int kb) {
    if constexpr (BIAS)
      return add_bias<1>(s, g, tab, kb - (i0 + 31 + off), kb + 4 * hh - iq - off);
    else
      return Affine{g.scale_log2, 0.0f};
  };
  auto values = [&](const uint16_t* vc, int b, Frag (&av)[DB][2]) {
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
  auto add_low = [&](const Frag (&av)[DB][2], const float (&s)[16], const Frag (&ph)[2]) {
    if constexpr (RES) {
      Frag pl[2];
      to_low_frags(s, ph, pl);
      accumulate(av, pl);
    }
  };

  // Tiles that every query of the workgroup sees whole: the next block's logits are on the matrix
  // cores while this block's exponentials are on the vector ALU.  Two tiles per turn, so that the
  // LDS buffers' places are constants.
  int kt = 0;
  if constexpr (sizeof(T) == 2) {
    const int whole = (g.causal ? min(m, q0 + off + 1) : m) / KT;
    f32x16_t next = f32x16_t{};
    if (whole > 0 && live) next = logits(lds, 0);
    auto tile = [&](int t, int buf) {
      const T *kc = lds + 2 * E * buf, *vc = kc + E, *kn = lds + 2 * E * (1 - buf);
      if (t + 1 < ntiles) fetch(t + 1, 1 - buf);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float s[16];
        Affine f;
        if (live) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = next[i];
          f = biased(s, t * KT + b * 32);
          raise_to(s, f);
        }
        if (b == NB - 1) {  // the next tile is in LDS
          wait_copies();
          __syncthreads();
        }
        if (live) {
          Frag av[DB][2], ph[2];
          next = b + 1 < NB ? logits(kc, b + 1) : logits(kn, 0);
          values(vc, b, av);
          weigh(s, f, ph);
          accumulate(av, ph);
          add_low(av, s, ph);
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
    const uint16_t *kc = Tl::operands(lds, kt & 1), *vc = kc + Tl::kSecond;
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
      const Affine f = biased(s, kb);
      if (kb + 31 > all_see) {
        asm volatile("");  // a branch: blocks that every query sees do not pay for it
        const int seen = last - kb - 4 * hh;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c_row(i, 0) > seen) s[i] = -INFINITY;
      }
      raise_to(s, f);
      weigh(s, f, ph);
      accumulate(av, ph);
      add_low(av, s, ph);
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
  const int64_t first = ((int64_t)(sq.begin + i0) * g.H + w.head) * D, step = (int64_t)g.H * D;
  store_rows<T, D>(lds + wave * 32 * D, o, inv, out + first, step, n - i0);
  if constexpr (RES)
    store_rows<T, D, true>(lds + wave * 32 * D, o, inv, out_res + first, step, n - i0);
}

// ---------------------------------------------------------------------------- backward

// dq pass: 128 queries of one head against the keys they see,
//   alpha = exp2(t - lse),  dP^T = V dout^T,  dS = alpha (dP - Delta),  dq^T += K^T dS^T,
// and Delta = <dout, out + out_res>, kept with lse log2(e) for the dk/dv pass, head by head.  The
// bias gradient sums dS by distance: a block that reaches into the table is written to LDS with
// its diagonals as rows, whose sums, one per lane, are added to the wave's sums by distance (with
// LDS atomics, 140 cycles each, the pass took 153 us for 4,096 tokens of 16 heads x 64, 66 without
// the gradient, and takes 76 this way); the other blocks go to a register per lane and side.  The
// workgroup's sums by bucket go to `partial`.  Every order is fixed.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 || D == 64 ? 2 : 1, 2)))
void seq_dq_kernel(SeqGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                   const T* __restrict__ v, const int32_t* __restrict__ cu_q,
                   const int32_t* __restrict__ cu_k, const float* __restrict__ table,
                   const int32_t* __restrict__ map, const T* __restrict__ out,
                   const T* __restrict__ out_res, const float* __restrict__ lse,
                   const T* __restrict__ dout, T* __restrict__ dq, float* __restrict__ delta,
                   float* __restrict__ lse2_out, float* __restrict__ partial) {
  constexpr int KT = kKeyTile<T, D>;
  using Tl = Tile<T, D, KT>;
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = KT / 32, E = Tl::kElems;
  __shared__ __attribute__((aligned(16))) T lds[Tl::kTwo];  // keys and values
  // for the bias gradient the waves' skewed blocks; the bias by distance; the waves' sums by
  // distance, 8 ends
  extern __shared__ __attribute__((aligned(16))) float room[];

  Work w;
  if (!work_of<false>(g.q_tiles, g.group, w)) return;
  const Place sq = place_of<kSeqTile, false>(cu_q, g.nq, cu_k, g.nk, g.B, g.causal,
                                             g.q_tiles.slots, w.slot);
  const int q0 = sq.tile * kSeqTile, n = sq.n, k0 = sq.other, m = sq.m;
  if (q0 >= n) {
    if (BIAS && partial != nullptr)
      for (int c = threadIdx.x; c < g.nb; c += kThreads)
        partial[((int64_t)w.slot * g.H + w.head) * g.nb + c] = 0.0f;
    return;
  }
  const int off = m - n;
  const int nkeys = g.causal ? min(m, min(q0 + kSeqTile, n) + off) : m;
  const int ntiles = nkeys > 0 ? (nkeys + KT - 1) / KT : 0;

  const T* kp = k + (int64_t)k0 * g.ks + w.u * D;
  const T* vp = v + (int64_t)k0 * g.vs + w.u * D;
  const uint32_t ksb = (uint32_t)g.ks * sizeof(T), vsb = (uint32_t)g.vs * sizeof(T);
  uint32_t ko[Tl::NC], vo[Tl::NC];
  Tl::copy_plan(ko, ksb);
  Tl::copy_plan(vo, vsb);
  auto fetch = [&](int kt, int buf) {
    const int64_t at = (int64_t)kt * KT;
    Tl::copy(lds + Tl::kPlace * buf, kp + at * g.ks, ko, ksb, m - kt * KT);
    Tl::copy(lds + Tl::kPlace * buf + E, vp + at * g.vs, vo, vsb, m - kt * KT);
  };
  if (ntiles > 0) fetch(0, 0);

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const int i0 = q0 + wave * 32, iq = i0 + (lane & 31);
  const bool qok = iq < n, live = i0 < n;
  const int64_t qrow = sq.begin + (qok ? iq : 0), row = qrow * g.H + w.head;
  const int stride = padded(g.span);
  float *tab = room, *all_sums = room, *ends = room, *skewed = room;
  if (BIAS && partial != nullptr) {
    tab = room + 4 * kSkewed;
    all_sums = tab + stride;
    ends = all_sums + 4 * stride;
  }
  const bool want_table = BIAS && partial != nullptr;
  if constexpr (BIAS) {
    fill_bias(tab, g, table, map, w.head);
    if (want_table)
      for (int i = threadIdx.x; i < 4 * kSkewed; i += kThreads) skewed[i] = 0.0f;
    if (want_table)
      for (int i = threadIdx.x; i < 4 * stride; i += kThreads) all_sums[i] = 0.0f;
  }
  Frag qf[KS], gf[KS];
  load_frag<T, D>(qf, q + qrow * g.qs + w.head * D, qok);
  load_frag<T, D>(gf, dout + row * D, qok);
  // Delta, and for the bias gradient how far the rounding of O takes it: 2^-16 of the root of its
  // terms' squares, four times the mean where the residual holds O's next bits (a channel is off
  // by 2^-18.7, by its weights' rounding as much again); in float32 the matrix cores lose up to
  // 2^-24 with every 16 keys, on one side
  float dl, trust = 0.0f;
  {
    Frag of[KS];
    load_frag<T, D>(of, out + row * D, qok);
    float part = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = frag_at(gf[ks], e), b = frag_at(of[ks], e);
        part = fmaf(a, b, part);
        trust = fmaf(a * b, a * b, trust);
      }
    if constexpr (BIAS)
      trust = sizeof(T) == 4 || out_res != nullptr ? sqrtf(pair_sum(trust)) * 0x1p-16f : 0.0f;
    if (out_res != nullptr) {
      load_frag<T, D>(of, out_res + row * D, qok);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int e = 0; e < 8; ++e) part = fmaf(frag_at(gf[ks], e), frag_at(of[ks], e), part);
    }
    dl = pair_sum(part);
  }
  // an empty row (lse = -inf) gets alpha = exp2(-inf) = 0
  const float lse_row = qok ? lse[row] : -INFINITY;
  const float lse2 = lse_row == -INFINITY ? INFINITY : lse_row * kLog2e;
  if (qok && hh == 0) {
    delta[(int64_t)w.head * g.nq + qrow] = dl;
    lse2_out[(int64_t)w.head * g.nq + qrow] = lse2;
  }
  const int last = g.causal ? min(m - 1, iq + off) : m - 1;
  const int wave_last = !live ? -1 : g.causal ? min(m - 1, min(i0 + 31, n - 1) + off) : m - 1;
  const int all_see = g.causal ? min(m - 1, i0 + off) : m - 1;

  f32x16_t acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x16_t{};
  float behind = 0.0f, ahead = 0.0f, inside = 0.0f, p_behind = 0.0f, p_ahead = 0.0f;

  // S^T = K Q^T and dP^T = V dout^T of a block
  auto products = [&](const uint16_t* kc, int b, f32x16_t& sa, f32x16_t& pa) {
    sa = f32x16_t{};
    pa = f32x16_t{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      sa = mfma(Tl::a_rows(kc, b * 32, ks), qf[ks], sa);
      pa = mfma(Tl::a_rows(kc + Tl::kSecond, b * 32, ks), gf[ks], pa);
    }
  };
  auto accumulate = [&](const uint16_t* kc, int b, const float (&ds)[16]) {
    Frag df[2];
    to_frags(ds, df);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        acc[db] = mfma(Tl::a_cols(kc, db * 32, b, p), df[p], acc[db]);
  };
  auto biased = [&](float (&s)[16], int kb) {
    if constexpr (BIAS)
      return add_bias<1>(s, g, tab, kb - (i0 + 31 + off), kb + 4 * hh - iq - off);
    else
      return Affine{g.scale_log2, 0.0f};
  };
  // alpha in place of the logits, and dS
  auto weigh = [&](float (&s)[16], const Affine& f, const f32x16_t& pa, float (&ds)[16]) {
    const float add = f.add - lse2;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], f.mul, add));
      ds[i] = s[i] * (pa[i] - dl);
    }
  };
  // dS by distance: blocks outside the table have one place, the others one per diagonal.  Where
  // lse and out are of these keys alone, a row's dS add up to what its Delta is off, of which
  // every place has alpha's share; the outer places, where alpha is largest, take theirs back at
  // the end.  With statistics of more keys than these the sum is no rounding, exceeds `trust` and
  // stays.  One text of 4,000 tokens, 4 heads x 64, the outer buckets' error: bf16 8e-7 (2.5e-6
  // without this), float32 7e-7 (1.4e-5).
  auto count = [&](const float (&p)[16], const float (&ds)[16], int kb) {
    if (!want_table) return;
    const int d_lo = kb - (i0 + 31 + off);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += ds[i];
    if (outside(g, d_lo)) {
      float all = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) all += p[i];
      if (d_lo >= g.rel_min) {
        ahead += sum;
        p_ahead += all;
      } else {
        behind += sum;
        p_behind += all;
      }
    } else {
      inside += sum;
      float* mine = skewed + wave * kSkewed;
      float* to = mine + (4 * hh - (lane & 31) + 31) * kSkew + 4 * hh;
#pragma unroll
      for (int i = 0; i < 16; ++i) to[c_row(i, 0) * (kSkew + 1)] = ds[i];
      if (lane < 63) {  // one diagonal per lane
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float4 x = *reinterpret_cast<const float4*>(mine + lane * kSkew + 4 * r);
          sum.x += x.x;
          sum.y += x.y;
          sum.z += x.z;
          sum.w += x.w;
        }
        all_sums[wave * stride + kPad + d_lo - g.rel_min + lane] +=
            (sum.x + sum.y) + (sum.z + sum.w);
      }
    }
  };
  wait_copies();
  __syncthreads();

  // As in the forward: tiles that every query sees whole, the next block's products beside this
  // block's vector work; then the tiles with a mask or a bias.
  int kt = 0;
  if constexpr (sizeof(T) == 2) {
    const int whole = q0 + kSeqTile <= n ? (g.causal ? min(m, max(q0 + off + 1, 0)) : m) / KT : 0;
    f32x16_t sa, pa;
    if (whole > 0) products(lds, 0, sa, pa);
    auto tile = [&](int t, int buf) {
      const T *kc = lds + 2 * E * buf, *kn = lds + 2 * E * (1 - buf);
      if (t + 1 < ntiles) fetch(t + 1, 1 - buf);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float s[16], ds[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = sa[i];
        const f32x16_t p0 = pa;
        const Affine f = biased(s, t * KT + b * 32);
        if (b == NB - 1) {  // the next tile is in LDS
          wait_copies();
          __syncthreads();
        }
        if (b + 1 < NB) products(kc, b + 1, sa, pa);
        else products(kn, 0, sa, pa);
        weigh(s, f, p0, ds);
        count(s, ds, t * KT + b * 32);
        accumulate(kc, b, ds);
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
    const uint16_t* kc = Tl::operands(lds, kt & 1);
    if (kt + 1 < ntiles) fetch(kt + 1, (kt + 1) & 1);
    const int kbase = kt * KT;
    const int nb = wave_last < kbase ? 0 : min(NB, (wave_last - kbase) / 32 + 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (b >= nb) break;
      f32x16_t sa, pa;
      products(kc, b, sa, pa);
      const int kb = kbase + b * 32;
      float s[16], ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = sa[i];
      const Affine f = biased(s, kb);
      weigh(s, f, pa, ds);
      if (kb + 31 > all_see || i0 + 31 >= n) {
        asm volatile("");
        const int seen = qok ? last - kb - 4 * hh : -1;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c_row(i, 0) > seen) s[i] = ds[i] = 0.0f;
      }
      count(s, ds, kb);
      accumulate(kc, b, ds);
    }
    wait_copies();
    __syncthreads();
  }
  if (live)
    store_rows<T, D>(lds + wave * 32 * D, acc, g.scale,
                     dq + ((int64_t)(sq.begin + i0) * g.H + w.head) * D, (int64_t)g.H * D, n - i0);
  if (want_table) {
    const float error = pair_sum(behind + inside + ahead);
    if (fabsf(error) <= trust) {
      behind -= p_behind * error;
      ahead -= p_ahead * error;
    }
    // the lanes' ends join in a fixed tree, the arrays in their order, then the distances of a
    // bucket: kThreads / width threads each
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      behind += __shfl_xor(behind, d);
      ahead += __shfl_xor(ahead, d);
    }
    if (lane == 0) {
      ends[2 * wave] = behind;
      ends[2 * wave + 1] = ahead;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < padded(g.span); i += kThreads) {
      float sum = 0.0f;
#pragma unroll
      for (int a = 0; a < 4; ++a) sum += all_sums[a * stride + i];
      tab[i] = sum;
    }
    __syncthreads();
    int* which = reinterpret_cast<int*>(all_sums);
    for (int i = threadIdx.x; i < padded(g.span); i += kThreads)
      which[i] = map[min(max(i - kPad, 0), g.span - 1)];
    __syncthreads();
    int width = 1;
    while (width < g.nb) width <<= 1;
    const int c = threadIdx.x % width, first = threadIdx.x / width, lanes = kThreads / width;
    float sum = 0.0f;
    for (int i = first; i < padded(g.span); i += lanes) sum += which[i] == c ? tab[i] : 0.0f;
    if (first == 0) {
      if (which[0] == c) sum += (ends[0] + ends[2]) + (ends[4] + ends[6]);
      if (which[padded(g.span) - 1] == c) sum += (ends[1] + ends[3]) + (ends[5] + ends[7]);
    }
    __syncthreads();
    tab[threadIdx.x] = sum;
    __syncthreads();
    if ((int)threadIdx.x < g.nb) {
      for (int j = 1; j < lanes; ++j) sum += tab[j * width + threadIdx.x];
      partial[((int64_t)w.slot * g.H + w.head) * g.nb + threadIdx.x] = sum;
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

// dk/dv pass (float32, and bf16 at 64 channels): 128 keys of one key head (wave w owns keys 32 w ..
// +31, lanes l and l ^ 32 share key l % 32) against the queries that see them, head by head of the
// group:
//   S = Q K^T,  dP = dout V^T,  dv^T += dout^T alpha,  dk^T += Q^T dS.
// With PARTS the (head, query tile) pairs of a key tile are dealt out to several workgroups,
// whose float32 sums seq_join_kernel adds.
template <typename T, int D, bool BIAS, bool PARTS>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 || D == 64 ? 2 : 1, 2)))
void seq_dkdv_kernel(SeqGeometry g, const T* __restrict__ q, const T* __restrict__ k,
                     const T* __restrict__ v, const int32_t* __restrict__ cu_q,
                     const int32_t* __restrict__ cu_k, const float* __restrict__ table,
                     const int32_t* __restrict__ map, const float* __restrict__ delta,
                     const float* __restrict__ lse2, const T* __restrict__ dout,
                     T* __restrict__ dk, T* __restrict__ dv, float* __restrict__ part_dk,
                     float* __restrict__ part_dv) {
  constexpr int QT = sizeof(T) == 2 ? 64 : 32;  // float32: room for two workgroups at 64 channels
  using Tl = Tile<T, D, QT>;
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = QT / 32, E = Tl::kElems;
  __shared__ __attribute__((aligned(16))) T lds[Tl::kTwo];       // queries and douts
  __shared__ __attribute__((aligned(16))) float stat[2][2][64];  // lse log2(e), Delta of a tile
  extern __shared__ float tab[];

  Work w;
  if (!work_of<false>(g.k_tiles, PARTS ? g.parts : 1, w)) return;
  const int part = PARTS ? w.head - w.u * g.parts : 0;
  const Place sk = place_of<kSeqTile, true>(cu_k, g.nk, cu_q, g.nq, g.B, g.causal, g.k_tiles.slots,
                                            w.slot);
  const int k0 = sk.tile * kSeqTile, m = sk.n, qbeg = sk.other, n = sk.m;
  if (k0 >= m) return;
  const int off = m - n;
  // first tile with a query that sees
  const int q_first = g.causal ? max(k0 - off, 0) / QT * QT : 0;
  const int per_head = n > q_first ? (n - q_first + QT - 1) / QT : 0;
  const int all = per_head * g.group;
  const int t0 = PARTS ? (int)((int64_t)all * part / g.parts) : 0;
  const int t1 = PARTS ? (int)((int64_t)all * (part + 1) / g.parts) : all;

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const uint32_t qsb = (uint32_t)g.qs * sizeof(T), gsb = (uint32_t)g.H * Tl::kRowBytes;
  uint32_t qo[Tl::NC], go[Tl::NC];
  Tl::copy_plan(qo, qsb);
  Tl::copy_plan(go, gsb);
  // Tiles are fetched in their order: the next one's head and number in it are counted on.
  int next_head = w.u * g.group + (t0 < t1 ? t0 / per_head : 0);
  int next_at = t0 < t1 ? t0 % per_head : 0;
  auto fetch = [&](int buf) {
    const int head = next_head, at = q_first + next_at * QT;
    if (++next_at == per_head) {
      next_at = 0;
      ++next_head;
    }
    const int64_t row = qbeg + at;
    Tl::copy(lds + Tl::kPlace * buf, q + row * g.qs + head * D, qo, qsb, n - at);
    Tl::copy(lds + Tl::kPlace * buf + E, dout + (row * g.H + head) * D, go, gsb, n - at);
    if (wave < 2)  // the rows' statistics; past the sequence's end the last row's
      copy_4(lds_offset(&stat[buf][wave][0]), wave == 0 ? lse2 : delta,
             (uint32_t)min(lane, n - at - 1) * 4u, (int64_t)head * g.nq + row);
  };
  int in_head = next_at, head = next_head;  // of tile `it`
  if (t0 < t1) fetch(0);

  const int j0 = k0 + wave * 32, jk = j0 + (lane & 31);
  const bool kok = jk < m, live = j0 < m;
  const int64_t krow = sk.begin + (kok ? jk : 0);
  Frag kf[KS], vf[KS];
  load_frag<T, D>(kf, k + krow * g.ks + w.u * D, kok);
  load_frag<T, D>(vf, v + krow * g.vs + w.u * D, kok);

  f32x16_t dka[DB], dva[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dka[db] = dva[db] = f32x16_t{};

  // S = Q K^T and dP = dout V^T of a block: the operands are read together, then multiplied
  auto products = [&](const uint16_t* qc, int b, f32x16_t& sa, f32x16_t& pa) {
    sa = f32x16_t{};
    pa = f32x16_t{};
    if constexpr (sizeof(T) == 2) {
      Frag aq[KS], ag[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        aq[ks] = Tl::a_rows(qc, b * 32, ks);
        ag[ks] = Tl::a_rows(qc + Tl::kSecond, b * 32, ks);
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        sa = mfma(aq[ks], kf[ks], sa);
        pa = mfma(ag[ks], vf[ks], pa);
      }
    } else {  // no room for them all
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        sa = mfma(Tl::a_rows(qc, b * 32, ks), kf[ks], sa);
        pa = mfma(Tl::a_rows(qc + Tl::kSecond, b * 32, ks), vf[ks], pa);
      }
    }
  };
  // alpha in place of the logits, and dS
  auto weigh = [&](int buf, int b, float (&s)[16], const Affine& f, const f32x16_t& pa,
                   float (&ds)[16]) {
#pragma unroll
    for (int blk = 0; blk < 4; ++blk) {
      const int at = b * 32 + 8 * blk + 4 * hh;
      const float4 l4 = *reinterpret_cast<const float4*>(&stat[buf][0][at]);
      const float4 d4 = *reinterpret_cast<const float4*>(&stat[buf][1][at]);
      const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = 4 * blk + j;
        s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], f.mul, f.add - lv[j]));
        ds[i] = s[i] * (pa[i] - dl[j]);
      }
    }
  };
  auto biased = [&](float (&s)[16], int qb) {
    if constexpr (BIAS)
      return add_bias<-1>(s, g, tab, j0 - (qb + 31 + off), jk - qb - 4 * hh - off);
    else
      return Affine{g.scale_log2, 0.0f};
  };
  auto accumulate = [&](const uint16_t* qc, int b, const float (&p)[16], const float (&ds)[16]) {
    Frag pf[2], df[2];
    to_frags(p, pf);
    to_frags(ds, df);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        dva[db] = mfma(Tl::a_cols(qc + Tl::kSecond, db * 32, b, i), pf[i], dva[db]);
        dka[db] = mfma(Tl::a_cols(qc, db * 32, b, i), df[i], dka[db]);
      }
  };
  wait_copies();

  int it = t0;
  while (it < t1) {
    const int qbase = q_first + in_head * QT;
    if constexpr (BIAS) {
      if (it == t0 || in_head == 0) {
        __syncthreads();  // the previous head's table is no longer read
        fill_bias(tab, g, table, map, head);
      }
    }
    __syncthreads();
    // Tiles of this head whose queries all exist and see all of the workgroup's keys: the next
    // block's products beside this block's vector work.
    // (From an even tile on, so that the LDS buffers' places are constants.)
    const int to_end = min(t1 - it, (n - qbase) / QT);  // full tiles up to the head's end
    const bool whole = to_end > 0 && ((it - t0) & 1) == 0 &&
                       (!g.causal || qbase + off >= k0 + kSeqTile - 1);
    if constexpr (!BIAS && sizeof(T) == 2) {
      if (whole) {
        f32x16_t sa, pa;
        auto tile = [&](int t, int buf) {
          const T *qc = lds + 2 * E * buf, *qn = lds + 2 * E * (1 - buf);
          if (t + 1 < t1) fetch(1 - buf);
  #pragma unroll
          for (int b = 0; b < NB; ++b) {
            float s[16], ds[16];
  #pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = sa[i];
            const f32x16_t p0 = pa;
            const Affine f = biased(s, 0);  // without a bias no place counts
            if (b == NB - 1) {  // the next tile is in LDS
              wait_copies();
              __syncthreads();
            }
            if (b + 1 < NB) products(qc, b + 1, sa, pa);
            else products(qn, 0, sa, pa);
            weigh(buf, b, s, f, p0, ds);
            accumulate(qc, b, s, ds);
          }
          __syncthreads();
        };
        products(lds, 0, sa, pa);
        const int end = it + to_end;
        in_head += to_end;
        if (in_head == per_head) {
          in_head = 0;
          ++head;
        }
        for (; it + 1 < end; it += 2) {
          tile(it, 0);
          tile(it + 1, 1);
        }
        if (it < end) tile(it++, 0);
        continue;
      }
    }
    const int buf = (it - t0) & 1;
    const uint16_t* qc = Tl::operands(lds, buf);
    if (it + 1 < t1) fetch(1 - buf);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int qb = qbase + b * 32;
      if (qb >= n || !live || (g.causal && qb + 31 + off < j0)) continue;
      f32x16_t sa, pa;
      products(qc, b, sa, pa);
      float s[16], ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = sa[i];
      weigh(buf, b, s, biased(s, qb), pa, ds);
      if (qb + 31 >= n || (g.causal && qb + off < j0 + 31)) {
        // queries before the key, and rows past the sequence's end
        asm volatile("");
        const int from = g.causal ? jk - off - qb - 4 * hh : 0, to = n - qb - 4 * hh;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c_row(i, 0) < from || c_row(i, 0) >= to) s[i] = ds[i] = 0.0f;
      }
      accumulate(qc, b, s, ds);
    }
    wait_copies();
    ++it;
    if (++in_head == per_head) {
      in_head = 0;
      ++head;
    }
  }
  __syncthreads();
  if (!live) return;
  if constexpr (PARTS) {
    if (!kok) return;
    const int64_t row = (((int64_t)part * g.nk + krow) * g.KH + w.u) * D;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      store_block(part_dk + row, db, dka[db], g.scale);
      store_block(part_dv + row, db, dva[db], 1.0f);
    }
  } else {
    const int64_t first = ((int64_t)(sk.begin + j0) * g.KH + w.u) * D, step = (int64_t)g.KH * D;
    store_rows<T, D>(lds + wave * 32 * D, dka, g.scale, dk + first, step, m - j0);
    store_rows<T, D>(lds + wave * 32 * D, dva, 1.0f, dv + first, step, m - j0);
  }
}

// dk/dv pass of bf16 at 128 channels, where a wave has no room for both sums: two waves share 32
// keys (lanes l and l ^ 32 of each share key l % 32):
//   waves 0 - 3:  S = Q K^T,  alpha,  dv^T += dout^T alpha
//   waves 4 - 7:  dP = dout V^T,  dS = alpha (dP - Delta),  dk^T += Q^T dS
// so that each has one operand and one sum in registers (two waves per SIMD) and two of the four
// products.  The second takes alpha from the first through LDS, one query tile later, in 24 bits
// (16 significant ones, cut off, next to the 8 that dS is rounded to), which is what its lanes hold
// of the same block.  Measured for 8,192 tokens, 16 heads x 128, all keys: both sums in one wave,
// one wave per SIMD, 1.44 ms (matrix cores 30% busy); in one wave at two waves per SIMD, operands
// read as they are used, 1.5 ms; dv and dk as two launches with S formed twice 1.32 ms; this
// 1.17 ms (41% busy; no less with alpha in float16, whose range loses weights below 2^-28).
template <bool BIAS, bool PARTS>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
void seq_dkdv_pair_kernel(
    SeqGeometry g, const uint16_t* __restrict__ q, const uint16_t* __restrict__ k,
    const uint16_t* __restrict__ v, const int32_t* __restrict__ cu_q,
    const int32_t* __restrict__ cu_k, const float* __restrict__ table,
    const int32_t* __restrict__ map, const float* __restrict__ delta,
    const float* __restrict__ lse2, const uint16_t* __restrict__ dout, uint16_t* __restrict__ dk,
    uint16_t* __restrict__ dv, float* __restrict__ part_dk, float* __restrict__ part_dv) {
  using T = uint16_t;
  constexpr int D = 128, QT = 64;
  using Tl = Tile<T, D, QT, 512>;
  using Frag = typename Type<T>::Frag;
  constexpr int KS = D / 16, DB = D / 32, NB = QT / 32, E = Tl::kElems;
  // three tiles of queries and douts: the first waves', the second waves', the next
  __shared__ __attribute__((aligned(16))) T lds[6 * E];
  __shared__ uint4 alpha[2][NB][4][3 * 64];  // by step
  __shared__ __attribute__((aligned(16))) float stat[3][2][64];  // lse log2(e), Delta of a tile
  extern __shared__ float tab[];

  Work w;
  if (!work_of<false>(g.k_tiles, PARTS ? g.parts : 1, w)) return;
  const int part = PARTS ? w.head - w.u * g.parts : 0;
  const Place sk = place_of<kSeqTile, true>(cu_k, g.nk, cu_q, g.nq, g.B, g.causal, g.k_tiles.slots,
                                            w.slot);
  const int k0 = sk.tile * kSeqTile, m = sk.n, qbeg = sk.other, n = sk.m;
  if (k0 >= m) return;
  const int off = m - n;
  // first tile with a query that sees
  const int q_first = g.causal ? max(k0 - off, 0) / QT * QT : 0;
  const int per_head = n > q_first ? (n - q_first + QT - 1) / QT : 0;
  const int all = per_head * g.group;
  const int t0 = PARTS ? (int)((int64_t)all * part / g.parts) : 0;
  const int t1 = PARTS ? (int)((int64_t)all * (part + 1) / g.parts) : all;

  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const uint32_t qsb = (uint32_t)g.qs * sizeof(T), gsb = (uint32_t)g.H * Tl::kRowBytes;
  uint32_t qo[Tl::NC], go[Tl::NC];
  Tl::copy_plan(qo, qsb);
  Tl::copy_plan(go, gsb);
  // The tile fetched next, its head and its number in it; the number of the one before it, and of
  // the one before that.
  int head = w.u * g.group + (t0 < t1 ? t0 / per_head : 0);
  int next_at = t0 < t1 ? t0 % per_head : 0, first_at = 0, second_at = 0;
  auto fetch = [&](int buf) {
    const int at = q_first + next_at * QT;
    const int64_t row = qbeg + at;
    Tl::copy(lds + 2 * E * buf, q + row * g.qs + head * D, qo, qsb, n - at);
    Tl::copy(lds + 2 * E * buf + E, dout + (row * g.H + head) * D, go, gsb, n - at);
    if (wave < 2)  // the rows' statistics; past the sequence's end the last row's
      copy_4(lds_offset(&stat[buf][wave][0]), wave == 0 ? lse2 : delta,
             (uint32_t)min(lane, n - at - 1) * 4u, (int64_t)head * g.nq + row);
  };
  auto count_on = [&] {
    second_at = first_at;
    first_at = next_at;
    if (++next_at == per_head) {
      next_at = 0;
      ++head;
    }
  };
  if (t0 < t1) fetch(0);
  const int head0 = head;
  count_on();

  const int pair = wave & 3;
  const bool second = wave >= 4;
  const int j0 = k0 + pair * 32, jk = j0 + (lane & 31);
  const bool kok = jk < m, live = j0 < m;
  const int64_t krow = sk.begin + (kok ? jk : 0);
  Frag wf[KS];  // K or V
  load_frag<T, D>(wf, (second ? v + krow * g.vs : k + krow * g.ks) + w.u * D, kok);
  f32x16_t sum[DB];  // dv or dk
#pragma unroll
  for (int db = 0; db < DB; ++db) sum[db] = f32x16_t{};
  wait_copies();

  // x of a block: S or dP
  auto products = [&](const T* rows, int b) {
    f32x16_t x = f32x16_t{};
    Frag a[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) a[ks] = Tl::a_rows(rows, b * 32, ks);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) x = mfma(a[ks], wf[ks], x);
    return x;
  };
  // Block b of the tile in LDS buffer `buf`, its alpha in place `half`; qb: its first query.
  auto block = [&](int buf, int half, int b, int qb, const f32x16_t& x) {
    const T* cols = lds + 2 * E * buf + (second ? 0 : E);
    float y[16];
    const float* st = &stat[buf][second ? 1 : 0][b * 32 + 4 * hh];
    uint4* al = &alpha[half][b][pair][lane];
    if (!second) {
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = x[i];
      Affine f = {g.scale_log2, 0.0f};
      if constexpr (BIAS)
        f = add_bias<-1>(y, g, tab, j0 - (qb + 31 + off), jk - qb - 4 * hh - off);
#pragma unroll
      for (int blk = 0; blk < 4; ++blk) {
        const float4 l4 = *reinterpret_cast<const float4*>(st + 8 * blk);
        const float lv[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = 4 * blk + j;
          y[i] = __builtin_amdgcn_exp2f(fmaf(y[i], f.mul, f.add - lv[j]));
        }
      }
      if (qb + 31 >= n || (g.causal && qb + off < j0 + 31)) {
        // queries before the key, and rows past the sequence's end
        asm volatile("");
        const int from = g.causal ? jk - off - qb - 4 * hh : 0, to = n - qb - 4 * hh;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c_row(i, 0) < from || c_row(i, 0) >= to) y[i] = 0.0f;
      }
      hand_over(al, y);
    } else {
      take_over(al, y);
#pragma unroll
      for (int blk = 0; blk < 4; ++blk) {
        const float4 d4 = *reinterpret_cast<const float4*>(st + 8 * blk);
        const float dl[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) y[4 * blk + j] *= x[4 * blk + j] - dl[j];
      }
    }
    Frag f[2];
    to_frags(y, f);
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        sum[db] = mfma(Tl::a_cols(cols, db * 32, b, p), f[p], sum[db]);
  };

  // Step i: the first waves work on tile t0 + i, the second ones on the tile before it.  Tile i is
  // in buffer i % 3, which the calls below have as a constant.
  const int steps = t1 - t0;
  auto run = [&](int step, int in, int out, int next) {
    __syncthreads();
    if constexpr (BIAS) {
      if (step < steps && (step == 0 || first_at == 0)) {
        fill_bias<512>(tab, g, table, map, step == 0 ? head0 : next_at == 0 ? head - 1 : head);
        __syncthreads();
      }
    }
    if (step + 1 < steps) fetch(next);
    const int half = (step & 1) ^ (second ? 1 : 0);  // the second waves: the step before
    auto tile = [&](int at, int buf) {
      const int qb = q_first + at * QT;
      if (g.causal && qb + QT - 1 + off < j0) return;  // the same for both waves
      const T* rows = lds + 2 * E * buf + (second ? E : 0);
      f32x16_t x = products(rows, 0);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x16_t y = f32x16_t{};
        if (b + 1 < NB) y = products(rows, b + 1);
        block(buf, half, b, qb + b * 32, x);
        x = y;
      }
    };
    if (live) {
      if (!second) {
        if (step < steps) tile(first_at, in);
      } else if (step > 0) {
        tile(second_at, out);
      }
    }
    count_on();
    wait_copies();
  };
  for (int step = 0; step <= steps; step += 3) {
    run(step, 0, 2, 1);
    if (step + 1 <= steps) run(step + 1, 1, 0, 2);
    if (step + 2 <= steps) run(step + 2, 2, 1, 0);
  }
  __syncthreads();
  if (!live) return;
  const float mul = second ? g.scale : 1.0f;
  if constexpr (PARTS) {
    if (!kok) return;
    float* to = (second ? part_dk : part_dv) + (((int64_t)part * g.nk + krow) * g.KH + w.u) * D;
#pragma unroll
    for (int db = 0; db < DB; ++db) store_block(to, db, sum[db], mul);
  } else {
    store_rows<T, D>(lds + wave * 32 * D, sum, mul,
                     (second ? dk : dv) + ((int64_t)(sk.begin + j0) * g.KH + w.u) * D,
                     (int64_t)g.KH * D, m - j0);
  }
}

// Adds the parts of dk and dv in their order and rounds: four values per thread, `count` groups of
// four in each part.
template <typename T>
__global__ __launch_bounds__(kThreads) void seq_join_kernel(int64_t count, int parts,
                                                            const float4* __restrict__ part_dk,
                                                            const float4* __restrict__ part_dv,
                                                            T* __restrict__ dk,
                                                            T* __restrict__ dv) {
  const int64_t i = (int64_t)(blockIdx.x / 2) * kThreads + threadIdx.x;
  if (i >= count) return;
  const float4* from = blockIdx.x % 2 == 0 ? part_dk : part_dv;
  T* to = (blockIdx.x % 2 == 0 ? dk : dv) + i * 4;
  float4 sum = from[i];
  for (int p = 1; p < parts; ++p) {
    const float4 x = from[p * count + i];
    sum.x += x.x;
    sum.y += x.y;
    sum.z += x.z;
    sum.w += x.w;
  }
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(to) = sum;
  } else {
    const uint16_t h[4] = {to_bf16(sum.x), to_bf16(sum.y), to_bf16(sum.z), to_bf16(sum.w)};
    *reinterpret_cast<uint2*>(to) = __builtin_bit_cast(uint2, h);
  }
}

// ---------------------------------------------------------------------------- launches

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
  return seq_launch(fn, seq_blocks(h.q_tiles, g.group), W * 64, bias ? padded(g.span) * 4 : 0, s, h,
                    (const T*)t.q, (const T*)t.k, (const T*)t.v, t.cu_q, t.cu_k, t.table, t.map,
                    out, res, lse);
}

template <typename T, int D>
hipError_t forward_d(const SeqGeometry& g, const SeqTensors& t, T* out, T* res, float* lse,
                     hipStream_t s) {
  // Eight waves halve the copies per product but leave half the workgroups: they pay where the
  // sequences are long and the workgroups many.  16 heads, 4 / 8 waves, us:
  //                            64 channels                      128 channels
  //   tokens              plain    bias   residual        plain    bias   residual
  //   one of 8,192      330/313  350/335  237/233 causal  513/495  529/516  377/363 causal
  //   two of 4,096      169/162  180/173  124/122 causal  261/253  270/262  196/188 causal
  //   four of 2,048      90/87    96/93    69/70  causal  138/138  141/142  111/110 causal
  //   32 of 512          55/60    61/64    52/63  causal   84/96    89/100   78/94  causal
  //   one of 4,096 x 8   59/75    71/84    75/102 causal   81/106   89/116  101/140 causal
  // One causal sequence of 16,384 at 64 channels is slower by 1% (residual 4%) with eight.
  const bool wide = g.nk >= 4096 * (int64_t)g.B && (int64_t)g.nq * g.H >= 256 * 512;
  if constexpr (sizeof(T) == 2) {
    if (wide) return forward_w<T, D, 8>(g, t, out, res, lse, s);
  }
  return forward_w<T, D, 4>(g, t, out, res, lse, s);
}

// The backward's workspace: Delta and lse log2(e) [heads][rows], the bias gradient's bucket sums,
// and the parts of dk and dv.
struct Workspace {
  size_t lse2, partial, part_dk, part_dv, bytes;
};
Workspace workspace_of(const SeqGeometry& g, bool want_table) {
  Workspace w;
  size_t at = round_256((size_t)g.nq * g.H * 4);
  w.lse2 = at;
  at *= 2;
  w.partial = at;
  if (want_table) at += round_256((size_t)g.q_tiles.slots * g.H * g.nb * 4);
  w.part_dk = at;
  const size_t part = g.parts > 1 ? round_256((size_t)g.parts * g.nk * g.KH * g.D * 4) : 0;
  w.part_dv = at + part;
  w.bytes = at + 2 * part;
  return w;
}

template <typename T, int D>
hipError_t backward_d(const SeqGeometry& g, const SeqTensors& t, const T* out, const T* res,
                      const float* lse, const T* dout, T* dq, T* dk, T* dv, float* d_table,
                      void* workspace, hipStream_t s) {
  const bool bias = g.nb > 0, want_table = bias && d_table != nullptr;
  const T *q = (const T*)t.q, *k = (const T*)t.k, *v = (const T*)t.v;
  const Workspace at = workspace_of(g, want_table);
  char* ws = (char*)workspace;
  float *delta = (float*)ws, *lse2 = (float*)(ws + at.lse2);
  float* partial = want_table ? (float*)(ws + at.partial) : nullptr;
  float* part_dk = g.parts > 1 ? (float*)(ws + at.part_dk) : nullptr;
  float* part_dv = g.parts > 1 ? (float*)(ws + at.part_dv) : nullptr;
  hipError_t e = hipSuccess;
  if (g.nq > 0) {
    const void* fn = bias ? (const void*)&seq_dq_kernel<T, D, true>
                          : (const void*)&seq_dq_kernel<T, D, false>;
    const size_t lds = !bias     ? 0
                       : partial ? 4 * (5 * (size_t)padded(g.span) + 8 + 4 * kSkewed)
                                 : 4 * (size_t)padded(g.span);
    e = seq_launch(fn, seq_blocks(g.q_tiles, g.group), kThreads, lds, s, g, q, k, v, t.cu_q,
                   t.cu_k, t.table, t.map, out, res, lse, dout, dq, delta, lse2, partial);
  }
  if (e == hipSuccess && want_table)
    e = seq_launch((const void*)&seq_table_kernel, g.H, kThreads, 0, s,
                   g.nq > 0 ? g.q_tiles.slots : 0, g.H, g.nb, (const float*)partial, d_table);
  if (e == hipSuccess && g.nk > 0) {
    const bool parts = g.parts > 1;
    const void* fn;
    constexpr bool kPair = sizeof(T) == 2 && D == 128;
    if constexpr (kPair)
      fn = parts ? (bias ? (const void*)&seq_dkdv_pair_kernel<true, true>
                         : (const void*)&seq_dkdv_pair_kernel<false, true>)
                 : (bias ? (const void*)&seq_dkdv_pair_kernel<true, false>
                         : (const void*)&seq_dkdv_pair_kernel<false, false>);
    else
      fn = parts ? (bias ? (const void*)&seq_dkdv_kernel<T, D, true, true>
                         : (const void*)&seq_dkdv_kernel<T, D, false, true>)
                 : (bias ? (const void*)&seq_dkdv_kernel<T, D, true, false>
                         : (const void*)&seq_dkdv_kernel<T, D, false, false>);
    e = seq_launch(fn, seq_blocks(g.k_tiles, g.parts), kPair ? 512 : kThreads,
                   bias ? (size_t)padded(g.span) * 4 : 0, s, g, q, k, v, t.cu_q, t.cu_k, t.table,
                   t.map, (const float*)delta, (const float*)lse2, dout, dk, dv, part_dk, part_dv);
  }
  if (e == hipSuccess && g.nk > 0 && g.parts > 1) {
    const int64_t count = (int64_t)g.nk * g.KH * D / 4;
    const int64_t blocks = (count + kThreads - 1) / kThreads;
    e = seq_launch((const void*)&seq_join_kernel<T>, 2 * blocks, kThreads, 0, s, count, g.parts,
                   (const float4*)part_dk, (const float4*)part_dv, dk, dv);
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

// Parts of the dk/dv pass.  Key heads x key tiles workgroups do the work of all heads of a group;
// where they are fewer than two per compute unit (four under a causal mask, where the first tiles
// have twice the average work), the (head, query tile) pairs are dealt out to up to 16 parts.  Key
// tiles are estimated from the rows and sequences.  A part has at least 256 queries of a head on
// average (1,900 tokens, 8 heads x 128, bf16: step of 99 us, 109 with parts of 128), in float32,
// whose tiles take longer than the join, 64 (1,721 tokens, 6 heads x 64: 234 us with parts of 256,
// 191 of 128, 170 of 64).
int seq_backward_parts(const SeqGeometry& g, bool bf16) {
  const int64_t blocks = (int64_t)g.KH * std::max<int64_t>(1, g.nk / kSeqTile);
  const int least = bf16 ? 256 : 64;
  const int64_t most = std::min<int64_t>(16, (int64_t)g.group * std::max(1, g.nq / g.B / least));
  return (int)std::max<int64_t>(1, std::min<int64_t>((g.causal ? 1024 : 512) / blocks, most));
}

size_t seq_backward_workspace(const SeqGeometry& g, bool want_table) {
  return workspace_of(g, want_table).bytes;
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
