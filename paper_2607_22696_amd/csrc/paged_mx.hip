// A paged cache held in 8 or 4 bits: the write of new tokens, their reading back, and the newest
// tokens' attention over the pages (include/dsa3d_mx.h), gfx950 kernels.
//
// A token's key or value of one head is D / 32 blocks of 32 elements (e4m3 or e2m1 floats) and a
// power of two each.  Elements are rounded and read by gfx950's scaled conversions.  Every value is
// a bf16 number exactly, and the products are those of paged.hip on bf16 operands.  (The scaled 8-bit
// products, v_mfma_scale_f32_32x32x64_f8f6f4, take the elements as they are, but not with a
// float32 sum: 64 terms of up to 1,024 came out up to 0.07 off, 2^-14 of the largest.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "paged_device.h"

namespace dsa3d {
namespace {

using namespace paged;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// The cache as the kernels take it: addresses of the first page.
struct MxPages {
  uint8_t *k, *v, *ks, *vs;
};

__device__ inline float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Elements as bf16: 8 channels of 8 bits from two words, or of 4 bits from one, times a power.
__device__ inline uint32_t two_of_8(uint32_t u, float power, bool upper) {
  return __builtin_bit_cast(uint32_t,
                            upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, power, true)
                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, power, false));
}
__device__ inline uint4 eight(uint32_t lo, uint32_t hi, float power) {
  return make_uint4(two_of_8(lo, power, false), two_of_8(lo, power, true),
                    two_of_8(hi, power, false), two_of_8(hi, power, true));
}
__device__ inline uint4 eight(uint32_t u, float power) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, power, 0),
                 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, power, 1),
                 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, power, 2),
                 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, power, 3);
  return make_uint4(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b),
                    __builtin_bit_cast(uint32_t, c), __builtin_bit_cast(uint32_t, d));
}

// A quarter of a key's or value's channels, a block or half of one, as W words of elements and the
// block's scale.
template <int BITS, int W>
struct Quarter {
  uint32_t w[W];
  // As narrow as in memory: widened where it is loaded, it is widened again at the end of a loop
  // that it is carried over, which waits for it there.
  uint8_t scale;

  __device__ inline void load(const uint8_t* at, const uint8_t* scale_at) {
    if constexpr (W >= 4) {
#pragma unroll
      for (int i = 0; i < W / 4; ++i)
        *reinterpret_cast<uint4*>(w + 4 * i) = *reinterpret_cast<const uint4*>(at + 16 * i);
    } else {
      *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(at);
    }
    scale = *scale_at;
  }
  __device__ inline uint4 eight_at(int chunk) const {  // channels 8 chunk .. + 7 of the quarter
    if constexpr (BITS == 8)
      return eight(w[2 * chunk], w[2 * chunk + 1], power_of(scale));
    else
      return eight(w[chunk], power_of(scale));
  }
};

// Alpha as an operand: 16 bits of it as two bf16 numbers, or a float32's three parts.  (One bf16
// number of it, the results divided by the sum of the rounded, takes less where products are the
// time, chunks of 512, 801 and 300 tokens beside three single ones 203 us instead of 252, and 64
// requests with 6 new tokens in 4 bits 86 instead of 91; but outputs are then off by 0.0020 to
// 0.0021 of their size instead of the 0.0016 that their own rounding makes.)
struct Two {
  bf16x8_t h, l;
};
template <typename T>
struct Alpha;
template <>
struct Alpha<uint16_t> {
  using Frag = Two;
  static __device__ inline Two of(const float* x) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y[2] = {x[2 * i], x[2 * i + 1]};
      h[i] = take_part(y);
      l[i] = take_part(y);
    }
    return {as_bf16x8(make_uint4(h[0], h[1], h[2], h[3])),
            as_bf16x8(make_uint4(l[0], l[1], l[2], l[3]))};
  }
};
template <>
struct Alpha<float> {
  using Frag = Split;
  static __device__ inline Split of(const float* x) {
    F32x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y.x[e] = x[e];
    return seq::split(y);
  }
};

// The products of exact bf16 keys and values with queries and alpha, which may be of parts.
__device__ inline f32x16_t times(const bf16x8_t& a, const bf16x8_t& b, const f32x16_t& c) {
  return mfma(a, b, c);
}
__device__ inline f32x16_t times(const bf16x8_t& a, const Two& b, f32x16_t c) {
  c = mfma(a, b.l, c);
  return mfma(a, b.h, c);
}
__device__ inline f32x16_t times(const bf16x8_t& a, const Split& b, f32x16_t c) {
  c = mfma(a, b.l, c);
  c = mfma(a, b.m, c);
  return mfma(a, b.h, c);
}

// A row's results to the output or, where its keys are in several parts, to the workspace.
template <typename T>
__device__ inline void store_4(T* to, const float4& y) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(to) = y;
  } else {
    const uint16_t h[4] = {to_bf16(y.x), to_bf16(y.y), to_bf16(y.z), to_bf16(y.w)};
    *reinterpret_cast<uint2*>(to) = __builtin_bit_cast(uint2, h);
  }
}

// Keeps a wave's own LDS accesses in their order (the LDS serves a wave in order).
__device__ inline void fence_wave() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The workgroup's key head, tile and part where parts are not dealt out.  A part of a head's keys
// stays on one XCD, whose L2 then serves it to the tiles of a request.
__device__ inline bool work_of_part(const PagedGeometry& g, Work& w, int& split) {
  if (!work_of(g.tiles, 1, w)) return false;
  split = w.u / g.KH;
  w.u -= split * g.KH;
  return true;
}

// Up to 64 requests, a lane each, with one load of their offsets and lengths.
struct Held {
  int begin, end, n, m, keys, tiles;
};
template <int ROWS>
__device__ inline Held held_by_lane(const PagedGeometry& g, const int32_t* cu_q,
                                    const int32_t* kv_lens) {
  const int lane = threadIdx.x & 63, b = min(lane, g.B - 1);
  const int raw = cu_q[b], raw_next = cu_q[b + 1], raw_m = kv_lens[b];  // three loads at once
  Held h;
  h.begin = b == 0 ? 0 : min(max(raw, 0), g.nq);
  h.end = min(max(raw_next, 0), g.nq);
  h.n = lane < g.B ? max(h.end - h.begin, 0) : 0;
  h.m = max(raw_m, 0);
  h.keys = h.n > 0 ? min(h.m, g.max_kv) : 0;
  h.tiles = h.n * g.group / ROWS + (h.n * g.group % ROWS != 0);
  return h;
}

// Deals numbers out to the lanes, `count` to each, those of size 3 first, then 2, 1 and 0, so that
// what is dealt out last is short.  The lane that has number `index`, and which of its numbers that
// is; behind the last one -1, and how far behind.
__device__ inline int lane_of(int index, int count, int size, int& nth) {
  int start = 0, before = 0;
#pragma unroll
  for (int c = 3; c >= 0; --c) {
    const int sum = prefix_sum(size == c ? count : 0);
    if (size == c) start = before + sum - count;
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  const uint64_t who = __ballot(index >= start && index < start + count);
  if (who == 0) {
    nth = index - before;
    return -1;
  }
  const int l = __builtin_ctzll(who);
  nth = index - __builtin_amdgcn_readlane(start, l);
  return l;
}

// The span of tile `tile` of lane l's request, or of the rows behind the last one (l = -1), which
// see nothing; false if there is no such tile.
template <int ROWS>
__device__ inline bool span_of(const PagedGeometry& g, const Held& h, int l, int tile, Span1& s) {
  if (l < 0) {
    s.b = g.B;
    s.begin = __builtin_amdgcn_readlane(h.end, g.B - 1);
    s.n = g.nq - s.begin;
    s.m = 0;
  } else {
    s.b = l;
    s.begin = __builtin_amdgcn_readlane(h.begin, l);
    s.n = __builtin_amdgcn_readlane(h.n, l);
    s.m = __builtin_amdgcn_readlane(h.m, l);
  }
  s.rows = s.n * g.group;
  if (tile > (s.rows - 1) / ROWS || s.rows == 0) return false;
  s.r0 = tile * ROWS;
  s.off = s.m - s.n;
  s.seen = min(s.m, g.max_kv);
  int hi = s.seen;
  if (g.causal)
    hi = min(hi, s.off + div_by(min(s.r0 + ROWS, s.rows) - 1, g.group_mul, g.group_shift) + 1);
  s.k_hi = max(hi, 0);
  return true;
}
// Part `split` of its keys, `len` of them.
__device__ inline void take_keys(Span1& s, int split, int len) {
  s.k_lo = (int)min((int64_t)split * len, (int64_t)s.k_hi);
  s.k_hi = (int)min((int64_t)s.k_hi, (int64_t)s.k_lo + len);
}

// What a workgroup works on.
struct Deal {
  Span1 s;
  int u, split, parts;  // key head; part of how many (the most there are where not dealt out)
  int nth, tiles;       // where dealt out and in parts: this one's number among the key head's
                        // parts with partial results; how far on the tile's next part is
};

// Partial results: [part][key head][row of the tile] of the parts that are dealt out, else [row of
// out][part]; log-sum-exps (base 2) and D channels in float32.  For each row of out, where they
// are: x the number of its tile's first part, y from there to the next, z how many (0: none, the
// row is in out), w key head x rows per tile + row of the tile.
struct Parts {
  int4* of;
  float *l, *o;
};
template <int ROWS>
__device__ inline int64_t part_row(const PagedGeometry& g, const Deal& w, int r, int64_t out_at) {
  return g.target > 0 ? ((int64_t)w.nth * g.KH + w.u) * ROWS + r : out_at * g.splits + w.split;
}
template <int ROWS>
__device__ inline int4 parts_of(const Deal& w, int r) {
  return make_int4(w.nth, w.tiles, w.parts, w.u * ROWS + r);
}

// Up to 64 requests' keys are divided by the sum of their lengths, and longer parts come first; a
// request's tiles over the same part follow each other, the last (under a causal mask the longest)
// first.  (A chunk of 400 of 30,000 tokens before 40 of 100 of 700, 32 / 8 heads, alpha in one bf16
// number: 784 us as they lie in parts chosen without the lengths, 712 longest first, 318 divided;
// chunks of 512, 801 and 300 of 16,000, 801 and 5,000 tokens beside three single ones 235 and 215.)
// More requests, of which a wave does not hold one a lane, come as they lie, in parts that the host
// chose: near what reading takes where they are alike (single tokens, 32 / 8 heads x 128, 128
// requests of 200 to 8,000 tokens: 219 us), but a long one among short ones is waited for (120,000
// tokens beside 63 requests of 200 to 2,000: 83 us, divided; beside 127: 532).
//
// Workgroups go round the XCDs by number.  Where the key heads are a multiple of 8 a head stays on
// one XCD, whose L2 serves a part to all tiles that read it.  Fewer lie on several, each of which
// reads the part (chunks as above with 8, 4, 2, 1 key heads and as many times 4 heads: 2.1, 2.5,
// 2.8, 3.6 times their products' time at the rate of large ones); whole heads on an XCD would leave
// six of them idle for 2 (four requests of 31,000 to 120,000 tokens, 16 / 2 heads, 4 bits: 45 us so,
// 30 spread out).
template <int ROWS>
__device__ inline bool deal(const PagedGeometry& g, const int32_t* cu_q, const int32_t* kv_lens,
                            Deal& d) {
  Span1& s = d.s;
  if (g.target == 0) {
    Work w;
    if (!work_of_part(g, w, d.split)) return false;
    d.u = w.u;
    d.parts = g.splits;
    d.nth = d.tiles = 0;
    return locate<ROWS>(g, cu_q, kv_lens, w.slot, d.split, s);
  }
  constexpr int STEP = 256;  // keys of the four waves' groups
  const int block = block_number(), index = block / g.KH;
  d.u = block - index * g.KH;
  const Held h = held_by_lane<ROWS>(g, cu_q, kv_lens);
  float all = (float)h.tiles * (float)h.keys;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) all += __shfl_xor(all, x);
  const float share = fminf(all / (float)g.target, (float)(1 << 30));
  const int most = max(((int)share + STEP) / STEP * STEP, g.part);  // more than a share
  const int parts = min(max(h.keys / most + (h.keys % most != 0), 1), g.splits);
  const int len = ((h.keys + parts - 1) / parts + STEP - 1) / STEP * STEP;
  int r;
  const int l = lane_of(index, h.tiles * parts, min((int)((int64_t)len * 4 / (most + 1)), 3), r);
  int tile = r;
  d.split = d.nth = d.tiles = 0;
  d.parts = 1;
  if (l >= 0) {
    const int tiles = __builtin_amdgcn_readlane(h.tiles, l);
    d.parts = __builtin_amdgcn_readlane(parts, l);
    d.split = r / tiles;
    tile = tiles - 1 - (r - d.split * tiles);
    if (d.split >= d.parts) return false;  // only where offsets decrease
    if (d.parts > 1) {
      const int mine = parts > 1 ? h.tiles * parts : 0;
      d.nth = __builtin_amdgcn_readlane(prefix_sum(mine) - mine, l) + r;
      d.tiles = tiles;
      if (d.nth < 0 || d.nth >= g.room) return false;  // likewise
    }
  }
  if (!span_of<ROWS>(g, h, l, tile, s)) return false;
  s.only = d.parts == 1;
  take_keys(s, d.split, l < 0 ? 0 : __builtin_amdgcn_readlane(len, l));
  return true;
}

// ------------------------------------------------------------------------- many rows

// 128 rows per workgroup, 32 per wave, tiles of 64 keys in LDS as bf16, two of them: a tile's
// elements are loaded two tiles ahead, converted once for all four waves, and the products of the
// next 32 keys run beside the softmax of these.  At 128 channels bf16 spills 32 to 47 registers, all of
// them around the last one or two tiles: the loop has none.
template <typename T, int D, int BITS, bool BIAS>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2)))
void mx_rows_kernel(PagedGeometry g, const T* __restrict__ q, MxPages c,
                    const int32_t* __restrict__ pages, const int32_t* __restrict__ kv_lens,
                    const int32_t* __restrict__ cu_q, const float* __restrict__ table,
                    const int32_t* __restrict__ map, T* __restrict__ out,
                    float* __restrict__ lse, Parts to) {
  constexpr int KT = 64, RB = D * BITS / 8, SB = D / 32;
  using Tl = Tile<uint16_t, D, KT>;
  using Frag = typename Type<T>::Frag;
  using Part = Quarter<BITS, RB / 16>;  // four lanes share a key
  constexpr int KS = D / 16, DB = D / 32, NB = KT / 32, E = Tl::kElems;
  __shared__ __attribute__((aligned(16))) uint16_t lds[4 * E];  // keys, values; twice
  __shared__ __attribute__((aligned(8))) uint16_t there[2][4];
  extern __shared__ float bias[];

  Deal w;
  if (!deal<kManyRows>(g, cu_q, kv_lens, w)) return;
  const Span1& s = w.s;
  const int ntiles = s.k_hi > s.k_lo ? (s.k_hi - s.k_lo + KT - 1) / KT : 0;
  const int lane = threadIdx.x & 63, wave = wave_id(), hh = lane >> 5;
  const int rw = s.r0 + wave * 32;
  const bool live = rw < s.rows;
  const Row x = row_of(g, s, w.u, rw + (lane & 31));
  Frag qf[KS];
  load_frag<T, D>(qf, q + x.q_at, x.ok);

  // A wave has 16 keys of a tile, a quarter of the channels per lane, in an order in which the chunks
  // that 8 lanes write to LDS meet in no bank.  Keys past the last repeat it, to be masked; one
  // without a place has the first page's first row, to be cleared.
  auto key_of_lane = [](int l) {
    return D == 128 ? (l & 1) | (l >> 3 & 1) << 1 | (l >> 1 & 3) << 2
                    : (l >> 3 & 1) | (l & 7) << 1;
  };
  const int key = wave * 16 + key_of_lane(lane & 15), part = lane >> 4;
  const int32_t* my_pages = pages + (int64_t)s.b * g.max_pages;
  auto key_of = [&](int kt) { return min(s.k_lo + kt * KT + key, s.k_hi - 1); };
  auto page_of = [&](int kt) {
    return my_pages[div_by((uint32_t)key_of(kt), g.page_mul, g.page_shift)];
  };
  Part kq, vq;
  auto load = [&](int kt, int p) {  // returns which of the wave's keys have a place, by lane
    const int j = key_of(kt), page = div_by((uint32_t)j, g.page_mul, g.page_shift);
    const bool ok = (uint32_t)p < (uint32_t)g.num_pages;
    const int64_t row =
        ok ? ((int64_t)p * g.KH + w.u) * g.page_size + (j - page * g.page_size) : 0;
    const int64_t at = row * RB + part * (RB / 4), sc = row * SB + part * SB / 4;
    kq.load(c.k + at, c.ks + sc);
    vq.load(c.v + at, c.vs + sc);
    return (uint32_t)__ballot(ok) & 0xffffu;
  };
  auto put = [&](uint32_t ok, int buf) {
    uint16_t* to = lds + 2 * E * buf;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const int at = Tl::at(key, part * (D / 4) + 8 * i);
      *reinterpret_cast<uint4*>(to + at) = kq.eight_at(i);
      *reinterpret_cast<uint4*>(to + E + at) = vq.eight_at(i);
    }
    uint32_t by_key = ok;
    if (ok != 0xffffu) {
      if ((ok >> (lane & 15) & 1) == 0) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
          *reinterpret_cast<uint4*>(to + E + Tl::at(key, part * (D / 4) + 8 * i)) =
              make_uint4(0, 0, 0, 0);
      }
      by_key = 0;
      for (int i = 0; i < 16; ++i) by_key |= (ok >> i & 1) << key_of_lane(i);
    }
    if (lane == 0) there[buf][wave] = (uint16_t)by_key;
  };
  uint32_t ok1 = 0;  // of the tile in kq and vq
  int next_page = 0;
  if (ntiles > 0) {
    const uint32_t ok0 = load(0, page_of(0));
    const int page1 = page_of(1);
    put(ok0, 0);
    ok1 = load(1, page1);
    next_page = page_of(2);
  }
  if constexpr (BIAS) fill_bias(bias, g, table, map, w.u);

  const int pos = s.off + x.i;
  const int last = min(g.causal ? min(s.seen - 1, pos) : s.seen - 1, s.k_hi - 1);
  const int all_see =
      min(g.causal ? min(s.seen - 1, s.off + div_by(rw, g.group_mul, g.group_shift))
                   : s.seen - 1, s.k_hi - 1);
  f32x16_t o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x16_t{};
  Softmax sm;
  const float scale = BIAS ? 1.0f : g.scale_log2;
  auto products = [&](const uint16_t* kc, int b) {
    f32x16_t acc = f32x16_t{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) acc = times(Tl::a_rows(kc, b * 32, ks), qf[ks], acc);
    return acc;
  };
  auto mask = [&](float (&y)[16], int kb, uint32_t bits) {
    if constexpr (BIAS) add_bias(y, g, bias, x.head - w.u * g.group, kb, pos);
    if (bits != ~0u || kb + 31 > all_see) {
      asm volatile("");  // a branch: blocks that every row sees do not pay for it
      const int seen = last - kb - 4 * hh;
      const uint32_t mine = bits >> (4 * hh);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (c_row(i, 0) > seen || (mine >> c_row(i, 0) & 1) == 0) y[i] = -INFINITY;
    }
  };
  auto accumulate = [&](const uint16_t* vc, int b, const float (&y)[16]) {
    const typename Alpha<T>::Frag pf[2] = {Alpha<T>::of(y), Alpha<T>::of(y + 8)};
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        o[db] = times(Tl::a_cols(vc, db * 32, b, p), pf[p], o[db]);
  };
  __syncthreads();
  // All tiles; LIVE: the wave has rows, else it only converts its share of them.  MORE: another
  // tile follows, which is converted first and whose first products end this one.
  auto run = [&](auto live_wave) {
    constexpr bool LIVE = decltype(live_wave)::value;
    f32x16_t next;
    if constexpr (LIVE) next = products(lds, 0);
    auto tile = [&](int kt, int buf, auto more) {
      constexpr bool MORE = decltype(more)::value;
      const uint16_t *kc = lds + 2 * E * buf, *kn = lds + 2 * E * (1 - buf);
      const uint2 bits = *reinterpret_cast<const uint2*>(there[buf]);
      if constexpr (MORE) {
        put(ok1, 1 - buf);
        __builtin_amdgcn_sched_barrier(0);  // the same registers, as in mx_keys_kernel
        ok1 = load(kt + 2, next_page);
        next_page = page_of(kt + 3);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float y[16];
        if constexpr (LIVE) {
#pragma unroll
          for (int i = 0; i < 16; ++i) y[i] = next[i];
          mask(y, s.k_lo + kt * KT + b * 32,
               __builtin_amdgcn_readfirstlane(b == 0 ? bits.x : bits.y));
          sm.raise_to(y, scale, o);
        }
        if (MORE && b == NB - 1) __syncthreads();  // the next tile is in LDS
        if constexpr (LIVE) {
          // ahead of the other workgroup's wave on this SIMD while the matrix cores have work: chunks
          // 251 and 245 us, at 64 channels 198 and 163, a prompt of 4,096 tokens 225 and 208
          __builtin_amdgcn_s_setprio(1);
          if constexpr (MORE) next = b + 1 < NB ? products(kc, b + 1) : products(kn, 0);
          else if (b + 1 < NB) next = products(kc, b + 1);
          sm.weigh(y, scale);
          accumulate(kc + E, b, y);
          __builtin_amdgcn_s_setprio(0);
        }
      }
      if constexpr (MORE) __syncthreads();  // and this one is free
    };
    int kt = 0;
    for (; kt + 2 < ntiles; kt += 2) {
      tile(kt, 0, std::true_type());
      tile(kt + 1, 1, std::true_type());
    }
    if (kt + 1 < ntiles) {
      tile(kt, 0, std::true_type());
      tile(kt + 1, 1, std::false_type());
    } else {
      tile(kt, 0, std::false_type());
    }
  };
  if (ntiles > 0) {
    if (live) run(std::true_type());
    else run(std::false_type());
  }
  const float ltot = pair_sum(sm.l);
  const float inv = ltot > 0.0f ? 1.0f / ltot : ltot;
  const float l2 = ltot == 0.0f ? -INFINITY : sm.base + __builtin_amdgcn_logf(ltot);
  if (!x.ok) return;
  if (s.only) {
#pragma unroll
    for (int db = 0; db < DB; ++db) store_block(out + x.out_at * D, db, o[db], inv);
    if (hh == 0 && lse != nullptr) lse[x.out_at] = l2 * kLn2;
    if (hh == 0 && g.splits > 1) to.of[x.out_at] = make_int4(0, 0, 0, 0);
  } else {
    const int r = wave * 32 + (lane & 31);
    const int64_t at = part_row<kManyRows>(g, w, r, x.out_at);
    if (ltot != 0.0f) {  // the join skips the parts of a row without keys
#pragma unroll
      for (int db = 0; db < DB; ++db) store_block(to.o + at * D, db, o[db], inv);
    }
    if (hh == 0) to.l[at] = l2;
    if (hh == 0 && w.split == 0) to.of[x.out_at] = parts_of<kManyRows>(w, r);
  }
}

// ------------------------------------------------------------------------- few rows

typedef float f32x4_t __attribute__((ext_vector_type(4)));

// 16 x 16 blocks of v_mfma_f32_16x16x32_bf16: lane l has row (column) l % 16 of an operand and 8 of
// the 32 contraction indices, those of quarter l / 16 of the wave; of the result column l % 16 and
// rows 4 (l / 16) .. + 3.
__device__ inline f32x4_t mfma16(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4_t times(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) {
  return mfma16(a, b, c);
}
__device__ inline f32x4_t times(const bf16x8_t& a, const Two& b, f32x4_t c) {
  c = mfma16(a, b.l, c);
  return mfma16(a, b.h, c);
}
__device__ inline f32x4_t times(const bf16x8_t& a, const Split& b, f32x4_t c) {
  c = mfma16(a, b.l, c);
  c = mfma16(a, b.m, c);
  return mfma16(a, b.h, c);
}

// x of the lanes 16 s .. 16 s + 15 in all four quarters, s = 0 .. 3.
__device__ inline void quarters(uint32_t x, uint32_t (&y)[4]) {
  const auto half = __builtin_amdgcn_permlane32_swap(x, x, false, false);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto two = __builtin_amdgcn_permlane16_swap(half[i], half[i], false, false);
    y[2 * i] = two[0];
    y[2 * i + 1] = two[1];
  }
}
// x joined over the four lanes that have the same column.
template <typename Join>
__device__ inline float over_quarters(float x, const Join& join) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  x = join(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return join(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float max_of(float x) {
  return over_quarters(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float sum_of(float x) {
  return over_quarters(x, [](float a, float b) { return a + b; });
}

// A wave's 32 rows of values in LDS: chunks of 8 channels XOR-permuted by the row, so that neither
// the writes (one chunk of 8 consecutive rows at a time, over 128 bytes of banks) nor the transposing
// reads (two neighbouring chunks of 8 consecutive rows, over 256) meet in a bank.
template <int D>
__device__ inline int value_at(int row, int chan) {
  const int f = D == 128 ? (row & 7) << 1 | (row >> 2 & 1) : row & 7;
  return row * D + (((chan >> 3) ^ f) << 3) + (chan & 7);
}
// Channels d0 .. d0 + 15 as rows, over the 32 keys in the order in which two results hold them:
// quarter h has keys 4 h .. + 3 and 16 + 4 h .. + 3.
template <int D>
__device__ inline bf16x8_t value_cols(const uint16_t* lds, int d0) {
  typedef short s4_t __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s4_t lds_s4_t;
  const int lane = threadIdx.x & 63, j = lane & 15;
  const int row = 4 * (lane >> 4) + (j >> 2), chan = d0 + 4 * (j & 3);
  const s4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t*)(lds + value_at<D>(row, chan)));
  const s4_t hi =
      __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t*)(lds + value_at<D>(row + 16, chan)));
  const uint2 ul = __builtin_bit_cast(uint2, lo), uh = __builtin_bit_cast(uint2, hi);
  return as_bf16x8(make_uint4(ul.x, ul.y, uh.x, uh.y));
}

// 16 RT rows per workgroup; its waves share out the keys in groups of 64 and read them each for
// itself, without a barrier until the end.  Lane l has a quarter of the channels of a group's keys
// 16 i + l % 16, which is the keys' operand (the contraction's order is free as long as the queries
// have it too).  Values pass, 32 keys at a time, through LDS that is the wave's own, to be read
// transposed.  The places of the next group's keys are looked up one group ahead, a key per lane,
// and its elements loaded as soon as this one's are converted.
//
// What bounds it is memory: single tokens of 64 requests, 32 / 8 heads x 128, read 554 MB in 8 bits
// in 104 us (5.3 TB/s; a copy reaches 4.9) and 286 MB in 4 bits in 56 us (5.1 TB/s; conversions
// issue 42% of the vector instructions' time).  Small calls wait for a chain: offsets and lengths,
// page numbers, elements, then 1.5 us per group.
template <typename T, int D, int BITS, bool BIAS, int RT>
__global__ __launch_bounds__(kThreads)
__attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 4)))
void mx_keys_kernel(PagedGeometry g, const T* __restrict__ q, MxPages c,
                    const int32_t* __restrict__ pages, const int32_t* __restrict__ kv_lens,
                    const int32_t* __restrict__ cu_q, const float* __restrict__ table,
                    const int32_t* __restrict__ map, T* __restrict__ out,
                    float* __restrict__ lse, Parts to) {
  constexpr int RB = D * BITS / 8, SB = D / 32, WAVES = kThreads / 64, ROWS = 16 * RT;
  // keys of a group: 32 where 64 would not leave enough registers (spilled ones are waited for
  // together with every load: 64 requests with 6 new tokens 168 us with 64, 125 with 32; with one
  // new token in float32 127 and 115)
  constexpr int KB = D == 128 && BITS == 8 && (RT == 2 || sizeof(T) == 4) ? 32 : 64, NI = KB / 16;
  constexpr uint64_t kAll = ~0ull >> (64 - KB);
  using Frag = typename Type<T>::Frag;
  using Part = Quarter<BITS, RB / 16>;
  constexpr int KS = D / 32, DC = D / 16, E = 32 * D;
  // each wave's half group of values; at the end the waves' results of 16 rows in float32
  __shared__ __attribute__((aligned(16))) uint16_t lds[WAVES * E];
  __shared__ float tops[WAVES][ROWS], totals[WAVES][ROWS];
  extern __shared__ float bias[];

  Deal w;
  if (!deal<ROWS>(g, cu_q, kv_lens, w)) return;
  const Span1& s = w.s;
  const int lane = threadIdx.x & 63, wave = wave_id(), quarter = lane >> 4, col = lane & 15;
  // Queries first, so that waiting for them does not wait for keys.  A column without a row has the
  // request's first one, and is never stored.
  Row x[RT];
  uint4 qw[RT][KS][sizeof(T) / 2];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    x[rt] = row_of(g, s, w.u, s.r0 + 16 * rt + col);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {  // channels quarter D / 4 + 8 ks .. + 7
      const T* from = q + x[rt].q_at + quarter * (D / 4) + 8 * ks;
#pragma unroll
      for (unsigned i = 0; i < sizeof(T) / 2; ++i)
        qw[rt][ks][i] = reinterpret_cast<const uint4*>(from)[i];
    }
  }
  const int first = s.k_lo + wave * KB;  // this wave's groups: first, first + 4 KB, ...
  const int groups = s.k_hi > first ? (s.k_hi - first + WAVES * KB - 1) / (WAVES * KB) : 0;
  // Key `lane` of group i, those past the last key repeat it, to be masked: its page number and,
  // from that, its row among all pages' rows, handed to the lanes that load it.  Returns which keys
  // have a row; the others' lanes load row 0.
  const int32_t* my_pages = pages + (int64_t)s.b * g.max_pages;
  auto key_of = [&](int i) { return min(first + i * (WAVES * KB) + lane % KB, s.k_hi - 1); };
  auto page_of = [&](int j) { return my_pages[div_by((uint32_t)j, g.page_mul, g.page_shift)]; };
  auto places = [&](int i, int p, uint32_t (&lo)[4], uint32_t (&hi)[4]) {
    const int j = key_of(i), page = div_by((uint32_t)j, g.page_mul, g.page_shift);
    const bool ok = (uint32_t)p < (uint32_t)g.num_pages;
    const int64_t row =
        ok ? ((int64_t)p * g.KH + w.u) * g.page_size + (j - page * g.page_size) : 0;
    quarters((uint32_t)row, lo);
    quarters((uint32_t)(row >> 32), hi);
    return (uint64_t)__ballot(ok) & kAll;
  };
  Part kq[NI], vq[NI];  // of keys 16 i + col of a group
  auto row_of_key = [](const uint32_t (&lo)[4], const uint32_t (&hi)[4], int i) {
    return (int64_t)((uint64_t)hi[i] << 32 | lo[i]);
  };
  auto load_keys = [&](const uint32_t (&lo)[4], const uint32_t (&hi)[4]) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int64_t row = row_of_key(lo, hi, i);
      kq[i].load(c.k + (row * RB + quarter * (RB / 4)), c.ks + (row * SB + quarter * SB / 4));
    }
  };
  auto load_values = [&](const uint32_t (&lo)[4], const uint32_t (&hi)[4], int half) {
#pragma unroll
    for (int i = 2 * half; i < 2 * half + 2; ++i) {
      const int64_t row = row_of_key(lo, hi, i);
      vq[i].load(c.v + (row * RB + quarter * (RB / 4)), c.vs + (row * SB + quarter * SB / 4));
    }
  };
  uint64_t there = 0;  // of the group in kq and vq
  int next_page = 0;   // of the group behind it
  if (groups > 0) {
    uint32_t lo[4], hi[4];
    there = places(0, page_of(key_of(0)), lo, hi);
    next_page = page_of(key_of(1));
    load_keys(lo, hi);
    load_values(lo, hi, 0);
    if constexpr (NI == 4) load_values(lo, hi, 1);
  }
  if constexpr (BIAS) fill_bias(bias, g, table, map, w.u);
  Frag qf[RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (sizeof(T) == 2) {
        qf[rt][ks] = as_bf16x8(qw[rt][ks][0]);
        asm volatile("" : "+v"(qf[rt][ks]));  // waited for here, not in the loop
      } else {
        F32x8 y;
        *reinterpret_cast<uint4*>(y.x) = qw[rt][ks][0];
        *reinterpret_cast<uint4*>(y.x + 4) = qw[rt][ks][1];
        qf[rt][ks] = seq::split(y);
        asm volatile("" : "+v"(qf[rt][ks].h), "+v"(qf[rt][ks].m), "+v"(qf[rt][ks].l));
      }
    }
  const int all_see =
      min(g.causal ? min(s.seen - 1, s.off + div_by(s.r0, g.group_mul, g.group_shift))
                   : s.seen - 1, s.k_hi - 1);
  f32x4_t o[RT][DC];
  float top[RT], base[RT], sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    top[rt] = -INFINITY;
    base[rt] = sum[rt] = 0.0f;
#pragma unroll
    for (int dc = 0; dc < DC; ++dc) o[rt][dc] = f32x4_t{};
  }
  const float scale = BIAS ? 1.0f : g.scale_log2;
  uint16_t* mine = lds + wave * E;
  if constexpr (BIAS) __syncthreads();

  // A group, keys kb .. kb + 63, whose elements are in kq and vq; MORE: these then get the next
  // group's (lo, hi), as soon as they are converted.
  auto group = [&](int kb, uint64_t bits, const uint32_t (&lo)[4], const uint32_t (&hi)[4],
                   auto more) {
    constexpr bool MORE = decltype(more)::value;
    f32x4_t acc[RT][NI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) acc[rt][i] = f32x4_t{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const bf16x8_t kf = as_bf16x8(kq[i].eight_at(ks));
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[rt][i] = times(kf, qf[rt][ks], acc[rt][i]);
      }
    // Loads moved up to before the conversions would need other registers, and copies of them that
    // wait at the loop's end.
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (MORE) load_keys(lo, hi);
    typename Alpha<T>::Frag pf[RT][NI / 2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      // element e is key kb + 16 (e / 4) + 4 quarter + e % 4
      float t[4 * NI];
#pragma unroll
      for (int e = 0; e < 4 * NI; ++e) t[e] = acc[rt][e / 4][e % 4];
      const int pos = s.off + x[rt].i;
      if constexpr (BIAS) {
        const float* tab = bias + (x[rt].head - w.u * g.group) * g.span;
#pragma unroll
        for (int e = 0; e < 4 * NI; ++e) {
          const int d = kb + 16 * (e / 4) + 4 * quarter + e % 4 - pos - g.rel_min;
          t[e] = fmaf(t[e], g.scale_log2, tab[min(max(d, 0), g.span - 1)]);
        }
      }
      if (bits != kAll || kb + KB - 1 > all_see) {
        asm volatile("");  // a branch: groups that every row sees do not pay for it
        const int last = min(g.causal ? min(s.seen - 1, pos) : s.seen - 1, s.k_hi - 1);
        const int seen = last - kb - 4 * quarter;
        const uint64_t have = bits >> (4 * quarter);
        const uint32_t word[2] = {(uint32_t)have, (uint32_t)(have >> 32)};
#pragma unroll
        for (int e = 0; e < 4 * NI; ++e)
          if (16 * (e / 4) + e % 4 > seen || (word[e / 8] >> (16 * (e / 4 % 2) + e % 4) & 1) == 0)
            t[e] = -INFINITY;
      }
      float mx = fmaxf(t[0], t[1]);
#pragma unroll
      for (int e = 2; e < 4 * NI; ++e) mx = fmaxf(mx, t[e]);
      mx = max_of(mx) * scale;  // scale > 0
      const bool raise = mx > top[rt] + kSlack;
      if (__any(raise)) {
        const float corr = raise ? __builtin_amdgcn_exp2f(top[rt] - mx) : 1.0f;
        if (raise) top[rt] = base[rt] = mx;
        sum[rt] *= corr;
#pragma unroll
        for (int dc = 0; dc < DC; ++dc) o[rt][dc] *= corr;
      }
#pragma unroll
      for (int e = 0; e < 4 * NI; ++e) {
        t[e] = __builtin_amdgcn_exp2f(fmaf(t[e], scale, -base[rt]));
        sum[rt] += t[e];
      }
#pragma unroll
      for (int i = 0; i < NI / 2; ++i) pf[rt][i] = Alpha<T>::of(t + 8 * i);
    }
#pragma unroll
    for (int half = 0; half < NI / 2; ++half) {
      if (!MORE && half == 1 && kb + 32 >= s.k_hi) break;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
          *reinterpret_cast<uint4*>(mine + value_at<D>(16 * i + col, quarter * (D / 4) + 8 * ks)) =
              vq[2 * half + i].eight_at(ks);
      const uint32_t have = (uint32_t)(bits >> (32 * half));
      if (have != ~0u) {  // what lies where a page number leads to no key may be NaN
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if ((have >> (16 * i + col) & 1) == 0) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
              *reinterpret_cast<uint4*>(
                  mine + value_at<D>(16 * i + col, quarter * (D / 4) + 8 * ks)) =
                  make_uint4(0, 0, 0, 0);
          }
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (MORE) load_values(lo, hi, half);
      fence_wave();
#pragma unroll
      for (int dc = 0; dc < DC; ++dc) {
        const bf16x8_t vf = value_cols<D>(mine, 16 * dc);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][dc] = times(vf, pf[rt][half], o[rt][dc]);
      }
      fence_wave();
    }
  };
  // The last group apart: with no load behind a condition the compiler counts those in flight, and
  // waits for no more than it needs.
  int i = 0;
  uint32_t lo[4], hi[4];
  for (; i + 1 < groups; ++i) {
    const uint64_t next_there = places(i + 1, next_page, lo, hi);
    next_page = page_of(key_of(i + 2));
    group(first + i * (WAVES * KB), there, lo, hi, std::true_type());
    there = next_there;
  }
  if (groups > 0) group(first + i * (WAVES * KB), there, lo, hi, std::false_type());

  // The waves' sums join over a common maximum, 16 rows at a time.
  const int count = min(s.rows - s.r0, ROWS);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float total = sum_of(sum[rt]);
    if (quarter == 0) {
      tops[wave][16 * rt + col] = top[rt];
      totals[wave][16 * rt + col] = total;
    }
  }
  __syncthreads();
  const auto most = [&](int r) {
    float y = tops[0][r];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) y = fmaxf(y, tops[i][r]);
    return y;
  };
  float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (rt > 0) __syncthreads();
    const float own =
        top[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top[rt] - most(16 * rt + col));
#pragma unroll
    for (int dc = 0; dc < DC; ++dc) {  // four channels, permuted against bank conflicts
      const int chunk = 4 * dc + quarter;
      const f32x4_t& y = o[rt][dc];
      *reinterpret_cast<float4*>(sums + (wave * 16 + col) * D + ((chunk ^ col) << 2)) =
          make_float4(y[0] * own, y[1] * own, y[2] * own, y[3] * own);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < min(count - 16 * rt, 16) * (D / 4); e += kThreads) {
      const int r = e / (D / 4), chunk = e % (D / 4), at_row = 16 * rt + r;
      const float tr = most(at_row);
      float total = 0.0f;
      float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < WAVES; ++i) {
        const float f = tops[i][at_row] == -INFINITY
                            ? 1.0f : __builtin_amdgcn_exp2f(tops[i][at_row] - tr);
        total = fmaf(totals[i][at_row], f, total);
        const float4 z =
            *reinterpret_cast<const float4*>(sums + (i * 16 + r) * D + ((chunk ^ r) << 2));
        y.x += z.x;
        y.y += z.y;
        y.z += z.z;
        y.w += z.w;
      }
      const float inv = total > 0.0f ? 1.0f / total : total;
      const float l2 = total == 0.0f
                           ? -INFINITY
                           : (tr == -INFINITY ? 0.0f : tr) + __builtin_amdgcn_logf(total);
      y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
      const Row z = row_of(g, s, w.u, s.r0 + at_row);
      if (s.only) {
        store_4(out + z.out_at * D + chunk * 4, y);
        if (chunk == 0 && lse != nullptr) lse[z.out_at] = l2 * kLn2;
        if (chunk == 0 && g.splits > 1) to.of[z.out_at] = make_int4(0, 0, 0, 0);
      } else {
        const int64_t at = part_row<ROWS>(g, w, at_row, z.out_at);
        if (total != 0.0f) store_4(to.o + at * D + chunk * 4, y);
        if (chunk == 0) to.l[at] = l2;
        if (chunk == 0 && w.split == 0) to.of[z.out_at] = parts_of<ROWS>(w, at_row);
      }
    }
  }
}

// ------------------------------------------------------------------------- join

// Joins the parts of each row, weights 2^(l - max l), as paged_join_kernel does, but for many parts
// with W waves per row, of which wave w has the parts w, w + W, ..., and with several loads on their
// way before the first is waited for (64 rows of 63 parts: 12.6 us with one wave and loads behind
// a branch, 4.0 so).  A part without keys has -inf, and its results were never written.  A wave
// looks at R rows at once and goes on with those that were not finished: a launch with many rows
// has few of them, and often none (chunks of 30 requests, 441,000 rows, none of them in parts:
// 1,633 us with one each, 1,580 with 8; 52,000 rows, half of them in three parts: 13 us either way).
//
// dealt: rows of a part over all key heads, and `most` parts have room; 0: parts are not dealt out,
// and every row has `most` of them.
template <typename T, int D, int W, int AT_ONCE, int R>
__global__ __launch_bounds__(kThreads) void mx_join_kernel(int64_t rows, int dealt, int64_t most,
                                                           Parts from, T* __restrict__ out,
                                                           float* __restrict__ lse) {
  constexpr int LANES = D / 4, SIDES = 64 / LANES, PER = kThreads / 64 / W;
  static_assert(W == 1 || R == 1, "several waves have one row");
  __shared__ float4 sums[W][LANES];
  __shared__ float tops[W], totals[W];
  const int wave = wave_id() % W, lane = threadIdx.x & 63;
  const int64_t row0 = ((int64_t)block_number() * PER + wave_id() / W) * R;
  if (row0 >= rows) return;  // a whole workgroup where W > 1
  const int side = lane / LANES, c = lane % LANES * 4;
  const int4 of = from.of[min(row0 + min(lane, R - 1), rows - 1)];
  uint64_t left = __ballot(lane < R && row0 + lane < rows && of.z != 0);
  for (; left != 0; left &= left - 1) {
    const int which = __builtin_ctzll(left);
    const int64_t row = row0 + which;
    int64_t first = row * most, step = 1;
    int parts = (int)most;
    if (dealt > 0) {
      const int nth = __builtin_amdgcn_readlane(of.x, which);
      const int next = __builtin_amdgcn_readlane(of.y, which);
      const int in_part = __builtin_amdgcn_readlane(of.w, which);
      parts = __builtin_amdgcn_readlane(of.z, which);
      // Where offsets decrease a row may have been nobody's, and `of` anything.
      if (nth < 0 || next < 0 || in_part < 0 || in_part >= dealt || parts < 0 ||
          nth + (int64_t)(parts - 1) * next >= most)
        continue;
      first = (int64_t)nth * dealt + in_part;
      step = (int64_t)next * dealt;
    }
    // lane l has part l W + wave
    const float mine =
        lane * W + wave < parts ? from.l[first + (lane * W + wave) * step] : -INFINITY;
    float top = mine;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if constexpr (W > 1) {
      tops[wave] = top;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < W; ++i) top = fmaxf(top, tops[i]);
    }
    const float weight = mine == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mine - top);
    float total = weight;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) total += __shfl_xor(total, d);
    // this wave's parts up to its last that is there
    const uint64_t some = __ballot(mine != -INFINITY);
    const int count = some == 0 ? 0 : 64 - __builtin_clzll(some);
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s0 = 0; s0 < count; s0 += AT_ONCE * SIDES) {
      float4 x[AT_ONCE];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        const int s = min(s0 + i * SIDES + side, count - 1) * W + wave;
        x[i] = *reinterpret_cast<const float4*>(from.o + (first + s * step) * D + c);
      }
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        const int s = s0 + i * SIDES + side;
        const float ws = __shfl(weight, s & 63), ls = __shfl(mine, s & 63);
        if (s < count && ls != -INFINITY) {
          sum.x = fmaf(ws, x[i].x, sum.x);
          sum.y = fmaf(ws, x[i].y, sum.y);
          sum.z = fmaf(ws, x[i].z, sum.z);
          sum.w = fmaf(ws, x[i].w, sum.w);
        }
      }
    }
#pragma unroll
    for (int d = 32; d >= LANES; d >>= 1) {
      sum.x += __shfl_xor(sum.x, d);
      sum.y += __shfl_xor(sum.y, d);
      sum.z += __shfl_xor(sum.z, d);
      sum.w += __shfl_xor(sum.w, d);
    }
    if constexpr (W > 1) {
      if (lane < LANES) sums[wave][lane] = sum;
      totals[wave] = total;
      __syncthreads();
      if (wave > 0 || lane >= LANES) return;  // R is 1
      sum = sums[0][lane];
#pragma unroll
      for (int i = 1; i < W; ++i) {
        const float4 y = sums[i][lane];
        sum.x += y.x;
        sum.y += y.y;
        sum.z += y.z;
        sum.w += y.w;
        total += totals[i];
      }
    }
    if (lane < LANES) {
      const float inv = total > 0.0f ? 1.0f / total : total;
      store_4(out + row * D + c, make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv));
    }
    if (lane == 0 && lse != nullptr) {
      const float base = top == -INFINITY ? 0.0f : top;
      lse[row] = total == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(total)) * kLn2;
    }
  }
}

// ------------------------------------------------------------------------- write and read

// Rows of k and v as chunks of 8 channels, a token's key first: chunk n is chunk n % per of token
// n / per.  A wave takes `steps` times 64 chunks that follow each other, a chunk per lane and step,
// and looks up the places of its tokens at once, a token per lane.
struct Rows {
  int per;                       // chunks of a token's key and value together, at least 16
  uint32_t per_mul, per_shift;   // chunk / per
};
constexpr int kMostSteps = 8;    // at most 64 kMostSteps / 16 + 1 tokens: a lane for each

// This lane's chunk: token, half (0: key, 1: value), head, first channel; and the token's place.
struct Chunk {
  int token, which, head, chan;
  bool ok;            // there is such a chunk
  int64_t place;      // the head's row among all pages' rows, -1: none
};

template <int STEPS>
__device__ inline void chunks_of(Chunk (&x)[STEPS], const PagedGeometry& g, const Rows& r,
                                 const int32_t* cu_q, const int32_t* kv_lens,
                                 const int32_t* pages) {
  const int lane = threadIdx.x & 63;
  const uint64_t base =
      ((uint64_t)(uint32_t)block_number() * (kThreads / 64) + wave_id()) * (64 * STEPS);
  const int first = (int)min(base / (uint32_t)r.per, (uint64_t)g.nq);
  const uint32_t skip = (uint32_t)(base - (uint64_t)(uint32_t)first * (uint32_t)r.per);
  // Token first + lane: the last request that begins at it or before (up to 64 of them are held by
  // a lane each), its position, its page.
  const int tok = first + lane < g.nq && first + lane >= first ? first + lane : g.nq - 1;
  const int ends = g.B <= 64 ? cu_at(cu_q, min(lane, g.B - 1) + 1, g.nq) : 0;
  int b = 0;
  for (int n = g.B + 1; n > 1; n -= n / 2) {
    const int mid = min(b + n / 2, g.B);
    if ((g.B <= 64 ? __shfl(ends, mid - 1) : cu_at(cu_q, mid, g.nq)) <= tok) b = mid;
  }
  int page = -1, row = 0;
  if (b < g.B) {
    const int begin = cu_at(cu_q, b, g.nq), n = max(cu_at(cu_q, b + 1, g.nq), begin) - begin;
    const int64_t at = (int64_t)kv_lens[b] - n + (tok - begin);
    if (tok >= begin && tok - begin < n && at >= 0 && at < (int64_t)g.max_pages * g.page_size) {
      const int nth = div_by((uint32_t)at, g.page_mul, g.page_shift);
      page = pages[(int64_t)b * g.max_pages + nth];
      row = (int)(at - (int64_t)nth * g.page_size);
      if (page < 0 || page >= g.num_pages) page = -1;
    }
  }
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const uint32_t n = skip + 64 * i + lane;
    const int nth = div_by(n, r.per_mul, r.per_shift), c = (int)n - nth * r.per;
    x[i].token = first + nth;
    x[i].ok = nth < g.nq - first;
    x[i].which = c >= r.per / 2;
    const int chan = (c - x[i].which * (r.per / 2)) * 8;
    x[i].head = chan / g.D;
    x[i].chan = chan - x[i].head * g.D;
    const int p = __shfl(page, nth), at = __shfl(row, nth);
    x[i].place = p < 0 ? -1 : ((int64_t)p * g.KH + x[i].head) * g.page_size + at;
  }
}

template <typename T>
__device__ inline void load_8(float (&x)[8], const T* at) {
  if constexpr (sizeof(T) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(at);
    const uint32_t h[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(h[i] << 16);
      x[2 * i + 1] = __uint_as_float(h[i] & 0xffff0000u);
    }
  } else {
    *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(at);
    *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(at + 4);
  }
}

// The largest magnitude's bits -> the block's scale byte.  With M 1.75 2^8 or 1.5 2^2, the least e
// with a <= M 2^e is a's exponent less 8 or 2, and one more where its mantissa is larger than M's:
// adding what M's mantissa leaves to a whole one carries then.  255 where the largest would round
// to 2^128 (a NaN's and an infinity's bits are larger still).
template <int BITS>
__device__ inline uint32_t scale_byte(uint32_t a) {
  constexpr uint32_t kUp = BITS == 8 ? 0x1fffffu : 0x3fffffu, kLess = BITS == 8 ? 8 : 2;
  constexpr uint32_t kOver = BITS == 8 ? 0x7f780000u : 0x7f600000u;
  const uint32_t e = (a + kUp) >> 23;
  return a >= kOver ? 255u : max(e, 10u + kLess) - kLess;
}

template <typename T, int D, int BITS, int STEPS>
__global__ __launch_bounds__(kThreads) void mx_append_kernel(
    PagedGeometry g, Rows r, const T* __restrict__ k, const T* __restrict__ v,
    const int32_t* __restrict__ cu_q, const int32_t* __restrict__ kv_lens,
    const int32_t* __restrict__ pages, MxPages to) {
  g.D = D;
  Chunk c[STEPS];
  chunks_of(c, g, r, cu_q, kv_lens, pages);
  float x[STEPS][8];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    if (c[i].ok && c[i].place >= 0) {
      load_8(x[i], (c[i].which ? v + c[i].token * g.vs : k + c[i].token * g.ks) +
                       c[i].head * D + c[i].chan);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    uint32_t a = 0;  // the block's largest: four lanes have it
#pragma unroll
    for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(x[i][e]) & 0x7fffffffu);
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xb1, 0xf, 0xf, true));  // ^ 1
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4e, 0xf, 0xf, true));  // ^ 2
    if (!c[i].ok || c[i].place < 0) continue;
    const uint32_t byte = scale_byte<BITS>(a);
    const bool none = byte == 255u;
    const float power = power_of(none ? 127u : byte);
    float (&y)[8] = x[i];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = none ? 0.0f : y[e];
    uint8_t* codes = c[i].which ? to.v : to.k;
    uint8_t* scales = c[i].which ? to.vs : to.ks;
    const int64_t at = c[i].place * D + c[i].chan;
    if constexpr (BITS == 8) {
      typedef short s2_t __attribute__((ext_vector_type(2)));
      uint32_t u[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        s2_t z = {0, 0};
        z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, y[4 * h], y[4 * h + 1], power, false);
        z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, y[4 * h + 2], y[4 * h + 3], power, true);
        u[h] = __builtin_bit_cast(uint32_t, z);
      }
      *reinterpret_cast<uint2*>(codes + at) = make_uint2(u[0], u[1]);
    } else {
      uint32_t u = 0;
      u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[0], y[1], power, 0);
      u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[2], y[3], power, 1);
      u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[4], y[5], power, 2);
      u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, y[6], y[7], power, 3);
      *reinterpret_cast<uint32_t*>(codes + at / 2) = u;
    }
    if (c[i].chan % 32 == 0) scales[at / 32] = (uint8_t)byte;
  }
}

template <typename T, int D, int BITS, int STEPS>
__global__ __launch_bounds__(kThreads) void mx_read_kernel(
    PagedGeometry g, Rows r, MxPages from, const int32_t* __restrict__ pages,
    const int32_t* __restrict__ kv_lens, const int32_t* __restrict__ cu_q, T* __restrict__ k,
    T* __restrict__ v) {
  g.D = D;
  Chunk c[STEPS];
  chunks_of(c, g, r, cu_q, kv_lens, pages);
  uint2 u[STEPS];
  uint8_t byte[STEPS];
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    u[i] = make_uint2(0, 0);
    byte[i] = 127;
    if (!c[i].ok || c[i].place < 0) continue;
    const uint8_t* codes = c[i].which ? from.v : from.k;
    const int64_t at = c[i].place * D + c[i].chan;
    byte[i] = (c[i].which ? from.vs : from.ks)[at / 32];
    if constexpr (BITS == 8)
      u[i] = *reinterpret_cast<const uint2*>(codes + at);
    else
      u[i].x = *reinterpret_cast<const uint32_t*>(codes + at / 2);
  }
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    if (!c[i].ok) continue;
    const float power = power_of(byte[i]);
    const uint4 y = BITS == 8 ? eight(u[i].x, u[i].y, power) : eight(u[i].x, power);
    T* to = (c[i].which ? v + c[i].token * g.vs : k + c[i].token * g.ks) + c[i].head * D +
            c[i].chan;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(to) = y;
    } else {  // a bf16 number is a float32 number's upper half
      *reinterpret_cast<uint4*>(to) =
          make_uint4(y.x << 16, y.x & 0xffff0000u, y.y << 16, y.y & 0xffff0000u);
      *reinterpret_cast<uint4*>(to + 4) =
          make_uint4(y.z << 16, y.z & 0xffff0000u, y.w << 16, y.w & 0xffff0000u);
    }
  }
}

template <typename T, int D, int BITS>
const void* append_fn(int steps) {
  return steps == 1   ? (const void*)&mx_append_kernel<T, D, BITS, 1>
         : steps == 4 ? (const void*)&mx_append_kernel<T, D, BITS, 4>
                      : (const void*)&mx_append_kernel<T, D, BITS, kMostSteps>;
}
template <typename T, int D, int BITS>
const void* read_fn(int steps) {
  return steps == 1   ? (const void*)&mx_read_kernel<T, D, BITS, 1>
         : steps == 4 ? (const void*)&mx_read_kernel<T, D, BITS, 4>
                      : (const void*)&mx_read_kernel<T, D, BITS, kMostSteps>;
}

// How rows are dealt out: one step per wave up to 4,096 of them (16 waves per compute unit), for the
// shortest chain; then four, or eight where there are more than 65,536 (7,597 tokens of 8 heads x
// 128 written to 4 bits: 13.1, 12.2, 13.1 us with 2, 4, 8 steps; 60,000 read: 89, 66, 64).
struct RowsPlan {
  Rows r;
  int steps;
  int64_t blocks;
};
RowsPlan plan_rows(const PagedGeometry& g) {
  RowsPlan p;
  p.r.per = 2 * g.KH * (g.D / 8);
  divisor(p.r.per, &p.r.per_mul, &p.r.per_shift);
  const int64_t steps = ((int64_t)g.nq * p.r.per + 63) / 64;
  p.steps = steps <= 4096 ? 1 : steps <= 65536 ? 4 : kMostSteps;
  const int each = p.steps * (kThreads / 64);
  p.blocks = (steps + each - 1) / each;
  return p;
}

// The form for the call's type, channels and bits.
typedef const void* (*Form)(int);
Form form(const PagedGeometry& g, bool bf16, int bits, Form b64_8, Form b128_8, Form b64_4,
          Form b128_4, Form f64_8, Form f128_8, Form f64_4, Form f128_4) {
  const Form all[2][2][2] = {{{f64_4, f64_8}, {f128_4, f128_8}},
                             {{b64_4, b64_8}, {b128_4, b128_8}}};
  return all[bf16][g.D == 128][bits == 8];
}

// Rows of partial results.
int64_t part_rows(const PagedGeometry& g) {
  return g.target > 0 ? g.room * g.KH * g.tile : (int64_t)g.splits * g.nq * g.H;
}

MxPages pages_of(const dsa3d_mx_cache& c) { return {c.k, c.v, c.k_scales, c.v_scales}; }

template <typename T, int D, int BITS>
hipError_t forward_d(const PagedGeometry& g, const T* q, const MxPages& c, const int32_t* pages,
                     const int32_t* kv_lens, const int32_t* cu_q, const float* table,
                     const int32_t* map, T* out, float* lse, void* ws, hipStream_t s) {
  const bool bias = g.nb > 0;
  const int64_t rows = (int64_t)g.nq * g.H;
  Parts p = {};
  if (g.splits > 1) {
    p.of = (int4*)ws;
    p.l = (float*)((char*)ws + round_256((size_t)rows * sizeof(int4)));
    p.o = (float*)((char*)p.l + round_256((size_t)part_rows(g) * 4));
  }
  const void* fn = g.tile == 16   ? (bias ? (const void*)&mx_keys_kernel<T, D, BITS, true, 1>
                                          : (const void*)&mx_keys_kernel<T, D, BITS, false, 1>)
                   : g.tile == 32 ? (bias ? (const void*)&mx_keys_kernel<T, D, BITS, true, 2>
                                          : (const void*)&mx_keys_kernel<T, D, BITS, false, 2>)
                                  : (bias ? (const void*)&mx_rows_kernel<T, D, BITS, true>
                                          : (const void*)&mx_rows_kernel<T, D, BITS, false>);
  hipError_t e = seq_launch(fn, g.blocks, kThreads,
                            bias ? (size_t)g.group * g.span * 4 : 0, s, g, q, c, pages, kv_lens,
                            cu_q, table, map, out, lse, p);
  if (e == hipSuccess && g.splits > 1) {
    constexpr int waves = kThreads / 64, look = 8;
    const bool many = rows > 16384 && g.splits <= 64;  // one wave has no more parts
    // One wave is better for few parts, four from 9 or so on: single tokens of n requests of 30,000
    // tokens, 32 / 8 heads x 128, us with one / four, n = 64 (2 parts) 672.7/675.8, 16 (6)
    // 180.6/181.3, 8 (12) 97.3/96.2, 4 (14) 57.2/56.5, 2 (29) 29.8/28.6, 1 (59) 25.4/24.0.  The host
    // knows only how many there may be: 16 leaves single tokens of 64 requests of up to 8,000 to one.
    const bool wide = !many && g.splits > 16;
    const int each = many ? waves * look : wide ? 1 : waves;
    e = seq_launch(many   ? (const void*)&mx_join_kernel<T, D, 1, 2, look>
                   : wide ? (const void*)&mx_join_kernel<T, D, waves, 8, 1>
                          : (const void*)&mx_join_kernel<T, D, 1, 4, 1>,
                   (rows + each - 1) / each, kThreads, 0, s, rows,
                   g.target > 0 ? g.KH * g.tile : 0, g.target > 0 ? g.room : g.splits, p, out, lse);
  }
  return e;
}

template <typename T>
hipError_t forward_t(const PagedGeometry& g, const void* q, const dsa3d_mx_cache& cache,
                     const int32_t* pages, const int32_t* kv_lens, const int32_t* cu_q,
                     const float* table, const int32_t* map, void* out, float* lse, void* ws,
                     hipStream_t s) {
  const MxPages c = pages_of(cache);
  const T* x = (const T*)q;
  T* y = (T*)out;
  if (cache.bits == 8)
    return g.D == 64
               ? forward_d<T, 64, 8>(g, x, c, pages, kv_lens, cu_q, table, map, y, lse, ws, s)
               : forward_d<T, 128, 8>(g, x, c, pages, kv_lens, cu_q, table, map, y, lse, ws, s);
  return g.D == 64
             ? forward_d<T, 64, 4>(g, x, c, pages, kv_lens, cu_q, table, map, y, lse, ws, s)
             : forward_d<T, 128, 4>(g, x, c, pages, kv_lens, cu_q, table, map, y, lse, ws, s);
}

}  // namespace

void set_plan_mx(PagedGeometry& g) {
  const MxPlan p = paged_mx_plan(g.nq, g.group, g.KH, g.B, g.max_kv, g.D);
  g.tile = p.tile;
  g.splits = p.splits;
  g.part = p.part;
  g.target = p.target;
  g.room = p.room;
  if (p.target > 0) {
    g.tiles = Spread{};
    g.blocks = g.KH * p.bound;
  } else {
    g.tiles = seq_spread(g.KH * g.splits, (int)((int64_t)g.nq * g.group / g.tile) + g.B + 1);
    g.blocks = seq_blocks(g.tiles, 1);
  }
}

size_t paged_mx_workspace(const PagedGeometry& g) {
  if (g.splits <= 1) return 0;
  const size_t n = part_rows(g);
  return round_256((size_t)g.nq * g.H * sizeof(int4)) + round_256(n * 4) + n * g.D * 4;
}

hipError_t launch_paged_forward_mx(const PagedGeometry& g, bool bf16, const void* q,
                                   const dsa3d_mx_cache& cache, const int32_t* pages,
                                   const int32_t* kv_lens, const int32_t* cu_q,
                                   const float* table, const int32_t* map, void* out, float* lse,
                                   void* ws, hipStream_t s) {
  if (g.nq == 0) return hipSuccess;
  return bf16 ? forward_t<uint16_t>(g, q, cache, pages, kv_lens, cu_q, table, map, out, lse, ws, s)
              : forward_t<float>(g, q, cache, pages, kv_lens, cu_q, table, map, out, lse, ws, s);
}

hipError_t launch_paged_append_mx(const PagedGeometry& g, bool bf16, const void* k, const void* v,
                                  const int32_t* cu_q, const int32_t* kv_lens,
                                  const int32_t* pages, const dsa3d_mx_cache& cache,
                                  hipStream_t s) {
  if (g.nq == 0) return hipSuccess;
  const RowsPlan p = plan_rows(g);
  const MxPages c = pages_of(cache);
  const void* fn = form(
      g, bf16, cache.bits, append_fn<uint16_t, 64, 8>, append_fn<uint16_t, 128, 8>,
      append_fn<uint16_t, 64, 4>, append_fn<uint16_t, 128, 4>, append_fn<float, 64, 8>,
      append_fn<float, 128, 8>, append_fn<float, 64, 4>, append_fn<float, 128, 4>)(p.steps);
  return seq_launch(fn, p.blocks, kThreads, 0, s, g, p.r, k, v, cu_q, kv_lens, pages, c);
}

hipError_t launch_paged_read_mx(const PagedGeometry& g, bool bf16, const dsa3d_mx_cache& cache,
                                const int32_t* pages, const int32_t* kv_lens, const int32_t* cu_q,
                                void* k, void* v, hipStream_t s) {
  if (g.nq == 0) return hipSuccess;
  const RowsPlan p = plan_rows(g);
  const MxPages c = pages_of(cache);
  const void* fn = form(
      g, bf16, cache.bits, read_fn<uint16_t, 64, 8>, read_fn<uint16_t, 128, 8>,
      read_fn<uint16_t, 64, 4>, read_fn<uint16_t, 128, 4>, read_fn<float, 64, 8>,
      read_fn<float, 128, 8>, read_fn<float, 64, 4>, read_fn<float, 128, 4>)(p.steps);
  return seq_launch(fn, p.blocks, kThreads, 0, s, g, p.r, c, pages, kv_lens, cu_q, k, v);
}

}  // namespace dsa3d
