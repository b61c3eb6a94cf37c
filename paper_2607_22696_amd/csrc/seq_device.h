// Device code shared by the sequence kernels (seqattn.hip, paged.hip): operand tiles in LDS, the
// matrix products, and the way from a block to its sequence.
//
// Products are those of winattn.hip: 32 x 32 blocks with the transposed result (S^T = K Q^T,
// O^T = V^T P^T), so that a lane owns one query's (or key's) column.  Operand fragments are the
// same for both storage types: lane l holds row (or column) l % 32 and the 8 consecutive
// contraction indices 8 (l / 32) .. +7 of a step of 16, multiplied by v_mfma_f32_32x32x16_bf16.
// The result's lane l holds column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4 in its element i.
//
// float32 operands are split into three bf16 parts, x = h + m + l exactly (each the nearest bf16 of
// what is left, so m <= 2^-8 and l <= 2^-17 of x's leading bit), and six of the nine products are
// summed in float32: the three left out are at most 2^-24 of the product together, of either sign,
// as much as one of its roundings.  (Parts cut off instead of rounded cost the same instructions
// and leave out up to 2^-21, always towards zero.)  Six bf16 products take 192 cycles where the
// eight v_mfma_f32_32x32x2_f32 of the same 16 indices take 512.  Tiles are split once per
// workgroup, into three bf16 tiles.  4,096 causal tokens, 8 heads x 128, forward: 594 us with
// float32 products, 467 with operands split as they are read, 389 this way (1,035 at two waves per
// SIMD, with 102 spilled registers).  Infinities, and values that round to one as a bf16 (3.39e38
// and more), have no such parts: they make NaN of what they reach.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "seq_internal.h"

namespace dsa3d {
namespace seq {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
struct F32x8 {
  float x[8];
};
struct Split {
  bf16x8_t h, m, l;
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.0f;    // base-2 headroom of a running maximum
constexpr float kHidden = -1e30f; // bias values at or below this hide a key

template <typename T>
struct Type;
template <>
struct Type<uint16_t> {  // bf16 bit patterns
  using Frag = bf16x8_t;
};
template <>
struct Type<float> {
  using Frag = Split;
};
// Rows of a tile of four waves: 64, or 32 where they would be 160 KB in float32.
template <typename T, int D>
constexpr int kKeyTile = sizeof(T) * D == 512 ? 32 : 64;

__device__ inline f32x16_t mfma(const bf16x8_t& a, const bf16x8_t& b, const f32x16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16_t mfma(const Split& a, const Split& b, f32x16_t c) {
  c = mfma(a.l, b.h, c);
  c = mfma(a.h, b.l, c);
  c = mfma(a.m, b.m, c);
  c = mfma(a.m, b.h, c);
  c = mfma(a.h, b.m, c);
  return mfma(a.h, b.h, c);
}
// Two floats as bf16, and what that leaves of them.
__device__ inline uint32_t take_part(float (&x)[2]) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t y = {x[0], x[1]};
  const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, bf16x2_t));
  x[0] -= __uint_as_float(u << 16);
  x[1] -= __uint_as_float(u & 0xffff0000u);
  return u;
}
__device__ inline Split split(const F32x8& a) {
  uint32_t h[4], m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[2] = {a.x[2 * i], a.x[2 * i + 1]};
    h[i] = take_part(x);
    m[i] = take_part(x);
    l[i] = take_part(x);
  }
  return {__builtin_bit_cast(bf16x8_t, make_uint4(h[0], h[1], h[2], h[3])),
          __builtin_bit_cast(bf16x8_t, make_uint4(m[0], m[1], m[2], m[3])),
          __builtin_bit_cast(bf16x8_t, make_uint4(l[0], l[1], l[2], l[3]))};
}

__device__ inline bf16x8_t as_bf16x8(const uint4& u) { return __builtin_bit_cast(bf16x8_t, u); }

__device__ inline uint16_t to_bf16(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// x combined with the value of lane l ^ 32 (v_permlane32_swap: no LDS traffic).
__device__ inline float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The wave's number within its workgroup, known to be the same for all its lanes.
__device__ inline int wave_id() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }

// Row of a 32-row block that element i of a result holds in this half of the wave.
__device__ inline int c_row(int i, int hh) { return 8 * (i / 4) + 4 * hh + (i % 4); }

__device__ inline uint32_t lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// 16 bytes per lane from base + off to LDS at `to` + 16 lane, without a register in between.  The
// compiler does not count it among the loads it waits for: the reader waits with wait_copies().
// (Its builtin has the compiler wait for every copy in flight before any LDS read.  m0 is reserved:
// the compiler keeps nothing in it, and nothing else in these kernels writes it.)
__device__ inline void copy_16(uint32_t to, const void* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}
// The same from an address per lane.
__device__ inline void copy_16(uint32_t to, const void* from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(to), "v"(from)
               : "memory");
}
// The same with 4 bytes per lane, from base + first floats + off bytes.
__device__ inline void copy_4(uint32_t to, const float* base, uint32_t off, int64_t first) {
  base += first;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}
__device__ inline void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A tile of ROWS rows x D channels in LDS, rows unpadded, the 16-byte chunks of a row XOR-permuted
// by a function of the row so that both operand reads are free of bank conflicts.  bf16: as
// winattn.hip's tiles (16-byte reads of one chunk of 16 consecutive rows, and the transposing
// 8-byte reads of 4 rows x 64 bytes).  float32: chunk ^ (row % 16), for which 16 consecutive rows'
// reads of one chunk touch all 64 banks, and a 4-byte read of 32 consecutive channels of one row
// touches 32 different ones.
template <typename T, int D, int ROWS, int THREADS = 256>
struct Tile {
  static constexpr bool kBf16 = sizeof(T) == 2;
  static constexpr int CH = 16 / sizeof(T);         // elements per 16-byte chunk
  static constexpr int KCH = D / CH;                // chunks per row
  static constexpr int NL = ROWS * KCH / THREADS;   // chunks per thread
  static constexpr int kStep = THREADS / KCH;       // rows between a thread's chunks
  static constexpr int kElems = ROWS * D;
  using Frag = typename Type<T>::Frag;
  static_assert(D == 64 || D == 128, "head_dim 64 or 128");
  static_assert(NL * THREADS == ROWS * KCH, "the threads share a tile evenly");

  static __device__ inline int at(int row, int chan) {
    if constexpr (kBf16) {
      const int f = D == 128 ? 4 * (row & 3) + ((row >> 2) & 3)
                             : 4 * ((row >> 1) & 1) + ((row >> 2) & 3);
      return row * D + (((chan >> 3) ^ f) << 3) + (chan & 7);
    } else {
      return row * D + (((chan >> 2) ^ (row & 15)) << 2) + (chan & 3);
    }
  }

  static __device__ inline int row_of_thread(int i) { return (int)threadIdx.x / KCH + i * kStep; }
  static __device__ inline int chan_of_thread() { return ((int)threadIdx.x % KCH) * CH; }

  // Tile rows through a table of tensor rows (negative: no such row, reads as zero).
  static __device__ inline void load(uint4 (&r)[NL], const T* src, int64_t stride,
                                     const int* tab) {
    int row[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) row[i] = tab[row_of_thread(i)];
#pragma unroll
    for (int i = 0; i < NL; ++i)
      r[i] = *reinterpret_cast<const uint4*>(src + (int64_t)max(row[i], 0) * stride +
                                             chan_of_thread());
#pragma unroll
    for (int i = 0; i < NL; ++i)
      if (row[i] < 0) r[i] = make_uint4(0, 0, 0, 0);
  }
  static __device__ inline void store(T* lds, const uint4 (&r)[NL]) {
#pragma unroll
    for (int i = 0; i < NL; ++i)
      *reinterpret_cast<uint4*>(lds + at(row_of_thread(i), chan_of_thread())) = r[i];
  }

  // Asynchronous staging: global_load_lds_dwordx4 puts 16 bytes per lane at consecutive LDS
  // addresses, 1 KiB per wave and instruction, so the permutation of a row's chunks is made in the
  // addresses read: the lane that writes position c of row r reads chunk c ^ f(r).
  static constexpr int kRowBytes = D * (int)sizeof(T);
  static constexpr int kRowsPerCopy = 1024 / kRowBytes;
  static constexpr int NC = ROWS * kRowBytes / (1024 * (THREADS / 64));  // copies per wave
  static_assert(NC >= 1, "every wave copies");
  static __device__ inline int copy_row(int i) {
    return (i * (THREADS / 64) + wave_id()) * kRowsPerCopy + ((int)threadIdx.x & 63) / KCH;
  }
  static __device__ inline uint32_t copy_to(const T* lds, int i) {
    return lds_offset(lds) + (i * (THREADS / 64) + wave_id()) * 1024;
  }
  static __device__ inline int copy_chunk(int row) {
    return (at(row, ((int)threadIdx.x % KCH) * CH) - row * D) * (int)sizeof(T);
  }
  // Byte offsets of this lane's sources from the tile's first row.
  static __device__ inline void copy_plan(uint32_t (&off)[NC], uint32_t stride_bytes) {
#pragma unroll
    for (int i = 0; i < NC; ++i)
      off[i] = (uint32_t)copy_row(i) * stride_bytes + copy_chunk(copy_row(i));
  }
  // Starts the copy of a tile whose row 0 is at src (uniform); rows from `valid` on repeat the last
  // valid one, to be masked.  Done once wait_copies() and a barrier have passed.
  static __device__ inline void copy(T* lds, const T* src, const uint32_t (&off)[NC],
                                     uint32_t stride_bytes, int valid) {
    if (valid >= ROWS) {
#pragma unroll
      for (int i = 0; i < NC; ++i) copy_16(copy_to(lds, i), src, off[i]);
    } else {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int row = copy_row(i);
        copy_16(copy_to(lds, i), src,
                (uint32_t)min(row, valid - 1) * stride_bytes + copy_chunk(row));
      }
    }
  }

  // Starts the copies of tile rows of two tensors that lie `tab` bytes from src and src2.
  static __device__ inline void copy(T* lds, const T* src, T* lds2, const T* src2,
                                     const int64_t* tab) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int row = copy_row(i);
      const int64_t at = tab[row] + copy_chunk(row);
      copy_16(copy_to(lds, i), reinterpret_cast<const char*>(src) + at);
      copy_16(copy_to(lds2, i), reinterpret_cast<const char*>(src2) + at);
    }
  }

  // Room for two tiles that belong together and for the next two, which are being copied: bf16
  // alternates between two places; float32 has one, which is free again once it is split.
  static constexpr int kTwo = (kBf16 ? 4 : 5) * ROWS * D, kPlace = kBf16 ? 2 * ROWS * D : 0;
  // from the first tile's operands to the second's
  static constexpr int kSecond = (kBf16 ? 1 : 3) * ROWS * D;
  // What the operands of the two tiles in place `buf` are read from: the tiles themselves, or the
  // three bf16 tiles that each of them is split into.
  static __device__ inline const uint16_t* operands(T* lds, int buf) {
    if constexpr (kBf16) {
      return lds + kPlace * buf;
    } else {
      using Part = Tile<uint16_t, D, ROWS, THREADS>;
      uint16_t* room = reinterpret_cast<uint16_t*>(lds + 2 * ROWS * D);
#pragma unroll
      for (int two = 0; two < 2; ++two)
#pragma unroll
        for (int i = 0; i < ROWS * D / 8 / THREADS; ++i) {
          const int at8 = (int)threadIdx.x + i * THREADS;
          const int row = at8 / (D / 8), c = at8 % (D / 8) * 8;
          const T* from = lds + two * ROWS * D;
          F32x8 x;
          *reinterpret_cast<float4*>(x.x) = *reinterpret_cast<const float4*>(from + at(row, c));
          *reinterpret_cast<float4*>(x.x + 4) =
              *reinterpret_cast<const float4*>(from + at(row, c + 4));
          const Split y = split(x);
          uint16_t* to = room + two * kSecond + Part::at(row, c);
          *reinterpret_cast<bf16x8_t*>(to) = y.h;
          *reinterpret_cast<bf16x8_t*>(to + ROWS * D) = y.m;
          *reinterpret_cast<bf16x8_t*>(to + 2 * ROWS * D) = y.l;
        }
      __syncthreads();
      return room;
    }
  }

  // Operand with tile rows as its rows: row r0 + l % 32, channels 16 ks + 8 (l / 32) .. +7.
  static __device__ inline Frag a_rows(const uint16_t* lds, int r0, int ks) {
    if constexpr (kBf16) {
      const int lane = threadIdx.x & 63, row = r0 + (lane & 31), c = ks * 16 + (lane >> 5) * 8;
      return as_bf16x8(*reinterpret_cast<const uint4*>(lds + at(row, c)));
    } else {
      using Part = Tile<uint16_t, D, ROWS, THREADS>;
      return {Part::a_rows(lds, r0, ks), Part::a_rows(lds + ROWS * D, r0, ks),
              Part::a_rows(lds + 2 * ROWS * D, r0, ks)};
    }
  }
  // Operand with channels as its rows: channel d0 + l % 32; tile rows 32 kb + 16 p + 4 (l / 32) +
  // {0..3, 8..11}, the order in which a result's elements 8 p .. 8 p + 7 hold them.  By
  // ds_read_b64_tr_b16 as in winattn.hip.
  static __device__ inline Frag a_cols(const uint16_t* lds, int d0, int kb, int p) {
    if constexpr (kBf16) {
      typedef short s4_t __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) s4_t lds_s4_t;
      const int lane = threadIdx.x & 63, j = lane & 15;
      const int row = kb * 32 + 16 * p + 4 * (lane >> 5) + (j >> 2);
      const int chan = d0 + 16 * ((lane >> 4) & 1) + 4 * (j & 3);
      const s4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t*)(lds + at(row, chan)));
      const s4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t*)(lds + at(row + 8, chan)));
      const uint2 ul = __builtin_bit_cast(uint2, lo), uh = __builtin_bit_cast(uint2, hi);
      return as_bf16x8(make_uint4(ul.x, ul.y, uh.x, uh.y));
    } else {
      using Part = Tile<uint16_t, D, ROWS, THREADS>;
      return {Part::a_cols(lds, d0, kb, p), Part::a_cols(lds + ROWS * D, d0, kb, p),
              Part::a_cols(lds + 2 * ROWS * D, d0, kb, p)};
    }
  }
  // The same operands straight from the tile, split as they are read.
  static __device__ inline Frag rows_of(const T* lds, int r0, int ks) {
    if constexpr (kBf16) {
      return a_rows(lds, r0, ks);
    } else {
      const int lane = threadIdx.x & 63, row = r0 + (lane & 31), c = ks * 16 + (lane >> 5) * 8;
      F32x8 f;
      *reinterpret_cast<float4*>(f.x) = *reinterpret_cast<const float4*>(lds + at(row, c));
      *reinterpret_cast<float4*>(f.x + 4) = *reinterpret_cast<const float4*>(lds + at(row, c + 4));
      return split(f);
    }
  }
  static __device__ inline Frag cols_of(const T* lds, int d0, int kb, int p) {
    if constexpr (kBf16) {
      return a_cols(lds, d0, kb, p);
    } else {
      const int lane = threadIdx.x & 63;
      F32x8 f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f.x[e] = lds[at(kb * 32 + 16 * p + 8 * (e / 4) + 4 * (lane >> 5) + (e % 4),
                        d0 + (lane & 31))];
      return split(f);
    }
  }
};

// This lane's row as the other operand: channels 16 ks + 8 (l / 32) .. +7, zero where !ok.
template <typename T, int D>
__device__ inline void load_frag(typename Type<T>::Frag (&f)[D / 16], const T* row, bool ok) {
  const int hh = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    if constexpr (sizeof(T) == 2) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (ok) u = *reinterpret_cast<const uint4*>(row + ks * 16 + hh * 8);
      f[ks] = as_bf16x8(u);
    } else {
      F32x8 x = {};
      if (ok) {
        *reinterpret_cast<float4*>(x.x) =
            *reinterpret_cast<const float4*>(row + ks * 16 + hh * 8);
        *reinterpret_cast<float4*>(x.x + 4) =
            *reinterpret_cast<const float4*>(row + ks * 16 + hh * 8 + 4);
      }
      f[ks] = split(x);
    }
  }
}

__device__ inline float frag_at(const bf16x8_t& f, int e) { return (float)f[e]; }
__device__ inline float frag_at(const Split& f, int e) {
  return (float)f.h[e] + ((float)f.m[e] + (float)f.l[e]);
}

// Sixteen result values as fragments (elements 8 p .. 8 p + 7) of the next product, rounded to
// the nearest bf16, or split.
__device__ inline void to_frags(const float (&x)[16], bf16x8_t (&f)[2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) f[p][e] = (__bf16)x[8 * p + e];
}
__device__ inline void to_frags(const float (&x)[16], Split (&f)[2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    F32x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y.x[e] = x[8 * p + e];
    f[p] = split(y);
  }
}
// x - bf16(x), exact in float32, rounded once: hi + lo carry x to within 2^-17 |x|.
__device__ inline void to_low_frags(const float (&x)[16], const bf16x8_t (&hi)[2],
                                    bf16x8_t (&lo)[2]) {
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) lo[p][e] = (__bf16)(x[8 * p + e] - (float)hi[p][e]);
}

// Sixteen values of a lane to LDS and back, 24 bits each: a float's upper three bytes (16
// significant bits, the rest cut off, and float32's range; a NaN stays one).  The wave's lanes are
// 16 bytes apart, its three pieces 64 lanes.
__device__ inline void hand_over(uint4* to, const float (&x)[16]) {
  uint32_t u[16], hi[8], lo[4];
#pragma unroll
  for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(x[i]);
#pragma unroll
  for (int i = 0; i < 8; ++i) hi[i] = __builtin_amdgcn_perm(u[2 * i + 1], u[2 * i], 0x07060302u);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    lo[i] = __builtin_amdgcn_perm(u[4 * i + 1], u[4 * i], 0x0c0c0501u) |
            __builtin_amdgcn_perm(u[4 * i + 3], u[4 * i + 2], 0x05010c0cu);
  to[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  to[64] = make_uint4(hi[4], hi[5], hi[6], hi[7]);
  to[128] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}
__device__ inline void take_over(const uint4* from, float (&x)[16]) {
  const uint4 a = from[0], b = from[64], c = from[128];
  const uint32_t hi[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}, lo[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    x[i] = __uint_as_float(__builtin_amdgcn_perm(
        hi[i / 2], lo[i / 4], (i % 2 ? 0x0706000cu : 0x0504000cu) | (uint32_t)(i % 4) << 8));
}
// Stores 16 values of channel block db (channels 32 db + 8 blk + 4 (l / 32) + j) times mul.
__device__ inline void store_block(float* row, int db, const f32x16_t& acc, float mul) {
  const int hh = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int blk = 0; blk < 4; ++blk)
    *reinterpret_cast<float4*>(row + db * 32 + 8 * blk + 4 * hh) =
        make_float4(acc[4 * blk] * mul, acc[4 * blk + 1] * mul, acc[4 * blk + 2] * mul,
                    acc[4 * blk + 3] * mul);
}

__device__ inline void store_block(uint16_t* row, int db, const f32x16_t& acc, float mul) {
  const int hh = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int blk = 0; blk < 4; ++blk) {
    __bf16 h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = (__bf16)(acc[4 * blk + j] * mul);
    *reinterpret_cast<uint2*>(row + db * 32 + 8 * blk + 4 * hh) = __builtin_bit_cast(uint2, h);
  }
}

// A wave's 32 results (lane l's column is row l % 32) times mul to the rows at `to`, `stride`
// elements apart, as far as there are `rows`.  bf16 rows pass through LDS, in the wave's own 32
// rows of `lds`, so that they are written whole, 16 bytes per lane; RES writes what the rounding
// to bf16 leaves instead.
template <typename T, int D, bool RES = false>
__device__ inline void store_rows(T* lds, const f32x16_t (&o)[D / 32], float mul, T* to,
                                  int64_t stride, int rows) {
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  if constexpr (sizeof(T) == 2) {
    using Rows = Tile<T, D, 32, 64>;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int blk = 0; blk < 4; ++blk) {
        __bf16 h[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x = o[db][4 * blk + j] * mul;
          h[j] = (__bf16)(RES ? x - (float)(__bf16)x : x);
        }
        *reinterpret_cast<uint2*>(lds + Rows::at(lane & 31, db * 32 + 8 * blk + 4 * hh)) =
            __builtin_bit_cast(uint2, h);
      }
    constexpr int PER = 64 / Rows::KCH;  // rows per instruction
    const int c = (lane % Rows::KCH) * 8;
#pragma unroll
    for (int i = 0; i < 32 / PER; ++i) {
      const int r = i * PER + lane / Rows::KCH;
      const uint4 u = *reinterpret_cast<const uint4*>(lds + Rows::at(r, c));
      if (r < rows) *reinterpret_cast<uint4*>(to + r * stride + c) = u;
    }
  } else if ((lane & 31) < rows) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) store_block(to + (lane & 31) * stride, db, o[db], mul);
  }
}

// ------------------------------------------------------------------- from blocks to sequences

// Rows of the sequence that holds tile `slot`.  Tiles have TILE rows (one row per token and
// `per` of them); sequence b's tiles are numbered from cu[b] per / TILE + b, which leaves room
// for them all without knowing the lengths on the host: floor(x + n) - floor(x) + 1 >= ceil(n).
// b = B stands for the rows behind the last sequence.
struct Slot {
  int b, begin, end, tile;  // rows begin .. end - 1 (tokens), tile number within the sequence
};

__device__ inline int cu_at(const int32_t* cu, int b, int total) {
  return b == 0 ? 0 : min(max(cu[b], 0), total);
}

// Largest b in 0 .. B with first(b) <= x, by 64-fold search: each lane looks at one candidate.
// Ends for any data; uniform over the wave.
template <typename First>
__device__ inline int search(int B, int x, const First& first) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B + 1;
  while (n > 1) {
    const int step = (n + 63) / 64, idx = lane * step;
    const bool ok = idx < n && first(lo + min(idx, n - 1)) <= x;
    const int cnt = max(__popcll(__ballot(ok)), 1);
    lo += (cnt - 1) * step;
    n = min(step, n - (cnt - 1) * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

template <int TILE>
__device__ inline Slot find_slot(const int32_t* cu, int B, int total, int per, int slot) {
  const auto first = [&](int b) { return cu_at(cu, b, total) * per / TILE + b; };
  Slot s;
  s.b = search(B, slot, first);
  s.begin = __builtin_amdgcn_readfirstlane(cu_at(cu, s.b, total));
  s.end = s.b < B ? __builtin_amdgcn_readfirstlane(max(cu_at(cu, s.b + 1, total), s.begin))
                  : total;
  s.tile = slot - (s.begin * per / TILE + s.b);
  if (s.tile < 0) {  // only where cu decreases: no rows
    s.tile = 0;
    s.end = s.begin;
  }
  return s;
}

// Keys of sequence b (none for the rows behind the last one).
__device__ inline void key_rows(const int32_t* cu, int b, int B, int total, int& begin, int& n) {
  begin = n = 0;
  if (b >= B) return;
  begin = __builtin_amdgcn_readfirstlane(cu_at(cu, b, total));
  n = __builtin_amdgcn_readfirstlane(max(cu_at(cu, b + 1, total) - begin, 0));
}

// The sums (largest) of x >= 0 over the wave's lanes up to each: by 1, 2, 4 and 8 lanes within rows
// of 16, then the first and third row's last lane to the next row, the second's to the two behind.
template <typename Join>
__device__ inline int prefix(int x, const Join& join) {
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = join(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  return join(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
}
__device__ inline int prefix_sum(int x) {
  return prefix(x, [](int a, int b) { return a + b; });
}
__device__ inline int prefix_max(int x) {
  return prefix(x, [](int a, int b) { return max(a, b); });
}

// A tile of one side's rows (queries, or keys where KEYS) and the sequence's rows of the other.
struct Place {
  int begin, n, tile;   // the sequence's rows on this side, the tile's number among them
  int other, m;         // and on the other side
};

// The tile of slot number `slot`.  Up to 63 sequences are held by a lane each, and slots number the
// tiles from the longest work to the shortest, so that what is dealt out last is short: the work of
// a tile, in tiles of the other side, is all of them, or under a causal mask one less with every
// tile from the last query's (first key's) on.  The slot's work is the largest that more than
// `slot` tiles reach.  More sequences: as they lie, late queries (early keys) first.  Texts of
// 1,024, 700, 2,048, 311 and 13 tokens, 16 heads x 64, biased step: 202 us as they lie, 191 so; 16
// causal ones of 1,024, 16 / 4 heads x 128, forward 95 and 89 us, eight of them, step 290 and 278;
// 32 of 512, 8 heads x 128, all keys, where there is nothing to order, 80 and 86.
template <int TILE, bool KEYS>
__device__ inline Place place_of(const int32_t* cu, int total, const int32_t* cu2, int total2,
                                 int B, int causal, int slots, int slot) {
  Place p = {};
  if (B >= 64) {
    const Slot s = find_slot<TILE>(cu, B, total, 1, KEYS ? slot : slots - 1 - slot);
    p.begin = s.begin;
    p.n = s.end - s.begin;
    p.tile = s.tile;
    key_rows(cu2, s.b, B, total2, p.other, p.m);
    return p;
  }
  const int lane = threadIdx.x & 63, b = min(lane, B);
  const int next = min(b + 1, B);  // four loads at once, none behind a branch
  const int raw0 = cu[b], raw1 = cu[next], raw2 = cu2[b], raw3 = cu2[next];
  const int begin = b == 0 ? 0 : min(max(raw0, 0), total);
  const int end = b < B ? min(max(raw1, 0), total) : total;
  const int other = b == 0 ? 0 : min(max(raw2, 0), total2);
  const int n = lane > B ? 0 : max(end - begin, 0);
  const int m = b < B ? max(min(raw3, total2) - other, 0) : 0;
  const int tiles = n / TILE + (n % TILE != 0), most = m / TILE + (m % TILE != 0);
  const int from = !causal ? tiles + most : KEYS ? tiles : most;
  const auto reach = [&](int c) {  // this sequence's tiles of work c and more
    return c <= 0 ? tiles : c > most ? 0 : min(max(from - c + 1, 0), tiles);
  };
  const auto all = [](int x) { return __builtin_amdgcn_readlane(prefix_sum(x), 63); };
  int lo = 0, hi = __builtin_amdgcn_readlane(prefix_max(most), 63);
  while (lo < hi) {
    const int c = (lo + hi + 1) / 2;
    if (all(reach(c)) > slot) lo = c;
    else hi = c - 1;
  }
  const int above = reach(lo + 1), here = reach(lo) - above;
  const int i = slot - all(above), before = prefix_sum(here) - here;
  const uint64_t who = __ballot(i >= before && i < before + here);
  if (who == 0) return p;  // behind the last tile
  const int l = __builtin_ctzll(who);
  const int rank = __builtin_amdgcn_readlane(above - before, l) + i;
  p.begin = __builtin_amdgcn_readlane(begin, l);
  p.n = __builtin_amdgcn_readlane(n, l);
  p.tile = KEYS ? rank : __builtin_amdgcn_readlane(tiles, l) - 1 - rank;
  p.other = __builtin_amdgcn_readlane(other, l);
  p.m = __builtin_amdgcn_readlane(m, l);
  return p;
}

// The bias by distance of one head, in base-2 units: -inf where it hides, 0 where it has no
// bucket.
__device__ inline float bias_of(const float* table, const int32_t* map, int heads, int buckets,
                                int head, int idx) {
  const int c = map[idx];
  if (c < 0 || c >= buckets) return 0.0f;
  const float x = table[(int64_t)c * heads + head];
  return x <= kHidden ? -INFINITY : x * kLog2e;
}

__device__ inline int block_number() { return (int)(blockIdx.x + blockIdx.y * kGridX); }

// Block -> (key head, slot, head within the group).  Blocks go to XCD x % 8, so the blocks of a
// key head stay on one XCD, whose L2 then serves its keys and values; with key heads that the 8
// XCDs do not share evenly, each head's tiles are dealt out over `parts` of them, so that early
// and late tiles (short and long ones under a causal mask) fall on each.  The long ones come first:
// late tiles of queries, early tiles of keys.
struct Work {
  int u, slot, head;  // head: u * per + the block's number among the `per` of its slot
};
template <bool LATE_FIRST = true>
__device__ inline bool work_of(const Spread& sp, int per, Work& w) {
  const int x = block_number() % 8;
  int r = block_number() / 8;
  const int j = r % per;
  r /= per;
  const int su = (r % sp.local) * 8 + x, nth = r / sp.local;
  if (nth >= sp.ranks) return false;  // behind the grid's last workgroup
  const int rank = LATE_FIRST ? sp.ranks - 1 - nth : nth;
  w.u = su % sp.units;
  w.slot = rank * sp.parts + su / sp.units;
  w.head = w.u * per + j;
  return w.slot < sp.slots;
}

}  // namespace seq
}  // namespace dsa3d
