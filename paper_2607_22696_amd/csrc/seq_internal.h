// Host-side launch interface of the sequence kernels (validated arguments only).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

#include "dsa3d_mx.h"

namespace dsa3d {

// How a launch deals (unit, slot) pairs out over the 8 XCDs (see work_of).
struct Spread {
  int units, slots;  // key heads; tiles of the packed rows
  int parts;         // parts a unit's slots are dealt to: units * parts is a multiple of 8
  int local;         // unit parts per XCD
  int ranks;         // slots of the largest part
};

struct SeqGeometry {
  int B, nq, nk;          // sequences, rows of q and of k
  int H, KH, group, D;    // heads, key heads, heads per key head
  int causal;
  int rel_min, span, nb;  // nb = 0: no bias
  float scale, scale_log2;
  int64_t qs, ks, vs;     // elements between token rows
  Spread q_tiles, k_tiles;
  int parts;              // parts of a key tile's queries in the dk/dv pass
};

constexpr int kSeqTile = 128;  // queries (forward, dq) or keys (dk, dv) per workgroup

Spread seq_spread(int units, int slots);
inline int64_t seq_blocks(const Spread& s, int per) {
  return 8ll * s.local * s.ranks * per;
}

// A launch has fewer than 2^32 threads in x, so more workgroups than kGridX lie in rows of that
// many (a multiple of 8: block n stays on XCD n % 8), the last of which may be wider than needed:
// workgroup blockIdx.x + blockIdx.y kGridX, which must not reach 2^31.
constexpr int kGridX = 1 << 22;
constexpr int64_t kMostBlocks = (1ll << 31) - kGridX;

template <typename... A>
hipError_t seq_launch(const void* fn, int64_t blocks, int threads, size_t lds, hipStream_t s,
                      A... args) {
  void* a[] = {(void*)&args...};
  const int64_t rows = (blocks + kGridX - 1) / kGridX;
  const dim3 grid((uint32_t)(rows > 1 ? kGridX : blocks), (uint32_t)rows);
  return hipLaunchKernel(fn, grid, dim3(threads), a, lds, s);
}

inline size_t round_256(size_t x) { return (x + 255) & ~size_t(255); }

struct SeqTensors {
  const void *q, *k, *v;
  const int32_t *cu_q, *cu_k;
  const float* table;
  const int32_t* map;
};

hipError_t launch_seq_forward(const SeqGeometry& g, bool bf16, const SeqTensors& t, void* out,
                              void* out_res, float* lse, hipStream_t stream);
int seq_backward_parts(const SeqGeometry& g, bool bf16);
size_t seq_backward_workspace(const SeqGeometry& g, bool want_table);
hipError_t launch_seq_backward(const SeqGeometry& g, bool bf16, const SeqTensors& t,
                               const void* out, const void* out_res, const float* lse,
                               const void* dout, void* dq, void* dk, void* dv, float* d_table,
                               void* workspace, hipStream_t stream);

// x / d as (x * mul) >> shift, exact for 0 <= x < 2^31: with 2^(s-1) < d <= 2^s and
// mul = floor(2^(31+s) / d) + 1, the product exceeds x 2^(31+s) / d by at most x < 2^31 <=
// 2^(31+s) / d, less than the step to the next whole quotient.
inline void divisor(int d, uint32_t* mul, uint32_t* shift) {
  int s = 0;
  while ((1ll << s) < d) ++s;
  *mul = d == 1 ? 1u : (uint32_t)((1ull << (31 + s)) / d + 1);
  *shift = d == 1 ? 0 : 31 + s;
}

struct PagedGeometry {
  int B, nq;
  int H, KH, group, D;
  int num_pages, page_size, max_pages, max_kv;
  uint32_t page_mul, page_shift;    // j / page_size as a product and a shift
  uint32_t group_mul, group_shift;  // row / group
  int causal;
  int rel_min, span, nb;
  float scale, scale_log2;
  int64_t qs, ks, vs;
  int tile;     // rows (tokens x heads of a group) per workgroup
  int splits;   // most parts of a tile's keys, and least keys of a part
  int part;
  Spread tiles;
  int64_t blocks;  // workgroups of the launch
  int target;      // > 0: parts by the lengths that the GPU sees (paged_rules.h)
  int64_t room;    // parts per key head with partial results, where target > 0
};

void set_plan(PagedGeometry& g);     // tile, splits, part, tiles and blocks
void set_plan_mx(PagedGeometry& g);  // and target and room, for a cache of 8 or 4 bits
size_t paged_workspace(const PagedGeometry& g);
hipError_t launch_paged_forward(const PagedGeometry& g, bool bf16, const void* q,
                                const void* k_pages, const void* v_pages, const int32_t* pages,
                                const int32_t* kv_lens, const int32_t* cu_q, const float* table,
                                const int32_t* map, void* out, float* lse, void* workspace,
                                hipStream_t stream);
hipError_t launch_paged_append(const PagedGeometry& g, bool bf16, const void* k, const void* v,
                               const int32_t* cu_q, const int32_t* kv_lens, const int32_t* pages,
                               void* k_pages, void* v_pages, hipStream_t stream);
size_t paged_mx_workspace(const PagedGeometry& g);
hipError_t launch_paged_forward_mx(const PagedGeometry& g, bool bf16, const void* q,
                                   const dsa3d_mx_cache& cache, const int32_t* pages,
                                   const int32_t* kv_lens, const int32_t* cu_q,
                                   const float* table, const int32_t* map, void* out, float* lse,
                                   void* workspace, hipStream_t stream);
hipError_t launch_paged_append_mx(const PagedGeometry& g, bool bf16, const void* k, const void* v,
                                  const int32_t* cu_q, const int32_t* kv_lens,
                                  const int32_t* pages, const dsa3d_mx_cache& cache,
                                  hipStream_t stream);
hipError_t launch_paged_read_mx(const PagedGeometry& g, bool bf16, const dsa3d_mx_cache& cache,
                                const int32_t* pages, const int32_t* kv_lens, const int32_t* cu_q,
                                void* k, void* v, hipStream_t stream);

}  // namespace dsa3d
