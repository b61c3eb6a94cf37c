// Host-side launch interface of the sequence kernels (validated arguments only).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

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
};

void set_plan(PagedGeometry& g);  // tile, splits, part and tiles
size_t paged_workspace(const PagedGeometry& g);
hipError_t launch_paged_forward(const PagedGeometry& g, bool bf16, const void* q,
                                const void* k_pages, const void* v_pages, const int32_t* pages,
                                const int32_t* kv_lens, const int32_t* cu_q, const float* table,
                                const int32_t* map, void* out, float* lse, void* workspace,
                                hipStream_t stream);
hipError_t launch_paged_append(const PagedGeometry& g, bool bf16, const void* k, const void* v,
                               const int32_t* cu_q, const int32_t* kv_lens, const int32_t* pages,
                               void* k_pages, void* v_pages, hipStream_t stream);

}  // namespace dsa3d
