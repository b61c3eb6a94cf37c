// How the paged attention deals its work out (host code; the figures were measured on one MI355X).
#pragma once

#include <algorithm>
#include <cstdint>

namespace dsa3d {

constexpr int kFewRows = 32, kManyRows = 128;
constexpr int kFewKeys = 128;   // keys per tile of the form with few rows: 32 per wave
constexpr int kMostParts = 64;  // of a tile's keys

struct PagedPlan {
  int tile;          // rows (tokens x heads of a group) per workgroup
  int splits, part;  // most parts of a tile's keys, and least keys of a part
};

// Rows per workgroup: 32 where the requests have no more on average, in which form single tokens
// are read fastest, else 128, which multiply each copied key with four times the rows.  Tiles of
// 32 / 128, us, 16 requests of 4,000 keys with n new tokens each: 32 / 8 heads x 128, n = 2 51/46,
// 8 60/50, 12 74/55, 64 211/111; 16 / 16 x 64, n = 2 53/56, 16 59/62, 64 87/73; one with 300 beside
// 15 of one 105/89, beside 63 261/314.  Parts of the keys (`splits` at most, of `part` keys at
// least, whole tiles; a tile whose keys fit one part has no join):
//  - few rows: reading is all, so the key heads, requests and parts make up to 2,048 workgroups,
//    which also evens out requests of different lengths, in parts of 1,024 keys, or of 512 where
//    that leaves the card half empty.  64 requests of 200 to 8,000 tokens, 32 / 8 heads x 128:
//    238 us in parts of 2,048 keys, 219 of 1,024, 215 of 512; one of 4,000: 63, 28, 19 us; four of
//    30,000: 105, 110, 113 us.
//  - many rows: a part's float32 results are written and read again, which weighs more than uneven
//    ends: parts of 4,096 keys, or as many as fill the card (512 workgroups).  1,024 new of 16,384
//    tokens: 340 us in parts of 2,048, 312 of 4,096; chunks of 512, 801, 300 and single tokens:
//    265 and 236 us.
inline PagedPlan paged_plan(int64_t tokens, int group, int kv_heads, int batch, int max_kv) {
  PagedPlan p;
  const int64_t rows = tokens * group;
  p.tile = rows <= (int64_t)kFewRows * batch ? kFewRows : kManyRows;
  const int64_t tiles =
      std::max<int64_t>((rows + p.tile - 1) / p.tile, std::min<int64_t>(batch, tokens));
  const int64_t units = std::max<int64_t>(1, tiles * kv_heads);
  int64_t splits;
  if (p.tile == kFewRows) {
    p.part = units * max_kv >= 512 * 1024 ? 1024 : 512;
    splits = std::min<int64_t>(2048 / units, max_kv / p.part);
  } else {
    const int64_t fill = (512 + units - 1) / units;
    splits = std::min<int64_t>(2048 / units, max_kv / 4096);
    p.part = 4096;
    if (splits < fill) {
      splits = std::min<int64_t>(fill, max_kv / 512);
      const int64_t even = std::max<int64_t>(512, max_kv / fill);
      p.part = (int)((even + kFewKeys - 1) / kFewKeys * kFewKeys);
    }
  }
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(splits, kMostParts));
  return p;
}

// The same over a cache of 8 or 4 bits.
constexpr int kDealt = 64;        // requests that a wave holds a lane each
constexpr int kMostPartsMx = 256;
constexpr int kLeastPartMx = 512;

struct MxPlan {
  int tile;          // 16, 32 or 128 rows per workgroup
  int splits, part;  // most parts of a tile's keys, and least keys of a part
  int target;        // > 0: parts go by the lengths that the GPU sees, about this many per key head
  int64_t bound;     // and are at most this many per key head,
  int64_t room;      // of which so many are of tiles that have several, and have partial results
};

// Rows per workgroup: 16 where the requests have no more on average, else as paged_plan.  Up to 64
// requests' keys are divided on the GPU, by all their lengths (more requests as by paged_plan, which
// fills the card where they are alike: see deal in paged_mx.hip), into parts of at least 512 keys
// (256: single tokens of 64 requests 111 and 112 us, drafts of 5 tokens of 16 20.0 and 22.3, 12
// biased ones 21.0 and 22.0), as many as there are workgroups at a time:
//  - two per compute unit, where few requests have parts of one length (four requests of 31,000 to
//    120,000 tokens, 16 / 2 heads, 4 bits: 24 us in 512 parts, 28 in 384, 29 in 768) and for many
//    rows, whose partial results cost most;
//  - else three, of which the longest go first (single tokens of 64 requests, 32 / 8 heads, 8 bits:
//    120 us in 512, 111 in 768, 113 in 1,280; 4 bits 74, 67, 67).
// The border goes by `all`, the workgroups without parts.  Single tokens of n requests, 32 / 8 heads
// x 128, 8 bits, us in 512 - all / 768 parts, of 30,000 tokens each and of 3,000 to 60,000: n = 4
// (all = 48) 56/59 and 57/66, 6 (64) 74/76 and 81/87, 7 (72) 87/99 and 91/104, 8 (88) 97/97 and
// 104/110, 12 (128) 157/138 and 159/160, 16 (168) 206/181 and 219/207; 64 with 2 / 1 heads (73) 98/96
// and 102/109.  The uneven ones of 7 and of 16 in float32 95/104 and 220/209, in 4 bits 56/63 and
// 122/117, at 64 channels 51/56 and 112/111, with 6 new tokens each 99/111 and 260/223.
//
// For many rows at most 16 parts, and 512 MiB of partial results if all rows had them, unless
// paged_plan had more.  Partial results are numbered over the parts of tiles that have several: the
// workspace does not grow with the longest cache that a call allows (64 requests with 8 new tokens
// each, 32 / 8 heads x 128, up to 131,072 tokens: 25 MiB; room for each row's most parts was 782).
inline MxPlan paged_mx_plan(int64_t tokens, int group, int kv_heads, int batch, int max_kv,
                            int head_dim) {
  const PagedPlan q = paged_plan(tokens, group, kv_heads, batch, max_kv);
  const int64_t rows = tokens * group;
  MxPlan p = {rows <= (int64_t)16 * batch ? 16 : q.tile, q.splits, q.part, 0, 0, 0};
  if (batch > kDealt) return p;
  p.part = kLeastPartMx;
  const int64_t slots = rows / p.tile + batch + 1, all = slots * kv_heads;
  const bool few = q.tile == kFewRows;
  p.target = (int)std::max<int64_t>(
      1, (!few ? 512 : all <= 96 ? 512 - all : 768) / kv_heads);
  const int64_t room = (int64_t)512 << 20, each = std::max<int64_t>(1, rows) * kv_heads * head_dim * 4;
  int64_t most =
      few ? kMostPartsMx : std::max<int64_t>(q.splits, std::min<int64_t>(16, room / each));
  if (batch == 1) {  // ceil(keys / part), part >= tiles keys / target
    const int64_t tiles = std::max<int64_t>(1, (rows + p.tile - 1) / p.tile);
    most = std::min(most, (p.target + tiles - 1) / tiles);
  }
  p.splits = (int)std::max<int64_t>(
      1, std::min<int64_t>({max_kv / p.part, p.target + 1, most}));
  // sum of ceil(keys / part) <= target + one per tile; 8 for the rounding of the GPU's sum
  p.bound = std::min<int64_t>(slots * p.splits, slots + p.target + 8);
  // ceil(keys / part) < 2 keys / part where it is 2 or more
  p.room = p.splits > 1 ? std::min<int64_t>(p.bound, 2 * (int64_t)p.target + 8) : 0;
  return p;
}

}  // namespace dsa3d
