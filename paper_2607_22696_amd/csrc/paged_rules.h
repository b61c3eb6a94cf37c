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

}  // namespace dsa3d
