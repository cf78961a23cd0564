// Which kernel takes a product: a function of sizes and types alone.  Host code.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace costa {

// Kinds of left operands.
enum Source : int { SRC_MX4, SRC_MX8, SRC_BF16, SRC_F16, SRC_F32 };
// bfloat16 parts that hold an element of each.
constexpr int parts_of(int src) { return src == SRC_F32 ? 3 : src == SRC_F16 ? 2 : 1; }

// How a product runs.
enum Variant : int { FEW_ROWS, TILES_BF16, TILES_SCALED, THIN };
struct ProductPlan {
  Variant variant;
  int bm, bn;   // tile of C (rows, columns)
  int splits;   // workgroups that share a tile's sum
};
constexpr int kCUs = 256;
constexpr int kFewWaves = 4;  // of a workgroup of the kernel for few rows
constexpr size_t kPartsMax = (size_t)256 << 20;  // bytes of a split sum's parts

inline int64_t up_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Most splits that the parts' memory allows.
inline int64_t splits_max(int64_t m, int64_t n) {
  return std::max<int64_t>((int64_t)(kPartsMax / 4) / std::max<int64_t>(m * n, 1), 1);
}

// Estimated time of a tiled product in us, from what MI355X measured.  A
// workgroup's step of k takes `step` us when the CU has w of them, max(alone, w *
// share): bfloat16, k by 64: 1.77 us for a 256x256 tile (one a CU), 0.57 a tile for
// several of 128x128, 0.39 of 128x64, not below 0.66 (the way from memory through
// shared memory); 4 bits, k by 256: 2.6 us at 256x256, 0.76 at 128x128, not below 1.0.
// Joining a split sum costs a launch and its parts' way to memory and back.  (It ranks
// tiles and splits of one call; as a time it holds for bfloat16 rows with k next to one
// another and for 4 bits.  A transposed float operand's step takes about twice as long: 35 us
// estimated, 66 measured for 100x64 over 524288; with an 8-bit operand, 29 and 31 to 38 for
// 1041x1999x2501.)
// (512x8192x8192 in bfloat16: 128x128 unsplit 88 us, 256x256 unsplit 232, split in four 86;
// 256x8192x8192: 128x128 split in four 53, 128x64 unsplit 72; 1024^3: 128x64 13, 128x128 17.)
// in_parts: the sums stay in parts, split or not, for a kernel that reads them anyway.
inline double tiled_time(bool scaled, int parts, int64_t bm, int64_t bn, int64_t splits, int64_t m, int64_t n, int64_t k,
                         bool in_parts = false) {
  const double size = (double)(bm * bn * parts) / 65536.0;
  const double share = scaled ? 0.2 + 2.4 * size : 0.22 + 1.55 * size, alone = scaled ? 1.0 : 0.66;
  const int64_t groups = up_div(m, bm) * up_div(n, bn) * splits, steps = up_div(up_div(k, scaled ? 256 : 64), splits);
  const double step = std::max(alone, (double)up_div(groups, kCUs) * share);
  const double way = (double)splits * m * n * 8e-6 / 4.0;
  return 3.0 + (double)steps * step + (in_parts ? way : splits > 1 ? 3.0 + way : 0.0);
}

inline ProductPlan plan_product(int src, bool k_next, int bbits, int64_t m, int64_t n, int64_t k, bool in_parts = false) {
  ProductPlan r{};
  if (src != SRC_MX4 && src != SRC_MX8 && k < 8) {
    r.variant = THIN;
    r.splits = 1;
    return r;
  }
  if (m <= 64 && k_next) {
    r.variant = FEW_ROWS;
    r.bm = m <= 16 ? 16 : m <= 32 ? 32 : 64;
    // (32 columns share a slab's way through shared memory; half as many workgroups)
    r.bn = m > 4 && n >= 64 * kCUs ? 32 : 16;
    const int64_t units = up_div(k, 1024 / bbits);
    const int64_t s = std::min(kCUs / std::max<int64_t>(up_div(n, r.bn), 1), units / (4 * kFewWaves));
    r.splits = (int)std::max<int64_t>(std::min(s, splits_max(m, n)), 1);
    return r;
  }
  // (the scaled kernel counts a tile's bytes in 32 bits)
  const bool scaled = src == SRC_MX4 && bbits == 4 && k <= 1 << 24;
  r.variant = scaled ? TILES_SCALED : TILES_BF16;
  const int parts = scaled ? 1 : parts_of(src);
  // (two steps of k each, at least)
  const int64_t most = std::min({splits_max(m, n), up_div(k, scaled ? 512 : 128), (int64_t)kCUs});
  double best = 0;
  for (const int bn : {256, 128, 64}) {
    if (scaled && bn == 64) continue;
    const int bm = bn == 256 && parts == 1 ? 256 : 128;
    const int64_t tiles = up_div(m, bm) * up_div(n, bn);
    // unsplit, in a few, or so that the workgroups are one to four for every CU
    for (int64_t c = 0; c < 8; ++c) {
      const int64_t s = std::min(c < 4 ? c + 1 : (c - 3) * kCUs / std::max<int64_t>(tiles, 1), most);
      if (s < 1) continue;
      const double t = tiled_time(scaled, parts, bm, bn, s, m, n, k, in_parts);
      if (r.splits == 0 || t < best) {
        best = t;
        r.bm = bm;
        r.bn = bn;
        r.splits = (int)s;
      }
    }
  }
  return r;
}

}  // namespace costa
