// Tiles, clusters and K-parts of a Newton-Schulz product (orth_product.cu): plain
// arithmetic without CUDA.
#pragma once

#include <stdint.h>

namespace oscars {

constexpr int kNsK = 64, kNsMaxBN = 256, kNsMaxStages = 8;
constexpr int kNsBox = 64 * 128;                   // one operand box: 64 rows of 128 bytes
constexpr int kNsEpiWarps = 8;
constexpr int kNsStg = 2048;                       // one staging box: 32 rows x 64 bytes
constexpr int kNsStgBytes = kNsEpiWarps * 2 * kNsStg;   // two per epilogue warp
constexpr int kNsBarBytes = 256;
constexpr int kNsSmem = 227 * 1024;
constexpr int kNsRing = kNsSmem - 1024 - kNsBarBytes - kNsStgBytes;

struct NsProduct {
  bool sym;                        // symmetric: M = N, square tiles
  int batch, M, N, K, a_halves, b_halves;
};
struct NsRoom {
  int sms, pairs, fours;           // CTAs, and clusters of two and of four, that run at once
};
struct NsShape {
  int cl, BN, mt, nt, split, full, stages;   // CTAs of a tile, its columns, tiles, K-parts, all tiles (not a triangle)
  int64_t units;                   // tiles of all matrices
};

inline int ns_stage_bytes(const NsProduct& a, int BN, int cl) { return (a.a_halves * 2 + a.b_halves * (BN / cl / 64)) * kNsBox; }
inline int ns_stages(const NsProduct& a, int BN, int cl, int split) {
  const int nk = ((a.K + kNsK - 1) / kNsK + split - 1) / split, bytes = ns_stage_bytes(a, BN, cl);
  int st = (kNsRing - (split > 1 ? 128 * BN * 4 : 0)) / bytes;   // beside the parts' sums
  st = st > kNsMaxStages ? kNsMaxStages : st;
  return st > nk ? (nk < 2 ? 2 : nk) : st;
}
// A CTA of a split tile owns BN / split columns, which the parts send it in whole groups of 32.
inline bool ns_split_fits(int BN, int split) { return BN % (32 * split) == 0; }

// The shape with the least estimated time: waves of tiles times the longer of a
// tile's products (2 BN clocks a K-block and product) and loads (52 bytes a clock
// into an SM), plus a tile's and a launch's fixed part, a split's exchange and a
// triangle's second write.  Symmetric products take square
// tiles: a triangle of them and their mirror images, or all of them where a wave has
// room (us a call, a triangle / all: 16 x 512 x 784 bf16 183 / 173, 4 x 768 x 768 bf16 124 /
// 119; with the K-blocks split, 512 x 784 fp32, 122 / 124).
inline NsShape ns_shape(const NsProduct& a, const NsRoom& has) {
  const int nk = (a.K + kNsK - 1) / kNsK, products = a.a_halves + a.b_halves - 1;
  double best = 0.0;
  NsShape to{};
  for (int c = 1; c <= 2; ++c) {
    const int mt = ((a.M + 127) / 128 + c - 1) / c * c;
    for (int bn = 64; bn <= kNsMaxBN; bn += 64) {
      if ((c == 2 && bn % 128) || (a.sym && bn != 128 * c)) continue;
      const int nt = (a.N + bn - 1) / bn;
      const int room = c == 2 ? has.pairs : has.sms;
      const double mma = 2.0 * bn * products, load = ns_stage_bytes(a, bn, c) / 52.0;
      for (int split = 1, full = 0; split <= (c == 1 ? 4 : 1); full ^= 1, split *= full ? 1 : 2) {
        if (full && (!a.sym || split > 1)) continue;
        const int64_t tiles = a.sym && !full ? nt * static_cast<int64_t>(nt + 1) / 2 : static_cast<int64_t>(mt / c) * nt;
        const int64_t units = a.batch * tiles;
        // a part has two K-blocks, and the clusters run at once
        if (split > 1 && (units > (split == 2 ? has.pairs : has.fours) || nk < 2 * split || !ns_split_fits(bn, split) ||
                          ns_stages(a, bn, c, split) < 2))
          continue;
        const double waves = split > 1 ? 1.0 : static_cast<double>((units + room - 1) / room);
        const double cost = waves * ((nk + split - 1) / split * (load > mma ? load : mma) + 600.0) + 12.0 * bn +
                            (c == 2 ? 1500.0 : 0.0) + (split > 1 ? 2500.0 : a.sym && !full && nt > 1 ? 6.0 * bn : 0.0);
        if (best == 0.0 || cost < best) {
          best = cost;
          to = NsShape{c, bn, mt, nt, split, full, 0, units};
        }
      }
    }
  }
  to.stages = ns_stages(a, to.BN, to.cl, to.split);
  return to;
}

}  // namespace oscars
