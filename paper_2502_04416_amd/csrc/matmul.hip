// Which kernel, tile and K split a product of matmul.h runs on.
#include "matmul.h"

#include <algorithm>

#include "../../include/cmoe.h"
#include "matmul_launch.h"

namespace cmoe {

namespace {

constexpr int CUS = 256;

struct Choice {
  Tile tile;
  int k_split;
};

struct Shape {
  bool a_columns, b_columns, dual, segments, splits;
};
constexpr Shape shape_of(Product kind) {
  return {kind == PRODUCT_DW, kind == PRODUCT_GATED || kind == PRODUCT_DOWN || kind == PRODUCT_DW || kind == PRODUCT_DHEAD, kind == PRODUCT_GATED,
          kind == PRODUCT_DX, kind != PRODUCT_LSE && kind != PRODUCT_DLOGITS};
}

// Relative time of a K step of 32 of a tile when the chip is full, and workgroups per CU.
constexpr double kStep[TILES] = {1.0, 0.60, 0.42, 2.6, 1.0};
constexpr int kPerCu[TILES] = {1, 2, 2, 2, 2};
constexpr double kTileCost = 16;             // prologue and epilogue, in steps of the large tile

Choice choose(Product kind, int dtype, bool ring, int64_t m, int64_t n, int64_t k, int pair, size_t slab_bytes) {
  const Shape sh = shape_of(kind);
  const int64_t steps = ((k + 31) / 32) * (sh.segments ? 2 : 1);
  const int64_t cols = sh.dual ? 2 * n : n;
  Choice best{ANY_128, 1};
  double best_cost = 1e300;
  const int forced_tile = tuning().mat_tile, forced_split = tuning().mat_split;
  const int first = ring ? RING_256 : ANY_128, last = ring ? RING_64 : ANY_32;
  for (int t = first; t <= last; ++t) {
    if (sh.a_columns && t == RING_64) continue;
    if (forced_tile >= first && forced_tile <= last && forced_tile != t && !(sh.a_columns && forced_tile == RING_64)) continue;
    const int64_t tiles = (m + kTiles[t].bm - 1) / kTiles[t].bm * ((cols + kTiles[t].bn - 1) / kTiles[t].bn) * pair;
    for (int split = 1; split <= 16; split *= 2) {
      if (split > 1 && (!sh.splits || pair > 1 || (size_t)split * m * cols * 4 > slab_bytes)) break;
      if (split > 1 && forced_split < 1 && steps / split < 8) break;
      if (forced_split >= 1 && split != forced_split && sh.splits && pair == 1) continue;
      const int64_t slots = (int64_t)CUS * kPerCu[t];
      const double rounds = (double)((tiles * split + slots - 1) / slots);
      // a last round that does not fill the chip still takes a tile's time; with one workgroup on a CU of two it is somewhat shorter
      const double fill = tiles * split <= CUS && kPerCu[t] == 2 ? 0.6 : 1.0;
      double cost = rounds * fill * kStep[t] * ((double)(steps + split - 1) / split + kTileCost);
      if (split > 1) cost += 8 + (double)split * m * cols * 8 / 4e12 / 0.68e-6;   // the slabs written and read, a launch
      if (cost < best_cost) best_cost = cost, best = {(Tile)t, split};
    }
  }
  (void)dtype;
  return best;
}

int64_t ranges_of(const Choice& c, int64_t n) { return (n + kTiles[c.tile].bn - 1) / kTiles[c.tile].bn * kTiles[c.tile].wgn; }

}  // namespace

int64_t lse_ranges(int dtype, int64_t m, int64_t n, int64_t k) {
  int64_t most = 0;
  for (int ring = 0; ring <= (dtype == CMOE_BF16); ++ring) most = std::max(most, ranges_of(choose(PRODUCT_LSE, dtype, ring, m, n, k, 1, 0), n));
  return most;
}

size_t matmul_slab_bytes(Product kind, int dtype, int64_t m, int64_t n, int64_t k) {
  if (!shape_of(kind).splits || m == 0 || n == 0) return 0;
  const size_t all = (size_t)1 << 40;
  const size_t one = (size_t)m * n * 4 * (shape_of(kind).dual ? 2 : 1);
  size_t most = 0;
  for (int ring = 0; ring <= (dtype == CMOE_BF16); ++ring)
    for (int pair = 1; pair <= (kind == PRODUCT_DW ? 2 : 1); ++pair) {
      const Choice c = choose(kind, dtype, ring, m, n, k, pair, all);
      if (c.k_split > 1) most = std::max(most, c.k_split * one);
    }
  return most;
}

hipError_t matmul(Product kind, int dtype, MatArgs p, size_t slab_bytes, hipStream_t s, int* ranges) {
  if (p.m <= 0 || p.n <= 0) return hipSuccess;
  if (!p.m_a) p.m_a = p.m;
  if (!p.n_b) p.n_b = p.n;
  if (!p.k_b) p.k_b = p.k;
  const Shape sh = shape_of(kind);
  auto wide = [](const void* q) { return ((uintptr_t)q & 15) == 0; };
  const bool ring = dtype == CMOE_BF16 && wide(p.a) && wide(p.a2) && wide(p.b) && wide(p.b2) && p.lda % 8 == 0 && p.ldb % 8 == 0 &&
                    (sh.a_columns ? p.m_a : p.k) % 8 == 0 && (sh.b_columns ? p.n_b : p.k) % 8 == 0;
  const Choice c = choose(kind, dtype, ring, p.m, p.n, p.k, kind == PRODUCT_DW && p.c2 ? 2 : 1, p.slab ? slab_bytes : 0);
  p.k_split = c.k_split;
  if (ranges) *ranges = (int)ranges_of(c, p.n);
  switch (kind) {
    case PRODUCT_GATED: return launch_gated(c.tile, dtype, p, s);
    case PRODUCT_DOWN: return launch_down(c.tile, dtype, p, s);
    case PRODUCT_DGATED: return launch_dgated(c.tile, dtype, p, s);
    case PRODUCT_DX: return launch_dx(c.tile, dtype, p, s);
    case PRODUCT_DW: return launch_dw(c.tile, dtype, p, s);
    case PRODUCT_LSE: return launch_lse(c.tile, dtype, p, s);
    case PRODUCT_DLOGITS: return launch_dlogits(c.tile, dtype, p, s);
    default: return launch_dhead(c.tile, dtype, p, s);
  }
}

}  // namespace cmoe
