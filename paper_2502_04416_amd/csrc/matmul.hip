// Which kernel, tile and K split a product of matmul.h runs on, and whether its operands are copied for it.
#include "matmul.h"

#include <algorithm>

#include "../../include/cmoe.h"
#include "matmul_launch.h"

namespace cmoe {

namespace {

constexpr int CUS = 256;

struct Shape {
  bool a_columns, b_columns, dual, segments, logits;
};
constexpr Shape shape_of(Product kind) {
  return {kind == PRODUCT_DW, kind == PRODUCT_GATED || kind == PRODUCT_DOWN || kind == PRODUCT_DW || kind == PRODUCT_DHEAD, kind == PRODUCT_GATED,
          kind == PRODUCT_DX, kind == PRODUCT_LSE || kind == PRODUCT_DLOGITS};
}

struct Choice {
  Tile tile;
  int full, k_split;
  bool copies;
  size_t slab;               // bytes
};

// What a tile takes, in us: a K step of 32 where it has a CU alone, and its share of one with others; its beginning and end; tiles to a CU.
// The ring's small tiles are bound by what a CU takes in, 62 KB a us, with two on it as with one.
struct Cost {
  double alone, share, ends;
  int per_cu;
};
constexpr Cost kBf16[TILES] = {{0.62, 0.69, 14, 1}, {0.265, 0.33, 6, 2}, {0.20, 0.21, 5, 2}, {0.3, 0.2, 5, 4}, {0.35, 0.3, 5, 2}};
constexpr Cost kFp32[TILES] = {{0, 0, 0, 1}, {0.82, 0.82, 8, 1}, {0.58, 0.58, 7, 1}, {0.82, 0.62, 6, 4}, {0.85, 0.7, 6, 2}};
constexpr double kLaunch = 4, kBytesPerUs = 4.5e6;

int64_t round8(int64_t n) { return (n + 7) / 8 * 8; }

// Bytes of the copies, and of what is read and written for them.
size_t copy_bytes(const Shape& sh, int planes, int64_t m, int64_t n, int64_t k, bool second) {
  const int64_t a = (sh.a_columns ? k * round8(m) : m * round8(k)) * (sh.segments ? 2 : 1);
  const int64_t b = (sh.b_columns ? k * round8(n) : n * round8(k)) * (second ? 2 : 1);
  return ((size_t)(a + b) * planes * 2 + 255) / 256 * 256;
}

// direct: bf16 operands that the ring can read where they are.  second: there is a second B.  plan: of logits, where it is settled.
// The tiles that fill the chip a whole number of times are left whole; the rest, if that is shorter, is split.
Choice weigh(Product kind, int dtype, bool direct, bool second, int64_t m, int64_t n, int64_t k, size_t workspace, const LogitsPlan* plan) {
  const Shape sh = shape_of(kind);
  const int pair = kind == PRODUCT_DW && second ? 2 : 1, planes = dtype == CMOE_F32 ? 3 : 1;
  const int64_t steps1 = ((k + 31) / 32) * (sh.segments ? 2 : 1);
  const int64_t cols = sh.dual ? 2 * n : n;
  const int forced_tile = tuning().mat_tile, forced_split = tuning().mat_split;
  const size_t copies = direct ? 0 : copy_bytes(sh, planes, m, n, k, second);
  const double copy_time = direct ? 0 : kLaunch + (double)copies * (planes == 3 ? 10.0 / 6 : 2) / kBytesPerUs;
  // the operands once, at the rate at which they arrive
  const double arrive = (double)(m * steps1 * 32 + cols * steps1 * 32) * (planes == 3 ? 4 : 2) / kBytesPerUs;
  // (the kernel for any operand loads 16 bytes at a time: operands that have not so many are copied too.  B may be up to 7 rows or K short of n and k.
  // Of logits one row of B has to be enough, so that the last piece of a vocabulary goes the way of all others, however narrow it is)
  const bool any = sh.logits ? k >= 8 : m * k >= 8 && std::max<int64_t>(n - 7, 1) * std::max<int64_t>(k - 7, 1) >= 8;
  Choice best{RING_128, 0, 1, !direct, 0};
  double best_cost = 1e300;
  auto can = [&](int t) {
    if (t > (direct ? RING_64 : ANY_32)) return false;
    const bool ring = t <= RING_64;
    if ((sh.a_columns && t == RING_64) || (planes == 3 && t == RING_256) || (!ring && !any)) return false;
    // logits have the bits of one order of sums in both passes (see LogitsPlan), and those of few rows are summed in two levels
    if (plan && !direct && any && ring == plan->in_place) return false;
    return !(sh.logits && t == RING_256 && m <= FEW_ROWS);
  };
  for (int t = RING_256; t < TILES; ++t) {
    if (!can(t) || (forced_tile >= 0 && forced_tile < TILES && forced_tile != t && can(forced_tile))) continue;
    const bool ring = t <= RING_64;
    const size_t room = ring ? copies : 0;
    if (room > workspace) continue;
    const int64_t steps = steps1;
    const int64_t tiles = (m + kTiles[t].bm - 1) / kTiles[t].bm * ((cols + kTiles[t].bn - 1) / kTiles[t].bn) * pair;
    const Cost& c = (dtype == CMOE_F32 ? kFp32 : kBf16)[t];
    const int64_t slots = (int64_t)CUS * c.per_cu, whole = tiles / slots * slots;
    for (int split = 1; split <= 32; ++split) {
      // (of logits either all tiles are split or none: which are last differs between the passes)
      const int64_t full = sh.logits && split > 1 ? 0 : whole, rest = tiles - full;
      if (plan && split != plan->k_split) continue;
      const size_t slab = split > 1 ? (size_t)rest * split * kTiles[t].bm * kTiles[t].bn * 4 : 0;
      if (split > 1 && (rest == 0 || room + slab > workspace)) break;
      if (split > 1 && !plan && forced_split < 1 && (steps / split < 6 || rest * (split - 1) >= slots)) break;
      if (!plan && forced_split >= 1 && split != forced_split && rest > 0) continue;
      const double part = (double)((steps + split - 1) / split);
      auto round = [&](double steps_of, int64_t on_a_cu) { return steps_of * std::max(c.alone, c.share * on_a_cu) + c.ends; };
      double cost = kLaunch + (double)(full / slots) * round((double)steps, c.per_cu);
      const int64_t parts = rest * split;
      cost += (double)(parts / slots) * round(part, c.per_cu) + (parts % slots ? round(part, (parts % slots + CUS - 1) / CUS) : 0);
      cost = std::max(cost, kLaunch + arrive);
      if (ring) cost += copy_time;
      if (split > 1) cost += kLaunch + (double)slab * 2 / kBytesPerUs;
      if (cost < best_cost) best_cost = cost, best = {(Tile)t, split > 1 ? (int)full : (int)(tiles / 8 * 8), split, ring && !direct, slab};
    }
  }
  return best;
}

// The same, remembered by a thread for the questions it has asked lately: a call asks each product's two or three times, for sizes and then to
// run it, and programs make the same calls over and over (1 us each to weigh, 5 in a backward pass of a few tokens).
Choice choose(Product kind, int dtype, bool direct, bool second, int64_t m, int64_t n, int64_t k, size_t workspace, const LogitsPlan* plan = nullptr) {
  struct Asked {
    int64_t m, n, k;
    size_t workspace;
    int how, tile, split, plan;
    bool operator==(const Asked& o) const {
      return m == o.m && n == o.n && k == o.k && workspace == o.workspace && how == o.how && tile == o.tile && split == o.split && plan == o.plan;
    }
  };
  constexpr int KEPT = 64;
  thread_local Asked asked[KEPT] = {};       // (m = 0 is never asked)
  thread_local Choice said[KEPT];
  const Asked q = {m, n, k, workspace, (kind << 3) | (dtype << 2) | (direct << 1) | (int)second, tuning().mat_tile, tuning().mat_split,
                   plan ? plan->k_split * 2 + plan->in_place : -1};
  uint64_t h = (uint64_t)m * 0x9E3779B97F4A7C15u + (uint64_t)n * 0xC2B2AE3D27D4EB4Fu + (uint64_t)k * 0x165667B19E3779F9u + (uint64_t)workspace * 0x27D4EB2F165667C5u +
               (uint64_t)(q.how * 64 + q.plan) * 0x85EBCA77C2B2AE63u;
  const int at = (int)((h ^ h >> 29) >> 20 & (KEPT - 1));
  if (!(asked[at] == q)) {
    said[at] = weigh(kind, dtype, direct, second, m, n, k, workspace, plan);
    asked[at] = q;
  }
  return said[at];
}

int64_t ranges_of(const Choice& c, int64_t n) { return (n + kTiles[c.tile].bn - 1) / kTiles[c.tile].bn * kTiles[c.tile].wgn; }

constexpr size_t EVERYTHING = (size_t)1 << 60;

bool has_second(Product kind) { return kind == PRODUCT_GATED || kind == PRODUCT_DX; }

template <typename T>
hipError_t prepare(const CopyArgs& args, uint32_t groups, hipStream_t s) {
  hipLaunchKernelGGL(matmul_prepare<T>, dim3(groups), dim3(256), 0, s, args);
  return hipGetLastError();
}

}  // namespace

LogitsPlan logits_plan(int dtype, int64_t m, int64_t n, int64_t k) {
  const Choice other = choose(PRODUCT_LSE, dtype, false, false, m, n, k, EVERYTHING);
  return {!other.copies, dtype == CMOE_BF16 && k % 8 == 0 ? choose(PRODUCT_LSE, dtype, true, false, m, n, k, EVERYTHING).k_split : other.k_split};
}

int64_t lse_ranges(int dtype, int64_t m, int64_t n, int64_t k, const LogitsPlan& plan) {
  int64_t most = 0;
  for (int direct = 0; direct <= (dtype == CMOE_BF16); ++direct) most = std::max(most, ranges_of(choose(PRODUCT_LSE, dtype, direct, false, m, n, k, EVERYTHING, &plan), n));
  return most;
}

size_t matmul_workspace_bytes(Product kind, int dtype, int64_t m, int64_t n, int64_t k, const LogitsPlan* plan) {
  if (m <= 0 || n <= 0) return 0;
  const Shape sh = shape_of(kind);
  size_t most = 0;
  for (int direct = 0; direct <= (dtype == CMOE_BF16); ++direct)
    for (int second = has_second(kind); second <= (has_second(kind) || kind == PRODUCT_DW); ++second) {
      const Choice c = choose(kind, dtype, direct, second, m, n, k, EVERYTHING, plan);
      most = std::max(most, (c.copies ? copy_bytes(sh, dtype == CMOE_F32 ? 3 : 1, m, n, k, second) : 0) + c.slab);
    }
  return (most + 15) / 16 * 16;
}

hipError_t matmul(Product kind, int dtype, MatArgs p, void* workspace, size_t workspace_bytes, hipStream_t s, int* ranges) {
  if (p.m <= 0 || p.n <= 0) return hipSuccess;
  if (!p.m_a) p.m_a = p.m;
  if (!p.n_b) p.n_b = p.n;
  if (!p.k_b) p.k_b = p.k;
  const Shape sh = shape_of(kind);
  const bool second = has_second(kind) || (kind == PRODUCT_DW && p.c2);
  auto wide = [](const void* q) { return ((uintptr_t)q & 15) == 0; };
  const bool direct = dtype == CMOE_BF16 && wide(p.a) && wide(p.a2) && wide(p.b) && wide(p.b2) && p.lda % 8 == 0 && p.ldb % 8 == 0 &&
                      (sh.a_columns ? p.m_a : p.k) % 8 == 0 && (sh.b_columns ? p.n_b : p.k) % 8 == 0;
  const Choice c = choose(kind, dtype, direct, second, p.m, p.n, p.k, workspace ? workspace_bytes : 0,
                          sh.logits ? &p.logits : nullptr);
  p.zs = kind == PRODUCT_DW && second ? 2 : 1;
  p.full = c.full, p.k_split = c.k_split, p.bm = kTiles[c.tile].bm, p.bn = kTiles[c.tile].bn;
  char* room = static_cast<char*>(workspace);
  if (c.copies) {
    const int planes = dtype == CMOE_F32 ? 3 : 1;
    CopyArgs args = {};
    uint32_t groups = 0;
    auto copy = [&](const void* from, int64_t ld, int64_t rows, int cols) {
      Copied& op = args.op[args.n++];
      op.from = from, op.to = reinterpret_cast<bf16_t*>(room), op.ld = ld, op.rows = rows, op.cols = cols, op.pitch = (int)round8(cols), op.first = groups;
      groups += (uint32_t)((rows * (op.pitch / 8) + 255) / 256);
      room += (size_t)rows * op.pitch * planes * 2;
      return op.to;
    };
    const int64_t a_rows = sh.a_columns ? p.k : p.m, b_rows = sh.b_columns ? p.k_b : p.n_b;
    const int a_cols = sh.a_columns ? p.m : p.k, b_cols = sh.b_columns ? p.n_b : p.k_b;
    p.a = copy(p.a, p.lda, a_rows, a_cols);
    if (sh.segments) p.a2 = copy(p.a2, p.lda, a_rows, a_cols);
    p.b = copy(p.b, p.ldb, b_rows, b_cols);
    if (second) p.b2 = copy(p.b2, p.ldb, b_rows, b_cols);
    p.lda = round8(a_cols), p.ldb = round8(b_cols);
    p.a_plane = a_rows * p.lda, p.b_plane = b_rows * p.ldb;
    // the zeros behind the columns are read
    if (sh.a_columns) p.m_a = (int)p.lda;
    else p.k = (int)p.lda;
    if (sh.b_columns) p.n_b = (int)p.ldb;
    else p.k_b = (int)p.ldb;
    if (groups)
      if (hipError_t e = dtype == CMOE_F32 ? prepare<float>(args, groups, s) : prepare<bf16_t>(args, groups, s)) return e;
    room = static_cast<char*>(workspace) + (room - static_cast<char*>(workspace) + 255) / 256 * 256;
  }
  if (c.k_split > 1) p.slab = reinterpret_cast<float*>(room);
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
