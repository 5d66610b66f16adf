// Launches of the products' kernels (host code); one translation unit per group of products instantiates them.
#pragma once
#include "lds_limit.h"
#include "matmul_device.h"

namespace cmoe {

// The ring's tiles and those of the kernel for any operand: rows, columns, columns of waves (the columns of a wave are a range of PRODUCT_LSE).
enum Tile { RING_256, RING_128, RING_64, ANY_64, ANY_32, TILES };
struct TileShape {
  int bm, bn, wgn;
};
constexpr TileShape kTiles[TILES] = {{256, 256, 2}, {128, 128, 2}, {64, 128, 2}, {64, 64, 2}, {32, 128, 4}};

template <class KERNEL>
hipError_t launch_tiles(KERNEL kernel, LdsLimit& limit, size_t lds, const MatArgs& p, int bno, hipStream_t s) {
  if (lds > 64 * 1024)
    if (hipError_t e = limit.raise(reinterpret_cast<const void*>(kernel), lds)) return e;
  const int64_t tiles = ((int64_t)p.m + p.bm - 1) / p.bm * (((int64_t)p.n + bno - 1) / bno) * p.zs;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(p.full + ((tiles - p.full) * p.k_split + 7) / 8 * 8)), dim3(256), lds, s, p);
  return hipGetLastError();
}

template <int BM, int BN, int STAGES, bool ACOL, bool BCOL, class EPI>
hipError_t launch_mat_ring(const MatArgs& p, hipStream_t s) {
  static LdsLimit limit;
  return launch_tiles(matmul_ring<BM, BN, STAGES, 2, 2, ACOL, BCOL, EPI>, limit, mat_ring_bytes<BM, BN, STAGES, 2, 2, EPI>(), p, EPI::DUAL ? BN / 2 : BN, s);
}
template <int BM, int BN, int WGM, int WGN, bool ACOL, bool BCOL, class EPI>
hipError_t launch_mat_any(const MatArgs& p, hipStream_t s) {
  static LdsLimit limit;
  return launch_tiles(matmul_any<BM, BN, WGM, WGN, ACOL, BCOL, EPI>, limit, mat_any_bytes<typename EPI::type, BM, BN, WGM, WGN, ACOL, BCOL>(), p, EPI::DUAL ? BN / 2 : BN, s);
}

template <bool ACOL, bool BCOL, class EPI>
hipError_t launch_product(Tile tile, const MatArgs& p, hipStream_t s) {
  hipError_t e = hipErrorInvalidValue;
  constexpr bool PLANES = planes_of<EPI>() > 1;
  if constexpr (!PLANES) {
    if (tile == RING_256) e = launch_mat_ring<256, 256, 5, ACOL, BCOL, EPI>(p, s);
  }
  if (tile == RING_128) e = launch_mat_ring<128, 128, PLANES ? 3 : 5, ACOL, BCOL, EPI>(p, s);
  if constexpr (!ACOL) {
    if (tile == RING_64) e = launch_mat_ring<64, 128, PLANES ? 4 : 6, ACOL, BCOL, EPI>(p, s);
  }
  if (tile == ANY_64) e = launch_mat_any<64, 64, 2, 2, ACOL, BCOL, EPI>(p, s);
  if (tile == ANY_32) e = launch_mat_any<32, 128, 1, 4, ACOL, BCOL, EPI>(p, s);
  if (e != hipSuccess || p.k_split == 1) return e;
  const int bno = EPI::DUAL ? p.bn / 2 : p.bn;
  const int64_t tiles = ((int64_t)p.m + p.bm - 1) / p.bm * (((int64_t)p.n + bno - 1) / bno) * p.zs;
  const unsigned split = (unsigned)(tiles - p.full);
  if constexpr (EPI::RANGES)
    hipLaunchKernelGGL(matmul_finish_ranges<typename EPI::type>, dim3(split, p.bm / 4), dim3(256), 0, s, p, kTiles[tile].wgn);
  else
    hipLaunchKernelGGL(matmul_finish<EPI>, dim3(split, (p.bm * bno / 8 + 255) / 256), dim3(256), 0, s, p);
  return hipGetLastError();
}

// By product and type; each in the translation unit of its group.
hipError_t launch_gated(Tile, int dtype, const MatArgs&, hipStream_t);
hipError_t launch_dgated(Tile, int dtype, const MatArgs&, hipStream_t);
hipError_t launch_down(Tile, int dtype, const MatArgs&, hipStream_t);
hipError_t launch_dx(Tile, int dtype, const MatArgs&, hipStream_t);
hipError_t launch_dw(Tile, int dtype, const MatArgs&, hipStream_t);
hipError_t launch_lse(Tile, int dtype, const MatArgs&, hipStream_t);
hipError_t launch_dlogits(Tile, int dtype, const MatArgs&, hipStream_t);
hipError_t launch_dhead(Tile, int dtype, const MatArgs&, hipStream_t);

}  // namespace cmoe
