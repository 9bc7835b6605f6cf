// train.hpp -- host helpers shared by the training operators' entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "gemm_tile.hpp"
#include "ppk1.hpp"

namespace pp {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t pad64(int64_t n) { return cdiv(n, 64) * 64; }
inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

inline pp_status launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? PP_OK : fail(PP_EHIP, std::string("launch: ") + hipGetErrorString(e));
}

// `planes` planes of [..][ld], plane_elems elements apart; rows, k as
// GemmOperand has them
inline GemmOperand operand(const void* base, int64_t plane_elems, int64_t ld, int64_t rows, int64_t k, int planes) {
  GemmOperand o;
  for (int q = 0; q < kMaxPlanes; ++q)
    o.plane[q] = static_cast<const uint8_t*>(base) + (q < planes ? q : 0) * plane_elems * 2;
  o.ld = ld;
  o.rows = static_cast<int32_t>(rows);
  o.k = static_cast<int32_t>(k);
  return o;
}

// The tiles of the products, and when each is used.  Measured on MI355X (us a
// step of 64 k, with every CU full / alone on its CU; us at either end of a
// tile):
//   256 x 256 phased                                     1.6 / 1.15      6
//   128 x 128, two workgroups a CU                       0.52 / 0.58     3.5
//   64 x 64, four steps in flight, two a CU              0.19 / 0.27     2.5
//   64 x 64, two groups of waves share the steps         0.23 / 0.19     4
//   32 x 32, four waves share the steps, two a CU        0.1 / 0.12      2.8
// The large tile wins wherever it fills the card (1310 TFLOP/s at 8192^3; the
// others 1040, 720, 630), the small ones where it would leave CUs without work:
// 4096^3 takes 104, 141, 218 and 267 us, 2048^3 43, 27, 28, 35 and 58,
// 1000 x 3008 x 1000 -, 35, 16, 14 and 21, 512 x 4608 x 512 80, 42, 20, 17 and 11,
// 256 x 960 x 256 -, 13, 6.5, 6.1 and 4.5.  Operands stored by rows of k cost 5 to
// 10 % each.
enum { kBig = 0, kMid = 1, kSmall = 2, kDeep = 3, kNarrow = 4, kTiles = 5 };
template <class T, bool AR, bool BR> using BigTile = GemmTile<T, 256, 256, 2, 4, 2, 1, true, AR, BR>;
template <class T, bool AR, bool BR> using MidTile = GemmTile<T, 128, 128, 2, 2, 2, 1, false, AR, BR>;
template <class T, bool AR, bool BR> using SmallTile = GemmTile<T, 64, 64, 2, 2, 4, 1, false, AR, BR>;
template <class T, bool AR, bool BR> using DeepTile = GemmTile<T, 64, 64, 2, 2, 4, 2, false, AR, BR>;
template <class T, bool AR, bool BR> using NarrowTile = GemmTile<T, 32, 32, 1, 1, 2, 4, false, AR, BR>;
constexpr int kTileEdge[kTiles] = {256, 128, 64, 64, 32};
constexpr int kTileWM[kTiles] = {2, 2, 2, 2, 1}, kTileWN[kTiles] = {4, 2, 2, 2, 1};   // waves' parts of a tile
constexpr int kCUs = 256;

// f(tile's type) for tile k; AR, BR: operands stored by rows of k
template <class T, bool AR, bool BR, class F>
void with_tile(int k, F&& f) {
  if (k == kBig)
    f(BigTile<T, AR, BR>());
  else if (k == kMid)
    f(MidTile<T, AR, BR>());
  else if (k == kSmall)
    f(SmallTile<T, AR, BR>());
  else if (k == kDeep)
    f(DeepTile<T, AR, BR>());
  else
    f(NarrowTile<T, AR, BR>());
}

// Modelled time in us of `tiles` tiles of `steps` steps on average, `most` at
// most.
inline double tile_time(int tile, double tiles, double steps, double most) {
  constexpr double full[kTiles] = {1.6, 0.52, 0.19, 0.23, 0.1}, alone[kTiles] = {1.15, 0.58, 0.27, 0.19, 0.12},
                   ends[kTiles] = {6., 3.5, 2.5, 4., 2.8};
  const double n = static_cast<double>(cdiv(static_cast<int64_t>(tiles), kCUs));
  // (a card in part idle clocks higher and shares its caches among fewer)
  const double step = alone[tile] + (std::max(full[tile], alone[tile]) - alone[tile]) * std::min(1., tiles / kCUs);
  const bool single = tile == kBig || tile == kDeep;   // one workgroup a CU
  return std::max(most * step, n > 1 ? n * steps * full[tile] : 0.) + ends[tile] * (single ? n : 0.5 + 0.5 * n);
}

inline int pick_tile(int64_t m, int64_t n, int64_t steps) {
  int best = kSmall;
  double least = 1e300;
  for (int k = 0; k < kTiles; ++k) {
    const double t = tile_time(k, static_cast<double>(cdiv(m, kTileEdge[k]) * cdiv(n, kTileEdge[k])), steps, steps);
    if (t < least) least = t, best = k;
  }
  return best;
}

// The same for a product whose sum over k may be split over workgroups: the
// partial sums are written to and read from memory (at about 3 TB/s) by one
// more launch (about 4 us).
struct SplitTile {
  int tile, splits;
};
inline SplitTile pick_split(int64_t m, int64_t n, int64_t steps, double* time = nullptr) {
  SplitTile best = {kSmall, 1};
  double least = 1e300;
  for (int k = 0; k < kTiles; ++k)
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (s > 1 && (steps / s < 4 || static_cast<double>(s) * m * n * 4 > 256e6)) break;
      const double per = static_cast<double>(cdiv(steps, s));
      double t = tile_time(k, static_cast<double>(cdiv(m, kTileEdge[k]) * cdiv(n, kTileEdge[k]) * s), per, per);
      if (s > 1) t += 4. + s * static_cast<double>(m) * n * 8e-6 / 3.;
      if (t < least) least = t, best = {k, s};
    }
  if (time) *time = least;
  return best;
}

}  // namespace pp
