// train.hpp -- host helpers shared by the training operators' entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "gemm_tile.hpp"
#include "ppk1.hpp"

namespace pp {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t pad64(int64_t n) { return cdiv(n, 64) * 64; }
inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// An entry point's body: no exception leaves it.
template <class F>
inline pp_status guarded(F&& f) {
  clear_error();
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(PP_EINVAL, std::string("out of host memory: ") + e.what());
  }
}

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

// The tiles of the products, and when each is used.  Measured on MI355X, us a
// step of 64 k with every CU full / alone on its CU, and us at either end of a
// tile; with one plane an operand, with two (three products), with three (six):
//   256 x 256 phased            1.6 / 1.15   6     4.8 / 3.45    6     9.6 / 6.9   6
//   192 x 192                   1.13 / 0.95  5     -                   -
//   128 x 128                   0.52 / 0.58  3.5   1.37 / 1.16   4.5   -
//   128 x 64                    -                  -                   1.5 / 1.25  2.5
//   64 x 64                     0.19 / 0.27  2.5   0.41 / 0.62   2.8   1.03 / 0.92 2
//   64 x 64, two groups of
//     waves share the steps     0.23 / 0.19  4     0.55 / 0.5    4     -
//   32 x 32, a wave's own steps 0.1 / 0.12   2.8   0.27 / 0.25   2.8   0.46 / 0.43 2.8
// (192 x 192: one plane, operands that are not stored by rows of k; for a
// triangle of tiles, which the large ones cover badly: 4096 x 4096 has 136 large
// ones, in a whole round with 120 CUs idle, and 253 of these.)
// The large tile wins wherever it fills the card (one plane, 8192^3: 1310
// TFLOP/s; 128 x 128 1040, 64 x 64 720), the small ones where it would leave CUs
// without work (512 x 512, k 4608: 80, 42, 20, 17 and 11 us).  All but the
// largest bring all planes of a step together: half the traffic and one barrier
// for three or six products, but as much LDS as there are planes.  512 x 512, k
// 4608, three products: 64 x 64 tiles 49 us, 32 x 32 21; one after the other 65
// and 39.  2048^3, six products: 128 x 64 98 us, 64 x 64 135; 128 x 128, one
// after the other, 145.  Operands stored by rows of k cost 5 to 10 % each.
enum { kBig = 0, kMid = 1, kSmall = 2, kDeep = 3, kNarrow = 4, kFit = 5, kTiles = 6 };
template <class T, bool AR, bool BR, int NP>
struct Tiles {
  using Big = GemmTile<T, 256, 256, 2, 4, 2, 1, true, AR, BR>;
  using Mid = std::conditional_t<NP == 2, GemmTile<T, 128, 128, 2, 4, 2, 1, false, AR, BR, 2>,
                                 std::conditional_t<NP == 3, GemmTile<T, 128, 64, 4, 2, 2, 1, false, AR, BR, 3>,
                                                    GemmTile<T, 128, 128, 2, 2, 2, 1, false, AR, BR>>>;
  using Small = GemmTile<T, 64, 64, 2, 2, NP == 1 ? 4 : 2, 1, false, AR, BR, NP>;
  using Deep = GemmTile<T, 64, 64, 2, 2, NP == 1 ? 4 : 2, 2, false, AR, BR, NP == 3 ? 1 : NP>;
  using Narrow = GemmTile<T, 32, 32, 1, 1, 2, NP == 3 ? 3 : 4, false, AR, BR, NP>;
};
// rows and columns of a tile, and its waves' parts of them
constexpr int tile_m(int, int k) { return k == kBig ? 256 : k == kFit ? 192 : k == kMid ? 128 : k == kNarrow ? 32 : 64; }
constexpr int tile_n(int np, int k) { return k == kMid && np == 3 ? 64 : tile_m(np, k); }
constexpr int tile_wm(int np, int k) { return k == kMid && np == 3 ? 4 : k == kNarrow ? 1 : 2; }
constexpr int tile_wn(int np, int k) { return k == kBig || k == kFit || (k == kMid && np == 2) ? 4 : k == kNarrow ? 1 : 2; }
constexpr int kCUs = 256;

// f(tile's type) for tile k; AR, BR: operands stored by rows of k; NP: planes;
// FIT: k may be kFit
template <class T, bool AR, bool BR, int NP, bool FIT = false, class F>
void with_tile(int k, F&& f) {
  using X = Tiles<T, AR, BR, NP>;
  if (k == kBig)
    f(typename X::Big());
  else if (k == kFit) {
    if constexpr (FIT) f(GemmTile<T, 192, 192, 2, 4, 2, 1>());
  } else if (k == kMid)
    f(typename X::Mid());
  else if (k == kSmall)
    f(typename X::Small());
  else if constexpr (NP < 3) {
    if (k == kDeep)
      f(typename X::Deep());
    else
      f(typename X::Narrow());
  } else
    f(typename X::Narrow());
}

// Modelled time in us of `tiles` tiles of `steps` k steps on average, `most` at
// most, with np planes an operand.
inline double tile_time(int np, int tile, double tiles, double steps, double most) {
  constexpr double full[3][kTiles] = {{1.6, 0.52, 0.19, 0.23, 0.1, 1.13}, {4.8, 1.37, 0.41, 0.55, 0.27, 1e9}, {9.6, 1.5, 1.03, 1e9, 0.46, 1e9}};
  constexpr double alone[3][kTiles] = {{1.15, 0.58, 0.27, 0.19, 0.12, 0.95}, {3.45, 1.16, 0.62, 0.5, 0.25, 1e9}, {6.9, 1.25, 0.92, 1e9, 0.43, 1e9}};
  constexpr double ends[3][kTiles] = {{6., 3.5, 2.5, 4., 2.8, 5.}, {6., 4.5, 2.8, 4., 2.8, 0.}, {6., 2.5, 2., 0., 2.8, 0.}};
  constexpr bool single[3][kTiles] = {{true, false, false, true, false, true}, {true, true, false, true, true, true}, {true, true, true, true, true, true}};
  const int q = np - 1;   // (single: one workgroup a CU)
  const double n = static_cast<double>(cdiv(static_cast<int64_t>(tiles), kCUs));
  // (a card in part idle clocks higher and shares its caches among fewer)
  const double step = alone[q][tile] + (std::max(full[q][tile], alone[q][tile]) - alone[q][tile]) * std::min(1., tiles / kCUs);
  return std::max(most * step, n > 1 ? n * steps * full[q][tile] : 0.) + ends[q][tile] * (single[q][tile] ? n : 0.5 + 0.5 * n);
}

inline int pick_tile(int np, int64_t m, int64_t n, int64_t steps) {
  int best = kSmall;
  double least = 1e300;
  for (int k = 0; k < kFit; ++k) {
    const double t = tile_time(np, k, static_cast<double>(cdiv(m, tile_m(np, k)) * cdiv(n, tile_n(np, k))), steps, steps);
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
inline SplitTile pick_split(int np, int64_t m, int64_t n, int64_t steps, double* time = nullptr) {
  SplitTile best = {kSmall, 1};
  double least = 1e300;
  for (int k = 0; k < kFit; ++k)
    for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (s > 1 && (steps / s < (np > 1 ? 2 : 4) || static_cast<double>(s) * m * n * 4 > 256e6)) break;
      const double per = static_cast<double>(cdiv(steps, s));
      double t = tile_time(np, k, static_cast<double>(cdiv(m, tile_m(np, k)) * cdiv(n, tile_n(np, k)) * s), per, per);
      if (s > 1) t += 4. + s * static_cast<double>(m) * n * 8e-6 / 3.;
      if (t < least) least = t, best = {k, s};
    }
  if (time) *time = least;
  return best;
}

}  // namespace pp
