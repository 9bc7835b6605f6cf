// train.hpp -- host helpers shared by the training operators' entry points.
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "gemm_nt.hpp"
#include "ppk1.hpp"

namespace pp {

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t pad64(int64_t n) { return cdiv(n, 64) * 64; }
inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

inline pp_status launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? PP_OK : fail(PP_EHIP, std::string("launch: ") + hipGetErrorString(e));
}

inline GemmOperand operand(const void* base, int64_t plane_elems, int64_t ld, int64_t rows, int planes) {
  GemmOperand o;
  for (int q = 0; q < kMaxPlanes; ++q)
    o.plane[q] = static_cast<const uint8_t*>(base) + (q < planes ? q : 0) * plane_elems * 2;
  o.ld = ld;
  o.rows = static_cast<int32_t>(rows);
  return o;
}
inline GemmOperand rows_from(GemmOperand o, int64_t r0, int64_t rows) {
  for (auto& p : o.plane) p = static_cast<const uint8_t*>(p) + r0 * o.ld * 2;
  o.rows = static_cast<int32_t>(rows);
  return o;
}

}  // namespace pp
