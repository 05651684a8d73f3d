// Rows grouped by request: the rows of request b in arrays of total_rows rows, from the running sums in row_offsets.
#ifndef MEPIC_ROWS_CUH_
#define MEPIC_ROWS_CUH_

#include <cuda_runtime.h>
#include <stdint.h>

namespace mepic_dev {

// Clamped into [0, total_rows] and to `most` rows; `bad` tells that something had to be clamped.
struct RowRange { int lo, n; bool bad; };
__device__ __forceinline__ RowRange rows_of(const int32_t* row_offsets, int b, int total_rows, int most) {
  const int a = __ldg(row_offsets + b), z = __ldg(row_offsets + b + 1);
  RowRange r;
  r.lo = min(max(a, 0), total_rows);
  const int hi = min(max(z, r.lo), total_rows);
  r.n = min(hi - r.lo, most);
  r.bad = a != r.lo || z != hi || hi - r.lo > most;
  return r;
}

}  // namespace mepic_dev

#endif
