// The requests of a step as the kernels over a paged cache see them, and the rotation of a pair.
#pragma once

#include "focus_attn.h"
#include "focus_common.h"
#include "focus_kernels.h"

namespace focus {

// Rows first .. first + n - 1 of the tensors are those of a request that are worked on; `count` is what row_start says.
struct RequestRows {
  int first, n, count;
};
__device__ __forceinline__ RequestRows clip_rows(const PagedBatch& b, int start, int end) {
  RequestRows q;
  q.first = min(max(start, 0), b.n_rows);
  q.count = max(min(end, b.n_rows) - q.first, 0);
  q.n = min(q.count, b.max_rows);
  return q;
}
// r: the same in all lanes
__device__ __forceinline__ RequestRows request_rows(const PagedBatch& b, int r) {
  if (b.row_start == nullptr) return clip_rows(b, r, r + 1);
  return clip_rows(b, uniform_load(b.row_start + r), uniform_load(b.row_start + r + 1));
}

// cos and sin in 64 bits.  angle = n pi/2 + r, |r| <= pi/4, with pi/2 in two parts whose first product is exact within the fused
// multiply-add, then Taylor's series to r^17 and r^16, whose rests at pi/4 are below 2^-56: some thirty operations.  32 bits are what is
// asked for, but of angles of 10^6 radians and more.
__device__ __forceinline__ void cos_sin(double angle, double& cosine, double& sine) {
  const double n = __builtin_rint(angle * 0.63661977236758134308);
  const double r = __builtin_fma(-n, 6.1232339957367658e-17, __builtin_fma(-n, 1.5707963267948966, angle)), z = r * r;
  const double s8[8] = {-1.0 / 6.0, 1.0 / 120.0, -1.0 / 5040.0, 1.0 / 362880.0, -1.0 / 39916800.0, 1.0 / 6227020800.0, -1.0 / 1307674368000.0,
                        1.0 / 355687428096000.0};
  const double c8[8] = {-1.0 / 2.0, 1.0 / 24.0, -1.0 / 720.0, 1.0 / 40320.0, -1.0 / 3628800.0, 1.0 / 479001600.0, -1.0 / 87178291200.0,
                        1.0 / 20922789888000.0};
  double s = s8[7], c = c8[7];
#pragma unroll
  for (int i = 6; i >= 0; --i) {
    s = __builtin_fma(s, z, s8[i]);
    c = __builtin_fma(c, z, c8[i]);
  }
  s = __builtin_fma(s * z, r, r);
  c = __builtin_fma(c, z, 1.0);
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  cosine = (quarter & 1) ? s : c;
  sine = (quarter & 1) ? c : s;
  if (quarter == 1 || quarter == 2) cosine = -cosine;
  if (quarter >= 2) sine = -sine;
}

}  // namespace focus
