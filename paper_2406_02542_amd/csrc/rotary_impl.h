// What the kernels that turn heads by their positions share (rotary.hip, append.hip).
#pragma once

#include "common.h"

namespace loki {

// cos and sin of x quarter turns, |x| reduced here; fp32 results.  Taylor polynomials on [-pi/4, pi/4]: the first
// term left out is below 2^-29.
__device__ __forceinline__ float2 cos_sin_quarters(double x) {
  const double k = rint(x);
  const float th = (float)(x - k) * 1.57079632679489662f, t2 = th * th;
  float s = fmaf(t2, 2.7557319224e-6f, -1.9841269841e-4f);
  s = fmaf(s, t2, 8.3333333333e-3f);
  s = fmaf(s, t2, -1.6666666667e-1f);
  s = fmaf(s * t2, th, th);
  float c = fmaf(t2, -2.7557319224e-7f, 2.4801587302e-5f);
  c = fmaf(c, t2, -1.3888888889e-3f);
  c = fmaf(c, t2, 4.1666666667e-2f);
  c = fmaf(c, t2, -0.5f);
  c = fmaf(c, t2, 1.0f);
  const int quarter = (int)((long long)k & 3);
  const float cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
  return make_float2(quarter == 1 || quarter == 2 ? -cs : cs, quarter >= 2 ? -sn : sn);
}

template <typename T>
__device__ __forceinline__ uint4 pack_chunk(const float (&f)[T::EPC]) {
  if constexpr (T::EPC == 8)
    return make_uint4(BF16::round2(f[0], f[1]), BF16::round2(f[2], f[3]), BF16::round2(f[4], f[5]), BF16::round2(f[6], f[7]));
  else
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

}  // namespace loki
