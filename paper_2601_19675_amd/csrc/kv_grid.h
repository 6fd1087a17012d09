// The grid of a row of the cache and the codes on it, as ptq_kv_cache_write defines them: what the kernels that write
// the cache share.  Not part of the C ABI.
#pragma once
#include "kv_cache.h"
#include "stored_rows.h"

namespace ptq {

// the largest over the LANES lanes of a row
template <int LANES, class T>
__device__ __forceinline__ T row_max(T v) {
  v = max(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, kDppSwapPairs, 0xf, 0xf, true));
  v = max(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, kDppSwapHalfQuads, 0xf, 0xf, true));
  if constexpr (LANES >= 8) v = max(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, kDppHalfMirror, 0xf, 0xf, true));
  if constexpr (LANES >= 16) v = max(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, kDppMirror, 0xf, 0xf, true));
  if constexpr (LANES >= 32) v = max(v, (T)__shfl_xor((int)v, 16));
  return v;
}

// what lane I of every four lanes has
template <int I>
__device__ __forceinline__ float of_four(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x55 * I, 0xf, 0xf, true));
}

// the quotient of d by a small whole number, correctly rounded: r = d - q by is exact, its share is added once
__device__ __forceinline__ double divided(double d, double by, double inv) {
  const double q = d * inv;
  return fma(fma(-q, by, d), inv, q);
}

// Bits tell a row's extremes, and whether all of it is finite: as signed numbers those of the largest value come last, as
// unsigned ones those of the value furthest below 0, if one is.
struct RowExtremes {
  int hi = 0;
  uint32_t lo = 0;
  __device__ __forceinline__ void take(float v) {
    hi = max(hi, __float_as_int(v));
    lo = max(lo, __float_as_uint(v));
  }
};

struct RowGrid {
  float scale, zero;
  float inv;      // 1 / scale, or 0 for a row that is not finite
  bool finite;
  bool odd;       // of any row of the wave: codes go by the quotient
};
template <int BITS>
__device__ __forceinline__ RowGrid row_grid(const RowExtremes& e) {
  constexpr double kTop = (1 << BITS) - 1;
  // a row with an infinity or a NaN: its scale becomes NaN, and so does whatever reads it; its codes 0 (x inv is NaN or 0)
  const bool finite = e.hi < 0x7f800000 && e.lo < 0xff800000u;
  const float hi = __int_as_float(e.hi);
  float lo = e.lo > 0x80000000u ? __uint_as_float(e.lo) : 0.f;
  float scale = finite ? (float)divided((double)hi - (double)lo, kTop, 1.0 / kTop) : 1.f;
  if (scale == 0.f) {   // nothing but zeros (or less than float32 can divide)
    lo = -1.f;
    scale = (float)(2.0 / kTop);
  }
  const float below[1] = {finite ? -lo : 0.f};
  float inv = __builtin_amdgcn_rcpf(scale), z[1];
  whole_codes<1>(below, inv, 1.f, scale, z);
  // both ends rounded away from 0 (the only codes past the grid), or no float32 reciprocal: by the quotient, and clamped
  const bool odd = __any((scale < 0x1p-110f) | (scale > 0x1p110f) | (finite && rintf(hi * inv) + z[0] > (float)kTop));
  return RowGrid{scale, z[0], finite ? inv : 0.f, finite, odd};
}

// Codes of N values of the row whose grid lane I of every four lanes has: the low bits of u.
template <int BITS, int I, int N>
__device__ __forceinline__ void row_codes_of(const float (&v)[N], const RowGrid& g, uint32_t (&code)[N]) {
  constexpr double kTop = (1 << BITS) - 1;
  const float inv_i = of_four<I>(g.inv), z_i = of_four<I>(g.zero);
  // 1.5 2^23 + a whole number has that number in its low bits, and adding it rounds there: code = rne(x inv + zero), which is rne(x / scale) + zero
  // as long as x inv + zero, off by less than 2^-14 (see whole_codes; the sum adds 2^-17), is not that close to a middle
  constexpr float kWhole = 12582912.f;
  const float from = z_i + kWhole;
  float u[N], far = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    u[e] = fmaf(v[e], inv_i, from);
    far = fmaxf(far, fabsf(fmaf(v[e], inv_i, from - u[e])));
  }
  if (__any(far > 0.5f - 0x1p-14f) | g.odd) {
    const float s = of_four<I>(g.scale), good = of_four<I>(g.finite ? 1.f : 0.f);
#pragma unroll
    for (int e = 0; e < N; ++e)
      u[e] = kWhole + (good != 0.f ? fminf((float)rint((double)v[e] / (double)s) + z_i, (float)kTop) : 0.f);
  }
#pragma unroll
  for (int e = 0; e < N; ++e) code[e] = __float_as_uint(u[e]);
}
// the low bytes of four numbers
__device__ __forceinline__ uint32_t byte_pair(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x0c0c0400u); }
__device__ __forceinline__ uint32_t four_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_amdgcn_perm(byte_pair(c, d), byte_pair(a, b), 0x05040100u);
}

}  // namespace ptq
