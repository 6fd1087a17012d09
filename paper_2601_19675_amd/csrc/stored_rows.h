// Rows of bfloat16 or float32 as the token kernels read and write them, and the rounding to whole codes they share.
// Not part of the C ABI.
#pragma once
#include "common.h"

namespace ptq {

__device__ __forceinline__ uint16_t f32_to_bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// the value that is stored for f, as float32
template <int DT>
__device__ __forceinline__ float as_stored(float f) {
  if constexpr (DT == PTQ_BF16) return (float)(__bf16)f;
  else return f;
}

// N consecutive elements that lie on element boundaries only: the device's loads and stores of up to 16 bytes take any
// address, and rows of odd length would otherwise go element by element.  Kept as whole words (bfloat16: two elements
// each).
template <int DT, int N>
struct Run {
  static constexpr int kWords = DT == PTQ_BF16 ? N / 2 : N;
  uint32_t w[kWords];
};
template <int WORDS, int ALIGN>
struct __attribute__((packed, aligned(ALIGN))) AnyWords {
  uint32_t w[WORDS];
};

// Elements [c, c + N) of a row of n, those past its end zero; widened by run_to_f32 once it is needed, so that several
// runs can be on their way together.  No branch around the load, behind which the compiler would wait for it: a lane
// past the end reads the row's first elements instead.  ODD: n may end inside a run, which is then put together from
// elements by the one lane that has it (and in rows of fewer than N elements).
template <int DT, int N, bool ODD>
__device__ __forceinline__ Run<DT, N> load_run(const void* row, int c, int n) {
  using ST = typename StoredType<DT>::type;
  constexpr int W = Run<DT, N>::kWords;
  const ST* q = static_cast<const ST*>(row);
  const bool whole = c + N <= n;
  Run<DT, N> r;
  if (!ODD || n >= N) {
    const AnyWords<W, sizeof(ST)> a = *reinterpret_cast<const AnyWords<W, sizeof(ST)>*>(q + (whole ? c : 0));
#pragma unroll
    for (int i = 0; i < W; ++i) r.w[i] = a.w[i];
  }
  if (ODD && !whole && c < n) {
#pragma unroll
    for (int i = 0; i < W; ++i) r.w[i] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < n) {
        if constexpr (DT == PTQ_BF16) r.w[i >> 1] |= (uint32_t)q[c + i] << (16 * (i & 1));
        else r.w[i] = __float_as_uint(q[c + i]);
      }
  }
  return r;
}
template <int DT, int N>
__device__ __forceinline__ void run_to_f32(const Run<DT, N>& r, int c, int n, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint32_t b;
    if constexpr (DT == PTQ_BF16) b = i & 1 ? r.w[i >> 1] & 0xffff0000u : r.w[i >> 1] << 16;
    else b = r.w[i];
    v[i] = __uint_as_float(c < n ? b : 0);
  }
}

template <int DT, int N, bool ODD>
__device__ __forceinline__ void store_run(void* row, int c, int n, const float (&v)[N]) {
  using ST = typename StoredType<DT>::type;
  constexpr int W = Run<DT, N>::kWords;
  ST* q = static_cast<ST*>(row) + c;
  if (c + N <= n) {
    AnyWords<W, sizeof(ST)> a;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (DT == PTQ_BF16) a.w[i] = (uint32_t)f32_to_bf16_bits(v[2 * i]) | ((uint32_t)f32_to_bf16_bits(v[2 * i + 1]) << 16);
      else a.w[i] = __float_as_uint(v[i]);
    }
    *reinterpret_cast<AnyWords<W, sizeof(ST)>*>(q) = a;
  } else if (ODD) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (c + i < n) {
        if constexpr (DT == PTQ_BF16) q[i] = f32_to_bf16_bits(v[i]);
        else q[i] = v[i];
      }
  }
}

// rne(times x / over) for N values, |result| <= 255.  inv is times / over to 1.5 * 2^-23 of itself (a reciprocal to the last bit and a
// rounding), so v = x inv is off by no more than 2^-22 |v| < 2^-14: only where v is that close to the middle of two codes does the
// quotient decide, in float64.  times x is exact there, and a quotient of two numbers of so few bits that is not a middle lies
// further from it than a float64 rounds.  (One value in 8000 needs it; the quotient for every value was two thirds of the work.)
// Where `over` is so small or large that it has no normal reciprocal, every value takes the quotient.  x and c are different arrays.
template <int N>
__device__ __forceinline__ void whole_codes(const float (&x)[N], float inv, float times, float over, float (&c)[N]) {
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float v = x[i] * inv;
    c[i] = rintf(v);
    far = fmaxf(far, fabsf(v - c[i]));
  }
  if (__any((far > 0.5f - 0x1p-14f) | (over < 0x1p-110f) | (over > 0x1p110f))) {   // (the wave's: or it would be computed for all)
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = (float)rint((double)times * (double)x[i] / (double)over);
  }
}

}  // namespace ptq
