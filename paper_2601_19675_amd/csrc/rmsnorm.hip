// Root-mean-square norm of token rows into 8 bits, with the residual's addition.
//
//   y = round(x + residual)      u = float32(y gamma)      A = max |u|
//   code = rne(127 u / A)        scale = A / 127 / sqrt(mean(y^2) + eps)
//
// A code does not depend on the root mean square, which only scales the row: one pass over the row finds A and the sum of
// squares, the row stays in registers, and the codes follow.  Bound: bytes (3 an element for bfloat16, 7 with the residual's
// way in and out).  A row of up to 2048 elements belongs to a wave, which then needs no barrier (few rows excepted); longer rows to
// a workgroup of 256 threads, beyond 16384 elements of 1024.  The sum of squares is float64: rows of any finite values have
// a finite norm, and the additions hide behind the memory.
//
// 16384 rows of 4096 bfloat16 with the residual's way in and out (470 MB): 80.7 us, 5.8 TB/s; 4096 rows of 11008 float32 (225 MB) 42 us,
// 5.4 TB/s; four rows of 4096 3.6 us, of which the launch is the most.
#include <algorithm>

#include "stored_rows.h"

namespace ptq {
namespace {

struct NormArgs {
  const void* X; const void* R; void* Y; const void* G; int8_t* C; float* S;
  int64_t ldx, ldr, ldy, ldc;
  int t, n;
  double eps;
  int normalize;
};

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
  v += dpp_move<kDppSwapPairs>(v);
  v += dpp_move<kDppSwapHalfQuads>(v);
  v += dpp_move<kDppHalfMirror>(v);
  v += dpp_move<kDppMirror>(v);
  v += __shfl_xor(v, 16);
  v += __shfl_xor(v, 32);
  return v;
}

// PER runs of eight elements a thread, ROW threads to a row
template <int DT, int PER, int ROW, bool ODD>
__global__ __launch_bounds__(ROW < 256 ? 256 : ROW) void rmsnorm_quantize_kernel(NormArgs a) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = ROW == kWave ? blockIdx.x * 4 + wave : blockIdx.x;
  const int at = ROW == kWave ? lane : tid;
  if (ROW == kWave && row >= a.t) return;
  float u[PER][8];
  uint32_t top = 0;   // bits of max |u|: infinities and NaN come last in this order
  double squares = 0.0;
  using ST = typename StoredType<DT>::type;
  const ST* X = static_cast<const ST*>(a.X) + row * a.ldx;
  const ST* R = static_cast<const ST*>(a.R) + row * a.ldr;
  // everything that the row needs is asked for before anything is used
  Run<DT, 8> x[PER], r[PER], g[PER];
#pragma unroll
  for (int p = 0; p < PER; ++p) x[p] = load_run<DT, 8, ODD>(X, (p * ROW + at) * 8, a.n);
  if (a.R) {
#pragma unroll
    for (int p = 0; p < PER; ++p) r[p] = load_run<DT, 8, ODD>(R, (p * ROW + at) * 8, a.n);
  }
  if (a.G) {
#pragma unroll
    for (int p = 0; p < PER; ++p) g[p] = load_run<DT, 8, ODD>(a.G, (p * ROW + at) * 8, a.n);
  }
#pragma unroll
  for (int p = 0; p < PER; ++p) run_to_f32<DT, 8>(x[p], (p * ROW + at) * 8, a.n, u[p]);
  if (a.R) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      float v[8];
      run_to_f32<DT, 8>(r[p], (p * ROW + at) * 8, a.n, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[p][i] = as_stored<DT>(u[p][i] + v[i]);
      // (a thread has read what it overwrites: the sum may go where one of its terms was)
      if (a.Y) store_run<DT, 8, ODD>(static_cast<ST*>(a.Y) + row * a.ldy, (p * ROW + at) * 8, a.n, u[p]);
    }
  }
  if (a.normalize) {
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) squares += (double)u[p][i] * (double)u[p][i];
  }
  if (a.G) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      float v[8];
      run_to_f32<DT, 8>(g[p], (p * ROW + at) * 8, a.n, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[p][i] *= v[i];
    }
  }
#pragma unroll
  for (int p = 0; p < PER; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(u[p][i]) & 0x7fffffffu);
  top = wave_max(top);
  if (a.normalize) squares = wave_sum(squares);
  if constexpr (ROW > kWave) {
    __shared__ uint32_t tops[ROW / kWave];
    __shared__ double sums[ROW / kWave];
    if (lane == 0) { tops[wave] = top; sums[wave] = squares; }
    __syncthreads();
    top = tops[0];
    squares = sums[0];
#pragma unroll
    for (int w = 1; w < ROW / kWave; ++w) { top = max(top, tops[w]); squares += sums[w]; }
  }
  const bool finite = top < 0x7f800000u;
  const float A = __uint_as_float(top);
  const float inv = 127.f * __builtin_amdgcn_rcpf(A);
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int c = (p * ROW + at) * 8, count = a.n - c;
    if (count <= 0) continue;
    float code[8];
    if (finite && top != 0) whole_codes<8>(u[p], inv, 127.f, A, code);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) code[i] = 0.f;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= ((uint32_t)(int)code[i] & 255u) << (8 * (i & 3));
    int8_t* out = a.C + row * a.ldc + c;
    if (!ODD || count >= 8) {
      *reinterpret_cast<uint2*>(out) = uint2{w[0], w[1]};
    } else {
      for (int i = 0; i < count; ++i) out[i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
  }
  if (at == 0) {
    double s = (double)A / 127.0;
    if (a.normalize && top != 0) s /= sqrt(squares / (double)a.n + a.eps);   // (a row of zeros has scale 0, also without an eps)
    a.S[row] = finite ? (float)s : __uint_as_float(0x7fc00000u);
  }
}

template <int DT, bool ODD>
void launch(const NormArgs& a, hipStream_t s) {
  const dim3 by_wave((unsigned)((a.t + 3) / 4)), by_row((unsigned)a.t);
  // A wave to a row, or a workgroup: 2048 columns, us: 4 rows 3.6 | 3.3, 256 rows 4.4 | 3.3, 4096 rows 9.8 | 11.0, 32768 rows 46 | 65; 1024 columns:
  // 4 rows 3.1 | 3.3, 256 rows 3.7 | 3.3, 32768 rows 30 | 60.
  if (a.n > 1024 && a.n <= 2048 && a.t <= 256) rmsnorm_quantize_kernel<DT, 1, 256, ODD><<<by_row, 256, 0, s>>>(a);
  else if (a.n <= 512) rmsnorm_quantize_kernel<DT, 1, 64, ODD><<<by_wave, 256, 0, s>>>(a);
  else if (a.n <= 1024) rmsnorm_quantize_kernel<DT, 2, 64, ODD><<<by_wave, 256, 0, s>>>(a);
  else if (a.n <= 2048) rmsnorm_quantize_kernel<DT, 4, 64, ODD><<<by_wave, 256, 0, s>>>(a);
  else if (a.n <= 4096) rmsnorm_quantize_kernel<DT, 2, 256, ODD><<<by_row, 256, 0, s>>>(a);
  else if (a.n <= 8192) rmsnorm_quantize_kernel<DT, 4, 256, ODD><<<by_row, 256, 0, s>>>(a);
  else if (a.n <= 12288) rmsnorm_quantize_kernel<DT, 6, 256, ODD><<<by_row, 256, 0, s>>>(a);
  else if (a.n <= 16384) rmsnorm_quantize_kernel<DT, 8, 256, ODD><<<by_row, 256, 0, s>>>(a);
  else rmsnorm_quantize_kernel<DT, 4, 1024, ODD><<<by_row, 1024, 0, s>>>(a);
}

}  // namespace

int64_t rmsnorm_max_columns() { return 8 * 4 * 1024; }

ptq_status rmsnorm_quantize_launch(const void* X, ptq_dtype dt, int64_t ldx, int64_t t, int64_t n, const void* residual,
                                   int64_t ldr, void* residual_out, int64_t ldo, const void* gamma, double eps, int normalize,
                                   int8_t* codes, int64_t ldc, float* scales, hipStream_t s) {
  // a launch has fewer than 2^32 threads, and a row up to 1024 of them
  constexpr int64_t kRows = 1 << 21;
  const int64_t size = dt == PTQ_BF16 ? 2 : 4;
  for (int64_t first = 0; first < t; first += kRows) {
    auto from = [&](const void* p, int64_t ld) { return p ? static_cast<const char*>(p) + first * ld * size : nullptr; };
    const NormArgs a{from(X, ldx), from(residual, ldr), const_cast<char*>(from(residual_out, ldo)), gamma, codes + first * ldc, scales + first,
                     ldx, ldr, ldo, ldc, (int)std::min(kRows, t - first), (int)n, eps, normalize};
    if (dt == PTQ_BF16) n % 8 ? launch<PTQ_BF16, true>(a, s) : launch<PTQ_BF16, false>(a, s);
    else n % 8 ? launch<PTQ_F32, true>(a, s) : launch<PTQ_F32, false>(a, s);
    PTQ_HIP_CHECK_LAUNCH();
  }
  return PTQ_OK;
}

}  // namespace ptq
