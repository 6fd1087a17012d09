// Pages of the quantized cache copied as they lie: to other pages of it (the page in which a forked sequence goes on, the moves of a
// compaction) or to those of another cache.
//
// Bound: bytes.  A page is six stretches of memory -- codes, scales and zeros of its keys and of its values -- which are cut into pieces of
// 4 KB; a wave copies a piece, four loads of 16 bytes a lane on their way.
//
// 12000 pages of 32 tokens, 8 heads of 128 channels in 4 bits (848 MB in and out): 173 us, 4.9 TB/s, the rate of a large copy; 24 pages in 8 bits 6.5
// us, all latency.
#include <algorithm>

#include "common.h"
#include "static_for.h"
#include "stored_rows.h"

namespace ptq {
namespace {

constexpr int kPiece = 4096;     // bytes of a wave
constexpr int kWaves = 4;

struct CopyArgs {
  const uint8_t* in[3]; uint8_t* out[3];     // codes, scales, zeros
  int64_t bytes[3];                          // of a page's keys, or of its values
  int64_t in_pages, out_pages;
  const int32_t *from, *to;
  int64_t n;
  uint32_t pieces[3];                        // of such a stretch
};

__global__ __launch_bounds__(kWaves * 64) void copy_pages_kernel(CopyArgs a, int64_t first) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t each = a.pieces[0] + a.pieces[1] + a.pieces[2];
  const int64_t unit = first + (int64_t)blockIdx.x * kWaves + wave, half = unit / each, i = half >> 1;
  if (i >= a.n) return;
  uint32_t piece = (uint32_t)(unit - half * each);
  const int32_t from = a.from[i], to = a.to[i];
  if ((uint32_t)from >= (uint64_t)a.in_pages || (uint32_t)to >= (uint64_t)a.out_pages) return;
  int k = 0;
  while (piece >= a.pieces[k]) piece -= a.pieces[k++];
  const int64_t bytes = a.bytes[k], at = (int64_t)piece * kPiece, which = half & 1;
  const uint8_t* in = a.in[k] + (which * a.in_pages + from) * bytes + at;
  uint8_t* out = a.out[k] + (which * a.out_pages + to) * bytes + at;
  const int left = (int)min(bytes - at, (int64_t)kPiece);
  using Line = AnyWords<4, 1>;
  if (left == kPiece) {
    Line v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const Line*>(in + (j * 64 + lane) * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<Line*>(out + (j * 64 + lane) * 16) = v[j];
    return;
  }
  const int whole = left & ~15;
  Line v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int b = (j * 64 + lane) * 16;
    if (b < whole) v[j] = *reinterpret_cast<const Line*>(in + b);
  }
  uint8_t rest = 0;
  if (lane < left - whole) rest = in[whole + lane];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int b = (j * 64 + lane) * 16;
    if (b < whole) *reinterpret_cast<Line*>(out + b) = v[j];
  }
  if (lane < left - whole) out[whole + lane] = rest;
}

}  // namespace

ptq_status kv_cache_copy_pages_launch(const uint8_t* from_codes, const float* from_scales, const uint8_t* from_zeros, int64_t from_pages,
                                      uint8_t* codes, float* scales, uint8_t* zeros, int64_t pages, int64_t page, int64_t hkv,
                                      int64_t row_bytes, const int32_t* from, const int32_t* to, int64_t n, hipStream_t s) {
  CopyArgs a{{from_codes, reinterpret_cast<const uint8_t*>(from_scales), from_zeros},
             {codes, reinterpret_cast<uint8_t*>(scales), zeros},
             {hkv * page * row_bytes, hkv * page * 4, hkv * page},
             from_pages, pages, from, to, n, {}};
  int64_t each = 0;
  for (int k = 0; k < 3; ++k) each += a.pieces[k] = (uint32_t)ceil_div(a.bytes[k], kPiece);
  // a launch has fewer than 2^32 threads
  const int64_t units = 2 * n * each, step = (int64_t)(1 << 23) * kWaves;
  for (int64_t first = 0; first < units; first += step)
    copy_pages_kernel<<<(unsigned)ceil_div(std::min(step, units - first), kWaves), kWaves * 64, 0, s>>>(a, first);
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

}  // namespace ptq
