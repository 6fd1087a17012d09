// A cache of keys and values that is quantized as it is written.
//
// Every (token, head) row of d values gets the library's asymmetric grid of its own (the one of ptq_quantize_layer):
//   lo = min(0, min x),  hi = max(0, max x),  (lo, hi) = (-1, 1) if the row is empty of anything else than 0,
//   scale = float32((hi - lo) / (2^bits - 1)),  zero = rne(-lo / scale),  code = clamp(rne(x / scale) + zero)
// and comes back as scale (code - zero).  Both ways are bound by bytes: a lane has eight values (16 bytes of bfloat16), a row
// d / 8 lanes.  The division that gives the scale is in float64, as the definition has it: the grid's width may need more
// than 24 bits.
//
// Four prompts of up to 8192 tokens, 32 heads of 128 channels, bfloat16 into 4 bits: 893 MB both ways in 217 us (write 124, read 96), 4.1
// TB/s; a large copy has 4.7.
#include <algorithm>

#include "kv_cache.h"
#include "static_for.h"
#include "stored_rows.h"

namespace ptq {
namespace {

constexpr int kRowsPerLane = 4;   // rows on their way per group of lanes

struct WriteArgs {
  const void* X[2];                // keys, values
  int64_t token[2], head[2];       // strides, elements
  const int32_t* slots;
  int t, d;
  KvCache c;
};

// the largest over the LANES lanes of a row
template <int LANES, class T>
__device__ __forceinline__ T row_max(T v) {
  v = max(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, kDppSwapPairs, 0xf, 0xf, true));
  v = max(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, kDppSwapHalfQuads, 0xf, 0xf, true));
  v = max(v, (T)__builtin_amdgcn_update_dpp(0, (int)v, kDppHalfMirror, 0xf, 0xf, true));
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

// LANES lanes to a row; consecutive groups take consecutive tokens of one head, whose rows lie side by side in a page.  Consecutive
// workgroups take the heads of the same tokens: a head's rows alone, 8 KB apart in a projection's output, would fall on few of the
// memory's channels (20000 tokens x 32 heads x 128 into 4 bits that way: 155 us).
template <int DT, int BITS, int LANES>
__global__ __launch_bounds__(256) void kv_write_kernel(WriteArgs a) {
  constexpr int kGroups = 256 / LANES;
  constexpr double kTop = (1 << BITS) - 1;
  using ST = typename StoredType<DT>::type;
  const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, which = blockIdx.y;
  const int tile = blockIdx.x / a.c.heads, head = blockIdx.x % a.c.heads;
  const int c = lane * 8;
  const ST* X = static_cast<const ST*>(which ? a.X[1] : a.X[0]) + head * (which ? a.head[1] : a.head[0]);
  const int64_t stride = which ? a.token[1] : a.token[0];
  const uint32_t places = (uint32_t)(a.c.pages << a.c.page_shift);
  const KvRows rows = kv_rows(a.c, which, head);
  Run<DT, 8> x[kRowsPerLane];
  int slot[kRowsPerLane];
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int token = (tile * kRowsPerLane + i) * kGroups + group, safe = min(token, a.t - 1);
    slot[i] = token < a.t ? a.slots[safe] : -1;
    x[i] = load_run<DT, 8, false>(X + safe * stride, c, a.d);
  }
  // Bits tell a row's extremes, and whether all of it is finite: as signed numbers those of the largest value come last, as
  // unsigned ones those of the value furthest below 0, if one is.
  int hi_bits = 0;
  uint32_t lo_bits = 0;
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    float v[8];
    run_to_f32<DT, 8>(x[i], c, a.d, v);
    int hi = 0;
    uint32_t lo = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi = max(hi, __float_as_int(v[e]));
      lo = max(lo, __float_as_uint(v[e]));
    }
    hi = row_max<LANES>(hi);
    lo = row_max<LANES>(lo);
    // the grids of the group's four rows are worked out side by side: lane i of every four has row i
    if ((lane & 3) == i) {
      hi_bits = hi;
      lo_bits = lo;
    }
  }
  // a row with an infinity or a NaN: its scale becomes NaN, and so does whatever reads it; its codes 0 (x inv is NaN or 0)
  const bool finite = hi_bits < 0x7f800000 && lo_bits < 0xff800000u;
  const float hi = __int_as_float(hi_bits);
  float lo = lo_bits > 0x80000000u ? __uint_as_float(lo_bits) : 0.f;
  float scale = finite ? (float)divided((double)hi - (double)lo, kTop, 1.0 / kTop) : 1.f;
  if (scale == 0.f) {   // nothing but zeros (or less than float32 can divide)
    lo = -1.f;
    scale = (float)(2.0 / kTop);
  }
  const float below[1] = {finite ? -lo : 0.f};
  float inv = __builtin_amdgcn_rcpf(scale), z[1];
  whole_codes<1>(below, inv, 1.f, scale, z);
  // both ends rounded away from 0 (the only codes past the grid), or no float32 reciprocal: by the quotient, and clamped
  const bool odd_grid = __any((scale < 0x1p-110f) | (scale > 0x1p110f) | (finite && rintf(hi * inv) + z[0] > (float)kTop));
  inv = finite ? inv : 0.f;
  {
    int mine = slot[0];
#pragma unroll
    for (int i = 1; i < kRowsPerLane; ++i) mine = (lane & 3) == i ? slot[i] : mine;
    if (lane < kRowsPerLane && (uint32_t)mine < places) {
      const int64_t row = kv_row(rows, (uint32_t)mine >> a.c.page_shift, mine & ((1 << a.c.page_shift) - 1));
      a.c.scales[row] = finite ? scale : __uint_as_float(0x7fc00000u);
      a.c.zeros[row] = (uint8_t)z[0];
    }
  }
  static_for<kRowsPerLane>([&](auto i_) {
    constexpr int i = decltype(i_)::value;
    const float inv_i = of_four<i>(inv), z_i = of_four<i>(z[0]);
    float v[8];
    run_to_f32<DT, 8>(x[i], c, a.d, v);
    // 1.5 2^23 + a whole number has that number in its low bits, and adding it rounds there: code = rne(x inv + zero), which is rne(x / scale) + zero
    // as long as x inv + zero, off by less than 2^-14 (see whole_codes; the sum adds 2^-17), is not that close to a middle
    constexpr float kWhole = 12582912.f;
    const float from = z_i + kWhole;
    float u[8], far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      u[e] = fmaf(v[e], inv_i, from);
      far = fmaxf(far, fabsf(fmaf(v[e], inv_i, from - u[e])));
    }
    if (__any(far > 0.5f - 0x1p-14f) | odd_grid) {
      const float s = of_four<i>(scale), good = of_four<i>(finite ? 1.f : 0.f);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        u[e] = kWhole + (good != 0.f ? fminf((float)rint((double)v[e] / (double)s) + z_i, (float)kTop) : 0.f);
    }
    auto byte_pair = [&](int e0, int e1) { return __builtin_amdgcn_perm(__float_as_uint(u[e1]), __float_as_uint(u[e0]), 0x0c0c0400u); };
    auto bytes = [&](int e0, int e1, int e2, int e3) { return __builtin_amdgcn_perm(byte_pair(e2, e3), byte_pair(e0, e1), 0x05040100u); };
    if ((uint32_t)slot[i] < places && c < a.d) {
      const int64_t row = kv_row(rows, (uint32_t)slot[i] >> a.c.page_shift, slot[i] & ((1 << a.c.page_shift) - 1));
      uint8_t* out = a.c.codes + row * a.c.row_bytes + lane * BITS;
      if constexpr (BITS == 8) *reinterpret_cast<uint2*>(out) = uint2{bytes(0, 1, 2, 3), bytes(4, 5, 6, 7)};
      else *reinterpret_cast<uint32_t*>(out) = bytes(0, 4, 1, 5) | (bytes(2, 6, 3, 7) << 4);
    }
  });
}

struct ReadArgs {
  void* X[2];
  int64_t token[2], head[2];
  const int32_t* table;
  int64_t ldt;
  const int32_t* cu;
  int64_t rows, max_kv;
  int d, first_tile;               // of places, in this launch
  KvCache c;
};

// The same layout the other way; four rows' page numbers, then their codes, are on their way together.
template <int DT, int BITS, int LANES>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a) {
  constexpr int kGroups = 256 / LANES;
  using ST = typename StoredType<DT>::type;
  const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, seq = blockIdx.z, which = blockIdx.y;
  const int tile = a.first_tile + blockIdx.x / a.c.heads, head = blockIdx.x % a.c.heads, c = lane * 8;
  const int64_t begin = a.cu[seq], end = a.cu[seq + 1];
  if (begin < 0 || end > a.rows) return;
  const int64_t length = min(end - begin, a.max_kv);
  ST* X = static_cast<ST*>(which ? a.X[1] : a.X[0]) + head * (which ? a.head[1] : a.head[0]);
  const int64_t stride = which ? a.token[1] : a.token[0];
  if ((int64_t)tile * kRowsPerLane * kGroups >= length) return;
  const KvRows rows = kv_rows(a.c, which, head);
  const int first = tile * kRowsPerLane * kGroups + group, inside = (1 << a.c.page_shift) - 1;
  int page[kRowsPerLane];
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int at = min(first + i * kGroups, (int)length - 1) >> a.c.page_shift;
    page[i] = a.table[seq * a.ldt + min((int64_t)at, a.ldt - 1)];
    page[i] = at < a.ldt && (uint32_t)page[i] < (uint64_t)a.c.pages ? page[i] : -1;
  }
  uint2 w[kRowsPerLane];
  float scale[kRowsPerLane];
  int zero[kRowsPerLane];
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int64_t r = kv_row(rows, max(page[i], 0), (first + i * kGroups) & inside);
    const uint8_t* in = a.c.codes + r * a.c.row_bytes + (c < a.d ? lane * BITS : 0);
    if constexpr (BITS == 8) w[i] = *reinterpret_cast<const uint2*>(in);
    else w[i].x = *reinterpret_cast<const uint32_t*>(in);
    scale[i] = a.c.scales[r];
    zero[i] = a.c.zeros[r];
  }
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    if (first + i * kGroups >= length) continue;
    const float s = page[i] < 0 ? 0.f : scale[i], z = (float)zero[i];   // a page that is not there: zeros
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t k;
      if constexpr (BITS == 8) k = ((e < 4 ? w[i].x : w[i].y) >> (8 * (e & 3))) & 255u;
      else k = (((e >> 1) & 1 ? (w[i].x >> 4) & 0x0f0f0f0fu : w[i].x & 0x0f0f0f0fu) >> (8 * (e >> 2) + 16 * (e & 1))) & 255u;
      v[e] = s * ((float)k - z);
    }
    store_run<DT, 8, false>(X + (begin + first + i * kGroups) * stride, c, a.d, v);
  }
}

KvCache cache_of(uint8_t* codes, float* scales, uint8_t* zeros, int64_t pages, int page, int hkv, int d, int bits) {
  return KvCache{codes, scales, zeros, pages, hkv, __builtin_ctz((unsigned)page), d * bits / 8};
}

// tokens or places of a workgroup, and such tiles in a launch, which has fewer than 2^32 threads
int tile_rows(int d) { return kRowsPerLane * (256 / (d <= 64 ? 8 : d <= 128 ? 16 : 32)); }
int64_t launch_tiles(int heads) { return (1 << 23) / heads; }

template <int DT, int BITS>
void write_lanes(const WriteArgs& all, hipStream_t s) {
  const int rows = tile_rows(all.d);
  const int64_t step = launch_tiles(all.c.heads) * rows;
  for (int64_t first = 0; first < all.t; first += step) {
    WriteArgs a = all;
    for (int i = 0; i < 2; ++i) a.X[i] = static_cast<const typename StoredType<DT>::type*>(all.X[i]) + first * all.token[i];
    a.slots += first;
    a.t = (int)std::min(step, all.t - first);
    const dim3 grid((unsigned)(ceil_div(a.t, rows) * a.c.heads), 2);
    if (a.d <= 64) kv_write_kernel<DT, BITS, 8><<<grid, 256, 0, s>>>(a);
    else if (a.d <= 128) kv_write_kernel<DT, BITS, 16><<<grid, 256, 0, s>>>(a);
    else kv_write_kernel<DT, BITS, 32><<<grid, 256, 0, s>>>(a);
  }
}
template <int DT, int BITS>
void read_lanes(const ReadArgs& all, int b, hipStream_t s) {
  // no sequence has more places than there are rows, whatever max_kv allows
  const int64_t tiles = ceil_div(std::min(all.max_kv, all.rows), tile_rows(all.d)), step = launch_tiles(all.c.heads);
  for (int64_t first = 0; first < tiles; first += step) {
    ReadArgs a = all;
    a.first_tile = (int)first;
    const dim3 grid((unsigned)(std::min(step, tiles - first) * a.c.heads), 2, (unsigned)b);
    if (a.d <= 64) kv_read_kernel<DT, BITS, 8><<<grid, 256, 0, s>>>(a);
    else if (a.d <= 128) kv_read_kernel<DT, BITS, 16><<<grid, 256, 0, s>>>(a);
    else kv_read_kernel<DT, BITS, 32><<<grid, 256, 0, s>>>(a);
  }
}

}  // namespace

ptq_status kv_cache_write_launch(const void* K, int64_t k_token, int64_t k_head, const void* V, int64_t v_token,
                                 int64_t v_head, ptq_dtype dt, int64_t t, int hkv, int d, const int32_t* slots, int bits,
                                 uint8_t* codes, float* scales, uint8_t* zeros, int64_t pages, int page, hipStream_t s) {
  const WriteArgs a{{K, V}, {k_token, v_token}, {k_head, v_head}, slots, (int)t, d,
                    cache_of(codes, scales, zeros, pages, page, hkv, d, bits)};
  if (dt == PTQ_BF16) bits == 8 ? write_lanes<PTQ_BF16, 8>(a, s) : write_lanes<PTQ_BF16, 4>(a, s);
  else bits == 8 ? write_lanes<PTQ_F32, 8>(a, s) : write_lanes<PTQ_F32, 4>(a, s);
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

ptq_status kv_cache_read_launch(const uint8_t* codes, const float* scales, const uint8_t* zeros, int64_t pages, int page,
                                int hkv, int d, int bits, const int32_t* table, int64_t ldt, int64_t b, const int32_t* cu_kv,
                                int64_t rows, int64_t max_kv, void* K, int64_t k_token, int64_t k_head, void* V,
                                int64_t v_token, int64_t v_head, ptq_dtype dt, hipStream_t s) {
  const ReadArgs a{{K, V}, {k_token, v_token}, {k_head, v_head}, table, ldt, cu_kv, rows, max_kv, d, 0,
                   cache_of(const_cast<uint8_t*>(codes), const_cast<float*>(scales), const_cast<uint8_t*>(zeros), pages, page, hkv, d, bits)};
  if (dt == PTQ_BF16) bits == 8 ? read_lanes<PTQ_BF16, 8>(a, (int)b, s) : read_lanes<PTQ_BF16, 4>(a, (int)b, s);
  else bits == 8 ? read_lanes<PTQ_F32, 8>(a, (int)b, s) : read_lanes<PTQ_F32, 4>(a, (int)b, s);
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

}  // namespace ptq
