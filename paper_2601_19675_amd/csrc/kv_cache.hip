// A cache of keys and values that is quantized as it is written.
//
// Every (token, head) row of d values gets the library's asymmetric grid of its own (the one of ptq_quantize_layer):
//   lo = min(0, min x),  hi = max(0, max x),  (lo, hi) = (-1, 1) if the row is empty of anything else than 0,
//   scale = float32((hi - lo) / (2^bits - 1)),  zero = rne(-lo / scale),  code = clamp(rne(x / scale) + zero)
// and comes back as scale (code - zero).  Both ways are bound by bytes: a lane has eight values (16 bytes of bfloat16), a row
// d / 8 lanes.  The division that gives the scale is in float64, as the definition has it: the grid's width may need more
// than 24 bits.
#include "kv_cache.h"
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

// min or max over the LANES lanes of a row
template <int LANES, bool MAX>
__device__ __forceinline__ float row_extreme(float v) {
  auto pick = [](float a, float b) { return MAX ? fmaxf(a, b) : fminf(a, b); };
  v = pick(v, dpp_move_f32<kDppSwapPairs>(v));
  v = pick(v, dpp_move_f32<kDppSwapHalfQuads>(v));
  v = pick(v, dpp_move_f32<kDppHalfMirror>(v));
  if constexpr (LANES >= 16) v = pick(v, dpp_move_f32<kDppMirror>(v));
  if constexpr (LANES >= 32) v = pick(v, __shfl_xor(v, 16));
  return v;
}

// the quotient of d by a small whole number, correctly rounded: r = d - q by is exact, its share is added once
__device__ __forceinline__ double divided(double d, double by, double inv) {
  const double q = d * inv;
  return fma(fma(-q, by, d), inv, q);
}

// LANES lanes to a row; consecutive groups take consecutive tokens of one head, whose rows lie side by side in a page
template <int DT, int BITS, int LANES>
__global__ __launch_bounds__(256) void kv_write_kernel(WriteArgs a) {
  constexpr int kGroups = 256 / LANES;
  constexpr double kTop = (1 << BITS) - 1;
  using ST = typename StoredType<DT>::type;
  const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, head = blockIdx.y, which = blockIdx.z;
  const int c = lane * 8;
  const ST* X = static_cast<const ST*>(which ? a.X[1] : a.X[0]) + head * (which ? a.head[1] : a.head[0]);
  const int64_t stride = which ? a.token[1] : a.token[0];
  const int64_t places = a.c.pages << a.c.page_shift;
  Run<DT, 8> x[kRowsPerLane];
  int slot[kRowsPerLane];
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int token = (blockIdx.x * kRowsPerLane + i) * kGroups + group;
    const int safe = min(token, a.t - 1);
    slot[i] = token < a.t ? a.slots[safe] : -1;
    x[i] = load_run<DT, 8, false>(X + safe * stride, c, a.d);
  }
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    float v[8];
    run_to_f32<DT, 8>(x[i], c, a.d, v);
    float lo = 0.f, hi = 0.f;
    bool finite = true;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo = fminf(lo, v[e]);
      hi = fmaxf(hi, v[e]);
      finite &= (__float_as_uint(v[e]) & 0x7f800000u) != 0x7f800000u;
    }
    // a row with an infinity or a NaN: its scale becomes NaN, and so does whatever reads it
    hi = finite ? hi : INFINITY;
    lo = row_extreme<LANES, false>(lo);
    hi = row_extreme<LANES, true>(hi);
    finite = hi < INFINITY;
    float scale = finite ? (float)divided((double)hi - (double)lo, kTop, 1.0 / kTop) : 1.f;
    if (scale == 0.f) {   // nothing but zeros (or less than float32 can divide)
      lo = -1.f;
      scale = (float)(2.0 / kTop);
    }
    const float lift = scale < 0x1p-60f ? 0x1p90f : 1.f;   // exact, and 1 / scale stays a normal number
    const float over = scale * lift, inv = 1.f / over;
    const float below[1] = {-lo * lift};
    float z[1], code[8];
    whole_codes<1>(below, inv, 1.f, over, z);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= lift;
    whole_codes<8>(v, inv, 1.f, over, code);
    const int zero = finite ? (int)z[0] : 0;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t k = finite ? (uint32_t)min(max((int)code[e] + zero, 0), (1 << BITS) - 1) : 0u;
      if constexpr (BITS == 8) w[e >> 2] |= k << (8 * (e & 3));
      else w[0] |= k << (4 * (e >> 1) + 16 * (e & 1));
    }
    if ((uint32_t)slot[i] >= (uint64_t)places) continue;
    const int64_t row = kv_row(a.c, which, slot[i] >> a.c.page_shift, head, slot[i] & ((1 << a.c.page_shift) - 1));
    if (c < a.d) {
      uint8_t* out = a.c.codes + row * a.c.row_bytes + lane * BITS;
      if constexpr (BITS == 8) *reinterpret_cast<uint2*>(out) = uint2{w[0], w[1]};
      else *reinterpret_cast<uint32_t*>(out) = w[0];
    }
    if (lane == 0) {
      a.c.scales[row] = finite ? scale : __uint_as_float(0x7fc00000u);
      a.c.zeros[row] = (uint8_t)zero;
    }
  }
}

struct ReadArgs {
  void* X[2];
  int64_t token[2], head[2];
  const int32_t* table;
  int64_t ldt;
  const int32_t* cu;
  int64_t rows, max_kv;
  int d;
  KvCache c;
};

template <int DT, int BITS, int LANES>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a) {
  constexpr int kGroups = 256 / LANES;
  using ST = typename StoredType<DT>::type;
  const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, seq = blockIdx.z;
  const int head = blockIdx.y >> 1, which = blockIdx.y & 1, c = lane * 8;
  const int64_t begin = a.cu[seq], end = a.cu[seq + 1];
  if (begin < 0 || end > a.rows) return;
  const int64_t length = min(end - begin, a.max_kv);
  ST* X = static_cast<ST*>(which ? a.X[1] : a.X[0]) + head * (which ? a.head[1] : a.head[0]);
  const int64_t stride = which ? a.token[1] : a.token[0];
  int64_t place[kRowsPerLane], row[kRowsPerLane];
  uint2 w[kRowsPerLane];
  float scale[kRowsPerLane];
  int zero[kRowsPerLane];
  if ((int64_t)blockIdx.x * kRowsPerLane * kGroups >= length) return;
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    place[i] = ((int64_t)blockIdx.x * kRowsPerLane + i) * kGroups + group;
    const int64_t at = min(place[i], length - 1) >> a.c.page_shift;
    const int page = at < a.ldt ? a.table[seq * a.ldt + at] : -1;
    row[i] = (uint32_t)page < (uint64_t)a.c.pages ? kv_row(a.c, which, page, head, (int)(place[i] & ((1 << a.c.page_shift) - 1))) : -1;
  }
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    const int64_t r = row[i] < 0 ? 0 : row[i];
    const uint8_t* in = a.c.codes + r * a.c.row_bytes + (c < a.d ? lane * BITS : 0);
    if constexpr (BITS == 8) w[i] = *reinterpret_cast<const uint2*>(in);
    else w[i].x = *reinterpret_cast<const uint32_t*>(in);
    scale[i] = a.c.scales[r];
    zero[i] = a.c.zeros[r];
  }
#pragma unroll
  for (int i = 0; i < kRowsPerLane; ++i) {
    if (place[i] >= length || c >= a.d) continue;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      int k;
      if constexpr (BITS == 8) k = ((e < 4 ? w[i].x : w[i].y) >> (8 * (e & 3))) & 255;
      else k = (w[i].x >> (4 * (e >> 1) + 16 * (e & 1))) & 15;
      v[e] = row[i] < 0 ? 0.f : scale[i] * (float)(k - zero[i]);
    }
    store_run<DT, 8, false>(X + (begin + place[i]) * stride, c, a.d, v);
  }
}

KvCache cache_of(uint8_t* codes, float* scales, uint8_t* zeros, int64_t pages, int page, int hkv, int d, int bits) {
  return KvCache{codes, scales, zeros, pages, hkv, __builtin_ctz((unsigned)page), d * bits / 8};
}

template <int DT, int BITS>
void write_lanes(const WriteArgs& a, hipStream_t s) {
  auto grid = [&](int lanes) { return dim3((unsigned)ceil_div(a.t, kRowsPerLane * (256 / lanes)), (unsigned)a.c.heads, 2); };
  if (a.d <= 64) kv_write_kernel<DT, BITS, 8><<<grid(8), 256, 0, s>>>(a);
  else if (a.d <= 128) kv_write_kernel<DT, BITS, 16><<<grid(16), 256, 0, s>>>(a);
  else kv_write_kernel<DT, BITS, 32><<<grid(32), 256, 0, s>>>(a);
}
template <int DT, int BITS>
void read_lanes(const ReadArgs& a, int b, hipStream_t s) {
  auto grid = [&](int lanes) {
    return dim3((unsigned)ceil_div(a.max_kv, kRowsPerLane * (256 / lanes)), (unsigned)(2 * a.c.heads), (unsigned)b);
  };
  if (a.d <= 64) kv_read_kernel<DT, BITS, 8><<<grid(8), 256, 0, s>>>(a);
  else if (a.d <= 128) kv_read_kernel<DT, BITS, 16><<<grid(16), 256, 0, s>>>(a);
  else kv_read_kernel<DT, BITS, 32><<<grid(32), 256, 0, s>>>(a);
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
  const ReadArgs a{{K, V}, {k_token, v_token}, {k_head, v_head}, table, ldt, cu_kv, rows, max_kv, d,
                   cache_of(const_cast<uint8_t*>(codes), const_cast<float*>(scales), const_cast<uint8_t*>(zeros), pages, page, hkv, d, bits)};
  if (dt == PTQ_BF16) bits == 8 ? read_lanes<PTQ_BF16, 8>(a, (int)b, s) : read_lanes<PTQ_BF16, 4>(a, (int)b, s);
  else bits == 8 ? read_lanes<PTQ_F32, 8>(a, (int)b, s) : read_lanes<PTQ_F32, 4>(a, (int)b, s);
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

}  // namespace ptq
