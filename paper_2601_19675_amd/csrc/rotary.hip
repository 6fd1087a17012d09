// Rotary positions: pairs of channels of a head, seen as points of a plane, are turned by the token's position times the pair's
// frequency,
//   y_a = scale (x_a cos - x_b sin),   y_b = scale (x_a sin + x_b cos),
// alone (Y may be X), or with the keys going on into the paged cache in the same launch.
//
// Bound: bytes, each channel once in and out.  A thread has the same four pairs of several heads of a token, so that cosines and sines are
// worked out once for all of them and stay in registers; consecutive threads have a head's row side by side, and consecutive workgroups
// the heads of the same tokens.  All of it is float64, which runs at float32's rate here and hides behind the memory: what
// is rounded to a key's type, and decides its codes, is the exact value but for 2^-50.
//
// 16384 tokens, 40 heads of 128 bfloat16 channels (336 MB): 68 to 70 us, 4.9 TB/s, the rate of a large copy; 16 tokens 3.5 to 3.7 us, all latency.  Four
// prompts of up to 4096 tokens, 32 heads of each kind, into 4 bits (401 MB): 111 to 118 us in kernel traces, 3.4 to 3.6 TB/s, some way from a copy.  (Eight pairs to a
// lane take 142 to 181 registers and leave two or three waves to a SIMD: 78, 4.8 and, traced, 137 us.)
#include <algorithm>
#include <cmath>

#include "kv_grid.h"
#include "rotary.h"
#include "static_for.h"

namespace ptq {
namespace {

constexpr int kHeadsAhead = 4;   // heads whose channels are on their way together
constexpr int kPairs = 4;        // of a lane

struct RotaryArgs {
  const void* X; void* Y;
  int64_t x_token, x_head, y_token, y_head;
  const int32_t* positions; const double* freq;
  int t, heads, d, rot, interleaved;
  int slices, per;                 // workgroups to a tile of tokens, and heads of each
  double scale;
};

// Which two runs of four channels a lane has, and whether they are pairs that turn (four frequencies from 4 lane on; rot % 16 == 0).
struct LaneRuns { int a, b; bool turns, apart; };   // apart: b is half of the turned channels behind a
__device__ __forceinline__ LaneRuns lane_runs(int lane, int rot, int interleaved) {
  const bool turns = 8 * lane < rot, apart = turns && !interleaved;
  return LaneRuns{apart ? 4 * lane : 8 * lane, apart ? 4 * lane + rot / 2 : 8 * lane + 4, turns, apart};
}
// cosines and sines of the lane's pairs; those of a lane without are not used
__device__ __forceinline__ void lane_angles(const LaneRuns& runs, int lane, int position, const double* freq, double scale, CosSin (&t)[kPairs]) {
  double f[kPairs];
#pragma unroll
  for (int e = 0; e < kPairs; ++e) f[e] = freq[runs.turns ? kPairs * lane + e : 0];
#pragma unroll
  for (int e = 0; e < kPairs; ++e) t[e] = cos_sin(position, f[e], scale);
}
__device__ __forceinline__ void turn_runs(float (&u)[kPairs], float (&v)[kPairs], const LaneRuns& runs, const CosSin (&t)[kPairs]) {
  if (!runs.turns) return;
  if (runs.apart) {
#pragma unroll
    for (int e = 0; e < kPairs; ++e) turn(u[e], v[e], t[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      turn(u[2 * e], u[2 * e + 1], t[e]);
      turn(v[2 * e], v[2 * e + 1], t[2 + e]);
    }
  }
}

// LANES lanes to a row of up to 8 LANES channels (d % 16 == 0, rot % 16 == 0); workgroup (tile, slice)
template <int DT, int LANES>
__device__ __forceinline__ void rotary_rows(const RotaryArgs& a, int tile, int slice) {
  constexpr int kTokens = 256 / LANES;
  using ST = typename StoredType<DT>::type;
  const int lane = threadIdx.x % LANES, token = tile * kTokens + threadIdx.x / LANES, safe = min(token, a.t - 1);
  const LaneRuns runs = lane_runs(lane, a.rot, a.interleaved);
  const int first = slice * a.per, last = min(a.heads, first + a.per);
  const ST* X = static_cast<const ST*>(a.X) + safe * a.x_token;
  ST* Y = static_cast<ST*>(a.Y) + safe * a.y_token;
  const int position = a.positions[safe];
  CosSin angles[kPairs];
  bool ready = false;
  for (int h0 = first; h0 < last; h0 += kHeadsAhead) {
    Run<DT, 4> x[kHeadsAhead][2];
#pragma unroll
    for (int i = 0; i < kHeadsAhead; ++i) {
      const ST* row = X + min(h0 + i, last - 1) * a.x_head;
      x[i][0] = load_run<DT, 4, false>(row, runs.a, a.d);
      x[i][1] = load_run<DT, 4, false>(row, runs.b, a.d);
    }
    if (!ready) lane_angles(runs, lane, position, a.freq, a.scale, angles);
    ready = true;
#pragma unroll
    for (int i = 0; i < kHeadsAhead; ++i) {
      float u[4], v[4];
      run_to_f32<DT, 4>(x[i][0], runs.a, a.d, u);
      run_to_f32<DT, 4>(x[i][1], runs.b, a.d, v);
      turn_runs(u, v, runs, angles);
      if (token < a.t && h0 + i < last) {
        store_run<DT, 4, false>(Y + (h0 + i) * a.y_head, runs.a, a.d, u);
        store_run<DT, 4, false>(Y + (h0 + i) * a.y_head, runs.b, a.d, v);
      }
    }
  }
}

template <int DT, int LANES>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
  rotary_rows<DT, LANES>(a, blockIdx.x / a.slices, blockIdx.x % a.slices);
}

// Any widths: a thread has one pair, or two channels that stay as they are, of a token's heads.  16384 tokens, 40 heads of bfloat16: 96 channels of
// which 24 turn 78 us (252 MB, 3.2 TB/s), 80 of which 20 turn 74; in whole runs, with 96 and 80 turning, 42 and 39.
template <int DT>
__global__ __launch_bounds__(256) void rotary_any_kernel(RotaryArgs a, int64_t first_tile) {
  using ST = typename StoredType<DT>::type;
  const int slice = blockIdx.x % a.slices, pairs = (a.d + 1) / 2;
  const int64_t i = (first_tile + blockIdx.x / a.slices) * 256 + threadIdx.x, token = i / pairs;
  if (token >= a.t) return;
  const int p = (int)(i - token * pairs);
  const bool turns = 2 * p < a.rot;
  const int ca = turns && !a.interleaved ? p : 2 * p, cb = turns && !a.interleaved ? p + a.rot / 2 : 2 * p + 1;
  const bool both = cb < a.d;
  const int last = min(a.heads, (slice + 1) * a.per);
  const ST* X = static_cast<const ST*>(a.X) + token * a.x_token;
  ST* Y = static_cast<ST*>(a.Y) + token * a.y_token;
  CosSin angle{1.0, 0.0};
  if (turns) angle = cos_sin(a.positions[token], a.freq[p], a.scale);
  for (int h0 = slice * a.per; h0 < last; h0 += kHeadsAhead) {
    ST x[kHeadsAhead][2];
#pragma unroll
    for (int k = 0; k < kHeadsAhead; ++k) {
      const ST* row = X + min(h0 + k, last - 1) * a.x_head;
      x[k][0] = row[ca];
      x[k][1] = row[both ? cb : ca];
    }
#pragma unroll
    for (int k = 0; k < kHeadsAhead; ++k) {
      if (h0 + k >= last) break;
      ST* row = Y + (h0 + k) * a.y_head;
      if (turns) {
        float u = (float)stored_to_f64<DT>(x[k][0]), v = (float)stored_to_f64<DT>(x[k][1]);
        turn(u, v, angle);
        if constexpr (DT == PTQ_BF16) {
          row[ca] = f32_to_bf16_bits(u);
          row[cb] = f32_to_bf16_bits(v);
        } else {
          row[ca] = u;
          row[cb] = v;
        }
      } else {
        row[ca] = x[k][0];
        if (both) row[cb] = x[k][1];
      }
    }
  }
}

struct RotaryCacheArgs {
  RotaryArgs q;                    // .t, .d, .rot, .positions ... are the keys' too
  const void* X[2];                // keys, values
  int64_t token[2], head[2];
  const int32_t* slots;
  int slices, per;                 // of the keys, and of the values
  KvCache c;
};

// Keys (turned) or values of a tile of tokens and a slice of heads into the cache: kv_cache.hip's rows, with the lanes' two runs.
template <int DT, int BITS, int LANES>
__device__ __forceinline__ void cache_rows(const RotaryCacheArgs& a, int tile, int slice, int which) {
  constexpr int kTokens = 256 / LANES;
  using ST = typename StoredType<DT>::type;
  const int lane = threadIdx.x % LANES, token = tile * kTokens + threadIdx.x / LANES, safe = min(token, a.q.t - 1);
  LaneRuns runs = lane_runs(lane, a.q.rot, a.q.interleaved);
  const int first = slice * a.per, last = min(a.c.heads, first + a.per);
  const ST* X = static_cast<const ST*>(which ? a.X[1] : a.X[0]) + safe * (which ? a.token[1] : a.token[0]);
  const int64_t stride = which ? a.head[1] : a.head[0];
  const int position = a.q.positions[safe], slot = token < a.q.t ? a.slots[safe] : -1;
  const bool there = (uint32_t)slot < (uint32_t)(a.c.pages << a.c.page_shift);
  const int place = there ? slot : 0;
  const uint32_t page = (uint32_t)place >> a.c.page_shift, offset = place & ((1 << a.c.page_shift) - 1);
  CosSin angles[kPairs];
  bool ready = which != 0;
  for (int h0 = first; h0 < last; h0 += kHeadsAhead) {
    Run<DT, 4> x[kHeadsAhead][2];
#pragma unroll
    for (int i = 0; i < kHeadsAhead; ++i) {
      const ST* row = X + min(h0 + i, last - 1) * stride;
      x[i][0] = load_run<DT, 4, false>(row, runs.a, a.q.d);
      x[i][1] = load_run<DT, 4, false>(row, runs.b, a.q.d);
    }
    if (!ready) lane_angles(runs, lane, position, a.q.freq, a.q.scale, angles);
    ready = true;
    float v[kHeadsAhead][2][4];
    RowExtremes most;
#pragma unroll
    for (int i = 0; i < kHeadsAhead; ++i) {
      run_to_f32<DT, 4>(x[i][0], runs.a, a.q.d, v[i][0]);
      run_to_f32<DT, 4>(x[i][1], runs.b, a.q.d, v[i][1]);
      if (!which) turn_runs(v[i][0], v[i][1], runs, angles);
      RowExtremes row;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[i][k][e] = as_stored<DT>(v[i][k][e]);
          row.take(v[i][k][e]);
        }
      row.hi = row_max<LANES>(row.hi);
      row.lo = row_max<LANES>(row.lo);
      if ((lane & 3) == i) most = row;
    }
    const RowGrid grid = row_grid<BITS>(most);
    auto row_at = [&](int head) { return kv_row(kv_rows(a.c, which, head), page, offset); };
    if (lane < kHeadsAhead && there && h0 + lane < last) {
      const int64_t row = row_at(h0 + lane);
      a.c.scales[row] = grid.finite ? grid.scale : __uint_as_float(0x7fc00000u);
      a.c.zeros[row] = (uint8_t)grid.zero;
    }
    static_for<kHeadsAhead>([&](auto i_) {
      constexpr int i = decltype(i_)::value;
      uint32_t u[2][4];
      row_codes_of<BITS, i>(v[i][0], grid, u[0]);
      row_codes_of<BITS, i>(v[i][1], grid, u[1]);
      const bool store = there && h0 + i < last && runs.a < a.q.d;   // (d % 16 == 0: a lane has both of its runs or neither)
      uint8_t* out = a.c.codes + row_at(store ? h0 + i : first) * a.c.row_bytes;
      if constexpr (BITS == 8) {
        if (store) {
          *reinterpret_cast<uint32_t*>(out + runs.a) = four_bytes(u[0][0], u[0][1], u[0][2], u[0][3]);
          *reinterpret_cast<uint32_t*>(out + runs.b) = four_bytes(u[1][0], u[1][1], u[1][2], u[1][3]);
        }
      } else {
        // a word has eight codes: bytes 0 and 2 are of the first four, 1 and 3 of the others, which the lane has itself or the one beside it
        auto half = [](const uint32_t (&c)[4]) {
          return __builtin_amdgcn_perm(0, byte_pair(c[0], c[1]), 0x0c010c00u) | (__builtin_amdgcn_perm(0, byte_pair(c[2], c[3]), 0x0c010c00u) << 4);
        };
        const uint32_t ha = half(u[0]), hb = half(u[1]);
        const bool second = lane & 1;
        const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(second ? ha : hb), kDppSwapPairs, 0xf, 0xf, true);
        const uint32_t low = !runs.apart || !second ? ha : other, high = !runs.apart ? hb : second ? hb : other;
        if (store) *reinterpret_cast<uint32_t*>(out + (runs.apart && second ? runs.b - 4 : runs.a) / 2) = low | (high << 8);
      }
    });
  }
}

template <int DT, int BITS, int LANES>
__global__ __launch_bounds__(256) void rotary_cache_kernel(RotaryCacheArgs a) {
  const int all = a.q.slices + 2 * a.slices, tile = blockIdx.x / all, part = blockIdx.x % all;
  if (part < a.q.slices) rotary_rows<DT, LANES>(a.q, tile, part);
  else cache_rows<DT, BITS, LANES>(a, tile, (part - a.q.slices) % a.slices, (part - a.q.slices) / a.slices);
}

int lanes_of(int64_t d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }

// Heads of a workgroup: as many as leave the device 8192 workgroups, between one round of loads and eight of them.  (The angles of a round's heads
// take as long as turning one head.  16384 tokens, 40 heads of 128 | four prompts into the cache, in us: with 2048 72 | 158, 4096 78 | 153, 8192
// 70 | 152, 16384 69 | 161.)
int heads_per(int64_t tiles, int64_t heads) {
  const int64_t most = std::min<int64_t>(8, ceil_div(std::max<int64_t>(1, tiles * heads / 8192), kHeadsAhead)), rounds = ceil_div(heads, kHeadsAhead);
  return (int)(ceil_div(rounds, ceil_div(rounds, most)) * kHeadsAhead);   // as many as that, and alike
}
// tiles of a launch, which has fewer than 2^32 threads
int64_t launch_tiles(int64_t slices) { return std::max<int64_t>(1, (1 << 23) / slices); }

template <int DT>
void rotary_typed(const RotaryArgs& all, hipStream_t s) {
  using ST = typename StoredType<DT>::type;
  RotaryArgs a = all;
  const bool runs = all.d % 16 == 0 && all.d <= 256 && all.rot % 16 == 0;
  const int lanes = lanes_of(all.d), tokens = 256 / lanes;
  const int64_t tiles = runs ? ceil_div(all.t, tokens) : ceil_div((int64_t)all.t * ((all.d + 1) / 2), 256);
  a.per = heads_per(tiles, all.heads);
  a.slices = (int)ceil_div(all.heads, a.per);
  const int64_t step = launch_tiles(a.slices);
  for (int64_t first = 0; first < tiles; first += step) {
    const int64_t n = std::min(step, tiles - first);
    const unsigned grid = (unsigned)(n * a.slices);
    if (!runs) {
      rotary_any_kernel<DT><<<grid, 256, 0, s>>>(a, first);
      continue;
    }
    a.X = static_cast<const ST*>(all.X) + first * tokens * a.x_token;
    a.Y = static_cast<ST*>(all.Y) + first * tokens * a.y_token;
    a.positions = all.positions + first * tokens;
    a.t = (int)std::min<int64_t>(n * tokens, all.t - first * tokens);
    if (lanes == 8) rotary_kernel<DT, 8><<<grid, 256, 0, s>>>(a);
    else if (lanes == 16) rotary_kernel<DT, 16><<<grid, 256, 0, s>>>(a);
    else rotary_kernel<DT, 32><<<grid, 256, 0, s>>>(a);
  }
}

template <int DT, int BITS>
void rotary_cache_typed(const RotaryCacheArgs& all, hipStream_t s) {
  using ST = typename StoredType<DT>::type;
  RotaryCacheArgs a = all;
  const int lanes = lanes_of(all.q.d), tokens = 256 / lanes;
  const int64_t tiles = ceil_div(all.q.t, tokens);
  const int64_t heads = all.q.heads + 2 * all.c.heads;
  a.q.per = std::min(all.q.heads, heads_per(tiles, heads));
  a.q.slices = (int)ceil_div(all.q.heads, a.q.per);
  a.per = std::min(all.c.heads, heads_per(tiles, heads));
  a.slices = (int)ceil_div(all.c.heads, a.per);
  const int64_t each = a.q.slices + 2 * a.slices, step = launch_tiles(each);
  for (int64_t first = 0; first < tiles; first += step) {
    const int64_t n = std::min(step, tiles - first), at = first * tokens;
    a.q.X = static_cast<const ST*>(all.q.X) + at * a.q.x_token;
    a.q.Y = static_cast<ST*>(all.q.Y) + at * a.q.y_token;
    a.q.positions = all.q.positions + at;
    a.slots = all.slots + at;
    for (int i = 0; i < 2; ++i) a.X[i] = static_cast<const ST*>(all.X[i]) + at * a.token[i];
    a.q.t = (int)std::min<int64_t>(n * tokens, all.q.t - at);
    const unsigned grid = (unsigned)(n * each);
    if (lanes == 8) rotary_cache_kernel<DT, BITS, 8><<<grid, 256, 0, s>>>(a);
    else if (lanes == 16) rotary_cache_kernel<DT, BITS, 16><<<grid, 256, 0, s>>>(a);
    else rotary_cache_kernel<DT, BITS, 32><<<grid, 256, 0, s>>>(a);
  }
}

}  // namespace

void rotary_frequencies(double* freq, int64_t rot, double base, ptq_rotary_scaling scaling, double factor, double context, double slow, double fast) {
  const double pi = 3.14159265358979323846;
  if (scaling == PTQ_ROTARY_BASE && rot > 2) base *= std::pow(factor, (double)rot / (double)(rot - 2));
  for (int64_t i = 0; i < rot / 2; ++i) {
    double f = std::pow(base, -2.0 * (double)i / (double)rot);
    if (scaling == PTQ_ROTARY_LINEAR) f /= factor;
    if (scaling == PTQ_ROTARY_TURNS) {
      const double turns = context * f / (2.0 * pi), kept = std::min(1.0, std::max(0.0, (turns - slow) / (fast - slow)));
      f *= kept + (1.0 - kept) / factor;
    }
    freq[i] = f;
  }
}

ptq_status rotary_launch(const void* X, int64_t x_token, int64_t x_head, ptq_dtype dt, int64_t t, int64_t heads, int64_t d,
                         const int32_t* positions, const double* freq, int64_t rot, double scale, int interleaved, void* Y,
                         int64_t y_token, int64_t y_head, hipStream_t s) {
  const RotaryArgs a{X, Y, x_token, x_head, y_token, y_head, positions, freq, (int)t, (int)heads, (int)d, (int)rot, interleaved, 1, 1, scale};
  dt == PTQ_BF16 ? rotary_typed<PTQ_BF16>(a, s) : rotary_typed<PTQ_F32>(a, s);
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

ptq_status rotary_kv_cache_write_launch(const void* Q, int64_t q_token, int64_t q_head, int64_t hq, const void* K, int64_t k_token,
                                        int64_t k_head, const void* V, int64_t v_token, int64_t v_head, ptq_dtype dt, int64_t t, int64_t hkv,
                                        int64_t d, const int32_t* positions, const double* freq, int64_t rot, double scale, int interleaved,
                                        const int32_t* slots, int bits, uint8_t* codes, float* scales, uint8_t* zeros, int64_t pages,
                                        int64_t page, void* Q_out, int64_t o_token, int64_t o_head, hipStream_t s) {
  RotaryCacheArgs a{};
  a.q = RotaryArgs{Q, Q_out, q_token, q_head, o_token, o_head, positions, freq, (int)t, (int)hq, (int)d, (int)rot, interleaved, 1, 1, scale};
  a.X[0] = K, a.X[1] = V;
  a.token[0] = k_token, a.token[1] = v_token, a.head[0] = k_head, a.head[1] = v_head;
  a.slots = slots;
  a.c = KvCache{codes, scales, zeros, pages, (int)hkv, __builtin_ctz((unsigned)page), (int)(d * bits / 8)};
  if (dt == PTQ_BF16) bits == 8 ? rotary_cache_typed<PTQ_BF16, 8>(a, s) : rotary_cache_typed<PTQ_BF16, 4>(a, s);
  else bits == 8 ? rotary_cache_typed<PTQ_F32, 8>(a, s) : rotary_cache_typed<PTQ_F32, 4>(a, s);
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

}  // namespace ptq
