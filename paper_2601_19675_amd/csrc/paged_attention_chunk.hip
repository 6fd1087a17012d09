// Attention over the paged quantized cache for chunks of tokens: more than 16 query rows that share a key head.
//
// Rows are the (token, head) pairs of a key head's group.  A wave has 32 of them, the columns of the 32 x 32 x 16 matrix
// instruction; the workgroup's eight waves (four for d > 128) go through the keys together, 64 at a time.  Half of them bring a tile's key
// codes, the other half its value codes: they are asked for a tile ahead, made float16 in registers once for all rows, and
// written to LDS as the matrix instructions want them -- keys [key][d] as the whole numbers code - zero, values [d][key], transposed
// with byte permutes.  What the page table, scales and zeros say of a tile is brought by the first wave another tile ahead.
//
//   S' = K Q'   (keys are rows, so a lane has scores of one query row, and they leave the instruction in the order in which the
//               second product takes them: no exchange)        y = ks S',   p = 2^(y f - M),   O' = V' p
//
// Q' is the row times a power of two that makes it fit float16, f = softmax_scale log2(e) over that power.  The running maximum moves
// only when a score is 2^8 above it; until then weights are below 2^8.  V' = vs 2^(7 - E) (code - zero) in float16, E the largest
// exponent of a value's scale so far (all products stay below 2^15; when E grows, sums shrink).  Roundings beside those to float16:
// float32.
//
// Bound: the matrix instructions (16 d flops a score) and the vector unit beside them (eight instruction slots a score, four of them
// the power of two) in about equal parts at d = 128.
#include <algorithm>

#include "paged_attention.h"
#include "stored_rows.h"

namespace ptq {
namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16v;

constexpr int kTile = 64;   // keys

template <int DP>
struct Chunk {
  static constexpr int kThreads = DP > 128 ? 256 : 512;
  static constexpr int kWaves = kThreads / 64, kRows = 32 * kWaves;
  static constexpr int kKeyPitch = DP <= 64 ? 128 : DP <= 128 ? 256 : 512;   // bytes of a key
  static constexpr int kKeyBytes = kTile * kKeyPitch, kValBytes = DP * kTile * 2;
  static constexpr int kBuffer = kKeyBytes + kValBytes;
  static constexpr int kHalf = kThreads / 2;
  static constexpr int kKeyUnits = (4 * DP + kHalf - 1) / kHalf;   // 16 codes of a key each, per thread
  static constexpr int kValUnits = (2 * DP + kHalf - 1) / kHalf;   // eight channels of four keys each
};
// 16-byte chunk c of a row lies at c ^ turn: rows that are read together are spread over the banks
template <int DP>
__device__ __forceinline__ int key_turn(int key) { return DP <= 64 ? (key & 7) ^ ((key >> 3) & 1) : key & 15; }
__device__ __forceinline__ int val_turn(int d) { return (d & 7) ^ ((d >> 3) & 7); }
// keeps the compiler from holding a register for every address that follows from v
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// what is known of a tile's keys before their codes
struct Meta {
  int64_t at[kTile];      // byte offset of the row's codes
  float ks[kTile];        // scale of the key; NaN also where the value's is not finite
  uint32_t kz[kTile];     // bits of 1024 + zero, twice
  uint16_t vz[kTile];     // ... of the value, once
  uint16_t vs[kTile];     // float16 of vs 2^(7 - E)
  uint64_t seen;          // keys that are there
  int e;                  // E
};

__device__ __forceinline__ int wave_max_int(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(v, v, kDppSwapPairs, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, kDppSwapHalfQuads, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, kDppHalfMirror, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, kDppMirror, 0xf, 0xf, false));
  return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
             max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

template <int BITS, int DP>
__global__ __launch_bounds__(Chunk<DP>::kThreads) void attend_chunk_kernel(AttendArgs a, int tiles) {
  using C = Chunk<DP>;
  constexpr int kSteps = DP / 16, kOut = DP / 32;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  Meta* metas = reinterpret_cast<Meta*>(smem + 2 * C::kBuffer);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, h = lane >> 5;

  // groups (sequence, key head) go round the dies, so that a group's row tiles share its codes in one L2; the last rows, which
  // see most, first
  const int items = tiles * a.splits, die = blockIdx.x & 7, idx = blockIdx.x >> 3;
  const int group = idx / items * 8 + die, item = idx % items;
  if (group >= a.b * a.c.heads) return;
  const int seq = group / a.c.heads, head = group % a.c.heads, tile = tiles - 1 - item % tiles, split = item / tiles;
  const Sequence q = sequence_of(a, seq);
  const int rows = min(q.queries, a.max_q) * a.group, row0 = tile * C::kRows;
  if (row0 >= rows) return;
  const int from = q.begin + split * a.split_keys;
  if (split > 0 && from >= q.end) return;

  // the keys that some row of the workgroup sees, in this split
  int lo, hi, lo_a, hi_a, lo_b, hi_b;
  visible(a, q, row0 / a.group, lo, hi);
  visible(a, q, (min(row0 + C::kRows, rows) - 1) / a.group, lo_b, hi_b);
  const int begin = max(from, lo & ~(kTile - 1)), end = min(min(hi_b, q.end), a.splits > 1 ? from + a.split_keys : q.end);
  const int count = end > begin ? (end - begin + kTile - 1) / kTile : 0;
  // ... and those that the wave's rows see: some of them [lo_a, hi_b), all of them [lo_b, hi_a)
  const int wrow = row0 + 32 * wave;
  const bool working = wrow < rows;
  if (working) {
    visible(a, q, wrow / a.group, lo_a, hi_a);
    visible(a, q, (min(wrow + 32, rows) - 1) / a.group, lo_b, hi_b);
  }

  const int row = wrow + r, token = q.first + row / a.group, qhead = head * a.group + row % a.group;
  const bool live = row < rows;
  visible(a, q, live ? row / a.group : 0, lo, hi);
  if (!live) hi = 0;
  f16x8 fq[kSteps];
  float factor;
  {
    Run<PTQ_BF16, 8> raw[kSteps];
    const uint16_t* Q = a.Q + (live ? token * a.q_token + qhead * a.q_head : 0);
    float top = 0.f;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) raw[u] = load_run<PTQ_BF16, 8, false>(Q, 16 * u + 8 * h, a.d);
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      float v[8];
      run_to_f32<PTQ_BF16, 8>(raw[u], 16 * u + 8 * h, live ? a.d : 0, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.f);
    }
    top = fmaxf(top, __shfl_xor(top, 32));
    const int e = __builtin_amdgcn_frexp_expf(top);
    factor = fmaxf(ldexpf(fabsf(a.scale), e - 15), 0x1p-126f);   // positive: a score that is not there is -inf times it
    const float lift = a.scale < 0.f ? -1.f : 1.f;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      float v[8];
      uint32_t w[4];
      run_to_f32<PTQ_BF16, 8>(raw[u], 16 * u + 8 * h, live ? a.d : 0, v);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = __builtin_bit_cast(uint32_t, to_f16(ldexpf(lift * v[2 * i], 15 - e), ldexpf(lift * v[2 * i + 1], 15 - e)));
      fq[u] = f16x8_of(w[0], w[1], w[2], w[3]);
    }
  }

  const int64_t plane = (a.c.pages * a.c.heads) << a.c.page_shift;
  const uint8_t* VC = a.c.codes + plane * a.c.row_bytes;
  const int32_t* table = a.table + seq * a.ldt;
  const int inside = (1 << a.c.page_shift) - 1;

  // ---- what comes before the codes: the first wave, a lane per key
  struct MetaLoad { int page; float ks, vs; int kz, vz; };
  auto page_of = [&](int t) {   // tile t's key `lane`
    const int key = begin + t * kTile + lane;
    const int p = table[min(key, q.length - 1) >> a.c.page_shift];
    return key < q.end && (uint32_t)p < (uint64_t)a.c.pages ? p : -1;
  };
  auto row_of = [&](int t, int page) -> int64_t {
    return page < 0 ? 0 : (((int64_t)page * a.c.heads + head) << a.c.page_shift) + ((begin + t * kTile + lane) & inside);
  };
  auto meta_load = [&](int t, int page) {
    const int64_t at = row_of(t, page);
    MetaLoad m{page, a.c.scales[at], a.c.scales[plane + at], a.c.zeros[at], a.c.zeros[plane + at]};
    return m;
  };
  int top_e = -1000;
  auto meta_store = [&](int t, const MetaLoad& m) {
    Meta& o = metas[t & 3];
    const bool there = m.page >= 0, good = fabsf(m.vs) < INFINITY && there;
    top_e = max(top_e, wave_max_int(good && m.vs != 0.f ? __builtin_amdgcn_frexp_expf(m.vs) : -1000));
    o.at[lane] = row_of(t, m.page) * a.c.row_bytes;
    o.ks[lane] = good ? m.ks : there ? __uint_as_float(0x7fc00000u) : 0.f;
    const uint32_t z = 0x6400u | m.kz;
    o.kz[lane] = z | (z << 16);
    o.vz[lane] = (uint16_t)(0x6400u | m.vz);
    o.vs[lane] = __builtin_bit_cast(uint16_t, (_Float16)(good ? ldexpf(m.vs, 7 - top_e) : 0.f));
    const uint64_t seen = __ballot(there);
    if (lane == 0) {
      o.seen = seen;
      o.e = top_e;
    }
  };

  // ---- codes of tile t: loads, then float16 in LDS
  constexpr int KW = BITS / 2, VW = BITS / 4;   // words of a unit: 16 codes | eight codes
  const bool key_half = wave < C::kWaves / 2;
  const int hid = tid % C::kHalf;
  struct Codes { uint32_t w[C::kKeyUnits * KW > C::kValUnits * 4 * VW ? C::kKeyUnits * KW : C::kValUnits * 4 * VW]; };
  auto codes_load = [&](int t, Codes& c) {
    const Meta& m = metas[t & 3];
    if (key_half) {
#pragma unroll
      for (int i = 0; i < C::kKeyUnits; ++i) {
        const int u = i * C::kHalf + hid, key = min(u / (DP / 16), kTile - 1), part = u % (DP / 16);
        const AnyWords<KW, 4> w = *reinterpret_cast<const AnyWords<KW, 4>*>(a.c.codes + m.at[key] + (16 * part < a.d ? part * 2 * BITS : 0));
#pragma unroll
        for (int j = 0; j < KW; ++j) c.w[i * KW + j] = w.w[j];
      }
    } else {
#pragma unroll
      for (int i = 0; i < C::kValUnits; ++i) {
        const int u = i * C::kHalf + hid, run = min(u / (DP / 8), kTile / 4 - 1), part = u % (DP / 8);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const AnyWords<VW, 4> w = *reinterpret_cast<const AnyWords<VW, 4>*>(VC + m.at[4 * run + k] + (8 * part < a.d ? part * BITS : 0));
#pragma unroll
          for (int j = 0; j < VW; ++j) c.w[(i * 4 + k) * VW + j] = w.w[j];
        }
      }
    }
  };
  auto codes_store = [&](int t, const Codes& c) {
    const Meta& m = metas[t & 3];
    char* buffer = smem + (t & 1) * C::kBuffer;
    if (key_half) {
#pragma unroll
      for (int i = 0; i < C::kKeyUnits; ++i) {
        const int u = i * C::kHalf + hid, key = u / (DP / 16), part = u % (DP / 16);
        if (key >= kTile) continue;
        const Zeros z = zeros_of<BITS>(m.kz[key]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          f16x8 f = row_codes<BITS>(&c.w[i * KW + j * (KW / 2)], z);
          if (DP != a.d && 16 * part >= a.d) f = f16x8_of(0, 0, 0, 0);
          *reinterpret_cast<f16x8*>(buffer + ((key * C::kKeyPitch + ((2 * part) ^ key_turn<DP>(key)) * 16) ^ (16 * j))) = f;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < C::kValUnits; ++i) {
        const int u = i * C::kHalf + hid, run = u / (DP / 8), part = u % (DP / 8);
        if (run >= kTile / 4) continue;
        const uint2 zz = *reinterpret_cast<const uint2*>(&m.vz[4 * run]), ss = *reinterpret_cast<const uint2*>(&m.vs[4 * run]);
        const uint32_t* w = &c.w[i * 4 * VW];
        uint32_t f[8][2];   // channel, pair of keys
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const Zeros z = zeros_of<BITS>(p ? zz.y : zz.x);
          const uint32_t *w0 = w + 2 * p * VW, *w1 = w0 + VW;
          if constexpr (BITS == 8) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint32_t even = perm(w1[j], w0[j], 0x05010400u), odd = perm(w1[j], w0[j], 0x07030602u);
              f[4 * j][p] = h2_sub(low_bytes(even), z.by1);
              f[4 * j + 1][p] = h2_sub(high_bytes(even), z.by1);
              f[4 * j + 2][p] = h2_sub(low_bytes(odd), z.by1);
              f[4 * j + 3][p] = h2_sub(high_bytes(odd), z.by1);
            }
          } else {
            uint32_t even[4], odd[4];   // channels 0, 2, 4, 6 | 1, 3, 5, 7
            nibble_pairs(perm(w1[0], w0[0], 0x05040100u), z, even);
            nibble_pairs(perm(w1[0], w0[0], 0x07060302u), z, odd);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              f[2 * j][p] = even[j];
              f[2 * j + 1][p] = odd[j];
            }
          }
          const f16x2 s = __builtin_bit_cast(f16x2, p ? ss.y : ss.x);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j][p] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, f[j][p]) * s);
        }
        // keys 4 run .. of a group of 16 go where the scores' order has them: runs 0, 2, 1, 3
        const int slot = (run >> 2) * 4 + (((run & 1) << 1) | ((run >> 1) & 1));
        const int base = opaque(part * 8 * kTile * 2 + (((slot >> 1) ^ val_turn(8 * part)) * 16) + (slot & 1) * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j)   // val_turn(8 part + j) = val_turn(8 part) ^ j
          *reinterpret_cast<uint2*>(buffer + C::kKeyBytes + (base ^ (16 * j)) + j * kTile * 2) = uint2{f[j][0], f[j][1]};
      }
    }
  };

  f32x16v acc[kOut];
#pragma unroll
  for (int n = 0; n < kOut; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
  float m = kNoScore, l = 0.f;   // m in units of 1 / factor
  int e = -1000;

  const int key_at = r * C::kKeyPitch + ((h ^ key_turn<DP>(r)) * 16), val_at = r * kTile * 2 + ((h ^ val_turn(r)) * 16);
  auto compute = [&](int t) {
    const int key0 = begin + t * kTile;
    const Meta& meta = metas[t & 3];
    const char* buffer = smem + (t & 1) * C::kBuffer;
    const int key_base = opaque(key_at), val_base = opaque(val_at);
    const uint64_t seen = meta.seen;
    const int now = __builtin_amdgcn_readfirstlane(meta.e);
    if (now != e) {   // (the first tile among others)
      const float f = e == -1000 ? 1.f : ldexpf(1.f, e - now);
#pragma unroll
      for (int n = 0; n < kOut; ++n) acc[n] *= f;
      e = now;
    }
    float y[2][16];
    float top = kNoScore;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      f32x16v s;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
      for (int u = 0; u < kSteps; ++u) {   // (turns of keys 32 apart are the same, and leave chunk bit 4 alone)
        const f16x8 f = *reinterpret_cast<const f16x8*>(buffer + (key_base ^ (32 * (u & 7))) + (u >> 3) * 256 + k * 32 * C::kKeyPitch);
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, fq[u], s, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 ks = *reinterpret_cast<const f32x4*>(&meta.ks[32 * k + 8 * j + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[k][4 * j + i] = s[4 * j + i] * ks[i];
      }
    }
    if (key0 < lo_b || key0 + kTile > hi_a || ~seen != 0) {   // some row does not see some key
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 32 * k + 8 * (i >> 2) + 4 * h + (i & 3), key = key0 + at;
          if (!(key >= lo && key < hi && ((seen >> at) & 1))) y[k][i] = -INFINITY;
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, y[k][i]);
    if (__any((top - m) * factor > 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = fmaxf(m, top), f = exp2_fast((m - next) * factor);
      m = next;
      l *= f;
#pragma unroll
      for (int n = 0; n < kOut; ++n) acc[n] *= f;
    }
    const float M = fmaxf(m * factor, kNoScore);   // (finite where nothing has been seen: -inf - M stays -inf)
    f16x8 weights[4];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = exp2_fast(fmaf(y[k][8 * u + 2 * i], factor, -M)), p1 = exp2_fast(fmaf(y[k][8 * u + 2 * i + 1], factor, -M));
          l += p0 + p1;
          w[i] = __builtin_bit_cast(uint32_t, to_f16(p0, p1));
        }
        weights[2 * k + u] = f16x8_of(w[0], w[1], w[2], w[3]);
      }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int n = 0; n < kOut; ++n) {
        // val_turn(32 n + r) = val_turn(r) ^ 4 (n & 1)
        const f16x8 f = *reinterpret_cast<const f16x8*>(buffer + C::kKeyBytes + (val_base ^ (32 * (u ^ (2 * (n & 1))))) + n * 32 * kTile * 2);
        acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, weights[u], acc[n], 0, 0, 0);
      }
  };

  if (count > 0) {
    MetaLoad ml;
    int next_page = -1;
    if (wave == 0) {
      meta_store(0, meta_load(0, page_of(0)));
      meta_store(1, meta_load(1, page_of(1)));
      next_page = page_of(2);
    }
    __syncthreads();
    Codes c;
    codes_load(0, c);
    codes_store(0, c);
    __syncthreads();
    for (int t = 0; t < count; ++t) {
      if (t + 1 < count) codes_load(t + 1, c);
      if (wave == 0) {
        ml = meta_load(t + 2, next_page);
        next_page = page_of(t + 3);
      }
      const int key0 = begin + t * kTile;
      if (working && key0 < hi_b && key0 + kTile > lo_a) compute(t);
      if (t + 1 < count) codes_store(t + 1, c);
      if (wave == 0) meta_store(t + 2, ml);
      __syncthreads();
    }
  }
  if (!live) return;
  l += __shfl_xor(l, 32);
  const float unit = e == -1000 ? 0.f : ldexpf(1.f, e - 7);
  if (a.splits > 1) {
    const int64_t at = ((int64_t)split * a.t + token) * a.hq + qhead;
    if (h == 0) {
      a.ml[2 * at] = m == kNoScore ? kNoScore : m * factor;
      a.ml[2 * at + 1] = l;
    }
#pragma unroll
    for (int n = 0; n < kOut; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 32 * n + 8 * j + 4 * h;
        if (d < a.d)
          *reinterpret_cast<f32x4*>(a.part + at * a.d + d) =
              f32x4{acc[n][4 * j] * unit, acc[n][4 * j + 1] * unit, acc[n][4 * j + 2] * unit, acc[n][4 * j + 3] * unit};
      }
  } else {
    const float inv = l == 0.f ? 0.f : unit / l;
    uint16_t* O = a.O + token * a.o_token + qhead * a.o_head;
#pragma unroll
    for (int n = 0; n < kOut; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float v[4] = {acc[n][4 * j] * inv, acc[n][4 * j + 1] * inv, acc[n][4 * j + 2] * inv, acc[n][4 * j + 3] * inv};
        const int d = 32 * n + 8 * j + 4 * h;
        if (d < a.d) store_run<PTQ_BF16, 4, false>(O, d, a.d, v);
      }
  }
}

template <int BITS, int DP>
bool chunk_launch(const AttendArgs& a, hipStream_t s) {
  using C = Chunk<DP>;
  constexpr int kBytes = 2 * C::kBuffer + 4 * (int)sizeof(Meta);
  if (!lds_opt_in<attend_chunk_kernel<BITS, DP>>(kBytes)) return false;
  const int tiles = (int)ceil_div((int64_t)a.max_q * a.group, C::kRows);
  const int64_t blocks = ceil_div((int64_t)a.b * a.c.heads, 8) * 8 * tiles * a.splits;
  if (blocks > INT32_MAX) return false;
  attend_chunk_kernel<BITS, DP><<<(unsigned)blocks, C::kThreads, kBytes, s>>>(a, tiles);
  return true;
}

}  // namespace

int paged_attention_chunk_rows(int64_t d) { return d > 128 ? Chunk<256>::kRows : Chunk<128>::kRows; }

ptq_status paged_attention_chunk_launch(const AttendArgs& a, int bits, hipStream_t s) {
  const bool launched = bits == 8 ? (a.d <= 64 ? chunk_launch<8, 64>(a, s) : a.d <= 96 ? chunk_launch<8, 96>(a, s)
                                     : a.d <= 128 ? chunk_launch<8, 128>(a, s) : chunk_launch<8, 256>(a, s))
                                  : (a.d <= 64 ? chunk_launch<4, 64>(a, s) : a.d <= 96 ? chunk_launch<4, 96>(a, s)
                                     : a.d <= 128 ? chunk_launch<4, 128>(a, s) : chunk_launch<4, 256>(a, s));
  return launched ? PTQ_OK : PTQ_ERR_HIP;
}

}  // namespace ptq
