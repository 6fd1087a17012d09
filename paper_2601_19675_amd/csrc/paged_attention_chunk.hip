// Attention over the paged quantized cache for chunks of tokens: more than 16 query rows that share a key head.
//
// Rows are the (token, head) pairs of a key head's group.  A wave has 32 of them, the columns of the 32 x 32 x 16 matrix
// instruction; the workgroup's eight waves (four for d > 128) go through the keys together, 64 at a time.  Half of them bring a tile's key
// codes, the other half its value codes: they are asked for two tiles ahead, made float16 in registers once for all rows, and
// written to LDS as the matrix instructions want them -- keys [key][d] as the whole numbers code - zero, values [d][key], transposed
// with byte permutes.  What the page table, scales and zeros say of a tile is brought by the waves in turn, four tiles ahead.
//
//   S' = K Q'   (keys are rows, so a lane has scores of one query row, and they leave the instruction in the order in which the
//               second product takes them: no exchange)        y = ks S',   p = 2^(y f - M),   O' = V' p
//
// Q' is the row times a power of two that makes it fit float16, f = softmax_scale log2(e) over that power.  The running maximum M, a whole
// number, moves only when one of the row's scores is 2^8 above it; until then weights are below 2^8.  V' = 2^4 vs (code - zero) in float16, whose
// normal numbers hold that for scales from 2^-18 up to 2^4 (4 bits: 2^8).  Roundings: weights and V' to float16, 2^-11 each, of which
// bfloat16 outputs see nothing; the sum of the weights is of the rounded ones, a channel of ones beside the values', so that the rounding of a
// weight drops out where the values are alike.  All sums are float32.
//
// A value's scale outside that range is brought to its nearer end by a power of two 2^x, which goes into the weights instead: from the first such key
// that a row sees on, M is the maximum of y f + x and the numerator's weights are 2^(y f + x - M), while the sum is that of 2^(y f - m), m a
// maximum of its own; the row joins them at its end.  This is decided by row, and nothing that other rows see enters into it: a key that a row does
// not see leaves its result as it is, bit by bit.  (Such a row, or a tile with such a key, nearly doubles its wave's turn: the case below takes 1470 us
// with all scales out of range.)
//
// Bound: a turn of one half of the workgroup, softmax (a score takes about eleven instruction slots, four of them the power of two) and the codes'
// way to float16, while the other half has the matrix unit (16 d flops a score).  At d = 128 a turn takes 2600 cycles, of which the matrix
// instructions are 1150; vector instructions are issued 44 % of the time, the matrix unit is busy 40 %: neither is full, a wave to a SIMD waits for
// its own results.  Chunks of 2048 and 1035 tokens against 16384 and 8283 keys, 32 heads of 128 channels over 8: 808 to 835 us by the card,
// 775 to 800 TFLOP/s of float16 products.
//
// Tiles of rows differ in how many keys they see.  Where that would leave compute units idle, all tiles of keys of all tiles of rows are laid
// end to end and dealt out in equal shares, and a second kernel joins what several workgroups have of a tile of rows.
#include <algorithm>

#include "paged_attention.h"
#include "static_for.h"
#include "stored_rows.h"

namespace ptq {
namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16v;

constexpr int kTile = 64;   // keys
// Workgroups that share the work, one to a compute unit.  It is counted in tiles of keys, and what comes before and after an item's
// tiles (queries and first codes 13000 cycles, outputs 8000, a tile 3200 to 5900) as kStart of them.
constexpr int kShares = kChunkShares, kStart = 4, kLeastShare = 2 * kStart;
constexpr int kValueLift = 4;         // V' = 2^kValueLift vs (code - zero)
constexpr int kMetas = 8, kMetaAhead = 4;   // tiles whose Meta is in LDS, and how far before its turn it is brought there

template <int DP>
struct Chunk {
  static constexpr int kThreads = DP > 128 ? 256 : 512;
  static constexpr int kWaves = kThreads / 64, kRows = 32 * kWaves;
  static constexpr int kKeyPitch = DP <= 64 ? 128 : DP <= 128 ? 256 : 512;   // bytes of a key
  static constexpr int kKeyBytes = kTile * kKeyPitch, kValBytes = DP * kTile * 2;
  static constexpr bool kTurns = DP <= 128;                  // two halves of the workgroup take turns at the matrix instructions
  static constexpr int kRing = 2;                            // tiles of codes in LDS
  static constexpr int kBuffers = kRing * (kKeyBytes + kValBytes);
  // Steps of d whose queries wait in LDS: at d = 128 the registers of two waves to a SIMD do not hold all of them beside what a turn needs
  // (and what the compiler spills goes to memory: 1584 us in place of 914)
  static constexpr int kQuerySteps = DP == 128 ? 4 : 0;
  static constexpr int kQueryBytes = kQuerySteps * 16 * 2 * kRows;
  static constexpr int kApartBytes = 2 * 4 * kThreads;       // what a row that has seen a value out of range keeps, by lane
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
  uint16_t vs[kTile];     // float16 of vs 2^(kValueLift - x)
  float x[kTile];         // 0, or what brings vs into range
  uint64_t seen;          // keys that are there
  int odd;                // whether an x is not 0
};

// the keys that some row of a tile of rows sees
template <int ROWS>
__device__ __forceinline__ void span_of(const AttendArgs& a, const Sequence& q, int tile, int& begin, int& end) {
  const int rows = min(q.queries, a.max_q) * a.group;
  int unused;
  visible(a, q, tile * ROWS / a.group, begin, unused);
  visible(a, q, (min((tile + 1) * ROWS, rows) - 1) / a.group, unused, end);
  begin = max(q.begin, begin & ~(kTile - 1));
  end = min(end, q.end);
}
// what a tile of rows counts for
template <int ROWS>
__device__ __forceinline__ int item_work(const AttendArgs& a, int seq, int tile) {
  const Sequence q = sequence_of(a, seq);
  if (tile * ROWS >= min(q.queries, a.max_q) * a.group) return 0;
  int begin, end;
  span_of<ROWS>(a, q, tile, begin, end);
  return kStart + max(0, end - begin + kTile - 1) / kTile;
}

template <int BITS, int DP>
__global__ __launch_bounds__(Chunk<DP>::kThreads) void attend_chunk_kernel(AttendArgs a, int tiles, int first_group) {
  using C = Chunk<DP>;
  constexpr int kSteps = DP / 16, kOut = DP / 32;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  Meta* metas = reinterpret_cast<Meta*>(smem + C::kBuffers + C::kQueryBytes + C::kApartBytes);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // the workgroup's share: `left` pieces of work from piece `off` of an item on; `at` is the item's place in the order of all
  int seq, head, tile, off = 0, left = INT32_MAX, at = 0, each = 1;
  int4 begun{0, 0, 0, 0};   // parts of the item that this share begins and does not end (0: there is none); its sequence, key head, tile
  int4* const begun_at = reinterpret_cast<int4*>(a.parts) + (blockIdx.x & 7) * (kShares / 8) + (blockIdx.x >> 3);
  if (a.splits > 1) {
    // consecutive shares on one die, where they find each other's codes in the L2
    const int pairs = a.b * tiles, lane = threadIdx.x & 63;
    int total = 0;   // of one key head
    for (int p0 = 0; p0 < pairs; p0 += kWave) total += p0 + lane < pairs ? item_work<C::kRows>(a, (p0 + lane) / tiles, (p0 + lane) % tiles) : 0;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) total += __shfl_xor(total, o);
    total = __builtin_amdgcn_readfirstlane(total);
    const int all = total * a.c.heads;
    each = max(kLeastShare, (all + kShares - 1) / kShares);
    const int64_t mine = ((blockIdx.x & 7) * (kShares / 8) + (blockIdx.x >> 3)) * (int64_t)each;
    if (mine >= all) {
      if (threadIdx.x == 0) *begun_at = begun;
      return;
    }
    left = min(each, all - (int)mine);
    head = (int)mine / total;
    const int within = (int)mine % total;
    int before = 0;
    for (int p0 = 0;; p0 += kWave) {   // the first item that reaches past `within`
      const int n = p0 + lane < pairs ? item_work<C::kRows>(a, (p0 + lane) / tiles, (p0 + lane) % tiles) : 0;
      int upto = n;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
      }
      const uint64_t past = __ballot(before + upto > within);
      if (past) {
        const int p = __builtin_ctzll(past);
        seq = (p0 + p) / tiles;
        tile = (p0 + p) % tiles;
        before += __builtin_amdgcn_readlane(upto, p) - __builtin_amdgcn_readlane(n, p);
        break;
      }
      before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    off = within - before;
    at = (int)mine - off;
  } else {
    // groups (sequence, key head) go round the dies, so that a group's row tiles share its codes in one L2; the last rows, which
    // see most, first
    const int die = blockIdx.x & 7, idx = blockIdx.x >> 3, group = first_group + idx / tiles * 8 + die;
    if (group >= a.b * a.c.heads) return;
    seq = group / a.c.heads, head = group % a.c.heads, tile = tiles - 1 - idx % tiles;
  }

  for (;;) {
  // (opaque: what follows from it is not kept in registers from one item to the next)
  const int tid = opaque(threadIdx.x), lane = tid & 63, r = lane & 31, h = lane >> 5;
  const Sequence q = sequence_of(a, seq);
  const int rows = min(q.queries, a.max_q) * a.group, row0 = tile * C::kRows;
  if (row0 >= rows) {   // (a share has something to do yet)
    if (a.splits == 1) return;
    tile = 0;
    if (++seq == a.b) {
      seq = 0;
      ++head;
    }
    continue;
  }

  // the keys that some row of the workgroup sees, and those of them in this share
  int lo, hi, lo_a, hi_a, lo_b, hi_b, begin, end;
  span_of<C::kRows>(a, q, tile, begin, end);
  const int whole = kStart + max(0, end - begin + kTile - 1) / kTile, take = min(whole - off, left);
  const bool alone = take == whole;
  end = min(end, begin + max(0, off + take - kStart) * kTile);
  begin += max(0, off - kStart) * kTile;
  const int count = end > begin ? (end - begin + kTile - 1) / kTile : 0;
  // ... and those that the wave's rows see: some of them [lo_a, hi_b), all of them [lo_b, hi_a)
  const int wrow = row0 + 32 * wave;
  const bool working = wrow < rows;
  if (working) {
    visible(a, q, wrow / a.group, lo_a, hi_a);
    visible(a, q, (min(wrow + 32, rows) - 1) / a.group, lo_b, hi_b);
  }

  const int64_t plane = (a.c.pages * a.c.heads) << a.c.page_shift;
  const uint8_t* VC = a.c.codes + plane * a.c.row_bytes;
  const int32_t* table = a.table + seq * a.ldt;
  const int inside = (1 << a.c.page_shift) - 1;

  // ---- what comes before the codes: a wave's tiles are every kWaves-th, a lane per key, so that it has that many tiles' time for its
  // loads
  struct MetaLoad { int page; float ks, vs; int kz, vz; };
  auto page_of = [&](int t) {   // tile t's key `lane`
    const int key = begin + t * kTile + lane;
    const int p = table[min(key, q.length - 1) >> a.c.page_shift];
    return key < end && (uint32_t)p < (uint64_t)a.c.pages ? p : -1;
  };
  auto row_of = [&](int t, int page) -> int64_t {
    return page < 0 ? 0 : (((int64_t)page * a.c.heads + head) << a.c.page_shift) + ((begin + t * kTile + lane) & inside);
  };
  auto meta_load = [&](int t, int page) {
    const int64_t at = row_of(t, page);
    MetaLoad m{page, a.c.scales[at], a.c.scales[plane + at], a.c.zeros[at], a.c.zeros[plane + at]};
    return m;
  };
  auto meta_store = [&](int t, const MetaLoad& m) {
    Meta& o = metas[t & (kMetas - 1)];
    // scales of mantissa 2^e, 0.5 <= mantissa < 1, that float16's normal numbers hold, 255 or 15 times as large too
    constexpr int kLow = -13 - kValueLift, kHigh = (BITS == 8 ? 8 : 12) - kValueLift;
    const bool there = m.page >= 0, good = there && fabsf(m.vs) < INFINITY;
    const int e = __builtin_amdgcn_frexp_expf(m.vs), near = min(max(e, kLow), kHigh);
    const int x = good && m.vs != 0.f ? e - near : 0;
    o.at[lane] = row_of(t, m.page) * a.c.row_bytes;
    o.ks[lane] = good ? m.ks : there ? __uint_as_float(0x7fc00000u) : 0.f;
    const uint32_t z = 0x6400u | m.kz;
    o.kz[lane] = z | (z << 16);
    o.vz[lane] = (uint16_t)(0x6400u | m.vz);
    o.vs[lane] = __builtin_bit_cast(uint16_t, (_Float16)(good ? ldexpf(m.vs, kValueLift - x) : 0.f));
    o.x[lane] = (float)x;
    const uint64_t seen = __ballot(there), odd = __ballot(x != 0);
    if (lane == 0) {
      o.seen = seen;
      o.odd = odd != 0;
    }
  };

  const int row = wrow + r, token = q.first + row / a.group, qhead = head * a.group + row % a.group;
  const bool live = row < rows;
  visible(a, q, live ? row / a.group : 0, lo, hi);
  if (!live) hi = 0;
  constexpr int kHeld = kSteps - C::kQuerySteps;   // steps of d of the queries in registers
  f16x8 fq[kHeld];
  char* const queries = smem + C::kBuffers + (wave * 64 + lane) * 16;   // the others: [step][wave][lane]
  float factor;
  MetaLoad ml;
  int next_page = -1;
  {
    // the wave's first tile of Meta, and the pages of the one after: asked for around the queries
    int page = -1;
    if (count > 0) {
      page = page_of(wave);
      next_page = page_of(wave + C::kWaves);
    }
    Run<PTQ_BF16, 8> raw[kSteps];
    const uint16_t* Q = a.Q + (live ? token * a.q_token + qhead * a.q_head : 0);
    float top = 0.f;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) raw[u] = load_run<PTQ_BF16, 8, false>(Q, 16 * u + 8 * h, a.d);
    if (count > 0) ml = meta_load(wave, page);
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
      if (u < kHeld) fq[u < kHeld ? u : 0] = f16x8_of(w[0], w[1], w[2], w[3]);
      else *reinterpret_cast<f16x8*>(queries + (u - kHeld) * C::kThreads * 16) = f16x8_of(w[0], w[1], w[2], w[3]);
    }
  }

  // ---- codes of tile t: loads, then float16 in LDS
  constexpr int KW = BITS / 2, VW = BITS / 4;   // words of a unit: 16 codes | eight codes
  const bool key_half = wave < C::kWaves / 2;
  const int hid = tid % C::kHalf;
  // (a vector, written as a whole: the compiler would merge the two halves' stores into an array, whose address is then not known, and send
  // them through memory, right behind the loads)
  constexpr int kCodeWords = C::kKeyUnits * KW > C::kValUnits * 4 * VW ? C::kKeyUnits * KW : C::kValUnits * 4 * VW;
  typedef uint32_t Codes __attribute__((ext_vector_type(kCodeWords)));
  auto codes_load = [&](int t) -> Codes {
    const Meta& m = metas[t & (kMetas - 1)];
    Codes c = 0u;
    if (key_half) {
      Codes k = 0u;
#pragma unroll
      for (int i = 0; i < C::kKeyUnits; ++i) {
        const int u = i * C::kHalf + hid, key = min(u / (DP / 16), kTile - 1), part = u % (DP / 16);
        const AnyWords<KW, 4> w = *reinterpret_cast<const AnyWords<KW, 4>*>(a.c.codes + m.at[key] + (16 * part < a.d ? part * 2 * BITS : 0));
#pragma unroll
        for (int j = 0; j < KW; ++j) k[i * KW + j] = w.w[j];
      }
      c = k;
    } else {
      Codes v = 0u;
#pragma unroll
      for (int i = 0; i < C::kValUnits; ++i) {
        const int u = i * C::kHalf + hid, run = min(u / (DP / 8), kTile / 4 - 1), part = u % (DP / 8);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const AnyWords<VW, 4> w = *reinterpret_cast<const AnyWords<VW, 4>*>(VC + m.at[4 * run + k] + (8 * part < a.d ? part * BITS : 0));
#pragma unroll
          for (int j = 0; j < VW; ++j) v[(i * 4 + k) * VW + j] = w.w[j];
        }
      }
      c = v;
    }
    return c;
  };
  auto key_buffer = [&](int t) { return smem + t % C::kRing * C::kKeyBytes; };
  auto val_buffer = [&](int t) { return smem + C::kRing * C::kKeyBytes + t % C::kRing * C::kValBytes; };
  // what codes_store needs of Meta: zeros of the keys, or zeros and scales of the values
  constexpr int kGridWords = C::kKeyUnits > 4 * C::kValUnits ? C::kKeyUnits : 4 * C::kValUnits;
  typedef uint32_t Grids __attribute__((ext_vector_type(kGridWords)));
  auto grids_load = [&](int t) -> Grids {
    const Meta& m = metas[t & (kMetas - 1)];
    Grids g = 0u;
    if (key_half) {
      Grids k = 0u;
#pragma unroll
      for (int i = 0; i < C::kKeyUnits; ++i) k[i] = m.kz[min((i * C::kHalf + hid) / (DP / 16), kTile - 1)];
      g = k;
    } else {
      Grids v = 0u;
#pragma unroll
      for (int i = 0; i < C::kValUnits; ++i) {
        const int run = min((i * C::kHalf + hid) / (DP / 8), kTile / 4 - 1);
        const uint2 z = *reinterpret_cast<const uint2*>(&m.vz[4 * run]), s = *reinterpret_cast<const uint2*>(&m.vs[4 * run]);
        v[4 * i] = z.x;
        v[4 * i + 1] = z.y;
        v[4 * i + 2] = s.x;
        v[4 * i + 3] = s.y;
      }
      g = v;
    }
    return g;
  };
  auto codes_store = [&](int t, const Codes c, const Grids grid) {
    if (key_half) {
      char* buffer = key_buffer(t);
#pragma unroll
      for (int i = 0; i < C::kKeyUnits; ++i) {
        const int u = i * C::kHalf + hid, key = u / (DP / 16), part = u % (DP / 16);
        if (key >= kTile) continue;
        const Zeros z = zeros_of<BITS>(grid[i]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t w[KW / 2];
#pragma unroll
          for (int n = 0; n < KW / 2; ++n) w[n] = c[i * KW + j * (KW / 2) + n];
          f16x8 f = row_codes<BITS>(w, z);
          if (DP != a.d && 16 * part >= a.d) f = f16x8_of(0, 0, 0, 0);
          *reinterpret_cast<f16x8*>(buffer + ((key * C::kKeyPitch + ((2 * part) ^ key_turn<DP>(key)) * 16) ^ (16 * j))) = f;
        }
      }
    } else {
      char* buffer = val_buffer(t);
#pragma unroll
      for (int i = 0; i < C::kValUnits; ++i) {
        const int u = i * C::kHalf + hid, run = u / (DP / 8), part = u % (DP / 8);
        if (run >= kTile / 4) continue;
        uint32_t w[4 * VW];
#pragma unroll
        for (int n = 0; n < 4 * VW; ++n) w[n] = c[i * 4 * VW + n];
        uint32_t f[8][2];   // channel, pair of keys
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const Zeros z = zeros_of<BITS>(grid[4 * i + p]);
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
          const f16x2 s = __builtin_bit_cast(f16x2, (uint32_t)grid[4 * i + 2 + p]);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j][p] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, f[j][p]) * s);
        }
        // keys 4 run .. of a group of 16 go where the scores' order has them: runs 0, 2, 1, 3
        const int slot = (run >> 2) * 4 + (((run & 1) << 1) | ((run >> 1) & 1));
        const int base = opaque(part * 8 * kTile * 2 + (((slot >> 1) ^ val_turn(8 * part)) * 16) + (slot & 1) * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j)   // val_turn(8 part + j) = val_turn(8 part) ^ j
          *reinterpret_cast<uint2*>(buffer + (base ^ (16 * j)) + j * kTile * 2) = uint2{f[j][0], f[j][1]};
      }
    }
  };

  f32x16v acc[kOut];
#pragma unroll
  for (int n = 0; n < kOut; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[n][i] = 0.f;
  float M = kNoScore;
  // of a row that has seen a value out of range: the sum of its weights (before, a negative number) and what that is relative to
  f32x2* const own = reinterpret_cast<f32x2*>(smem + C::kBuffers + C::kQueryBytes) + threadIdx.x;
  *own = f32x2{-1.f, kNoScore};
  bool apart = false;   // whether a row of the wave has
  // the sum of the weights, in every element (the first one is used): one more channel of the values, which are 1 there
  f32x16v sum;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum[i] = 0.f;
  const f16x8 ones = f16x8_of(0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u);

  const int key_at = r * C::kKeyPitch + ((h ^ key_turn<DP>(r)) * 16), val_at = r * kTile * 2 + ((h ^ val_turn(r)) * 16);
  // What the matrix instructions do in one go: the values of tile t - 1 (with its weights), then the scores of tile t, either may be
  // missing.  Groups of instructions -- the channels' blocks of 16 keys; two steps of d of both halves of the keys -- whose operands are
  // read from LDS kReadAhead groups before: for itself the compiler reads each operand right before its instruction and waits.
  constexpr int kReadAhead = 1, kGroups = 4 + kSteps / 2, kPer = kOut > 4 ? kOut : 4;
  auto multiply = [&](auto had_, auto has_, int t, const f16x8 (&weights)[4], f32x16v (&s)[2]) {
    constexpr int kFirst = decltype(had_)::value ? 0 : 4, kLast = decltype(has_)::value ? kGroups : 4;
    const char *keys = key_buffer(t), *vals = val_buffer(t + C::kRing - 1);
    const int key_base = opaque(key_at), val_base = opaque(val_at);
    f16x8 f[kReadAhead + 1][kPer], fql[kReadAhead + 1][2];
    auto read = [&](auto g_) {
      constexpr int g = decltype(g_)::value, at = g % (kReadAhead + 1);
      if constexpr (g < 4) {
#pragma unroll
        for (int n = 0; n < kOut; ++n)   // val_turn(32 n + r) = val_turn(r) ^ 4 (n & 1)
          f[at][n] = *reinterpret_cast<const f16x8*>(vals + (val_base ^ (32 * (g ^ (2 * (n & 1))))) + n * 32 * kTile * 2);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {    // (turns of keys 32 apart are the same, and leave chunk bit 4 alone)
          const int u = 2 * (g - 4) + (i >> 1), k = i & 1;
          f[at][i] = *reinterpret_cast<const f16x8*>(keys + (key_base ^ (32 * (u & 7))) + (u >> 3) * 256 + k * 32 * C::kKeyPitch);
          if (k == 0 && u >= kHeld) fql[at][i >> 1] = *reinterpret_cast<const f16x8*>(queries + (u - kHeld) * C::kThreads * 16);
        }
      }
    };
    static_for<kReadAhead>([&](auto i_) {
      constexpr int g = kFirst + decltype(i_)::value;
      if constexpr (g < kLast) read(std::integral_constant<int, g>{});
    });
    static_for<kLast - kFirst>([&](auto i_) {
      constexpr int g = kFirst + decltype(i_)::value, at = g % (kReadAhead + 1);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (g + kReadAhead < kLast) read(std::integral_constant<int, g + kReadAhead>{});
      if constexpr (g < 4) {
#pragma unroll
        for (int n = 0; n < kOut; ++n) acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[at][n], weights[g], acc[n], 0, 0, 0);
        sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(ones, weights[g], sum, 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int u = 2 * (g - 4) + (i >> 1), k = i & 1;
          if (u == 0) s[k] = f32x16v{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          s[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f[at][i], u < kHeld ? fq[u < kHeld ? u : 0] : fql[at][i >> 1], s[k], 0, 0, 0);
        }
      }
    });
    __builtin_amdgcn_sched_barrier(0);
  };
  // Some value of the tile is out of range, or was of one before.  A row that sees such a value, or has, adds up its weights here, relative to a
  // maximum of their own, and goes on with log2 of weight times 2^x for a score; any other row keeps its scores.  Returns what they are to be multiplied
  // by.  (Four at a time: the registers hold no more.)
  auto out_of_range = [&](const Meta& meta, f32x16v (&s)[2]) {
    float top = -INFINITY;
    int sees = 0;
    auto four = [&](int j) {
      __builtin_amdgcn_sched_barrier(0);
      return *reinterpret_cast<const f32x4*>(&meta.x[8 * j + opaque(4 * h)]);
    };
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const f32x4 x = four(j);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y = s[j >> 2][4 * (j & 3) + i];
        sees |= (x[i] != 0.f) & (y != -INFINITY);
        top = fmaxf(top, y);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    sees |= __shfl_xor(sees, 32);
    top = fmaxf(top, __shfl_xor(top, 32)) * factor;
    f32x2 kept = *own;
    if (sees && kept[0] < 0.f) kept = f32x2{sum[0], M};
    const bool mine = !(kept[0] < 0.f);
    apart = __any(mine);
    const float m = top > kept[1] + 8.f ? ceilf(top) : kept[1];
    float more = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const f32x4 x = four(j);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y = s[j >> 2][4 * (j & 3) + i];
        more += exp2_fast(fmaf(y, factor, -m));
        s[j >> 2][4 * (j & 3) + i] = mine ? fmaf(y, factor, x[i]) : y;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    more += __shfl_xor(more, 32);
    if (mine) *own = f32x2{kept[0] * exp2_fast(kept[1] - m) + more, m};
    return mine ? 1.f : factor;
  };
  // the weights of tile t; what has been summed so far is brought to their maximum
  auto soften = [&](int t, f32x16v (&s)[2], f16x8 (&weights)[4]) {
    const int key0 = begin + t * kTile;
    const Meta& meta = metas[t & (kMetas - 1)];
    const uint64_t seen = meta.seen;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 ks = *reinterpret_cast<const f32x4*>(&meta.ks[32 * k + 8 * j + 4 * h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[k][4 * j + i] *= ks[i];
      }
    if (key0 < lo_b || key0 + kTile > hi_a || ~seen != 0) {   // some row does not see some key
      // counted from the half wave's first key: what is left are constants
      const int from_ = opaque(lo - key0 - 4 * h), to_ = opaque(hi - key0 - 4 * h);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t there = (uint32_t)(seen >> (32 * k)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 8 * (i >> 2) + (i & 3);
          s[k][i] = (32 * k + at >= from_) & (32 * k + at < to_) & (int)((there >> at) & 1) ? s[k][i] : -INFINITY;
        }
      }
    }
    float f = factor;
    if (apart | (__builtin_amdgcn_readfirstlane(meta.odd) != 0)) f = out_of_range(meta, s);
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[k][i]);
    top *= f;
    if (__any(top > M + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = top > M + 8.f ? ceilf(top) : M, shrink = exp2_fast(M - next);
      M = next;
      sum *= shrink;
#pragma unroll
      for (int n = 0; n < kOut; ++n) acc[n] *= shrink;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = exp2_fast(fmaf(s[k][8 * u + 2 * i], f, -M)), p1 = exp2_fast(fmaf(s[k][8 * u + 2 * i + 1], f, -M));
          w[i] = __builtin_bit_cast(uint32_t, to_f16(p0, p1));
        }
        weights[2 * k + u] = f16x8_of(w[0], w[1], w[2], w[3]);
      }
  };
  auto meet = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  if (count > 0) {
    int mine = wave;   // the wave's tile of Meta
    auto meta_next = [&]() {
      meta_store(mine, ml);
      mine += C::kWaves;
      ml = meta_load(mine, next_page);
      next_page = page_of(mine + C::kWaves);
    };
    static_assert(kMetaAhead <= C::kWaves, "");
    if (wave < kMetaAhead) meta_next();
    meet();
    // Tile t's codes are asked for two tiles before they are written to LDS, a tile before its turn.  Two tiles to a trip of the loop; those
    // past the last are like any other, with keys that nobody sees.
    const int trips = (count + 1) / 2;
    Codes c0 = codes_load(0), c1 = codes_load(1);
    codes_store(0, c0, grids_load(0));
    c0 = codes_load(2);
    meet();
    auto meta_due = [&](int t) {
      if (mine == t + kMetaAhead) meta_next();
    };
    f32x16v s[2];
    f16x8 weights[4];
    constexpr std::true_type yes;
    constexpr std::false_type no;
    if constexpr (C::kTurns) {
      // One half of the waves -- one on each SIMD -- multiplies (the values of the tile before, the keys of this one) while the other
      // half works out weights and makes the next tile's codes float16; then they change places.  The first half writes the
      // keys, the second the values: a slot is written when both halves have read what was in it.
      // (All waves in step, with a barrier per tile and one tile's codes on their way: 1006 us in place of 914 for two chunks of up to 2048
      // tokens, 32 heads of 128 channels, 16384 keys.)
      const bool second = wave >= C::kWaves / 2;
      if (second) meet();
      if (working) multiply(no, yes, 0, weights, s);
      meet();
      for (int i = 0, t = 0; i < trips; ++i, t += 2) {
        Grids g = grids_load(t + 1);
        if (working) soften(t, s, weights);
        codes_store(t + 1, c1, g);
        meet();
        c1 = codes_load(t + 3);
        meta_due(t);
        if (working) multiply(yes, yes, t + 1, weights, s);
        meet();
        g = grids_load(t + 2);
        if (working) soften(t + 1, s, weights);
        codes_store(t + 2, c0, g);
        meet();
        c0 = codes_load(t + 4);
        meta_due(t + 1);
        if (working) multiply(yes, yes, t + 2, weights, s);
        meet();
      }
      if (!second) meet();
    } else {
      auto turn = [&](int t) {
        if (!working) return;
        multiply(no, yes, t, weights, s);
        soften(t, s, weights);
        multiply(yes, no, t + 1, weights, s);
      };
      for (int i = 0, t = 0; i < trips; ++i, t += 2) {
        turn(t);
        codes_store(t + 1, c1, grids_load(t + 1));
        c1 = codes_load(t + 3);
        meta_due(t);
        meet();
        turn(t + 1);
        codes_store(t + 2, c0, grids_load(t + 2));
        c0 = codes_load(t + 4);
        meta_due(t + 1);
        meet();
      }
    }
  }
  if (live) {
    // numerator and sum have powers of two of their own; what they differ by may be more than a float32 holds
    const f32x2 kept = apart ? *own : f32x2{-1.f, 0.f};
    const bool mine = !(kept[0] < 0.f);
    const float l = mine ? kept[0] : sum[0], of = mine ? kept[1] : M;   // the sum, and what it is relative to
    const int up = (int)fminf(fmaxf(M - of, -600.f), 600.f);
    const float inv = l == 0.f ? 0.f : ldexpf(1.f / l, up / 2 - kValueLift), rest = ldexpf(1.f, up - up / 2);
    auto output = [&](int n, int j) {
      return f32x4{acc[n][4 * j] * inv * rest, acc[n][4 * j + 1] * inv * rest, acc[n][4 * j + 2] * inv * rest, acc[n][4 * j + 3] * inv * rest};
    };
    if (!alone) {
      // (an item that begins here is the share's last, one that began before is its first)
      const int64_t slot_row = (int64_t)(2 * ((at + off) / each) + (off == 0)) * a.slot_rows + (row - row0);
      if (h == 0) {
        a.ml[2 * slot_row] = of;
        a.ml[2 * slot_row + 1] = l;
      }
#pragma unroll
      for (int n = 0; n < kOut; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int d = 32 * n + 8 * j + 4 * h;
          if (d < a.d) *reinterpret_cast<f32x4*>(a.part + slot_row * a.d + d) = output(n, j);
        }
    } else {
      uint16_t* O = a.O + token * a.o_token + qhead * a.o_head;
#pragma unroll
      for (int n = 0; n < kOut; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 o = output(n, j);
          const float v[4] = {o[0], o[1], o[2], o[3]};
          const int d = 32 * n + 8 * j + 4 * h;
          if (d < a.d) store_run<PTQ_BF16, 4, false>(O, d, a.d, v);
        }
    }
  }
  if (a.splits == 1) return;
  if (off == 0 && !alone) begun = int4{(at + whole - 1) / each - at / each + 1, seq, head, tile};
  left -= take;
  if (left <= 0) break;
  at += whole;
  off = 0;
  ++tile;
  meet();   // the next item's codes go where this one's were
  }
  if (threadIdx.x == 0) *begun_at = begun;
}

// Joins what the shares have of an item that one of them begins, means of their keys' values and what those weigh: a thread has four channels
// of a row.
template <int DP>
__global__ __launch_bounds__(256) void join_chunk_kernel(AttendArgs a) {
  using C = Chunk<DP>;
  const int4 begun = reinterpret_cast<const int4*>(a.parts)[blockIdx.x];
  const int parts = begun.x, seq = begun.y, head = begun.z, tile = begun.w;
  const int i = blockIdx.y * 256 + threadIdx.x, local = i / (DP / 4), c = i % (DP / 4) * 4;
  if (parts == 0 || c >= a.d) return;
  const Sequence q = sequence_of(a, seq);
  const int row = tile * C::kRows + local;
  if (row >= min(q.queries, a.max_q) * a.group) return;
  float top = kNoScore, sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  auto some = [&](int p0, auto n_) {   // parts p0, p0 + 1, ...; those past the last count nothing
    constexpr int n = decltype(n_)::value;
    f32x4 v[n];
    f32x2 ml[n];
    float t = top;
#pragma unroll
    for (int j = 0; j < n; ++j) {   // the first is in its share's second place, the others in their shares' first
      const int p = min(p0 + j, parts - 1);
      const int64_t at = (int64_t)(2 * (blockIdx.x + p) + (p == 0)) * a.slot_rows + local;
      v[j] = *reinterpret_cast<const f32x4*>(a.part + at * a.d + c);
      ml[j] = *reinterpret_cast<const f32x2*>(a.ml + 2 * at);
    }
#pragma unroll
    for (int j = 0; j < n; ++j) t = fmaxf(t, ml[j][0]);
    const float before = exp2_fast(top - t) * sum;
    float w[n], all = before;
#pragma unroll
    for (int j = 0; j < n; ++j) {
      w[j] = p0 + j < parts ? exp2_fast(ml[j][0] - t) * ml[j][1] : 0.f;
      all += w[j];
    }
    const float inv = all == 0.f ? 0.f : 1.f / all;   // a row that has seen nothing: zeros
    o *= before * inv;
#pragma unroll
    for (int j = 0; j < n; ++j) o += (w[j] * inv) * v[j];
    top = t;
    sum = all;
  };
  int p = 0;
  for (; parts - p > 4; p += 16) some(p, std::integral_constant<int, 16>{});
  if (p < parts) some(p, std::integral_constant<int, 4>{});
  const float v[4] = {o[0], o[1], o[2], o[3]};
  const int64_t token = q.first + row / a.group, qhead = head * a.group + row % a.group;
  store_run<PTQ_BF16, 4, false>(a.O + token * a.o_token + qhead * a.o_head, c, a.d, v);
}

template <int BITS, int DP>
bool chunk_launch(const AttendArgs& a, hipStream_t s) {
  using C = Chunk<DP>;
  constexpr int kBytes = C::kBuffers + C::kQueryBytes + C::kApartBytes + kMetas * (int)sizeof(Meta);
  if (!lds_opt_in<attend_chunk_kernel<BITS, DP>>(kBytes)) return false;
  const int tiles = (int)ceil_div((int64_t)a.max_q * a.group, C::kRows);
  if (a.splits > 1) {
    attend_chunk_kernel<BITS, DP><<<kShares, C::kThreads, kBytes, s>>>(a, tiles, 0);
    join_chunk_kernel<DP><<<dim3(kShares, C::kRows * (DP / 4) / 256), 256, 0, s>>>(a);
    return true;
  }
  // A launch has fewer than 2^32 threads; eight groups of up to 2^27 rows, two threads to a row, fit one.
  const int64_t eights = ceil_div((int64_t)a.b * a.c.heads, 8), step = std::max<int64_t>(1, (1 << 19) / tiles);
  for (int64_t first = 0; first < eights; first += step)
    attend_chunk_kernel<BITS, DP><<<(unsigned)(std::min(step, eights - first) * 8 * tiles), C::kThreads, kBytes, s>>>(a, tiles, (int)(8 * first));
  return true;
}

}  // namespace

ChunkItems paged_attention_chunk_items(const AttendArgs& a) {
  const int64_t rows = a.d > 128 ? Chunk<256>::kRows : Chunk<128>::kRows;
  static_assert(Chunk<128>::kRows <= kChunkRows && Chunk<64>::kRows == Chunk<128>::kRows, "");
  const int64_t tiles = (int64_t)a.b * ceil_div((int64_t)a.max_q * a.group, rows), busy = (int64_t)a.t * a.group / rows + a.b;
  return ChunkItems{tiles * a.c.heads, std::min(tiles, busy) * a.c.heads};
}

ptq_status paged_attention_chunk_launch(const AttendArgs& a, int bits, hipStream_t s) {
  const bool launched = bits == 8 ? (a.d <= 64 ? chunk_launch<8, 64>(a, s) : a.d <= 96 ? chunk_launch<8, 96>(a, s)
                                     : a.d <= 128 ? chunk_launch<8, 128>(a, s) : chunk_launch<8, 256>(a, s))
                                  : (a.d <= 64 ? chunk_launch<4, 64>(a, s) : a.d <= 96 ? chunk_launch<4, 96>(a, s)
                                     : a.d <= 128 ? chunk_launch<4, 128>(a, s) : chunk_launch<4, 256>(a, s));
  return launched ? PTQ_OK : PTQ_ERR_HIP;
}

}  // namespace ptq
