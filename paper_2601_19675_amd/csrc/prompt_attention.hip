// Softmax attention of whole prompts, packed one behind the other, on bfloat16 queries, keys and values.
//
// Rows are the (token, head) pairs of a key head's group.  A wave has 32 of them, the columns of the 32 x 32 x 16 matrix instruction, and
// goes through the keys 64 at a time:
//
//   S' = K Q'   (keys are rows, so a lane has scores of one query row, and they leave the instruction in the order in which the
//               second product takes them: no exchange)        p = 2^(s f - M),   O' = V' p,   f = softmax_scale log2(e)
//
// Keys and values go from memory straight into LDS, as they lie: a row's 16-byte chunks in another order, so that rows that are read
// together are spread over the banks.  Keys are read by row, values by the LDS reads that transpose (four keys of a channel a lane).  The running
// maximum M, a whole number, moves only when one of the row's scores is 2^8 above it; weights are rounded to bfloat16 (2^-8 of each), and the sum of
// the weights is of the rounded ones, so that the rounding drops out where the values are alike.  Scores, maxima and sums are float32.
//
// A wave works out the scores of the next tile beside the weights of this one, and then sums the values beside the new scores' maximum, so that the matrix
// unit and the vector unit have something to do at any time; four waves share the tiles in LDS, and two workgroups (three for d <= 64) a
// compute unit, so that one's beginning and end hide behind the other's middle.  (Workgroups of eight such waves, in turn with
// these: 703 and 712 us for the long prompts below, but 135 and 94 for 21 packed ones of up to 2001 tokens, 17.5 and 12.7 for 333 tokens.)
//
// 8192 and 4142 tokens, 32 heads of 128 channels over 8, causal (690 GFLOP): 680 to 720 us, 960 to 1010 TFLOP/s.  Counters of one launch (744 us under the
// profiler): 1.64 GHz, the matrix unit busy 55 % of the cycles, the vector unit 54 %, no bank conflicts.  Neither unit is full and the clock is low, which
// looks like the card's power, though power itself was not measured.  333 tokens: 12.4 us, six tiles of keys one after the other on 88 of 256
// compute units.
//
// A key that a row does not see leaves it as it is, whatever it holds: its score is replaced.  A value that is not finite would meet a weight of 0
// all the same (0 times it is not 0): a workgroup that ends with anything not finite starts over, takes such values out of the tiles that it
// reads, and adds them at the end for the rows that see them.  Sums that are not finite even so are too large for float32 (weights are up to
// 2^8, values up to 2^128): it starts over once more, and those rows have a maximum 2^kLift above the one that they ended with.
#include <algorithm>

#include "lds_dma.h"
#include "paged_attention.h"
#include "static_for.h"
#include "stored_rows.h"

namespace ptq {
namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16v;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

constexpr int kTile = 64;   // keys
// 2^24 keys with values below 2^128 and weights of 2^(8 - kLift) are within float32.  (A weight below 2^(kLift - 126) of the largest is lost.)
constexpr float kLift = 34.f;

struct PromptArgs {
  const uint16_t *Q, *K, *V; uint16_t* O;   // bfloat16
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  const int32_t* cu;
  float scale;                              // softmax_scale log2(e)
  int t, b, hkv, group, d, max_n, causal, window;
  int tiles;                                // of rows, of the longest prompt there may be
  int ways;                                 // dies that share a group
};

template <int DP, int WAVES>
struct Prompt {
  static constexpr int kThreads = 64 * WAVES, kWaves = WAVES, kRows = 32 * kWaves;
  static constexpr int kPitch = DP <= 64 ? 128 : DP <= 128 ? 256 : 512;     // bytes of a key, or of a value
  static constexpr int kBytes = kTile * kPitch;
  static constexpr int kRing = 2;                                           // tiles of each in LDS
  static constexpr int kLds = 2 * kRing * kBytes;
  static constexpr int kRequests = kBytes / 1024 / kWaves;                  // of 1024 bytes, of a wave for a tile
};
// what a turn (see there) has to do
enum {
  kHad = 1, kMore = 2,        // there is a tile t, a tile t + 1
  kMask = 4,                  // some row does not see all of tile t + 1
};
// 16-byte chunk c of row `key` lies at c ^ turn
template <int DP>
__device__ __forceinline__ int key_turn(int key) { return DP <= 64 ? (key & 7) ^ ((key >> 3) & 1) : key & 15; }
// (four keys' chunks, two at a time, meet in a transposing read)
template <int DP>
__device__ __forceinline__ int val_turn(int key) { return DP <= 64 ? (key & 2) << 1 : (key & 3) << 2; }
// keeps the compiler from holding a register for every address that follows from v
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2)); }
__device__ __forceinline__ bf16x8 bf16x8_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d}); }

// DMA: rows of K and V begin at multiples of 16 bytes; otherwise they go through registers
template <int DP, int WAVES, bool DMA>
__global__ __launch_bounds__((Prompt<DP, WAVES>::kThreads), DP > 128 ? 1 : DP > 64 || !DMA ? 2 : 3) void prompt_kernel(PromptArgs a, int64_t first_item) {
  using C = Prompt<DP, WAVES>;
  constexpr int kSteps = DP / 16, kOut = DP / 32, kRing = C::kRing;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;

  // Groups (prompt, key head) go round the dies, so that a group's row tiles share its keys and values in one L2; where there are too few of them for that,
  // several dies share a group.  The last rows, which see most, first.  (Consecutive workgroups of a die go to its shader engines in turn,
  // however busy those are, so neighbours have to be alike: with the groups next to each other, of which some are short, 1233 us in place of 925.)
  const int64_t block = first_item + blockIdx.x, idx = block >> 3;
  const int each = (a.tiles + a.ways - 1) / a.ways, nth = (int)(idx % each);
  const int64_t unit = idx / each * 8 + (block & 7), group = unit / a.ways;
  const int tile = a.tiles - 1 - (nth * a.ways + (int)(unit % a.ways)), seq = (int)(group / a.hkv), head = (int)(group % a.hkv);
  if (group >= (int64_t)a.b * a.hkv || tile < 0) return;
  const int64_t from64 = a.cu[seq], to64 = a.cu[seq + 1];
  if (from64 < 0 || to64 > a.t || to64 <= from64) return;
  const int first = (int)from64, n = min((int)(to64 - from64), a.max_n), rows = n * a.group, row0 = tile * C::kRows;
  if (row0 >= rows) return;

  // keys [lo, hi) that token i sees
  auto sees = [&](int i, int& lo, int& hi) {
    hi = a.causal ? min(n, i + 1) : n;
    lo = a.window > 0 ? max(0, i - a.window + 1) : 0;
  };
  int begin, end, unused;
  sees(row0 / a.group, begin, unused);
  sees((min(row0 + C::kRows, rows) - 1) / a.group, unused, end);
  begin &= ~(kTile - 1);
  const int count = (end - begin + kTile - 1) / kTile;      // a row sees itself: at least one
  const int wrow = row0 + 32 * wave;
  // tiles [plain0, plain1) are those of which every row of the workgroup sees all keys
  int plain0, plain1;
  {
    int lo_b, hi_a;
    sees(row0 / a.group, unused, hi_a);
    sees((min(row0 + C::kRows, rows) - 1) / a.group, lo_b, unused);
    plain0 = max(0, lo_b - begin + kTile - 1) / kTile;
    plain1 = max(0, hi_a - begin) / kTile;
  }

  // ---- keys and values of a tile, into LDS
  const uint16_t* const keys0 = a.K + (int64_t)(first + begin) * a.k_token + head * a.k_head;
  const uint16_t* const vals0 = a.V + (int64_t)(first + begin) * a.v_token + head * a.v_head;
  auto key_slot = [&](int t) { return t % kRing * C::kBytes; };
  auto val_slot = [&](int t) { return (kRing + t % kRing) * C::kBytes; };
  // which chunk of which key the lane brings with the wave's request i
  uint32_t key_off[C::kRequests], val_off[C::kRequests];
#pragma unroll
  for (int i = 0; i < C::kRequests; ++i) {
    const int at = ((wave * C::kRequests + i) * 64 + lane) * 16, row = at / C::kPitch, pos = at % C::kPitch / 16;
    const int kc = pos ^ key_turn<DP>(row), vc = pos ^ val_turn<DP>(row);
    key_off[i] = 8 * kc < a.d ? (uint32_t)row * (uint32_t)a.k_token * 2 + 16 * kc : 0xffffff00u;   // past every descriptor's end: zeros
    val_off[i] = 8 * vc < a.d ? (uint32_t)row * (uint32_t)a.v_token * 2 + 16 * vc : 0xffffff00u;
  }
  // (a descriptor is scalar work: nothing that a request has to wait for)
  auto tile_at = [&](const uint16_t* from, int64_t token, int t) __attribute__((always_inline)) {
    const int left = n - (begin + t * kTile);   // keys
    const uint32_t bytes = ((uint32_t)(min(left, kTile) - 1) * (uint32_t)token + (uint32_t)a.d) * 2u;
    const uint64_t at = (uint64_t)(from + (int64_t)t * kTile * token);
    return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)(left > 0 ? bytes : 0u), 0x00020000};
  };
  auto bring_one = [&](const i32x4& tile, const uint16_t* from, int64_t token, const uint32_t (&off)[C::kRequests], int t, int slot, int i) __attribute__((always_inline)) {
    if constexpr (DMA) {
      request_to_lds_waiting(tile, off[i], lds + slot + (wave * C::kRequests + i) * 1024);
    } else {
      const int at = ((wave * C::kRequests + i) * 64 + lane) * 16, row = at / C::kPitch, pos = at % C::kPitch / 16;
      const int chunk = pos ^ (slot < kRing * C::kBytes ? key_turn<DP>(row) : val_turn<DP>(row)), key = t * kTile + row;
      const bool there = begin + key < n && 8 * chunk < a.d;
      AnyWords<4, 2> w = *reinterpret_cast<const AnyWords<4, 2>*>(from + (there ? key * token + 8 * chunk : 0));
      *reinterpret_cast<u32x4*>(smem + slot + at) = there ? u32x4{w.w[0], w.w[1], w.w[2], w.w[3]} : u32x4{0, 0, 0, 0};
    }
  };
  auto bring = [&](const uint16_t* from, int64_t token, const uint32_t (&off)[C::kRequests], int t, int slot) __attribute__((always_inline)) {
    const i32x4 tile = tile_at(from, token, t);
#pragma unroll
    for (int i = 0; i < C::kRequests; ++i) bring_one(tile, from, token, off, t, slot, i);
  };
  auto bring_keys = [&](int t) __attribute__((always_inline)) { bring(keys0, a.k_token, key_off, t, key_slot(t)); };
  auto bring_vals = [&](int t) __attribute__((always_inline)) { bring(vals0, a.v_token, val_off, t, val_slot(t)); };
  // until all but the last N tiles that this wave has asked for are there (keys and values count one each)
  auto arrived = [&](auto n_) __attribute__((always_inline)) {
    if constexpr (DMA) wait_requests<decltype(n_)::value * C::kRequests>();
  };
  auto meet = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // ---- the wave's queries
  const int row = wrow + r, token = first + row / a.group, qhead = head * a.group + row % a.group;
  const bool live = row < rows;
  int lo, hi;
  sees(live ? row / a.group : 0, lo, hi);
  if (!live) hi = 0;
  bf16x8 fq[kSteps];
  {
    const uint16_t* Q = a.Q + (live ? token * a.q_token + qhead * a.q_head : 0);
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const Run<PTQ_BF16, 8> q = load_run<PTQ_BF16, 8, false>(Q, 16 * u + 8 * h, a.d);
      const bool in = live && 16 * u + 8 * h < a.d;
      fq[u] = bf16x8_of(in ? q.w[0] ^ flip : 0, in ? q.w[1] ^ flip : 0, in ? q.w[2] ^ flip : 0, in ? q.w[3] ^ flip : 0);
    }
  }
  const float factor = fmaxf(fabsf(a.scale), 0x1p-126f);   // positive: a score that is not there is -inf times it

  f32x16v acc[kOut];
  float M, sum[4];   // the sums are of the weights of the lane's keys, every fourth pair
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3f803f80u);

  // a lane's place in a tile of keys: row r, chunk h; of values: keys 4 h + j of 16, channels 4 (lane & 3) of 16 (lane >> 4 & 1) on
  const int j = (lane & 15) >> 2, vchunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  const int key_at = r * C::kPitch + ((h ^ key_turn<DP>(r)) * 16);
  const int val_at = (4 * h + j) * C::kPitch + ((vchunk ^ val_turn<DP>(j)) * 16) + 8 * (lane & 1);
  // channels 32 k + .. of keys 16 g + 4 h .. and 16 g + 8 + 4 h ..: what an instruction takes of the values
  auto value = [&](int at, int g, int k) __attribute__((always_inline)) {
    using P = __attribute__((address_space(3))) s16x4*;
    const uint32_t p = lds + (uint32_t)(DP <= 64 ? at ^ (64 * k) : (at ^ (64 * (k & 3))) + (k >> 2) * 256) + g * 16 * C::kPitch;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)p), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(p + 8 * C::kPitch));
    const uint2 u = __builtin_bit_cast(uint2, x), w = __builtin_bit_cast(uint2, y);
    return bf16x8_of(u.x, u.y, w.x, w.y);
  };
  // values of tile t that are not finite become 0
  auto clean = [&](int t) __attribute__((always_inline)) {
#pragma unroll 1
    for (int at = threadIdx.x * 16; at < C::kBytes; at += C::kThreads * 16) {
      u32x4 v = *reinterpret_cast<u32x4*>(smem + val_slot(t) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
        if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
      }
      *reinterpret_cast<u32x4*>(smem + val_slot(t) + at) = v;
    }
    meet();
  };
  // ... and are added here for the wave's rows that see them (a weight is positive: an infinity stays what it is)
  auto add_cleaned = [&]() {
#pragma unroll 1
    for (int key0 = begin; key0 < end; key0 += kTile) {
      int odd = 0;
#pragma unroll 1
      for (int i = lane; i < kTile * (a.d / 8); i += kWave) {
        const int key = min(key0 + i / (a.d / 8), n - 1), c = i % (a.d / 8) * 8;
        const Run<PTQ_BF16, 8> v = load_run<PTQ_BF16, 8, false>(a.V + (int64_t)(first + key) * a.v_token + head * a.v_head, c, a.d);
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= ((v.w[e] & 0x7f80u) == 0x7f80u) | ((v.w[e] & 0x7f800000u) == 0x7f800000u);
      }
      if (!__any(odd)) continue;
#pragma unroll 1
      for (int key = max(key0, lo); key < min(min(key0 + kTile, end), hi); ++key) {
        const uint16_t* V = a.V + (int64_t)(first + key) * a.v_token + head * a.v_head;
#pragma unroll
        for (int k = 0; k < kOut; ++k)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int c = 32 * k + 8 * (i >> 2) + 4 * h + (i & 3);
            const float v = c < a.d ? bf16_bits_to_f32(V[c]) : 0.f;
            acc[k][i] += fabsf(v) < INFINITY ? 0.f : v;
          }
      }
    }
  };

  uint32_t weights[16];   // pairs of bfloat16
  constexpr int kScores = 2 * kSteps, kAll = kScores + 4 * kOut, kAhead = 4;
  static_assert(2 * 2 * C::kRequests <= kAll, "");   // (every request has its place in a turn)
  // One turn: the scores of tile t + 1 beside the weights of tile t, then the values of tile t beside the maximum of the new scores.  A matrix
  // instruction takes as long as what vector instructions a pair of weights takes, and they run side by side; so they are laid out in turn, with the
  // operands read from LDS kAhead instructions before.
  bf16x8 f[kAhead + 1];
  auto turn = [&](auto what_, int t, f32x16v (&cur)[2], f32x16v (&next)[2]) __attribute__((always_inline)) {
    constexpr int what = decltype(what_)::value;
    constexpr bool had = what & kHad, more = what & kMore, mask = what & kMask;
    constexpr int kFirst = more ? 0 : kScores, kLast = had ? kAll : kScores;
    const int key_base = opaque(key_slot(t + 1) + key_at), val_base = opaque(val_slot(t + kRing) + val_at);
    auto read = [&](auto m_) __attribute__((always_inline)) {
      constexpr int m = decltype(m_)::value, at = m % (kAhead + 1);
      if constexpr (m < kScores) {    // (turns of keys 32 apart are the same, and leave chunk bit 4 alone)
        constexpr int u = m % kSteps, k = m / kSteps;
        f[at] = *reinterpret_cast<const bf16x8*>(smem + (key_base ^ (32 * (u & 7))) + (u >> 3) * 256 + k * 32 * C::kPitch);
      } else {
        f[at] = value(val_base, (m - kScores) / kOut, (m - kScores) % kOut);
      }
    };
    i32x4 vals{}, keys{};   // the tiles that are asked for
    if constexpr (had && more) {
      vals = tile_at(vals0, a.v_token, t + kRing - 1);
      keys = tile_at(keys0, a.k_token, t + kRing);
    }
    static_for<kAhead>([&](auto i_) __attribute__((always_inline)) {
      constexpr int m = kFirst + decltype(i_)::value;
      if constexpr (m < kLast) read(std::integral_constant<int, m>{});
    });
    const int key0 = begin + (t + 1) * kTile;   // counted from the half wave's first key: what is left are constants
    const int from_ = opaque(lo - key0 - 4 * h), to_ = opaque(hi - key0 - 4 * h);
    float top[2] = {-INFINITY, -INFINITY};
    auto highest = [&](auto e_) __attribute__((always_inline)) {
      constexpr int e = decltype(e_)::value, k = e / 16, i = e % 16, at = 32 * k + 8 * (i >> 2) + (i & 3);
      if constexpr (mask) next[k][i] = ((at >= from_) & (at < to_)) ? next[k][i] : -INFINITY;
      top[e & 1] = fmaxf(top[e & 1], next[k][i]);
    };
    static_for<kLast - kFirst>([&](auto i_) __attribute__((always_inline)) {
      constexpr int m = kFirst + decltype(i_)::value, at = m % (kAhead + 1);
      if constexpr (m % 2 == 0) __builtin_amdgcn_sched_barrier(0);
      if constexpr (m + kAhead < kLast) read(std::integral_constant<int, m + kAhead>{});
      // slots of tiles that everybody has read are filled again, early in the turn, but a request at a time: several would wait for each other
      constexpr int n = m / 2;
      if constexpr (had && more && n < 2 * C::kRequests && m == 2 * n) {
        if constexpr (n < C::kRequests) bring_one(vals, vals0, a.v_token, val_off, t + kRing - 1, val_slot(t + kRing - 1), n);
        else bring_one(keys, keys0, a.k_token, key_off, t + kRing, key_slot(t + kRing), n - C::kRequests);
      }
      if constexpr (m < kScores) {
        constexpr int u = m % kSteps, k = m / kSteps;
        if (u == 0) next[k] = f32x16v{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        next[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[at], fq[u], next[k], 0, 0, 0);
      } else {
        constexpr int g = (m - kScores) / kOut, k = (m - kScores) % kOut;
        acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[at], bf16x8_of(weights[4 * g], weights[4 * g + 1], weights[4 * g + 2], weights[4 * g + 3]), acc[k], 0, 0, 0);
      }
      if constexpr (had && m < kScores) {
        constexpr int from = 16 * m / kScores, to = 16 * (m + 1) / kScores;
        static_for<to - from>([&](auto j_) __attribute__((always_inline)) {
          constexpr int w = from + decltype(j_)::value, k = w / 8, e = w % 8 * 2;
          weights[w] = bf16_pair(exp2_fast(fmaf(cur[k][e], factor, -M)), exp2_fast(fmaf(cur[k][e + 1], factor, -M)));
          sum[w & 3] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, weights[w]), ones, sum[w & 3], false);
        });
      } else if constexpr (more && m >= kScores) {
        constexpr int from = 32 * (m - kScores) / (4 * kOut), to = 32 * (m + 1 - kScores) / (4 * kOut);
        static_for<to - from>([&](auto j_) __attribute__((always_inline)) { highest(std::integral_constant<int, from + decltype(j_)::value>{}); });
      }
    });
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!more) return;
    if constexpr (!had) static_for<32>([&](auto e_) __attribute__((always_inline)) { highest(e_); });
    // what has been summed so far is brought to the new maximum
    float most = fmaxf(top[0], top[1]) * factor;
    if (__any(most > M + 8.f)) {
      most = fmaxf(most, __shfl_xor(most, 32));
      const float to = most > M + 8.f ? ceilf(most) : M, shrink = exp2_fast(M - to);
      M = to;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] *= shrink;
#pragma unroll
      for (int k = 0; k < kOut; ++k) acc[k] *= shrink;
    }
  };
  // ... of the last tile: there are no scores beside its weights
  auto last_weights = [&](f32x16v (&cur)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      weights[w] = bf16_pair(exp2_fast(fmaf(cur[w / 8][w % 8 * 2], factor, -M)), exp2_fast(fmaf(cur[w / 8][w % 8 * 2 + 1], factor, -M)));
      sum[w & 3] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, weights[w]), ones, sum[w & 3], false);
    }
  };

  M = kNoScore;
#pragma unroll 1
  for (int go = 0;; ++go) {
    const bool careful = go > 0;
#pragma unroll
    for (int k = 0; k < kOut; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[k][i] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = 0.f;
    f32x16v s0[2], s1[2];
    // asked for in the order K0, V0, K1, V1, ...
    bring_keys(0);
#pragma unroll
    for (int t = 0; t < kRing - 1; ++t) {
      bring_vals(t);
      bring_keys(t + 1);
    }
    arrived(std::integral_constant<int, 2 * kRing - 2>{});
    meet();
    turn(std::integral_constant<int, kMore | kMask>{}, -1, s0, s0);
    // the values of tile t and the keys of the next are there, and everybody has those before them behind him
    auto next_tiles = [&](int t) __attribute__((always_inline)) {
      arrived(std::integral_constant<int, 2 * kRing - 4>{});
      meet();
      if (careful) clean(t);
    };
    int t = 0;
    auto turns = [&](auto mask_, int to) __attribute__((always_inline)) {   // up to the scores of tile `to`
      constexpr std::integral_constant<int, kHad | kMore | decltype(mask_)::value> what{};
      for (; t + 1 < to; t += 2) {
        next_tiles(t);
        turn(what, t, s0, s1);
        next_tiles(t + 1);
        turn(what, t + 1, s1, s0);
      }
      if (t < to) {
        next_tiles(t);
        turn(what, t, s0, s1);
        s0[0] = s1[0], s0[1] = s1[1];
        ++t;
      }
    };
    turns(std::integral_constant<int, kMask>{}, min(plain0 - 1, count - 1));
    turns(std::integral_constant<int, 0>{}, min(plain1 - 1, count - 1));
    turns(std::integral_constant<int, kMask>{}, count - 1);
    next_tiles(t);
    last_weights(s0);
    turn(std::integral_constant<int, kHad>{}, t, s0, s1);
    arrived(std::integral_constant<int, 0>{});   // nothing comes into LDS that is somebody else's by then
    if (go < 2) {
      float odd = 0.f;   // NaN if anything is not finite
#pragma unroll
      for (int k = 0; k < kOut; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd = fmaf(acc[k][i], 0.f, odd);
      // (in the second go only rows whose weights are numbers gain by another)
      const uint64_t again = __ballot(live && odd != 0.f && (!careful || fabsf((sum[0] + sum[1]) + (sum[2] + sum[3])) < INFINITY));
      const uint32_t again_rows = (uint32_t)again | (uint32_t)(again >> 32);
      M = careful && (again_rows >> r & 1) ? M + kLift : kNoScore;
      meet();
      int* const vote = reinterpret_cast<int*>(smem);
      if (lane == 0) vote[wave] = again != 0;
      meet();
      int any = 0;
#pragma unroll
      for (int w = 0; w < C::kWaves; ++w) any |= vote[w];
      meet();
      if (__builtin_amdgcn_readfirstlane(any) != 0) continue;
    }
    if (careful) add_cleaned();
    break;
  }
  float l = (sum[0] + sum[1]) + (sum[2] + sum[3]);
  l += __shfl_xor(l, 32);
  if (!live) return;
  const float inv = l == 0.f ? __uint_as_float(0x7fc00000u) : 1.f / l;   // (a row sees itself: its weights are not all 0 unless its scores are -inf)
  uint16_t* O = a.O + token * a.o_token + qhead * a.o_head;
#pragma unroll
  for (int k = 0; k < kOut; ++k)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float v[4] = {acc[k][4 * q] * inv, acc[k][4 * q + 1] * inv, acc[k][4 * q + 2] * inv, acc[k][4 * q + 3] * inv};
      const int c = 32 * k + 8 * q + 4 * h;
      if (c < a.d) store_run<PTQ_BF16, 4, false>(O, c, a.d, v);
    }
}

template <int DP, int WAVES, bool DMA>
bool prompt_form_launch(const PromptArgs& all, hipStream_t s) {
  using C = Prompt<DP, WAVES>;
  if (!lds_opt_in<prompt_kernel<DP, WAVES, DMA>>(C::kLds)) return false;
  PromptArgs a = all;
  a.tiles = (int)ceil_div((int64_t)a.max_n * a.group, C::kRows);
  const int64_t groups = (int64_t)a.b * a.hkv;
  a.ways = 1;
  while (a.ways < 8 && ceil_div(groups * a.ways, 8) * 8 * 20 > groups * a.ways * 21) a.ways *= 2;   // a twentieth of the dies' time idle at most
  // (8000 tokens, 28 heads over 4: 871 us with a die to a group, 486 so; 16 over 1: 1625 and 277)
  // a launch has fewer than 2^32 threads
  const int64_t items = ceil_div(a.tiles, a.ways) * ceil_div(groups * a.ways, 8) * 8, step = 1 << 22;
  for (int64_t first = 0; first < items; first += step)
    prompt_kernel<DP, WAVES, DMA><<<(unsigned)std::min(step, items - first), C::kThreads, C::kLds, s>>>(a, first);
  return true;
}
template <int DP, int WAVES>
bool prompt_launch(const PromptArgs& a, hipStream_t s) {
  const bool lines = (uintptr_t)a.K % 16 == 0 && (uintptr_t)a.V % 16 == 0 && a.k_token % 8 == 0 && a.k_head % 8 == 0 && a.v_token % 8 == 0 &&
                     a.v_head % 8 == 0 && a.k_token < (1 << 24) && a.v_token < (1 << 24);
  return lines ? prompt_form_launch<DP, WAVES, true>(a, s) : prompt_form_launch<DP, WAVES, false>(a, s);
}

}  // namespace

ptq_status prompt_attention_launch(const void* Q, int64_t q_token, int64_t q_head, const void* K, int64_t k_token, int64_t k_head,
                                   const void* V, int64_t v_token, int64_t v_head, int64_t t, int64_t hq, int64_t hkv, int64_t d,
                                   const int32_t* cu, int64_t b, int64_t max_n, double softmax_scale, int causal, int64_t window, void* O,
                                   int64_t o_token, int64_t o_head, hipStream_t s) {
  PromptArgs a{};
  a.Q = static_cast<const uint16_t*>(Q), a.K = static_cast<const uint16_t*>(K), a.V = static_cast<const uint16_t*>(V);
  a.O = static_cast<uint16_t*>(O);
  a.q_token = q_token, a.q_head = q_head, a.k_token = k_token, a.k_head = k_head, a.v_token = v_token, a.v_head = v_head;
  a.o_token = o_token, a.o_head = o_head, a.cu = cu;
  a.scale = (float)(softmax_scale * 1.4426950408889634);
  a.t = (int)t, a.b = (int)b, a.hkv = (int)hkv, a.group = (int)(hq / hkv), a.d = (int)d, a.max_n = (int)max_n, a.causal = causal;
  a.window = (int)std::min<int64_t>(window, INT32_MAX / 2);
  const bool launched = d <= 64 ? prompt_launch<64, 4>(a, s) : d <= 96 ? prompt_launch<96, 4>(a, s)
                        : d <= 128 ? prompt_launch<128, 4>(a, s) : prompt_launch<256, 4>(a, s);
  if (!launched) return PTQ_ERR_HIP;
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

}  // namespace ptq
