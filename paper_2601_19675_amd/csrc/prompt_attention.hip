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
// A key that a row does not see leaves it as it is, whatever it holds: its score is replaced.  A value that is not finite would meet a weight of 0
// all the same (0 times it is not 0): a workgroup that ends with anything not finite starts over, takes such values out of the tiles that it
// reads, and adds them at the end for the rows that see them.
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
typedef __attribute__((__vector_size__(2 * sizeof(uint16_t)))) uint16_t u16x2;

constexpr int kTile = 64;   // keys

struct PromptArgs {
  const uint16_t *Q, *K, *V; uint16_t* O;   // bfloat16
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
  const int32_t* cu;
  float scale;                              // softmax_scale log2(e)
  int t, b, hkv, group, d, max_n, causal, window;
  int tiles;                                // of rows, of the longest prompt there may be
};

// TURNS: eight waves, two to a SIMD, one half of which multiplies while the other works out weights
template <int DP, bool TURNS>
struct Prompt {
  static constexpr int kThreads = TURNS ? 512 : 256, kWaves = kThreads / 64, kRows = 32 * kWaves;
  static constexpr int kPitch = DP <= 64 ? 128 : DP <= 128 ? 256 : 512;     // bytes of a key, or of a value
  static constexpr int kBytes = kTile * kPitch;
  static constexpr int kRing = TURNS ? 4 : DP > 128 ? 2 : 2;                // tiles of each in LDS
  static constexpr int kLds = 2 * kRing * kBytes;
  static constexpr int kRequests = kBytes / 1024 / kWaves;                  // of 1024 bytes, of a wave for a tile
  static constexpr int kRequestRows = 1024 / kPitch;
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
template <int DP, bool TURNS, bool DMA>
__global__ __launch_bounds__((Prompt<DP, TURNS>::kThreads)) void prompt_kernel(PromptArgs a, int64_t first_item) {
  using C = Prompt<DP, TURNS>;
  constexpr int kSteps = DP / 16, kOut = DP / 32, kRing = C::kRing;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;

  // Groups (prompt, key head) go round the dies, so that a group's row tiles share its keys and values in one L2; the last rows, which see
  // most, first.  (Consecutive workgroups of a die go to its shader engines in turn, however busy those are: they have to be alike.)
  const int64_t block = first_item + blockIdx.x, idx = block >> 3, group = idx / a.tiles * 8 + (block & 7);
  if (group >= (int64_t)a.b * a.hkv) return;
  const int tile = a.tiles - 1 - (int)(idx % a.tiles), seq = (int)(group / a.hkv), head = (int)(group % a.hkv);
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
  auto tile_at = [&](const uint16_t* from, int64_t token, int t) {
    const int left = n - (begin + t * kTile);   // keys
    const uint32_t bytes = ((uint32_t)(min(left, kTile) - 1) * (uint32_t)token + (uint32_t)a.d) * 2u;
    const uint64_t at = (uint64_t)(from + (int64_t)t * kTile * token);
    return i32x4{(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)(left > 0 ? bytes : 0u), 0x00020000};
  };
  auto bring_one = [&](const i32x4& tile, const uint16_t* from, int64_t token, const uint32_t (&off)[C::kRequests], int t, int slot, int i) {
    if constexpr (DMA) {
      request_to_lds(tile, off[i], lds + slot + (wave * C::kRequests + i) * 1024);
    } else {
      const int at = ((wave * C::kRequests + i) * 64 + lane) * 16, row = at / C::kPitch, pos = at % C::kPitch / 16;
      const int chunk = pos ^ (slot < kRing * C::kBytes ? key_turn<DP>(row) : val_turn<DP>(row)), key = t * kTile + row;
      const bool there = begin + key < n && 8 * chunk < a.d;
      AnyWords<4, 2> w = *reinterpret_cast<const AnyWords<4, 2>*>(from + (there ? key * token + 8 * chunk : 0));
      *reinterpret_cast<u32x4*>(smem + slot + at) = there ? u32x4{w.w[0], w.w[1], w.w[2], w.w[3]} : u32x4{0, 0, 0, 0};
    }
  };
  auto bring = [&](const uint16_t* from, int64_t token, const uint32_t (&off)[C::kRequests], int t, int slot) {
    const i32x4 tile = tile_at(from, token, t);
#pragma unroll
    for (int i = 0; i < C::kRequests; ++i) bring_one(tile, from, token, off, t, slot, i);
  };
  auto bring_keys = [&](int t) { bring(keys0, a.k_token, key_off, t, key_slot(t)); };
  auto bring_vals = [&](int t) { bring(vals0, a.v_token, val_off, t, val_slot(t)); };
  // until all but the last N tiles that this wave has asked for are there (keys and values count one each)
  auto arrived = [&](auto n_) {
    if constexpr (DMA) wait_requests<decltype(n_)::value * C::kRequests>();
  };
  auto meet = [&]() {
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
  auto value = [&](int at, int g, int k) {
    using P = __attribute__((address_space(3))) s16x4*;
    const uint32_t p = lds + (uint32_t)(DP <= 64 ? at ^ (64 * k) : (at ^ (64 * (k & 3))) + (k >> 2) * 256) + g * 16 * C::kPitch;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)p), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(p + 8 * C::kPitch));
    const uint2 u = __builtin_bit_cast(uint2, x), w = __builtin_bit_cast(uint2, y);
    return bf16x8_of(u.x, u.y, w.x, w.y);
  };
  // values of tile t that are not finite become 0
  auto clean = [&](int t) {
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

  // What the matrix instructions do in one go: the values of tile t - 1 (with its weights), then the scores of tile t, either may be
  // missing.  Groups of instructions -- the channels' blocks of 16 keys; two steps of d of both halves of the keys -- whose operands are
  // read from LDS kReadAhead groups before; the first ones' may be read apart (read_), before the barrier that the others have to wait for.
  constexpr int kGroups = 4 + kSteps / 2, kPer = kOut > 4 ? kOut : 4, kReadAhead = DP > 128 ? 1 : 2;
  bf16x8 f[kReadAhead + 1][kPer];
  auto multiply = [&](auto had_, auto has_, auto read_, auto multiply_, int t, const bf16x8 (&weights)[4], f32x16v (&s)[2]) {
    constexpr int kFirst = decltype(had_)::value ? 0 : 4, kLast = decltype(has_)::value ? kGroups : 4;
    const int key_base = opaque(key_slot(t) + key_at), val_base = opaque(val_slot(t + kRing - 1) + val_at);
    auto read = [&](auto g_) {
      constexpr int g = decltype(g_)::value, at = g % (kReadAhead + 1);
      if constexpr (g < 4) {
#pragma unroll
        for (int k = 0; k < kOut; ++k) f[at][k] = value(val_base, g, k);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {    // (turns of keys 32 apart are the same, and leave chunk bit 4 alone)
          const int u = 2 * (g - 4) + (i >> 1), k = i & 1;
          f[at][i] = *reinterpret_cast<const bf16x8*>(smem + (key_base ^ (32 * (u & 7))) + (u >> 3) * 256 + k * 32 * C::kPitch);
        }
      }
    };
    if constexpr (decltype(read_)::value)
      static_for<kReadAhead>([&](auto i_) {
        constexpr int g = kFirst + decltype(i_)::value;
        if constexpr (g < kLast) read(std::integral_constant<int, g>{});
      });
    if constexpr (!decltype(multiply_)::value) return;
    constexpr bool kBrings = TURNS && decltype(had_)::value && decltype(has_)::value;
    i32x4 vals{}, keys{};
    if constexpr (kBrings) {
      vals = tile_at(vals0, a.v_token, t + kRing - 2);
      keys = tile_at(keys0, a.k_token, t + kRing - 1);
    }
    static_for<kLast - kFirst>([&](auto i_) {
      constexpr int g = kFirst + decltype(i_)::value, at = g % (kReadAhead + 1);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (g + kReadAhead < kLast) read(std::integral_constant<int, g + kReadAhead>{});
      // slots of tiles that both halves have read are filled again beside the products, a request at a time: several would wait for each other
      constexpr int i = (g * 2 * C::kRequests + kGroups - 1) / kGroups;
      if constexpr (kBrings && i < 2 * C::kRequests && i * kGroups / (2 * C::kRequests) == g) {
        if constexpr (i < C::kRequests) bring_one(vals, vals0, a.v_token, val_off, t + kRing - 2, val_slot(t + kRing - 2), i);
        else bring_one(keys, keys0, a.k_token, key_off, t + kRing - 1, key_slot(t + kRing - 1), i - C::kRequests);
      }
      if constexpr (g < 4) {
#pragma unroll
        for (int k = 0; k < kOut; ++k) acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[at][k], weights[g], acc[k], 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int u = 2 * (g - 4) + (i >> 1), k = i & 1;
          if (u == 0) s[k] = f32x16v{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
          s[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[at][i], fq[u], s[k], 0, 0, 0);
        }
      }
    });
    __builtin_amdgcn_sched_barrier(0);
  };
  // the weights of tile t; what has been summed so far is brought to their maximum
  auto soften = [&](auto mask_, int t, f32x16v (&s)[2], bf16x8 (&weights)[4]) {
    if constexpr (decltype(mask_)::value) {
      const int key0 = begin + t * kTile;
      // counted from the half wave's first key: what is left are constants
      const int from_ = opaque(lo - key0 - 4 * h), to_ = opaque(hi - key0 - 4 * h);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 32 * k + 8 * (i >> 2) + (i & 3);
          s[k][i] = ((at >= from_) & (at < to_)) ? s[k][i] : -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[k][i]);
    top *= factor;
    if (__any(top > M + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = top > M + 8.f ? ceilf(top) : M, shrink = exp2_fast(M - next);
      M = next;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] *= shrink;
#pragma unroll
      for (int k = 0; k < kOut; ++k) acc[k] *= shrink;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = bf16_pair(exp2_fast(fmaf(s[k][8 * u + 2 * i], factor, -M)), exp2_fast(fmaf(s[k][8 * u + 2 * i + 1], factor, -M)));
          sum[i] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i]), ones, sum[i], false);
        }
        weights[2 * k + u] = bf16x8_of(w[0], w[1], w[2], w[3]);
      }
    // here, and not where they are used: behind the barrier they would stand before the wave's matrix instructions
#pragma unroll
    for (int g = 0; g < 4; ++g) asm volatile("" : "+v"(weights[g]));
  };

  constexpr std::true_type yes;
  constexpr std::false_type no;
#pragma unroll 1
  for (bool careful = false;; careful = true) {
#pragma unroll
    for (int k = 0; k < kOut; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[k][i] = 0.f;
    M = kNoScore;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = 0.f;
    f32x16v s[2];
    bf16x8 weights[4];
    // asked for in the order K0, V0, K1, V1, ...
    bring_keys(0);
#pragma unroll
    for (int t = 0; t < (TURNS ? kRing - 1 : 0); ++t) {
      bring_vals(t);
      bring_keys(t + 1);
    }
    if constexpr (TURNS) {
      // Phases: the first half of the waves multiplies in the even ones -- values of tile t - 1 and keys of tile t in phase 2 t -- and works
      // out weights in the odd ones; the second half is a phase behind.
      const bool second = wave >= C::kWaves / 2;
      static_assert(2 * C::kRequests <= kGroups, "");
      arrived(std::integral_constant<int, 2 * kRing - 2>{});
      meet();
      if (second) {
        arrived(std::integral_constant<int, 2 * kRing - 3>{});
        meet();
        if (careful) clean(0);
      }
      multiply(no, yes, yes, yes, 0, weights, s);
      auto until_weights = [&](auto mask_, auto last_, int t) {
        // the values of tile t have to be there a phase before their turn
        if (second) arrived(std::integral_constant<int, 2 * kRing - 4>{});
        else arrived(std::integral_constant<int, 2 * kRing - 3>{});
        meet();
        if (careful && !second) clean(t);
        soften(mask_, t, s, weights);
        multiply(yes, std::integral_constant<bool, !decltype(last_)::value>{}, yes, no, t + 1, weights, s);
        if (second) arrived(std::integral_constant<int, 2 * kRing - 5>{});
        else arrived(std::integral_constant<int, 2 * kRing - 4>{});
        meet();
        if (careful && second && !decltype(last_)::value) clean(t + 1);
      };
      int t = 0;
      for (; t < min(plain0, count - 1); ++t) {
        until_weights(yes, no, t);
        multiply(yes, yes, no, yes, t + 1, weights, s);
      }
      for (; t < min(plain1, count - 1); ++t) {
        until_weights(no, no, t);
        multiply(yes, yes, no, yes, t + 1, weights, s);
      }
      for (; t < count - 1; ++t) {
        until_weights(yes, no, t);
        multiply(yes, yes, no, yes, t + 1, weights, s);
      }
      until_weights(yes, yes, t);
      multiply(yes, no, no, yes, count, weights, s);
      if (!second) meet();
    } else {
      // all waves in step: tile t's values and the next one's keys are asked for when everybody has the slots' tiles behind him
      for (int t = 0; t < count; ++t) {
        arrived(std::integral_constant<int, 0>{});
        meet();
        bring_vals(t);
        bring_keys(t + 1);
        multiply(no, yes, yes, yes, t, weights, s);
        soften(yes, t, s, weights);
        arrived(std::integral_constant<int, 1>{});
        meet();
        if (careful) clean(t);
        multiply(yes, no, yes, yes, t + 1, weights, s);
      }
    }
    arrived(std::integral_constant<int, 0>{});   // nothing comes into LDS that is somebody else's by then
    if (careful) {
      add_cleaned();
      break;
    }
    float odd = 0.f;   // NaN if anything is not finite
#pragma unroll
    for (int k = 0; k < kOut; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd = fmaf(acc[k][i], 0.f, odd);
    meet();
    int* const vote = reinterpret_cast<int*>(smem);
    if (lane == 0) vote[wave] = 0;
    if (live && odd != 0.f) vote[wave] = 1;
    meet();
    int any = 0;
#pragma unroll
    for (int w = 0; w < C::kWaves; ++w) any |= vote[w];
    if (__builtin_amdgcn_readfirstlane(any) == 0) break;
    meet();
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

template <int DP, bool TURNS, bool DMA>
bool prompt_form_launch(const PromptArgs& all, hipStream_t s) {
  using C = Prompt<DP, TURNS>;
  if (!lds_opt_in<prompt_kernel<DP, TURNS, DMA>>(C::kLds)) return false;
  PromptArgs a = all;
  a.tiles = (int)ceil_div((int64_t)a.max_n * a.group, C::kRows);
  // a launch has fewer than 2^32 threads
  const int64_t items = (int64_t)a.tiles * ceil_div((int64_t)a.b * a.hkv, 8) * 8, step = 1 << 22;
  for (int64_t first = 0; first < items; first += step)
    prompt_kernel<DP, TURNS, DMA><<<(unsigned)std::min(step, items - first), C::kThreads, C::kLds, s>>>(a, first);
  return true;
}
template <int DP, bool TURNS>
bool prompt_launch(const PromptArgs& a, hipStream_t s) {
  const bool lines = (uintptr_t)a.K % 16 == 0 && (uintptr_t)a.V % 16 == 0 && a.k_token % 8 == 0 && a.k_head % 8 == 0 && a.v_token % 8 == 0 &&
                     a.v_head % 8 == 0 && a.k_token < (1 << 24) && a.v_token < (1 << 24);
  return lines ? prompt_form_launch<DP, TURNS, true>(a, s) : prompt_form_launch<DP, TURNS, false>(a, s);
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
  const bool launched = d <= 64 ? prompt_launch<64, true>(a, s) : d <= 96 ? prompt_launch<96, true>(a, s)
                        : d <= 128 ? prompt_launch<128, true>(a, s) : prompt_launch<256, false>(a, s);
  if (!launched) return PTQ_ERR_HIP;
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

}  // namespace ptq
