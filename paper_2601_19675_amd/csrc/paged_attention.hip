// Attention over the paged quantized cache, for up to 16 query rows that share a key head: single tokens, or a few of them.
//
//   score_j = softmax_scale ks_j (q . (code_j - zero_j)),   O = sum_j p_j vs_j (code'_j - zero'_j) / sum_j p_j,   p_j = exp(score_j - max)
//
// Bound: the cache's bytes, read once.  The 16 columns of the matrix instruction are the query rows of a key head (heads of the
// group times tokens), so the codes are loaded and made float16 once for all of them.  A workgroup's four waves share out
// its keys, 32 of a wave at a time, each with a running maximum, and meet in LDS.  Where there is more to do than a wave of workgroups
// per sequence and key head would share evenly, the contexts of all sequences are laid end to end (128 keys a block) and dealt out in
// equal shares, two workgroups to a compute unit; what a sequence got from several workgroups meets in a second kernel.
// Nothing is staged: a lane loads the codes that it feeds to the matrix instruction.  Keys: row = lane, d / 4 codes side by side.  Values
// have to come as eight keys of one channel: a lane takes d / 16 channels of eight keys and transposes them with byte
// permutes; which channels a row of the instruction stands for is free, and so is the order of keys, which is that in which the scores
// leave the first product.
//
// 16 single tokens against up to 32768 keys, 32 heads of 128 channels over 8, 4 bits: 372 MB in 92.6 us, 4.0 TB/s (a large copy: 4.7).  Four against
// 700, 32 heads of their own, 8 bits: 13.0 us: 128 workgroups on 256 compute units, four trips to memory one after the other (sequence, page,
// codes, output), between them the five to six blocks of 32 keys that a wave has one after the other.
//
// What the vector unit does to a code is what the kernel would be bound by else, so codes go in as c 2^-24 (8 bits: one byte permute to
// a pair) or 16 c 2^-24 (4 bits: a mask), and the zeros' share is taken out of the sums: q . (c - z) = q . c - z sum q, and
// sum p (c' - z') = sum p c' - sum p z', the latter one more instruction in the same form, so that codes that equal their zeros
// give exact zeros.  The instruction sums such small numbers as if they were 2^-14 at least: its sums are good to 2^-21 of
// the terms for 16 c and for 8 bits (scores), to 2^-17 for the values' channels that come as c of 4 bits.
//
// The value's scale goes into the weight: with vs = mant 2^e, e enters the exponent that the running maximum is taken of, so
// that the weights that are rounded to float16 are at most 2^8 whatever the scales are (rounding: 2^-11 of a weight, the
// precision that bfloat16 outputs do not see), and is taken out of the sum of the weights again, which stays float32.  A row that sees a value's
// scale beyond 2^-40 or 2^40, where that would leave float32's range, adds up its weights relative to a maximum of their own instead, in a second walk
// through the keys (the cases above then take 145 and 18.5 us).
//
// With SHARED the sequences' keys begin behind the prefix that their group has in common (ptq_paged_attention_shared), and the parts that
// paged_attention_chunk.hip has left of the prefix join theirs at the end, or in a kernel of their own where a sequence is shared out.  64 sequences, 151 to 732
// keys of their own, 8 key heads of 128 channels in 8 bits (58 MB of codes): 26 us with the join.
#include <algorithm>

#include "paged_attention.h"
#include "static_for.h"
#include "stored_rows.h"

namespace ptq {
namespace {

constexpr int kRows = 16, kBlock = 32, kWaves = 4, kShareBlock = kWaves * kBlock;
constexpr int kFarExponent = 40;   // of a value's scale that the sum of the weights does not go through

// blocks that a sequence counts for in the shares: one at least, if it has queries (somebody has to write their zeros)
__device__ __forceinline__ int share_blocks(const AttendArgs& a, const Sequence& q) {
  return q.queries == 0 ? 0 : max(1, (q.end - q.begin + kShareBlock - 1) / kShareBlock);
}
// ... in the shares that SHARED has
template <bool SHARED>
__device__ __forceinline__ int shared_out(const AttendArgs& a, const Sequence& q) {
  const int blocks = share_blocks(a, q);
  return SHARED && blocks <= a.few_blocks ? 0 : blocks;
}
// a sequence, of one that shares a prefix what is behind it
template <bool SHARED>
__device__ __forceinline__ Sequence own_of(const AttendArgs& a, int s) {
  Sequence q = sequence_of(a, s);
  if constexpr (SHARED) q.begin = min(max(q.begin, shared_of(a, s)), q.end);
  return q;
}
// The parts that a (token, head) has of its prefix: where row p of them is.
struct PrefixParts {
  const float *part, *ml;
  int64_t first;
  int step, most, parts;
  __device__ __forceinline__ int64_t row(int p) const { return p == 0 ? first : min(first + (2 * p - 1) * (int64_t)step, (int64_t)most); }
};
__device__ __forceinline__ PrefixParts prefix_parts(const AttendArgs& a, int seq, int64_t at) {
  PrefixParts r{a.alone, a.alone_ml, at, 0, INT32_MAX, 0};
  if (shared_of(a, seq) == 0) return r;
  const int2 where = a.where[at];
  if (where.x >= 0) {
    r.part = a.pre_part;
    r.ml = a.pre_ml;
    r.step = a.slot_rows;
    // (where sequences do not lie one after the other, nobody may have written `where`: whatever it holds, what is read is part of the workspace)
    r.most = 2 * kChunkShares * a.slot_rows - 1;
    r.first = min(where.x, r.most);
  }
  r.parts = where.x < 0 ? 1 : min(max(where.y, 0), kChunkShares);
  return r;
}
struct __attribute__((packed, aligned(4))) Four { float e[4]; };
// 2^-e, by its bits: those of 1, and -2^23 times e (which the compiler makes two instructions)
__device__ __forceinline__ float power_below(int e) {
  float f;
  asm("v_mad_i32_i24 %0, %1, %2, 1.0" : "=v"(f) : "v"(e), "s"(-(1 << 23)));
  return f;
}

template <int BITS, int DP>
struct Shape {
  static constexpr int kKeyCodes = DP / 4;                    // of a key, per lane
  static constexpr int kKeyWords = kKeyCodes * BITS / 32;
  static constexpr int kValCodes = DP / 16;                   // of a value, per lane
  static constexpr int kValWords = kValCodes * BITS / 32;     // 0: half a word
};

// eight codes of a key, in order, as c 2^-24 (8 bits) or 16 c 2^-24
template <int BITS>
__device__ __forceinline__ f16x8 key_codes(const uint32_t* w) {
  if constexpr (BITS == 8) {
    return f16x8_of(perm(0, w[0], 0x0c010c00u), perm(0, w[0], 0x0c030c02u), perm(0, w[1], 0x0c010c00u), perm(0, w[1], 0x0c030c02u));
  } else {
    return f16x8_of((w[0] << 4) & 0x00f000f0u, w[0] & 0x00f000f0u, (w[0] >> 4) & 0x00f000f0u, (w[0] >> 8) & 0x00f000f0u);
  }
}

// HALVES: pages of 16 tokens and more, so that each half of a block lies in one page, whose number is the wave's (addresses are scalar
// work); WHOLE: d == DP
template <int BITS, int DP, bool HALVES, bool WHOLE, bool SHARED>
__global__ __launch_bounds__(kWaves * 64, DP > 128 || !HALVES ? 1 : 2) void attend_rows_kernel(AttendArgs a) {
  using S = Shape<BITS, DP>;
  constexpr int kSteps = DP / 32;      // matrix instructions to a score
  constexpr int kOut = DP / 16;        // ... to an output
  constexpr int kCodeExp = BITS == 8 ? 24 : 20;   // a key's code c goes in as c 2^-kCodeExp
  extern __shared__ __attribute__((aligned(16))) float smem[];
  float (*lds_o)[kRows][DP + 4] = reinterpret_cast<float (*)[kRows][DP + 4]>(smem);
  f32x4 (*lds_ml)[kRows] = reinterpret_cast<f32x4 (*)[kRows]>(smem + kWaves * kRows * (DP + 4));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int head = blockIdx.y;
  // the workgroup's share: blocks [off, off + left) of sequence seq and on, `before` blocks before that sequence
  int seq = blockIdx.z, off = 0;
  int before = 0, share = 1, left = INT32_MAX;
  const bool mixed = SHARED && a.mixed, whole = a.splits == 1 || (mixed && (int)blockIdx.z < a.b);
  const int nth = mixed ? (int)blockIdx.z - a.b : (int)blockIdx.x, all = mixed ? (int)gridDim.z - a.b : (int)gridDim.x;   // of the workgroups with shares
  if (!whole) {
    int total = 0;
    for (int s0 = 0; s0 < a.b; s0 += kWave) total += s0 + lane < a.b ? shared_out<SHARED>(a, own_of<SHARED>(a, s0 + lane)) : 0;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) total += __shfl_xor(total, o);
    total = __builtin_amdgcn_readfirstlane(total);
    share = max(a.least_share, (total + all - 1) / all);
    const int64_t mine = (int64_t)nth * share;
    if (mine >= total) return;
    left = min(share, total - (int)mine);
    for (int s0 = 0;; s0 += kWave) {   // the first sequence that reaches past `mine`
      const int n = s0 + lane < a.b ? shared_out<SHARED>(a, own_of<SHARED>(a, s0 + lane)) : 0;
      int upto = n;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const int v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
      }
      const uint64_t past = __ballot(before + upto > mine);
      if (past) {
        const int s = __builtin_ctzll(past);
        seq = s0 + s;
        before += __builtin_amdgcn_readlane(upto, s) - __builtin_amdgcn_readlane(n, s);
        break;
      }
      before += __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    off = (int)mine - before;
  }

  for (;; ++seq) {
  if (seq >= a.b) return;
  const Sequence q = own_of<SHARED>(a, seq);
  const int queries = min(q.queries, a.max_q), rows = queries * a.group;
  const int blocks = share_blocks(a, q);
  if (rows == 0 || (SHARED && (blocks > a.few_blocks) == whole)) {   // (not this workgroup's)
    if (whole) return;
    continue;
  }
  const int take = min(blocks - off, left);
  const int from = q.begin + off * kShareBlock, to = min(q.end, from + take * kShareBlock);
  const bool alone = take == blocks;   // nobody else has keys of this sequence
  const int part = alone ? 0 : nth - before / share;

  // the lane's query row, d as the keys have it: channels [g DP / 4, (g + 1) DP / 4)
  const int token = q.first + r / a.group, qhead = head * a.group + r % a.group;
  const bool live = r < rows;
  f16x8 fq[kSteps];
  float factor, qsum = 0.f;
  {
    float v[kSteps][8], top = 0.f;
    const uint16_t* Q = a.Q + (live ? token * a.q_token + qhead * a.q_head : 0);
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int c = g * (DP / 4) + 8 * u;
      run_to_f32<PTQ_BF16, 8>(load_run<PTQ_BF16, 8, false>(Q, c, a.d), c, live ? a.d : 0, v[u]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = fabsf(v[u][i]);
        top = fmaxf(top, x < INFINITY ? x : 0.f);
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    // a power of two of the row's own brings it below 2^15: bfloat16's eight bits are float16's too, but its exponents are not
    const int e = __builtin_amdgcn_frexp_expf(top);
    factor = ldexpf(a.scale, e - 15 + kCodeExp);
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f16x2 p = to_f16(ldexpf(v[u][2 * i], 15 - e), ldexpf(v[u][2 * i + 1], 15 - e));
        qsum += (float)p[0] + (float)p[1];
        w[i] = __builtin_bit_cast(uint32_t, p);
      }
      fq[u] = f16x8_of(w[0], w[1], w[2], w[3]);
    }
    qsum += __shfl_xor(qsum, 16);
    qsum += __shfl_xor(qsum, 32);
    qsum = ldexpf(qsum, -kCodeExp);
  }
  int lo, hi, lo_all, hi_all, unused;   // the row's keys; those that every row sees
  visible(a, q, live ? r / a.group : 0, lo, hi);
  visible(a, q, 0, unused, hi_all);
  visible(a, q, queries - 1, lo_all, unused);
  hi_all = min(hi_all, to);

  const int64_t plane = (a.c.pages * a.c.heads) << a.c.page_shift;   // rows of the keys, before those of the values
  const int32_t* table = a.table + seq * a.ldt;
  const int inside = (1 << a.c.page_shift) - 1, row_bytes = a.c.row_bytes;

  // what a block of 32 keys needs of the page table (-1: not there), and what the cache holds of it.  Key 4 g + i and 16 + 4 g + i
  // (i < 4) are the lane's own where scores and values are concerned, key r and 16 + r where it feeds a key's row.
  struct Pages { int key[2], own[HALVES ? 1 : 8]; };
  struct Block {
    uint32_t k[2][S::kKeyWords], v[8][S::kValWords > 0 ? S::kValWords : 1];
    Four ks[2], vs[2];
    uint32_t kz[2], vz[2];
  };
  auto page_of = [&](int key) {
    const int p = table[min(key, q.length - 1) >> a.c.page_shift];
    return ((key < to) & ((uint32_t)p < (uint64_t)a.c.pages)) ? p : -1;
  };
  auto pages_of = [&](int key0) {
    Pages p;
    if constexpr (HALVES) {
#pragma unroll
      for (int i = 0; i < 2; ++i) p.key[i] = page_of(key0 + 16 * i);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) p.key[i] = page_of(key0 + 16 * i + r);
#pragma unroll
      for (int i = 0; i < 8; ++i) p.own[i] = page_of(key0 + 16 * (i >> 2) + 4 * g + (i & 3));
    }
    return p;
  };
  auto row_of = [&](int page, int key) -> int64_t {
    return page < 0 ? 0 : (((int64_t)page * a.c.heads + head) << a.c.page_shift) + (key & inside);
  };
  // a lane's part of a row of codes, in bytes
  const int key_part = g * (S::kKeyCodes * BITS / 8), val_all = S::kValWords > 0 ? r * S::kValCodes * BITS / 8 : r * 2;
  const int val_part = WHOLE || val_all < row_bytes ? val_all : 0;
  auto key_load = [&](const uint8_t* in, uint32_t at, uint32_t (&k)[S::kKeyWords]) {
    if constexpr (WHOLE) {
      const AnyWords<S::kKeyWords, 4> w = *reinterpret_cast<const AnyWords<S::kKeyWords, 4>*>(in + at + key_part);
#pragma unroll
      for (int j = 0; j < S::kKeyWords; ++j) k[j] = w.w[j];
    } else {   // eight codes at a time; those past d meet zeros of the query
#pragma unroll
      for (int u = 0; u < kSteps; ++u) {
        const int part = key_part + u * BITS;
        const AnyWords<BITS / 4, 4> w = *reinterpret_cast<const AnyWords<BITS / 4, 4>*>(in + at + (part < row_bytes ? part : 0));
#pragma unroll
        for (int j = 0; j < BITS / 4; ++j) k[u * (BITS / 4) + j] = w.w[j];
      }
    }
  };
  auto val_load = [&](const uint8_t* in, uint32_t at, uint32_t (&v)[S::kValWords > 0 ? S::kValWords : 1]) {
    if constexpr (S::kValWords > 0) {
      const AnyWords<S::kValWords, 4> w = *reinterpret_cast<const AnyWords<S::kValWords, 4>*>(in + at);
#pragma unroll
      for (int j = 0; j < S::kValWords; ++j) v[j] = w.w[j];
    } else {
      v[0] = *reinterpret_cast<const uint16_t*>(in + at);
    }
  };
  auto fetch = [&](int key0, const Pages& p, Block& b) {
    if constexpr (HALVES) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t row = row_of(p.key[i], key0 + 16 * i);
        const uint8_t* kc = a.c.codes + row * row_bytes;
        const uint8_t* vc = kc + plane * row_bytes;
        const float* ks = a.c.scales + row;
        const uint8_t* kz = a.c.zeros + row;
        key_load(kc, r * row_bytes, b.k[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) val_load(vc + j * row_bytes, 4 * g * row_bytes + val_part, b.v[4 * i + j]);
        b.ks[i] = *reinterpret_cast<const Four*>(reinterpret_cast<const char*>(ks) + 16u * g);
        b.vs[i] = *reinterpret_cast<const Four*>(reinterpret_cast<const char*>(ks + plane) + 16u * g);
        b.kz[i] = reinterpret_cast<const AnyWords<1, 1>*>(kz + 4u * g)->w[0];
        b.vz[i] = reinterpret_cast<const AnyWords<1, 1>*>(kz + plane + 4u * g)->w[0];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) key_load(a.c.codes + row_of(p.key[i], key0 + 16 * i + r) * row_bytes, 0, b.k[i]);
      b.kz[0] = b.kz[1] = b.vz[0] = b.vz[1] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t row = row_of(p.own[i], key0 + 16 * (i >> 2) + 4 * g + (i & 3));
        b.ks[i >> 2].e[i & 3] = a.c.scales[row];
        b.vs[i >> 2].e[i & 3] = a.c.scales[plane + row];
        b.kz[i >> 2] |= (uint32_t)a.c.zeros[row] << (8 * (i & 3));
        b.vz[i >> 2] |= (uint32_t)a.c.zeros[plane + row] << (8 * (i & 3));
        val_load(a.c.codes + (plane + row) * row_bytes, val_part, b.v[i]);
      }
    }
  };

  f32x4 acc[kOut], acc_z[BITS == 8 ? 1 : 2] = {};   // (4 bits: for channels as c 2^-24, and as 16 c 2^-24)
#pragma unroll
  for (int i = 0; i < kOut; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kNoScore, l = 0.f;
  float furthest = 0.f;   // of the exponents of the value's scales that have been seen

  // log2 of the weights, with the exponents of their value's scales in them, and the latter's mantissas and exponents
  auto score = [&](int key0, const Pages& p, const Block& b, float (&x)[8], float (&mant)[8], int (&e)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < kSteps; ++u)
        s = __builtin_amdgcn_mfma_f32_16x16x32_f16(key_codes<BITS>(&b.k[i][u * (BITS / 4)]), fq[u], s, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int n = 4 * i + j;
        const float vs = b.vs[i].e[j];
        e[n] = __builtin_amdgcn_frexp_expf(vs);
        mant[n] = __builtin_amdgcn_frexp_mantf(vs);
        x[n] = fmaf(fmaf(-(float)((b.kz[i] >> (8 * j)) & 255u), qsum, s[j]), b.ks[i].e[j] * factor, (float)e[n]);
      }
    }
    bool all = (key0 >= lo_all) & (key0 + kBlock <= hi_all);
    if constexpr (HALVES) all &= (p.key[0] >= 0) & (p.key[1] >= 0);
    if (!HALVES || !all) {   // some row does not see some key
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = key0 + 16 * (i >> 2) + 4 * g + (i & 3);
        const bool seen = (key >= lo) & (key < min(hi, to)) & ((HALVES ? p.key[i >> 2] : p.own[HALVES ? 0 : i]) >= 0);
        mant[i] = seen ? mant[i] : 0.f;
        x[i] = seen ? x[i] : -INFINITY;
        e[i] = seen ? e[i] : 0;
      }
    }
  };
  auto compute = [&](int key0, const Pages& p, const Block& b) {
    float x[8], mant[8];
    int e[8];
    score(key0, p, b, x, mant, e);
    float top = kNoScore;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      top = fmaxf(top, x[i]);
      furthest = fmaxf(furthest, fabsf((float)e[i]));
    }
    // the maximum moves only when one of the row's own scores is 2^8 above it: until then weights stay small enough, and what other rows see does
    // not change a bit of this one
    if (__any(top > m + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = top > m + 8.f ? top : m, f = exp2_fast(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (f32x4& z : acc_z) z *= f;
#pragma unroll
      for (int i = 0; i < kOut; ++i) acc[i] *= f;
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float p0 = exp2_fast(x[i] - m), p1 = exp2_fast(x[i + 1] - m);
      l = fmaf(p0, power_below(e[i]), l);
      l = fmaf(p1, power_below(e[i + 1]), l);
      w[i >> 1] = __builtin_bit_cast(uint32_t, to_f16(p0 * mant[i], p1 * mant[i + 1]));
    }
    const f16x8 weights = f16x8_of(w[0], w[1], w[2], w[3]);
#pragma unroll
    for (int n = 0; n < (BITS == 8 ? 1 : 2); ++n) {
      const uint32_t z0 = b.vz[0] << (4 * n), z1 = b.vz[1] << (4 * n);
      acc_z[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16x8_of(perm(0, z0, 0x0c010c00u), perm(0, z0, 0x0c030c02u), perm(0, z1, 0x0c010c00u),
                                                                 perm(0, z1, 0x0c030c02u)), weights, acc_z[n], 0, 0, 0);
    }
    // channel by channel: eight keys of it
    if constexpr (BITS == 8) {
#pragma unroll
      for (int j = 0; j < S::kValWords; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t f[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) f[k] = perm(b.v[2 * k + 1][j], b.v[2 * k][j], 0x0c040c00u + 0x00010001u * c);
          acc[4 * j + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16x8_of(f[0], f[1], f[2], f[3]), weights, acc[4 * j + c], 0, 0, 0);
        }
    } else {
      constexpr int kHalves = S::kValWords > 0 ? 2 * S::kValWords : 1;
#pragma unroll
      for (int j = 0; j < kHalves; ++j) {   // a half word: channels 0, 2, 4, 6 or 1, 3, 5, 7 of eight, the second and fourth 16-fold
        uint32_t f[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t pair = perm(b.v[2 * k + 1][j >> 1], b.v[2 * k][j >> 1], j & 1 ? 0x07060302u : 0x05040100u), u = pair >> 8;
          f[k][0] = pair & 0x000f000fu;
          f[k][1] = pair & 0x00f000f0u;
          f[k][2] = u & 0x000f000fu;
          f[k][3] = u & 0x00f000f0u;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
          acc[4 * j + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16x8_of(f[0][c], f[1][c], f[2][c], f[3][c]), weights, acc[4 * j + c], 0, 0, 0);
      }
    }
  };

  // blocks wave, wave + 4, ...: the next one's codes and the page numbers of the one after are on their way during a block (two blocks'
  // codes, where the registers hold them, brought nothing)
  int key0 = from + wave * kBlock;
  if (key0 < to) {
    constexpr int kStep = kWaves * kBlock, kAhead = 1, kBuffers = kAhead + 1;
    Pages p[kBuffers + 1];
    Block b[kBuffers];
#pragma unroll
    for (int i = 0; i <= kAhead; ++i) p[i] = pages_of(key0 + i * kStep);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(key0 + i * kStep, p[i], b[i]);
    bool more = true;
    while (more) {
      static_for<kBuffers>([&](auto i_) {
        constexpr int i = decltype(i_)::value;
        if (!more) return;
        p[kBuffers] = pages_of(key0 + kBuffers * kStep);
        fetch(key0 + kAhead * kStep, p[(i + kAhead) % kBuffers], b[(i + kAhead) % kBuffers]);
        compute(key0, p[i], b[i]);
        p[i] = p[kBuffers];
        key0 += kStep;
        more = key0 < to;
      });
    }
  }
  float of = m;   // what the sum of the weights is relative to
  if (__builtin_expect(__any(furthest > kFarExponent), 0)) {   // rows that see a scale out of range: the sum once more, relative to a maximum of its own
    furthest = fmaxf(furthest, __shfl_xor(furthest, 16));
    furthest = fmaxf(furthest, __shfl_xor(furthest, 32));
    float sum = 0.f, top = kNoScore;
    for (key0 = from + wave * kBlock; key0 < to; key0 += kWaves * kBlock) {
      Block b;
      const Pages p = pages_of(key0);
      fetch(key0, p, b);
      float x[8], mant[8], most = kNoScore;
      int e[8];
      score(key0, p, b, x, mant, e);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] -= (float)e[i];
        most = fmaxf(most, x[i]);
      }
      most = fmaxf(most, __shfl_xor(most, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      const float next = fmaxf(top, most);
      sum *= exp2_fast(top - next);
      top = next;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += exp2_fast(x[i] - top);
    }
    l = furthest > kFarExponent ? sum : l;
    of = furthest > kFarExponent ? top : m;
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // the waves' parts meet: row 4 g + i of instruction n is lane 4 g + i's channel n
#pragma unroll
  for (int n = 0; n < kOut; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = 4 * g + i;
      int c;
      if constexpr (BITS == 8) c = s * S::kValCodes + n;
      else if constexpr (S::kValWords > 0) c = s * S::kValCodes + 8 * (n >> 3) + 2 * (n & 3) + ((n >> 2) & 1);
      else c = 8 * (s >> 1) + 2 * n + (s & 1);
      lds_o[wave][r][c] = BITS == 4 && (n & 1) ? (acc[n][i] - acc_z[BITS == 8 ? 0 : 1][i]) * 0x1p20f : (acc[n][i] - acc_z[0][i]) * 0x1p24f;
    }
  if (g == 0) lds_ml[wave][r] = f32x4{m, l, of, 0.f};
  __syncthreads();
  for (int i = threadIdx.x; i < rows * (DP / 4); i += kWaves * 64) {
    const int row = i / (DP / 4), c = i % (DP / 4) * 4;
    if (c >= a.d) continue;
    float top = kNoScore, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    f32x4 ml[kWaves];
    bool same = true;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      ml[w] = lds_ml[w][row];
      top = fmaxf(top, ml[w][0]);
      same &= ml[w][2] == ml[w][0];
    }
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = exp2_fast(ml[w][0] - top);
      sum += f * ml[w][1];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += f * lds_o[w][row][c + j];
    }
    if (!same) {   // numerator and sum have powers of two of their own; what they differ by may be more than a float32 holds
      float top_l = kNoScore;
      sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top_l = fmaxf(top_l, ml[w][2]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum += exp2_fast(ml[w][2] - top_l) * ml[w][1];
      const float half = exp2_fast(0.5f * (top - top_l)), inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = o[j] * inv * half * half;
      top = top_l;
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;   // a row that sees nothing: zeros
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] *= inv;
    }
    const int tok = q.first + row / a.group, h = head * a.group + row % a.group;
    if constexpr (SHARED) {
      if (whole) {   // all there is of the sequence's own keys: the prefix's parts join them here, sixteen at a time
        const PrefixParts pre = prefix_parts(a, seq, (int64_t)tok * a.hq + h);
        for (int p0 = 0; p0 < pre.parts; p0 += 16) {
          f32x4 v[16];
          f32x2 ml[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int64_t at = pre.row(min(p0 + j, pre.parts - 1));
            v[j] = *reinterpret_cast<const f32x4*>(pre.part + at * a.d + c);
            ml[j] = *reinterpret_cast<const f32x2*>(pre.ml + 2 * at);
          }
          float next = top;
#pragma unroll
          for (int j = 0; j < 16; ++j) next = fmaxf(next, ml[j][0]);
          const float before = exp2_fast(top - next) * sum;
          float w[16], all = before;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            w[j] = p0 + j < pre.parts ? exp2_fast(ml[j][0] - next) * ml[j][1] : 0.f;
            all += w[j];
          }
          const float inv = all == 0.f ? 0.f : 1.f / all;   // a row that has seen nothing: zeros
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            o[i] *= before * inv;
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i] += (w[j] * inv) * v[j][i];
          }
          top = next;
          sum = all;
        }
        store_run<PTQ_BF16, 4, false>(a.O + tok * a.o_token + h * a.o_head, c, a.d, o);
        continue;
      }
    }
    if (SHARED || !alone) {
      const int64_t at = ((int64_t)part * a.t + tok) * a.hq + h;
      *reinterpret_cast<f32x4*>(a.part + at * a.d + c) = f32x4{o[0], o[1], o[2], o[3]};
      if (c == 0) {
        a.ml[2 * at] = top;
        a.ml[2 * at + 1] = sum;
      }
    } else {
      store_run<PTQ_BF16, 4, false>(a.O + tok * a.o_token + h * a.o_head, c, a.d, o);
    }
  }
  if (whole) {
    if (mixed && head == 0)   // nothing to join
      for (int i = threadIdx.x; i < queries; i += kWaves * 64) a.parts[q.first + i] = 0;
    return;
  }
  if (off == 0 && head == 0) {
    const int parts = alone ? 1 : (before + blocks - 1) / share - before / share + 1;
    for (int i = threadIdx.x; i < queries; i += kWaves * 64) a.parts[q.first + i] = parts;
  }
  left -= take;
  if (left <= 0) return;
  before += blocks;
  off = 0;
  __syncthreads();   // the next sequence's parts go where this one's were
  }
}

// Joins the splits' parts of a (token, head), means of their keys' values and what those weigh: a lane looks at one part's maximum and sum, and has
// four channels of all parts.
__global__ __launch_bounds__(64) void attend_join_kernel(AttendArgs a) {
  const int tok = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, c = lane * 4;
  int seq = 0;   // the sequence that the token belongs to
  for (int n = a.b; n > 1;) {
    const int half = n >> 1;
    if (a.cu_q[seq + half] <= tok) seq += half;
    n -= half;
  }
  const Sequence q = sequence_of(a, seq);
  if (tok < q.first || tok - q.first >= min(q.queries, a.max_q)) return;
  const int parts = a.parts[tok];
  if (parts == 1) return;   // written by the one workgroup that had it
  const int64_t first = (int64_t)tok * a.hq + h, step = (int64_t)a.t * a.hq;
  float top = kNoScore, sum = 0.f;
  for (int s = lane; s < parts; s += 64) top = fmaxf(top, a.ml[2 * (first + s * step)]);
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const float* part = a.part + first * a.d + (c < a.d ? c : 0);
  for (int s0 = 0; s0 < parts; s0 += 64) {
    const int s = min(s0 + lane, parts - 1);
    float f = s0 + lane < parts ? exp2_fast(a.ml[2 * (first + s * step)] - top) * a.ml[2 * (first + s * step) + 1] : 0.f;
    float all = f;
#pragma unroll
    for (int n = 1; n < kWave; n <<= 1) all += __shfl_xor(all, n);
    all += sum;
    const float inv = all == 0.f ? 0.f : 1.f / all;   // a row that sees nothing: zeros
    o *= sum * inv;
    f *= inv;
    sum = all;
    const int here = min(64, parts - s0);
    for (int i = 0; i < here; i += 8) {   // (f is 0 past the last part)
      f32x4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const f32x4*>(part + (s0 + min(i + j, here - 1)) * step * a.d);
#pragma unroll
      for (int j = 0; j < 8; ++j) o += __shfl(f, i + j) * v[j];
    }
  }
  if (c >= a.d) return;
  const float v[4] = {o[0], o[1], o[2], o[3]};
  store_run<PTQ_BF16, 4, false>(a.O + tok * a.o_token + h * a.o_head, c, a.d, v);
}

// Joins the parts of a (token, head) that shares a prefix: those of the prefix, then those of what is behind it.  As above.
__global__ __launch_bounds__(64) void shared_join_kernel(AttendArgs a) {
  const int tok = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, c = lane * 4;
  const int seq = last_not_above(a.cu_q, 0, a.b, tok);
  const Sequence q = sequence_of(a, seq);
  if (tok < q.first || tok - q.first >= min(q.queries, a.max_q)) return;
  const int own = min(a.parts[tok], a.splits);
  if (own <= 0) return;   // written by the one workgroup that had it
  const int64_t first = (int64_t)tok * a.hq + h, step = (int64_t)a.t * a.hq;
  const PrefixParts pre = prefix_parts(a, seq, first);
  const int parts = pre.parts + own, cc = c < a.d ? c : 0;
  auto row_of = [&](int p) { return p < pre.parts ? pre.row(p) : first + (p - pre.parts) * step; };
  auto ml_of = [&](int p) { return *reinterpret_cast<const f32x2*>((p < pre.parts ? pre.ml : a.ml) + 2 * row_of(p)); };
  auto part_of = [&](int p) { return *reinterpret_cast<const f32x4*>((p < pre.parts ? pre.part : a.part) + row_of(p) * a.d + cc); };
  float top = kNoScore, sum = 0.f;
  for (int s = lane; s < parts; s += 64) top = fmaxf(top, ml_of(s)[0]);
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < parts; s0 += 64) {
    const int s = min(s0 + lane, parts - 1);
    const f32x2 ml = ml_of(s);
    float f = s0 + lane < parts ? exp2_fast(ml[0] - top) * ml[1] : 0.f;
    float all = f;
#pragma unroll
    for (int n = 1; n < kWave; n <<= 1) all += __shfl_xor(all, n);
    all += sum;
    const float inv = all == 0.f ? 0.f : 1.f / all;   // a row that sees nothing: zeros
    o *= sum * inv;
    f *= inv;
    sum = all;
    const int here = min(64, parts - s0);
    for (int i = 0; i < here; i += 8) {   // (f is 0 past the last part)
      f32x4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = part_of(s0 + min(i + j, here - 1));
#pragma unroll
      for (int j = 0; j < 8; ++j) o += __shfl(f, i + j) * v[j];
    }
  }
  if (c >= a.d) return;
  const float v[4] = {o[0], o[1], o[2], o[3]};
  store_run<PTQ_BF16, 4, false>(a.O + tok * a.o_token + h * a.o_head, c, a.d, v);
}

constexpr int kFewKeys = 2048;         // behind a prefix: one workgroup's
constexpr int64_t kPartRows = 65536;   // rows times splits at most: what the workspace holds

int64_t most_splits(int64_t rows, int64_t max_kv) {
  return std::max<int64_t>(1, std::min<int64_t>(ceil_div(max_kv, 256), kPartRows / std::max<int64_t>(rows, 1)));
}

constexpr int64_t kLongKeys = 4096, kMostSharedTiles = 4096;
constexpr int kShares = 512;          // workgroups that share the contexts: two to a compute unit
int64_t shares(int64_t hkv) { return std::max<int64_t>(1, kShares / hkv); }

template <int BITS, int DP, bool HALVES, bool WHOLE, bool SHARED>
bool rows_form_launch(const AttendArgs& a, hipStream_t s) {
  constexpr int kBytes = kWaves * kRows * (DP + 4 + 4) * (int)sizeof(float);
  if (!lds_opt_in<attend_rows_kernel<BITS, DP, HALVES, WHOLE, SHARED>>(kBytes)) return false;
  dim3 grid = a.splits > 1 ? dim3((unsigned)shares(a.c.heads), (unsigned)a.c.heads, 1) : dim3(1, (unsigned)a.c.heads, (unsigned)a.b);
  if (SHARED && a.mixed) grid = dim3(1, (unsigned)a.c.heads, (unsigned)(a.b + shares(a.c.heads)));
  attend_rows_kernel<BITS, DP, HALVES, WHOLE, SHARED><<<grid, kWaves * 64, kBytes, s>>>(a);
  return true;
}
template <int BITS, int DP, bool SHARED>
bool rows_launch(const AttendArgs& a, hipStream_t s) {
  if (a.c.page_shift < 4) return rows_form_launch<BITS, DP, false, false, SHARED>(a, s);
  return a.d == DP ? rows_form_launch<BITS, DP, true, true, SHARED>(a, s) : rows_form_launch<BITS, DP, true, false, SHARED>(a, s);
}
template <bool SHARED>
bool rows_launch_any(const AttendArgs& a, int bits, hipStream_t s) {
  return bits == 8 ? (a.d <= 64 ? rows_launch<8, 64, SHARED>(a, s) : a.d <= 128 ? rows_launch<8, 128, SHARED>(a, s) : rows_launch<8, 256, SHARED>(a, s))
                   : (a.d <= 64 ? rows_launch<4, 64, SHARED>(a, s) : a.d <= 128 ? rows_launch<4, 128, SHARED>(a, s) : rows_launch<4, 256, SHARED>(a, s));
}

}  // namespace

// which form is taken is not known here: what the larger one needs
size_t paged_attention_workspace_bytes(int64_t hq, int64_t d, int64_t t, int64_t max_kv) {
  const int64_t rows = hq * t, splits = most_splits(rows, max_kv);
  const int64_t rows_form = splits <= 1 ? 0 : splits * rows * (d + 2) + t;
  const int64_t chunk_form = max_kv < kSharedChunkKeys ? 0 : 2 * kChunkShares * std::min<int64_t>(kChunkRows, rows) * (d + 2) + 4 * kChunkShares;
  return align_up((size_t)std::max(rows_form, chunk_form) * sizeof(float), 256);
}

namespace {
AttendArgs attend_args(const void* Q, int64_t q_token, int64_t q_head, int64_t t, int64_t hq, int64_t d, const int32_t* cu_q, int64_t b,
                       int64_t max_q, const uint8_t* codes, const float* scales, const uint8_t* zeros, int64_t pages, int64_t page, int64_t hkv,
                       int bits, const int32_t* table, int64_t ldt, const int32_t* kv_lens, int64_t max_kv, double softmax_scale, int causal,
                       int64_t window, void* O, int64_t o_token, int64_t o_head) {
  AttendArgs a{};
  a.Q = static_cast<const uint16_t*>(Q);
  a.O = static_cast<uint16_t*>(O);
  a.q_token = q_token, a.q_head = q_head, a.o_token = o_token, a.o_head = o_head;
  a.cu_q = cu_q, a.table = table, a.kv_lens = kv_lens, a.ldt = ldt;
  a.c = KvCache{const_cast<uint8_t*>(codes), const_cast<float*>(scales), const_cast<uint8_t*>(zeros), pages, (int)hkv,
                __builtin_ctz((unsigned)page), (int)(d * bits / 8)};
  a.scale = (float)(softmax_scale * 1.4426950408889634);
  a.t = (int)t, a.b = (int)b, a.hq = (int)hq, a.group = (int)(hq / hkv), a.d = (int)d, a.max_q = (int)max_q, a.max_kv = (int)max_kv;
  a.causal = causal, a.window = (int)std::min<int64_t>(window, INT32_MAX / 2);
  return a;
}
}  // namespace

ptq_status paged_attention_launch(const void* Q, int64_t q_token, int64_t q_head, int64_t t, int64_t hq, int64_t d,
                                  const int32_t* cu_q, int64_t b, int64_t max_q, const uint8_t* codes, const float* scales,
                                  const uint8_t* zeros, int64_t pages, int64_t page, int64_t hkv, int bits,
                                  const int32_t* table, int64_t ldt, const int32_t* kv_lens, int64_t max_kv,
                                  double softmax_scale, int causal, int64_t window, void* O, int64_t o_token, int64_t o_head,
                                  void* ws, hipStream_t s) {
  AttendArgs a = attend_args(Q, q_token, q_head, t, hq, d, cu_q, b, max_q, codes, scales, zeros, pages, page, hkv, bits, table, ldt, kv_lens, max_kv,
                             softmax_scale, causal, window, O, o_token, o_head);
  const bool rows_form = max_q * a.group <= kRows;
  // the keys a split has to get through: those in the window, if there is one
  const int64_t keys = window > 0 ? std::min<int64_t>(max_kv, (int64_t)a.window + max_q + 63) : max_kv;
  if (rows_form) {
    // Shares cost a second kernel and its launch (4 us), which 2048 keys in one workgroup take (6 us from 256 keys on): shorter contexts
    // stay whole, and so do more sequences and heads than four rounds of workgroups.
    a.splits = keys < 2048 || b * hkv >= 4 * kShares || b * ceil_div(max_kv, kShareBlock) > INT32_MAX / 2 ? 1 : (int)most_splits(hq * t, max_kv);
    // 256 keys at least to a share (two contexts of 4129, 32 heads of 128 channels over 8: 17.3 us, with 512 21.3; from four contexts of 8192
    // on no difference), and a sequence's parts fit the workspace
    a.least_share = a.splits > 1 ? (int)std::max<int64_t>(2, ceil_div(ceil_div(max_kv, kShareBlock), a.splits - 1)) : 1;
  } else {
    // Workgroups run in rounds, one to a compute unit, and the host does not know how much each has to do.  Shares cost each workgroup
    // a second item's queries and half done outputs, and a second kernel: they are taken where the last round would leave a fifth of the
    // compute units idle or more, and for a single round of long contexts, which are seldom the same.  us, whole | in shares, contexts of one length (of
    // different ones, down to a fifth), 128 channels: 8 items of 2048 keys 78 | 45, 256 of 2048 84 | 97 (84 | 91), of 4096 162 | 174 (159 | 143), of
    // 16384 643 | 656 (598 | 430); 400 of 16384 (849 | 813); 512 of 16384 1208 | 1248 (774 | 846); 768 of 8192 874 | 912; 64 channels: 212 of 5000
    // (154 | 118), 324 of 2500 161 | 131, 576 of 5000 431 | 390; a chunk of 512 beside 15 single tokens, all of 32768: 192 of the 1024 tiles that max_q
    // alone would say, 3000 | 945.
    const ChunkItems items = paged_attention_chunk_items(a);
    const int64_t rounds = ceil_div(items.busy, kChunkShares), idle = rounds * kChunkShares - items.busy;
    const bool shared = keys >= kSharedChunkKeys && (5 * idle >= rounds * kChunkShares || (rounds == 1 && keys >= kLongKeys));
    // (every workgroup looks through all tiles for its share, and counts work in 32 bits)
    a.splits = !shared || items.tiles / hkv > kMostSharedTiles || items.tiles * ceil_div(max_kv, 64) > INT32_MAX / 4 ? 1 : 2;
    a.slot_rows = (int)std::min<int64_t>(kChunkRows, hq * t);
  }
  const int64_t part_rows = rows_form ? a.splits * t * hq : 2 * kChunkShares * a.slot_rows;
  a.part = static_cast<float*>(ws);
  a.ml = a.part + part_rows * d;
  a.parts = reinterpret_cast<int*>(a.ml + part_rows * 2);
  if (rows_form) {
    if (!rows_launch_any<false>(a, bits, s)) return PTQ_ERR_HIP;
  } else {
    const ptq_status rc = paged_attention_chunk_launch(a, bits, s);
    if (rc != PTQ_OK) return rc;
  }
  if (rows_form && a.splits > 1) attend_join_kernel<<<dim3((unsigned)t, (unsigned)hq), 64, 0, s>>>(a);
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

// parts of what is behind the prefixes, of the prefixes (shares', and tiles of rows that a share has alone), what begins in a share, the parts'
// maxima and sums, where a row's first part is, how many a token has; or what the call without prefixes needs
namespace {
struct SharedPlan { int64_t splits, own_rows, prefix_rows, slot_rows, floats; };
SharedPlan shared_plan(int64_t hq, int64_t d, int64_t t, int64_t max_kv) {
  SharedPlan p;
  const int64_t rows = hq * t;
  p.splits = most_splits(rows, max_kv);
  p.own_rows = p.splits * rows;
  p.slot_rows = std::min<int64_t>(kChunkRows, rows);
  p.prefix_rows = 2 * kChunkShares * p.slot_rows;
  p.floats = (p.own_rows + p.prefix_rows + rows) * (d + 2) + 2 * rows + t + 4 * kChunkShares;
  return p;
}
}  // namespace
namespace {
// Whether prefixes gone through apart take less time than every sequence's whole way, in us as measured and by what the bounds say.  Every sequence by itself: 15, and
// 0.135 to a megabyte of codes (pages that several name are in the caches).  Apart: 25, 1.7e-4 for a key of a prefix, a key head and a tile of 256 rows of 128 channels,
// 0.25 for each of a row's parts beyond 32, and what is behind the prefixes as before.  A prefix that a die's L2 holds (4 MB) is read from there by all
// sequences as fast.  32 heads of 128 channels over 8, 8 bits, apart | by itself: 8 behind 1000 keys 27 | 18, 64 41 | 28; 4 behind 8192 32 | 27, 8
// 32 | 36, 16 33 | 54; 4 behind 32768 52 | 53, 8 52 | 88, 64 80 | 498.  16 heads over 1: 16 behind 32768 94 | 38.  32 over 32: 8 behind 2048 35 | 31, 12 39 | 47.  The
// numbers are fitted to caches some of whose scales lie below 2^-18 (apart: 4 or 8 behind 32768 73, 64 116), and cautious elsewhere.  Misses seen: 16 in two
// groups behind 8192 with up to 7800 keys of their own 71 | 66; 256 channels, 16 heads over 4, 64 behind 2048 111 | 61, 16 behind 8192 100 | 63, both gone
// through apart; 4 bits, 8 behind 32768 50 | 66, 16 behind 8192 32 | 41, neither; 2 of 64 of 8400 keys behind 8192 227 | 198, apart, as if all were behind it.
bool prefixes_pay(const AttendArgs& a, int bits) {
  const double key = (double)a.c.heads * a.d * 2 * bits / 8 * 1e-6;   // megabytes
  const double tiles = (double)ceil_div((int64_t)a.t * a.group, 256) + a.groups - 1, prefix = a.max_shared;
  if (prefix * key <= 4.0) return false;
  const double parts = std::min(kChunkShares / (a.c.heads * tiles), prefix / 128);
  const double each = 15 + 0.135 * a.b * key * a.max_kv;
  const double apart = 25 + 1.7e-4 * a.c.heads * tiles * prefix * a.d / 128 + 0.25 * std::max(0.0, parts - 32) + 0.135 * a.b * key * (a.max_kv - prefix);
  return apart < each;
}
}  // namespace
size_t paged_attention_shared_workspace_bytes(int64_t hq, int64_t d, int64_t t, int64_t max_kv) {
  return std::max(align_up((size_t)shared_plan(hq, d, t, max_kv).floats * sizeof(float), 256), paged_attention_workspace_bytes(hq, d, t, max_kv));
}

ptq_status paged_attention_shared_launch(const void* Q, int64_t q_token, int64_t q_head, int64_t t, int64_t hq, int64_t d,
                                         const int32_t* cu_q, int64_t b, int64_t max_q, const uint8_t* codes, const float* scales,
                                         const uint8_t* zeros, int64_t pages, int64_t page, int64_t hkv, int bits, const int32_t* table,
                                         int64_t ldt, const int32_t* kv_lens, int64_t max_kv, const int32_t* cu_groups, const int32_t* shared,
                                         int64_t groups, int64_t max_shared, double softmax_scale, int causal, void* O, int64_t o_token,
                                         int64_t o_head, void* ws, hipStream_t s) {
  AttendArgs a = attend_args(Q, q_token, q_head, t, hq, d, cu_q, b, max_q, codes, scales, zeros, pages, page, hkv, bits, table, ldt, kv_lens, max_kv,
                             softmax_scale, causal, 0, O, o_token, o_head);
  a.cu_groups = cu_groups, a.shared = shared, a.groups = (int)groups, a.max_shared = (int)std::min(max_shared, max_kv);
  // Chunks of tokens are bound by their products, which are no fewer with a prefix in common, and prefixes of less than a block are not gone
  // through apart.  Every workgroup looks through all tiles of rows for its share, and counts work in 32 bits, with whole shares up to six times of it.
  if (max_q * a.group > kRows || a.max_shared < 64 || groups == 0 || paged_attention_prefix_tiles(a) > kMostSharedTiles ||
      paged_attention_prefix_work(a) > INT32_MAX / 8 || !prefixes_pay(a, bits))
    return paged_attention_launch(Q, q_token, q_head, t, hq, d, cu_q, b, max_q, codes, scales, zeros, pages, page, hkv, bits, table, ldt, kv_lens,
                                  max_kv, softmax_scale, causal, 0, O, o_token, o_head, ws, s);
  const SharedPlan p = shared_plan(hq, d, t, max_kv);
  const int64_t rows = hq * t;
  AttendArgs pre = a;
  a.part = static_cast<float*>(ws);
  pre.part = a.part + p.own_rows * d;
  pre.alone = pre.part + p.prefix_rows * d;
  pre.parts = reinterpret_cast<int*>(pre.alone + rows * d);
  a.ml = pre.alone + rows * d + 4 * kChunkShares;
  pre.ml = a.ml + 2 * p.own_rows;
  pre.alone_ml = pre.ml + 2 * p.prefix_rows;
  pre.where = reinterpret_cast<int2*>(pre.alone_ml + 2 * rows);
  a.parts = reinterpret_cast<int*>(pre.where + rows);
  pre.splits = 2;
  a.slot_rows = pre.slot_rows = (int)p.slot_rows;
  a.pre_part = pre.part, a.pre_ml = pre.ml;
  a.alone = pre.alone, a.alone_ml = pre.alone_ml, a.where = pre.where;
  // What is behind the prefixes is seldom long, and with one workgroup to a sequence and key head the parts join there: 25 us and no second kernel in place of
  // 42 and 11 (64 sequences, 8 key heads, 151 to 732 keys behind a prefix).  The difference of the two bounds says how long it
  // seems to be.  A sequence behind a short prefix, or of no group, has more than that: it goes in shares beside the others, if the bounds leave room for one.
  // (8 behind 32768 keys and one of 33000 by itself: 88 us, with a workgroup to each 359.  Where there is none it costs 2 us: 64 behind 32768 87 and 85.)
  const int64_t own = max_kv - a.max_shared;
  const bool never = b * hkv >= 4 * kShares || b * ceil_div(max_kv, kShareBlock) > INT32_MAX / 2 || p.splits == 1;
  a.mixed = !never && own < kFewKeys && max_kv > kFewKeys;
  a.splits = never || (own < kFewKeys && !a.mixed) ? 1 : (int)p.splits;
  a.few_blocks = a.mixed ? kFewKeys / kShareBlock : a.splits > 1 ? 0 : INT32_MAX;
  a.least_share = a.splits > 1 ? (int)std::max<int64_t>(2, ceil_div(ceil_div(max_kv, kShareBlock), a.splits - 1)) : 1;
  const ptq_status rc = paged_attention_prefix_launch(pre, bits, s);
  if (rc != PTQ_OK) return rc;
  if (!rows_launch_any<true>(a, bits, s)) return PTQ_ERR_HIP;
  if (a.splits > 1) shared_join_kernel<<<dim3((unsigned)t, (unsigned)hq), 64, 0, s>>>(a);
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

}  // namespace ptq
