// What the two forms of attention over the paged 8- or 4-bit cache share (paged_attention.hip: single tokens and their
// kind; paged_attention_chunk.hip: chunks of tokens).  Not part of the C ABI.
//
// Codes become float16 exactly, by their bits: those of c itself are the float16 c 2^-24 (below float16's normal numbers, which
// the matrix instructions take as they are), 0x6400 | c is 1024 + c.  Products with them are exact, so the grids' scales can
// stay float32 and outside the matrix instructions.
#pragma once
#include "kv_cache.h"

namespace ptq {

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;

constexpr float kNoScore = -3e38f;       // a running maximum before the first score
constexpr uint32_t kF16Of1024 = 0x64646464u;

struct AttendArgs {
  const uint16_t* Q; uint16_t* O;        // bfloat16
  int64_t q_token, q_head, o_token, o_head;
  const int32_t* cu_q; const int32_t* table; const int32_t* kv_lens;
  int64_t ldt;
  KvCache c;
  float scale;                           // softmax_scale log2(e): scores are powers of two
  int t, b, hq, group, d, max_q, max_kv, causal, window;
  int splits;                            // > 1: workgroups have shares of the work, and partial results go to part and ml
  int least_share;                       // rows form: blocks of 128 keys that a workgroup takes at least
  int slot_rows;                         // chunk form: rows of a part
  // rows form: [part][token][head][...]; chunk form: [share][item it ends, item it begins][row][...]
  float* part;                           // [...][d]: the mean of the part's values
  float* ml;                             // [...][2]: a maximum, the sum of the weights relative to it
  int* parts;                            // rows form: [token], how many there are; chunk form: [share][4], see there
};

// a sequence's queries and keys
struct Sequence {
  int first, queries, length;            // first token, new tokens, keys that the table and max_kv reach
  int place;                             // of the first query, among all keys that the sequence is said to have
  int begin, end;                        // keys that some query sees lie in [begin, end), begin a multiple of 64
};
__device__ __forceinline__ Sequence sequence_of(const AttendArgs& a, int s) {
  Sequence q;
  const int64_t from = a.cu_q[s], to = a.cu_q[s + 1];
  q.first = (int)from;
  q.queries = from >= 0 && to <= a.t && to > from ? (int)(to - from) : 0;
  const int64_t most = min((int64_t)a.max_kv, a.ldt << a.c.page_shift);
  const int keys = max(0, a.kv_lens[s]);
  q.place = keys - q.queries;
  q.length = (int)min((int64_t)keys, most);
  q.end = q.length;
  q.begin = 0;
  if (a.window > 0) q.begin = max(0, q.place - a.window + 1) & ~63;
  q.begin = min(q.begin, q.end);
  return q;
}
// keys [lo, hi) that query i of a sequence sees
__device__ __forceinline__ void visible(const AttendArgs& a, const Sequence& q, int i, int& lo, int& hi) {
  const int place = q.place + i;
  hi = a.causal ? max(0, min(q.length, place + 1)) : q.length;
  lo = a.window > 0 ? max(0, place - a.window + 1) : 0;
}

__device__ __forceinline__ uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }
__device__ __forceinline__ uint32_t h2_sub(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, a) - __builtin_bit_cast(f16x2, b));
}
// a / 16 - b; contracted into one instruction, and exact either way
__device__ __forceinline__ uint32_t h2_sixteenth_sub(uint32_t a, uint32_t b) {
  const f16x2 s = {(_Float16)0.0625f, (_Float16)0.0625f};
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, a), s, -__builtin_bit_cast(f16x2, b)));
}
// float16 pairs 1024 + byte 0 | 1 (or 2 | 3) of w
__device__ __forceinline__ uint32_t low_bytes(uint32_t w) { return perm(kF16Of1024, w, 0x04010400u); }
__device__ __forceinline__ uint32_t high_bytes(uint32_t w) { return perm(kF16Of1024, w, 0x04030402u); }
__device__ __forceinline__ f16x8 f16x8_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(f16x8, u32x4{a, b, c, d});
}

// what is subtracted from a pair of values: z holds the bits of 1024 + zero twice or for two rows
struct Zeros {
  uint32_t by1;    // 1024 + zero
  uint32_t by16;   // 64 + zero
};
template <int BITS>
__device__ __forceinline__ Zeros zeros_of(uint32_t z) {
  Zeros r{z, 0};
  if constexpr (BITS == 4) r.by16 = h2_sub(z, 0x63806380u);   // 960
  return r;
}
// four pairs from the nibbles of w: bits 0..3 | 16..19, 4..7 | 20..23, ...
__device__ __forceinline__ void nibble_pairs(uint32_t w, const Zeros& z, uint32_t (&p)[4]) {
  const uint32_t u = w >> 8;
  p[0] = h2_sub((w & 0x000f000fu) | 0x64006400u, z.by1);
  p[1] = h2_sixteenth_sub((w & 0x00f000f0u) | 0x64006400u, z.by16);
  p[2] = h2_sub((u & 0x000f000fu) | 0x64006400u, z.by1);
  p[3] = h2_sixteenth_sub((u & 0x00f000f0u) | 0x64006400u, z.by16);
}
// eight codes of a row, in order
template <int BITS>
__device__ __forceinline__ f16x8 row_codes(const uint32_t* w, const Zeros& z) {
  if constexpr (BITS == 8) {
    return f16x8_of(h2_sub(low_bytes(w[0]), z.by1), h2_sub(high_bytes(w[0]), z.by1), h2_sub(low_bytes(w[1]), z.by1),
                    h2_sub(high_bytes(w[1]), z.by1));
  } else {
    uint32_t p[4];
    nibble_pairs(w[0], z, p);
    return f16x8_of(p[0], p[1], p[2], p[3]);
  }
}

__device__ __forceinline__ f16x2 to_f16(float a, float b) {
  return __builtin_convertvector(f32x2{a, b}, f16x2);   // to nearest
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr int kChunkShares = 256, kChunkRows = 256;   // workgroups that have shares; query rows of a workgroup at most
constexpr int kSharedChunkKeys = 2048;                 // shorter contexts are not shared out
// tiles of rows of all sequences and key heads: by max_q, and those of them that can hold a row of the tokens there are
struct ChunkItems { int64_t tiles, busy; };
ChunkItems paged_attention_chunk_items(const AttendArgs& a);
ptq_status paged_attention_chunk_launch(const AttendArgs& a, int bits, hipStream_t s);

}  // namespace ptq
