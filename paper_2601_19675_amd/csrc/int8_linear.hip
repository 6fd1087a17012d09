// Product of 8-bit tokens with an 8-bit weight:  O = (sum_k A[i][k] W[j][k]) a_scale[i] w_scale[j] + bias[j].
//
// Both operands have k side by side, which is how the matrix instructions want them: 16 bytes of a row are a lane's operand,
// no transposition and no unpacking.  Sums are 32-bit integers, hence exact and independent of the order (n <= 131056 keeps
// 128 * 128 * n below 2^31); the epilogue converts, scales twice and adds, each rounded to float32.
//
// With few tokens the weight's bytes are the bound: its rows go straight from memory into registers (skinny_kernel).  Beyond
// that the products are: tiles of W rows x tokens staged in LDS (tile_kernel).  form_of has the rule.
#include <algorithm>

#include "lds_dma.h"
#include "stored_rows.h"

namespace ptq {
namespace {

typedef __attribute__((__vector_size__(16 * sizeof(int)))) int i32x16;

struct LinearArgs {
  const int8_t* A; const float* as; const int8_t* W; const float* ws; const float* bias; void* O;
  int64_t lda, ldw, ldo;
  int t, m, n;
};

// N consecutive outputs of a token
template <int DT, int N>
__device__ __forceinline__ void store_outputs(const LinearArgs& a, int token, int row, float as, const int (&sum)[N],
                                              const float (&ws)[N], const float (&bias)[N]) {
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = (float)sum[i] * as * ws[i] + bias[i];
  store_run<DT, N, true>(static_cast<typename StoredType<DT>::type*>(a.O) + token * a.ldo, row, a.m, v);
}
// scales and biases of N consecutive rows of W (past the last: its own)
template <int N>
__device__ __forceinline__ void load_channels(const LinearArgs& a, int row, float (&ws)[N], float (&bias)[N]) {
  const float* b = a.bias ? a.bias : a.ws;   // no branch around a load
  if (row + N <= a.m) {
    const AnyWords<N, 4> x = *reinterpret_cast<const AnyWords<N, 4>*>(a.ws + row), y = *reinterpret_cast<const AnyWords<N, 4>*>(b + row);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      ws[i] = __uint_as_float(x.w[i]);
      bias[i] = __uint_as_float(y.w[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = min(row + i, a.m - 1);
      ws[i] = a.ws[at];
      bias[i] = b[at];
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) bias[i] = a.bias ? bias[i] : 0.f;
}

// ---- few tokens ---------------------------------------------------------------------------------------------
// A workgroup takes 16 rows of W; its eight waves share out the 64-byte steps of k and meet in LDS.  Every byte of W is read
// once, eight loads of 16 bytes a lane on their way: one trip to memory for n = 4096.  The tokens (columns of the matrix
// instruction, TB x 16 of them) come from the L2.  One token, 4096 x 4096: 5.3 us for 16.8 MB (3.6 at the rate of a copy).
constexpr int kSkinnyWaves = 8, kSkinnyAhead = 8;

template <int DT, int TB>
__global__ __launch_bounds__(kSkinnyWaves * 64) void skinny_kernel(LinearArgs a) {
  __shared__ i32x4 part[kSkinnyWaves][TB][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int row0 = blockIdx.x * 16;
  const int8_t* W = a.W + (int64_t)min(row0 + r, a.m - 1) * a.ldw;
  const int8_t* A[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) A[b] = a.A + (int64_t)min(b * 16 + r, a.t - 1) * a.lda;
  i32x4 acc[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) acc[b] = i32x4{0, 0, 0, 0};
  constexpr int kAhead = TB > 2 ? kSkinnyAhead / 2 : kSkinnyAhead;
  const int steps = (a.n + 63) / 64;
  for (int s0 = wave; s0 < steps; s0 += kSkinnyWaves * kAhead) {
    i32x4 w[kAhead], x[kAhead][TB];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int k = (s0 + i * kSkinnyWaves) * 64 + g * 16, at = k < a.n ? k : 0;
      w[i] = *reinterpret_cast<const i32x4*>(W + at);
#pragma unroll
      for (int b = 0; b < TB; ++b) x[i][b] = *reinterpret_cast<const i32x4*>(A[b] + at);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int k = (s0 + i * kSkinnyWaves) * 64 + g * 16;
      if (k >= a.n) w[i] = i32x4{0, 0, 0, 0};
#pragma unroll
      for (int b = 0; b < TB; ++b) acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[i][b], acc[b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int b = 0; b < TB; ++b) part[wave][b][lane] = acc[b];
  __syncthreads();
  if (wave >= TB) return;
  i32x4 sum = part[0][wave][lane];
#pragma unroll
  for (int w = 1; w < kSkinnyWaves; ++w) sum += part[w][wave][lane];
  const int token = wave * 16 + r, row = row0 + 4 * g;   // the instruction's columns are tokens, four rows to a lane
  if (token >= a.t || row >= a.m) return;
  float ws[4], bias[4];
  load_channels<4>(a, row, ws, bias);
  const int s[4] = {sum[0], sum[1], sum[2], sum[3]};
  store_outputs<DT, 4>(a, token, row, a.as[token], s, ws, bias);
}

// ---- tiles --------------------------------------------------------------------------------------------------
// Four waves, each 32 WM rows of W x 32 WN tokens on 32 x 32 x 32 instructions; the block tile is twice that both ways.
// Stages of SK = 128 bytes of k go from memory straight into LDS, into a ring: whole lines (with 64 bytes the second half of a line
// was fetched again a stage later: 0.39 in place of 0.30 us per 128 bytes of a 128 x 128 tile), a row's chunks of 16 bytes at c ^ turn(r), which
// spreads the rows that a read touches together over all banks (the request applies it on the memory's side).  The next
// operands are read from LDS beside the products; behind the barrier, where nobody needs a stage any more, its slot is asked to be
// filled with the one RING stages on.
//
// The sums leave through LDS, 32 tokens of a wave at a time: a lane of the matrix instruction has four rows of W in a run of eight for
// one token, and a store wants whole lines of a token.
//
// If n is not a multiple of 128 the stage that holds the rest comes first, with its lanes past n sent out of the buffer's range
// (zeros): the main loop does not have to know about it.
//
// 8192 tokens x 11008 x 4096: 353 us, 2.1 POP/s, the rate of a large library product.  333 tokens x 4096 x 11008: 27.7 us, 1.1 POP/s: 192 tiles of
// 86 stages that take 0.26 us each, of which the products are 0.11.

__device__ __forceinline__ int turn(int r) { return (r & 7) ^ ((r >> 3) & 1); }

constexpr int SK = 128;   // bytes of k in a stage
template <int WM, int WN, int RING>
constexpr int tile_lds_bytes() { return RING * (64 * WM + 64 * WN) * SK; }

struct TilePlan {
  int tiles_m, tiles_t, splits, stages;   // stages: of all k, per split at most stages_each
  int stages_each;
  int* partial;                           // splits > 1: [split][64 WN tiles_t][64 WM tiles_m]
};

// which tile and split a block works on: the blocks of a die (consecutive numbers modulo 8) get consecutive tiles, eight token
// tiles deep, whose operands they share in the die's L2
__device__ __forceinline__ void tile_of_block(const TilePlan& p, int id, int total, int& tm, int& tt, int& split) {
  const int die = id & 7, each = total >> 3, rest = total & 7;
  int i = die * each + min(die, rest) + (id >> 3);
  const int tiles = p.tiles_m * p.tiles_t;
  split = i / tiles;
  i -= split * tiles;
  const int deep = 8, group = i / (deep * p.tiles_m);
  const int first = group * deep, here = min(deep, p.tiles_t - first);
  i -= group * deep * p.tiles_m;
  tm = i / here;
  tt = first + i % here;
}

// DT < 0: the sums of a split, into p.partial
template <int DT, int WM, int WN, int RING>
__global__ __launch_bounds__(256) void tile_kernel(LinearArgs a, TilePlan p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  typedef __attribute__((address_space(3))) char lds_char;
  typedef __attribute__((address_space(3))) i32x4 lds_i32x4;
  lds_char* lds = (lds_char*)smem;
  const uint32_t lbase = (uint32_t)(uintptr_t)lds;
  constexpr int kPartW = 64 * WM * SK, kSlot = kPartW + 64 * WN * SK, kChunks = SK / 16, kSteps = SK / 32;
  constexpr bool kWholeStage = WM * WN <= 4;
  constexpr int LW = WM * SK / 64, L = LW + WN * SK / 64, F = kWholeStage ? L : L / 2;   // requests of a stage, and how many of them go first
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wt = wave & 1, h = lane >> 5;
  int tm, tt, split;
  tile_of_block(p, blockIdx.x, gridDim.x, tm, tt, split);
  const int m0 = tm * 64 * WM, t0 = tt * 64 * WN;
  const int first = split * p.stages_each, last = min(first + p.stages_each, p.stages);
  const int nstage = last - first;

  i32x16 acc[WM][WN];
#pragma unroll
  for (int x = 0; x < WM; ++x)
#pragma unroll
    for (int y = 0; y < WN; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0;

  const int whole = a.n / SK, rest = a.n % SK;
  const int k0 = (rest ? (first == 0 ? 0 : first - 1) : first) * SK;   // of the first stage that is whole
  auto extent = [&](int rows, int64_t ld, int k) { return (int64_t)(rows - 1) * ld + a.n - k; };
  const int rows_w = min(64 * WM, a.m - m0), rows_t = min(64 * WN, a.t - t0);
  const int8_t* W0 = a.W + (int64_t)m0 * a.ldw;
  const int8_t* A0 = a.A + (int64_t)t0 * a.lda;
  i32x4 dw = buffer_at(W0 + k0, extent(rows_w, a.ldw, k0)), dt = buffer_at(A0 + k0, extent(rows_t, a.lda, k0));

  // request q of a stage: 1 KB of rows; the wave's share is every fourth
  uint32_t vo[L];
  auto row_of = [&](int q) { return (4 * (q < LW ? q : q - LW) + wave) * (64 / kChunks) + lane / kChunks; };
  auto chunk_of = [&](int q) { return (lane & (kChunks - 1)) ^ turn(row_of(q)); };
#pragma unroll
  for (int q = 0; q < L; ++q) vo[q] = (uint32_t)(row_of(q) * (int)(q < LW ? a.ldw : a.lda) + 16 * chunk_of(q));
  const uint32_t wbase = lbase + wave * 1024;
  auto place = [](int q) constexpr { return (uint32_t)(q < LW ? q * 4096 : kPartW + (q - LW) * 4096); };
  int asked = 0;   // stages asked for; those past the last one are asked of an empty buffer
  auto advance = [&](i32x4& d) {
    const uint64_t base = (((uint64_t)(uint32_t)d[1] << 32) | (uint32_t)d[0]) + SK;
    d[0] = (int)__builtin_amdgcn_readfirstlane((uint32_t)base);
    d[1] = (int)__builtin_amdgcn_readfirstlane((uint32_t)(base >> 32));
    d[2] = asked < nstage ? d[2] - SK : 0;
  };

  // prologue: all stages of the ring but the last, and the first half of that
  auto ask = [&](int q, uint32_t slot, uint32_t v) {
    if (q < LW) request_to_lds(dw, v, wbase + slot + place(q));
    else request_to_lds(dt, v, wbase + slot + place(q));
  };
  const bool rest_first = rest != 0 && first == 0;
  if (rest_first) {
    const i32x4 sw = dw, st = dt;
    dw = buffer_at(W0 + whole * SK, extent(rows_w, a.ldw, whole * SK));
    dt = buffer_at(A0 + whole * SK, extent(rows_t, a.lda, whole * SK));
#pragma unroll
    for (int q = 0; q < L; ++q) ask(q, 0, 16 * chunk_of(q) < rest ? vo[q] : 0x80000000u);
    dw = sw;
    dt = st;
    ++asked;
    if (asked >= nstage) dw[2] = dt[2] = 0;
    asm volatile("s_nop 4" : "+s"(dw), "+s"(dt));
  }
  static_for<RING - 1>([&](auto s_) {
    constexpr int s = decltype(s_)::value;
    if (s == 0 && rest_first) return;
#pragma unroll
    for (int q = 0; q < L; ++q) ask(q, s * kSlot, vo[q]);
    ++asked;
    advance(dw);
    advance(dt);
  });
#pragma unroll
  for (int q = 0; q < F; ++q) ask(q, (RING - 1) * kSlot, vo[q]);
  wait_requests<(RING - 2) * L + F>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");   // no read of LDS above the barrier

  // where a lane finds its operands inside a slot, per 32 bytes of k
  uint32_t aw[kSteps][WM], at[kSteps][WN];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
#pragma unroll
    for (int T = 0; T < WM; ++T) {
      const int row = wm * 32 * WM + 32 * T + (lane & 31);
      aw[k][T] = row * SK + ((16 * (h ^ turn(row))) ^ (32 * k));
    }
#pragma unroll
    for (int U = 0; U < WN; ++U) {
      const int row = wt * 32 * WN + 32 * U + (lane & 31);
      at[k][U] = kPartW + row * SK + ((16 * (h ^ turn(row))) ^ (32 * k));
    }
  }
  auto read_one = [&](uint32_t at_) { return *(lds_i32x4*)(lds + at_); };

  // The products of 32 bytes of k on (fw, ft) while the next operands are read from `slot` (half HALF of the stage), and P
  // requests, q0 onwards, go into slot `dst`, spread over the products.
  auto half = [&](auto half_, auto q0_, auto p_, const i32x4 (&fw)[WM], const i32x4 (&ft)[WN], i32x4 (&nw)[WM], i32x4 (&nt)[WN],
                  uint32_t slot, uint32_t dst) {
    constexpr int HALF = decltype(half_)::value, Q0 = decltype(q0_)::value, P = decltype(p_)::value;
    static_for<WM>([&](auto x_) {
      constexpr int x = decltype(x_)::value;
      nw[x] = read_one(slot + aw[HALF][x]);
      if constexpr (x < WN) nt[x] = read_one(slot + at[HALF][x]);
#pragma unroll
      for (int y = 0; y < WN; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[x], ft[y], acc[x][y], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < P; ++j)
        if (j * WM / (P ? P : 1) == x) ask(Q0 + j, dst, vo[Q0 + j]);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  using std::integral_constant;
  // every wave has read a slot and everybody's requests for the next stage have arrived
  auto meet = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wait_requests<(RING - 2) * L>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  int s = 0;
  uint32_t slot = 0;   // where stage s lies
  // (there is one stage at least: no way around the loops, on which the sums would have to be copied)
  if constexpr (kWholeStage) {
    // A half of a stage is too little here to hide the way from LDS (128 cycles of products, some 200 to the operands): the whole
    // next stage is read beside the products of one.
    struct Operands { i32x4 w[kSteps][WM], t[kSteps][WN]; } f0, f1;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
#pragma unroll
      for (int T = 0; T < WM; ++T) f0.w[k][T] = read_one(aw[k][T]);
#pragma unroll
      for (int U = 0; U < WN; ++U) f0.t[k][U] = read_one(at[k][U]);
    }
    ++asked;
    advance(dw);
    advance(dt);
    auto stage = [&](const Operands& now, Operands& then) {
      const uint32_t next = slot + kSlot == RING * kSlot ? 0 : slot + kSlot;
      meet();
      static_for<kSteps * WM>([&](auto g_) {
        constexpr int g = decltype(g_)::value, k = g / WM, x = g % WM;
        then.w[k][x] = read_one(next + aw[k][x]);
#pragma unroll
        for (int y = 0; y < WN; ++y)
          if (y * WM / WN == x) then.t[k][y] = read_one(next + at[k][y]);
#pragma unroll
        for (int y = 0; y < WN; ++y) acc[x][y] = __builtin_amdgcn_mfma_i32_32x32x32_i8(now.w[k][x], now.t[k][y], acc[x][y], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < L; ++q)
          if (q * kSteps * WM / L == g) ask(q, slot, vo[q]);
        __builtin_amdgcn_sched_barrier(0);
      });
      ++asked;
      advance(dw);
      advance(dt);
      slot = next;
    };
    while (true) {
      stage(f0, f1);
      if (++s >= nstage) break;
      stage(f1, f0);
      if (++s >= nstage) break;
    }
  } else {
    i32x4 fw[2][WM], ft[2][WN];
#pragma unroll
    for (int T = 0; T < WM; ++T) fw[0][T] = read_one(aw[0][T]);
#pragma unroll
    for (int U = 0; U < WN; ++U) ft[0][U] = read_one(at[0][U]);
    do {
      const uint32_t before = slot == 0 ? (RING - 1) * kSlot : slot - kSlot, next = slot + kSlot == RING * kSlot ? 0 : slot + kSlot;
      static_for<kSteps>([&](auto k_) {
        constexpr int k = decltype(k_)::value, now = k & 1, then = 1 - now;
        if constexpr (k == 0) {
          half(integral_constant<int, 1>{}, integral_constant<int, F>{}, integral_constant<int, L - F>{}, fw[now], ft[now], fw[then], ft[then], slot, before);
          ++asked;
          advance(dw);
          advance(dt);
        } else if constexpr (k + 1 < kSteps) {
          half(integral_constant<int, k + 1>{}, integral_constant<int, 0>{}, integral_constant<int, 0>{}, fw[now], ft[now], fw[then], ft[then], slot, slot);
        } else {
          meet();
          half(integral_constant<int, 0>{}, integral_constant<int, 0>{}, integral_constant<int, F>{}, fw[now], ft[now], fw[then], ft[then], next, slot);
        }
      });
      slot = next;
    } while (++s < nstage);
  }
  wait_requests<0>();   // nothing may land in this LDS after the workgroup has left it

  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  constexpr int kPitch = 32 * WM * 4 + 16;             // bytes of a token; the odd 16 spread the tokens over the banks
  constexpr int kLanes = 4 * WM, kTokens = 64 / kLanes;  // eight outputs a lane
  static_assert(4 * 32 * kPitch <= tile_lds_bytes<WM, WN, RING>(), "");
  lds_char* area = lds + wave * 32 * kPitch;
  const int col = 8 * (lane % kLanes), row = m0 + wm * 32 * WM + col;
  float ws[8], bias[8];
  float as[WN][32 / kTokens];
  if constexpr (DT >= 0) {
    load_channels<8>(a, row, ws, bias);
#pragma unroll
    for (int U = 0; U < WN; ++U)
#pragma unroll
      for (int i = 0; i < 32 / kTokens; ++i) as[U][i] = a.as[min(t0 + wt * 32 * WN + 32 * U + i * kTokens + lane / kLanes, a.t - 1)];
  }
#pragma unroll
  for (int U = 0; U < WN; ++U) {
#pragma unroll
    for (int T = 0; T < WM; ++T)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(lds_i32x4*)(area + (lane & 31) * kPitch + (32 * T + 8 * q + 4 * h) * 4) =
            i32x4{acc[T][U][4 * q], acc[T][U][4 * q + 1], acc[T][U][4 * q + 2], acc[T][U][4 * q + 3]};
#pragma unroll
    for (int i = 0; i < 32 / kTokens; ++i) {
      const int token = wt * 32 * WN + 32 * U + i * kTokens + lane / kLanes;
      const i32x4 lo = *(lds_i32x4*)(area + (i * kTokens + lane / kLanes) * kPitch + col * 4);
      const i32x4 hi = *(lds_i32x4*)(area + (i * kTokens + lane / kLanes) * kPitch + col * 4 + 16);
      if constexpr (DT < 0) {
        int* out = p.partial + ((int64_t)split * p.tiles_t * 64 * WN + t0 + token) * (p.tiles_m * 64 * WM) + row;
        *reinterpret_cast<i32x4*>(out) = lo;
        *reinterpret_cast<i32x4*>(out + 4) = hi;
      } else if (t0 + token < a.t && row < a.m) {
        const int v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        store_outputs<DT, 8>(a, t0 + token, row, as[U][i], v, ws, bias);
      }
    }
  }
}

// adds the splits' sums and writes the outputs: eight outputs of a token a thread, four splits on their way together
template <int DT>
__global__ __launch_bounds__(64) void split_sum_kernel(LinearArgs a, const int* __restrict__ partial, int splits, int rows, int cols) {
  const int row = (blockIdx.x * 64 + threadIdx.x) * 8, token = blockIdx.y;
  if (row >= a.m) return;
  int v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int* in = partial + (int64_t)token * cols + row;
  float ws[8], bias[8];
  load_channels<8>(a, row, ws, bias);
  for (int s = 0; s < splits; s += 4) {
    i32x4 x[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int* p = in + (int64_t)min(s + i, splits - 1) * rows * cols;
      x[i][0] = *reinterpret_cast<const i32x4*>(p);
      x[i][1] = *reinterpret_cast<const i32x4*>(p + 4);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (s + i < splits) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += x[i][e >> 2][e & 3];
      }
  }
  store_outputs<DT, 8>(a, token, row, a.as[token], v, ws, bias);
}

constexpr int kSkinnyTokens = 64;   // that skinny_kernel has columns for
struct Form {
  int tile;   // -1: few tokens
  TilePlan plan;
};
// Tiles of 64 wm rows of W x 64 wn tokens, one workgroup to a compute unit, and what they take: us from a workgroup's start to its
// end beside its stages, and us a 128-byte stage with up to 64 workgroups at work and with 256 (measured, n = 4096 and 11008; the
// products of a stage alone are 0.85, 0.21 and 0.11 us at 2.4 GHz; a full chip runs at less, and its tiles share the L2s).
struct TileShape { int wm, wn; double fixed, low, full; };
constexpr int kUnits = 256;
constexpr TileShape kTiles[] = {{4, 4, 10.0, 1.03, 1.70}, {2, 2, 5.0, 0.30, 0.55}, {1, 2, 5.0, 0.20, 0.30}};

// The tile and the number of splits of k with the least time by these numbers.  us measured for n = 4096, m = 4096 (tiles in the order
// above): 512 tokens 45, 18.4, 14.8; 1024 tokens 46, 23.0, 27.7; 4096 tokens 65, 86, 113; 333 tokens and n = 11008 98, 29.2 in two splits,
// 29.3.  Splits cost the partial sums' way through memory and a second kernel; only the smallest tile is worth them (few tokens, small m).
Form form_of(int64_t t, int64_t m, int64_t n) {
  Form f{};
  const int64_t stages = ceil_div(n, SK);
  double best = 1e300;
  for (int i = 0; i < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++i) {
    const TileShape& T = kTiles[i];
    const int64_t tm = ceil_div(m, 64 * T.wm), tt = ceil_div(t, 64 * T.wn);
    for (int64_t splits = 1; splits == 1 || (T.wm == 1 && splits <= 16 && stages / splits >= 4 && tm * tt * splits <= kUnits); ++splits) {
      const int64_t each = ceil_div(stages, splits), used = ceil_div(stages, each), blocks = tm * tt * used;
      auto round_us = [&](int64_t at_work) {
        return T.fixed + (double)each * (T.low + (T.full - T.low) * std::max(0.0, ((double)at_work - 64.0) / 192.0));
      };
      const int64_t last = blocks % kUnits;
      const double us = (double)(blocks / kUnits) * round_us(kUnits) + (last ? round_us(last) : 0.0) +
                        (used > 1 ? 6.0 + 0.0066 * (double)(blocks * T.wm * T.wn) : 0.0);
      if (us < best) {
        best = us;
        f.tile = i;
        f.plan = TilePlan{(int)tm, (int)tt, (int)used, (int)stages, (int)each, nullptr};
      }
    }
  }
  if (t <= kSkinnyTokens) {
    // The few-token kernel by what it took, in us, beside tiles (m x n: tokens, few-token kernel | tiles): 4096 x 4096: 16 5.8 | 10.1, 32 7.8 | 10.4,
    // 64 12.3 | 10.9; 11008 x 4096: 8 10.8 | 10.8, 16 12.9 | 11.0, 64 28.9 | 12.0; 4096 x 11008: 16 13.2 | 14.8, 32 19.2 | 15.2.  The
    // estimate for tiles is a sixth high where they are so few.
    const double few = 2.0 + (double)m * (double)n / 16777216.0 * (2.6 + 0.1 * (double)t + (t <= 16 ? 0.0 : t <= 32 ? 1.0 : 3.0));
    if (few < 0.85 * best) f.tile = -1;
  }
  return f;
}

template <int DT, int WM, int WN, int RING>
ptq_status tile_launch(const LinearArgs& a, const TilePlan& p, hipStream_t s) {
  constexpr int kBytes = tile_lds_bytes<WM, WN, RING>();
  const unsigned blocks = (unsigned)(p.tiles_m * p.tiles_t * p.splits);
  if (!p.partial) {
    if (!lds_opt_in<tile_kernel<DT, WM, WN, RING>>(kBytes)) return PTQ_ERR_HIP;
    tile_kernel<DT, WM, WN, RING><<<blocks, 256, kBytes, s>>>(a, p);
  } else if constexpr (WM == 1) {   // (the larger tiles are not split)
    if (!lds_opt_in<tile_kernel<-1, WM, WN, RING>>(kBytes)) return PTQ_ERR_HIP;
    tile_kernel<-1, WM, WN, RING><<<blocks, 256, kBytes, s>>>(a, p);
    split_sum_kernel<DT><<<dim3((unsigned)ceil_div(a.m, 512), (unsigned)a.t), 64, 0, s>>>(a, p.partial, p.splits, p.tiles_t * 64 * WN,
                                                                                         p.tiles_m * 64 * WM);
  }
  return PTQ_OK;
}

template <int DT>
ptq_status launch(const LinearArgs& a, void* ws, hipStream_t s) {
  Form f = form_of(a.t, a.m, a.n);
  if (f.tile < 0) {
    const dim3 grid((unsigned)ceil_div(a.m, 16));
    if (a.t <= 16) skinny_kernel<DT, 1><<<grid, kSkinnyWaves * 64, 0, s>>>(a);
    else if (a.t <= 32) skinny_kernel<DT, 2><<<grid, kSkinnyWaves * 64, 0, s>>>(a);
    else skinny_kernel<DT, 4><<<grid, kSkinnyWaves * 64, 0, s>>>(a);
    return PTQ_OK;
  }
  TilePlan& p = f.plan;
  if ((int64_t)p.tiles_m * p.tiles_t * p.splits > INT32_MAX) return PTQ_ERR_SHAPE;
  p.partial = p.splits > 1 ? static_cast<int*>(ws) : nullptr;
  switch (f.tile) {
    case 0: return tile_launch<DT, 4, 4, 2>(a, p, s);
    case 1: return tile_launch<DT, 2, 2, 4>(a, p, s);
    default: return tile_launch<DT, 1, 2, 4>(a, p, s);
  }
}

}  // namespace

int64_t int8_linear_max_columns() { return 131056; }

size_t int8_linear_workspace_bytes(int64_t m, int64_t n, int64_t t) {
  if (m <= 0 || n <= 0 || t <= 0) return 0;
  const Form f = form_of(t, m, n);
  if (f.tile < 0 || f.plan.splits <= 1) return 0;
  return (size_t)f.plan.splits * f.plan.tiles_m * f.plan.tiles_t * 64 * 64 * kTiles[f.tile].wm * kTiles[f.tile].wn * sizeof(int);
}

ptq_status int8_linear_launch(const int8_t* A, int64_t lda, const float* a_scales, int64_t t, const int8_t* W, int64_t ldw,
                              const float* w_scales, int64_t m, int64_t n, const float* bias, void* O, ptq_dtype odt,
                              int64_t ldo, void* ws, hipStream_t s) {
  const LinearArgs a{A, a_scales, W, w_scales, bias, O, lda, ldw, ldo, (int)t, (int)m, (int)n};
  const ptq_status rc = odt == PTQ_BF16 ? launch<PTQ_BF16>(a, ws, s) : launch<PTQ_F32>(a, ws, s);
  if (rc != PTQ_OK) return rc;
  PTQ_HIP_CHECK_LAUNCH();
  return PTQ_OK;
}

}  // namespace ptq
