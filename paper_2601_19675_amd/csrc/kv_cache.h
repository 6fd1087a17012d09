// The paged 8- or 4-bit cache of keys and values as its kernels address it.  Not part of the C ABI.
//
//   codes   [2][pages][heads][page][d bits / 8] bytes     scales  [2][pages][heads][page] float32
//   zeros   [2][pages][heads][page] bytes                  keys first, then values
#pragma once
#include "common.h"

namespace ptq {

struct KvCache {
  uint8_t* codes;
  float* scales;
  uint8_t* zeros;
  int64_t pages;
  int heads, page_shift, row_bytes;
};

// row of (keys 0 or values 1, page, head, place in the page): an index into scales and zeros, times row_bytes into codes
__device__ __forceinline__ int64_t kv_row(const KvCache& c, int which, int64_t page, int head, int offset) {
  return ((((int64_t)which * c.pages + page) * c.heads + head) << c.page_shift) + offset;
}

// one operand of a lane exchange inside 16 lanes (see dpp_move)
template <int CTRL>
__device__ __forceinline__ float dpp_move_f32(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

}  // namespace ptq
