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

// Rows of one head, keys (0) or values (1): place `offset` of a page is row first + page * per_page + offset, an index into scales and
// zeros, times row_bytes into codes.
struct KvRows {
  int64_t first;
  uint32_t per_page;
};
__device__ __forceinline__ KvRows kv_rows(const KvCache& c, int which, int head) {
  return KvRows{((int64_t)which * c.pages * c.heads + head) << c.page_shift, (uint32_t)c.heads << c.page_shift};
}
__device__ __forceinline__ int64_t kv_row(const KvRows& r, uint32_t page, uint32_t offset) {
  return r.first + (int64_t)((uint64_t)page * r.per_page + offset);
}

}  // namespace ptq
