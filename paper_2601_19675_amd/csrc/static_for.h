// A loop whose index is a compile-time constant.  Not part of the C ABI.
#pragma once
#include <type_traits>
#include <utility>

namespace ptq {

// f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>)
template <class F, int... Is>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, Is...>) {
  (f(std::integral_constant<int, Is>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for_impl(f, std::make_integer_sequence<int, N>{});
}

}  // namespace ptq
