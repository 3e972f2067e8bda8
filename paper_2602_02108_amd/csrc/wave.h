// What kernels do across the lanes of a wave.
#pragma once
#include <type_traits>

#include "common.h"

namespace oomb {

// Sums, maxima and running sums over the lanes of a wave: six steps between registers (lanes 1, 2, 4, 8 to the left inside rows of 16, then row by row).
template <typename V, typename F> __device__ __forceinline__ V wave_upto(V x, V none, F f) {
  auto moved = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false));
  };
  using std::integral_constant;
  x = f(x, moved(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{}));   // row_shr:1
  x = f(x, moved(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{}));
  x = f(x, moved(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{}));
  x = f(x, moved(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{}));
  x = f(x, moved(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{}));   // row_bcast:15 into rows 1 and 3
  x = f(x, moved(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{}));   // row_bcast:31 into rows 2 and 3
  return x;
}
template <typename V> __device__ __forceinline__ V last_lane(V x) { return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63)); }

}  // namespace oomb
