// Rows of bf16 or float32 values four at a time, sums over the lanes of a head and the rotation of eight
// values by four angles: what the kernels that norm, rotate and store rows share.
#pragma once

#include <type_traits>

#include "common.h"

namespace omnitide {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

// Four values of a row in storage: float32 as they are, bf16 in words 0 and 1.
template <bool F32>
__device__ inline u32x4 load_quad(const uint8_t* row, int dim) {
  if constexpr (F32) return *reinterpret_cast<const u32x4*>(row + 4 * dim);
  const u32x2 t = *reinterpret_cast<const u32x2*>(row + 2 * dim);
  return u32x4{t[0], t[1], 0, 0};
}

template <bool F32>
__device__ inline floatx4 unpack_quad(u32x4 w) {
  if constexpr (F32) return __builtin_bit_cast(floatx4, w);
  return floatx4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u),
                 __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
}

__device__ inline uint32_t pack_bf16(float lo, float hi) {
  const __bf16 a = static_cast<__bf16>(lo), b = static_cast<__bf16>(hi);
  return static_cast<uint32_t>(__builtin_bit_cast(uint16_t, a)) |
         (static_cast<uint32_t>(__builtin_bit_cast(uint16_t, b)) << 16);
}

template <bool F32>
__device__ inline void store_quad(uint8_t* row, int dim, floatx4 v) {
  if constexpr (F32)
    __builtin_nontemporal_store(v, reinterpret_cast<floatx4*>(row + 4 * dim));
  else
    __builtin_nontemporal_store(u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])},
                                reinterpret_cast<u32x2*>(row + 2 * dim));
}

// Sum over the 8 or 16 lanes of a head, the same in each of them.
template <int LPH>
__device__ inline float head_sum(float v) {
  auto move = [](float x, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value,
                                                      0xf, 0xf, false));
  };
  v += move(v, std::integral_constant<int, 0xb1>{});    // lane ^ 1
  v += move(v, std::integral_constant<int, 0x4e>{});    // lane ^ 2
  v += move(v, std::integral_constant<int, 0x141>{});   // mirrored in 8 lanes: the other quad
  if constexpr (LPH == 16) v += move(v, std::integral_constant<int, 0x140>{});  // in 16 lanes
  return v;
}

// Turns the eight values of a lane, four pairs, by (c, s): HALF pairs x with y, the other style neighbours.
template <bool HALF>
__device__ inline void turn_quads(floatx4& x, floatx4& y, floatx4 c, floatx4 s) {
  if constexpr (HALF) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float u = x[e], v = y[e];
      x[e] = fmaf(u, c[e], -v * s[e]);
      y[e] = fmaf(u, s[e], v * c[e]);
    }
  } else {
    float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float u = f[2 * e], v = f[2 * e + 1];
      f[2 * e] = fmaf(u, c[e], -v * s[e]);
      f[2 * e + 1] = fmaf(u, s[e], v * c[e]);
    }
    x = floatx4{f[0], f[1], f[2], f[3]};
    y = floatx4{f[4], f[5], f[6], f[7]};
  }
}

}  // namespace
}  // namespace omnitide
