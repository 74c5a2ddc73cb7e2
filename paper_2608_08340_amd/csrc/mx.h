// Element types of the microscaled format (oprag.h): codes, scales and the values they stand for.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "oprag_internal.h"

namespace oprag {
namespace dev {

// 2^(c - 127) as fp32 (c = 0: the subnormal 2^-127; c = 255: NaN).
__device__ __forceinline__ float mx_scale(unsigned c) {
  return __uint_as_float(c == 255u ? 0x7fc00000u : c == 0u ? 0x00400000u : c << 23);
}

// Magnitude of code bits below the sign: with F fraction bits a code is a float of bias 1, whose
// subnormals and normals an exact product with 2^126 moves to their values.
template <int BITS>
__device__ __forceinline__ float mx_decode(unsigned code) {
  constexpr unsigned kSign = 1u << (BITS - 1);
  constexpr int kFrac = BITS - 3;  // two exponent bits
  const float mag = __uint_as_float((code & (kSign - 1)) << (23 - kFrac)) * 0x1p126f;
  return (code & kSign) ? -mag : mag;
}

template <int DT>
__device__ __forceinline__ float load_as_f32(const void* p, long long i) {
  if constexpr (DT == kDtypeF32) {
    return static_cast<const float*>(p)[i];
  } else if constexpr (DT == kDtypeBF16) {
    return __uint_as_float((unsigned)static_cast<const unsigned short*>(p)[i] << 16);
  } else {
    return (float)static_cast<const _Float16*>(p)[i];
  }
}

// Rounds to nearest even.
template <int DT>
__device__ __forceinline__ void store_from_f32(void* p, long long i, float v) {
  if constexpr (DT == kDtypeF32) {
    static_cast<float*>(p)[i] = v;
  } else if constexpr (DT == kDtypeBF16) {
    static_cast<__bf16*>(p)[i] = (__bf16)v;
  } else {
    asm("" : "+v"(v));  // a product fused with its conversion (fma_mix, + 0) would turn -0 into 0
    static_cast<_Float16*>(p)[i] = (_Float16)v;
  }
}

// `keep`, and in the lanes whose group of four within sixteen MASK names `take` of the lane eight away.
template <int MASK>
__device__ __forceinline__ unsigned swap_eight(unsigned keep, unsigned take) {
  return (unsigned)__builtin_amdgcn_update_dpp((int)keep, (int)take, 0x128, 0xf, MASK, false);
}

}  // namespace dev

// Calls f(std::integral_constant<int, dtype>) for a run-time dtype.
template <typename F>
hipError_t with_dtype(int dtype, F&& f) {
  switch (dtype) {
    case kDtypeF32: return f(std::integral_constant<int, kDtypeF32>{});
    case kDtypeBF16: return f(std::integral_constant<int, kDtypeBF16>{});
    case kDtypeF16: return f(std::integral_constant<int, kDtypeF16>{});
    default: return hipErrorInvalidValue;
  }
}
template <typename F>
hipError_t with_bits(int bits, F&& f) {
  switch (bits) {
    case 4: return f(std::integral_constant<int, 4>{});
    case 6: return f(std::integral_constant<int, 6>{});
    default: return hipErrorInvalidValue;
  }
}

}  // namespace oprag
