// Rows to the microscaled format and back (oprag_mx_quantize, oprag_mx_values).
#include <algorithm>

#include "mx.h"

namespace oprag {
namespace {

using namespace dev;

// One thread per block of 32 elements.
template <int DT, int BITS>
__global__ __launch_bounds__(256) void quantize_kernel(const void* __restrict__ x, long long ld, MxRows out) {
  const long long total = out.rows * out.nb, stride = (long long)gridDim.x * 256;
  for (long long b = (long long)blockIdx.x * 256 + threadIdx.x; b < total; b += stride) {
    const long long row = b / out.nb;
    const int d0 = (int)(b - row * out.nb) * 32, w = min(32, out.dim - d0);
    const long long at = row * ld + d0;
    unsigned top = 0;
    for (int i = 0; i < w; ++i) top = max(top, __float_as_uint(load_as_f32<DT>(x, at + i)) & 0x7fffffffu);
    const bool bad = top >= 0x7f800000u;
    const int c = max((int)(top >> 23) - 2, 0);
    const float inv = __uint_as_float((unsigned)(254 - c) << 23);  // 2^(127 - c), c <= 252
    unsigned char* dst = out.codes + b * (4 * BITS);
    unsigned long long word = 0;
    int have = 0;
    for (int i = 0; i < 32; ++i) {
      const unsigned code = i < w && !bad ? mx_encode<BITS>(load_as_f32<DT>(x, at + i) * inv) : 0u;
      word |= (unsigned long long)code << have;
      have += BITS;
      for (; have >= 8; have -= 8, word >>= 8) *dst++ = (unsigned char)word;
    }
    out.scales[b] = (unsigned char)(bad ? 255 : c);
  }
}

// One thread per element.
template <int DT, int BITS>
__global__ __launch_bounds__(256) void values_kernel(MxRows r, void* __restrict__ out, long long ld) {
  const long long total = r.rows * r.dim, stride = (long long)gridDim.x * 256;
  for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < total; t += stride) {
    const long long row = t / r.dim;
    const int d = (int)(t - row * r.dim);
    const long long b = row * r.nb + d / 32;
    const int bit = (d % 32) * BITS;
    const unsigned char* p = r.codes + b * (4 * BITS) + bit / 8;
    unsigned v = p[0] >> (bit % 8);
    if (bit % 8 + BITS > 8) v |= (unsigned)p[1] << (8 - bit % 8);
    store_from_f32<DT>(out, row * ld + d, mx_decode<BITS>(v & ((1u << BITS) - 1)) * mx_scale(r.scales[b]));
  }
}

unsigned grid_for(long long threads) { return (unsigned)std::min<long long>((threads + 255) / 256, 1 << 16); }

}  // namespace

hipError_t launch_mx_quantize(const void* x, int dtype, long long ld, const MxRows& out, hipStream_t s) {
  return with_dtype(dtype, [&](auto dt) {
    return with_bits(out.bits, [&](auto bits) {
      quantize_kernel<dt(), bits()><<<grid_for(out.rows * out.nb), 256, 0, s>>>(x, ld, out);
      return hipGetLastError();
    });
  });
}

hipError_t launch_mx_values(const MxRows& rows, void* out, int dtype, long long ld, hipStream_t s) {
  return with_dtype(dtype, [&](auto dt) {
    return with_bits(rows.bits, [&](auto bits) {
      values_kernel<dt(), bits()><<<grid_for(rows.rows * rows.dim), 256, 0, s>>>(rows, out, ld);
      return hipGetLastError();
    });
  });
}

}  // namespace oprag
