// The gradient of the products of quantised rows (oprag_mx_scores_grad): G X or G^T X.
#include <algorithm>

#include "mx.h"

namespace oprag {
namespace {

using namespace dev;

// One thread per output element.
template <int DT, int BITS>
__global__ __launch_bounds__(256) void grad_kernel(const void* __restrict__ g, long long row_step, long long col_step,
                                                   long long m, MxRows x, float* __restrict__ out, long long out_ld) {
  const long long total = m * x.dim, stride = (long long)gridDim.x * 256;
  for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < total; t += stride) {
    const long long row = t / x.dim;
    const int d = (int)(t - row * x.dim), bit = (d % 32) * BITS;
    double sum = 0.0;  // a long index has more terms than fp32 adds exactly enough in a row
    for (long long k = 0; k < x.rows; ++k) {
      const long long b = k * x.nb + d / 32;
      const unsigned char* p = x.codes + b * (4 * BITS) + bit / 8;
      unsigned v = p[0] >> (bit % 8);
      if (bit % 8 + BITS > 8) v |= (unsigned)p[1] << (8 - bit % 8);
      sum += (double)load_as_f32<DT>(g, row * row_step + k * col_step) * (mx_decode<BITS>(v & ((1u << BITS) - 1)) * mx_scale(x.scales[b]));
    }
    out[row * out_ld + d] = (float)sum;
  }
}

}  // namespace

size_t mx_grad_workspace_bytes(long long, const MxRows&) { return 0; }

hipError_t launch_mx_grad(const void* grad, int dtype, long long ld, bool transposed, long long m, const MxRows& x,
                          float* out, long long out_ld, void*, hipStream_t s) {
  const unsigned grid = (unsigned)std::min<long long>((m * x.dim + 255) / 256, 1 << 16);
  return with_dtype(dtype, [&](auto dt) {
    return with_bits(x.bits, [&](auto bits) {
      grad_kernel<dt(), bits()><<<grid, 256, 0, s>>>(grad, transposed ? 1 : ld, transposed ? ld : 1, m, x, out, out_ld);
      return hipGetLastError();
    });
  });
}

}  // namespace oprag
