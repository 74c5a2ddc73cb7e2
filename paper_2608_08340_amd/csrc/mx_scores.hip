// Inner products of rows in the microscaled format (oprag_mx_scores).
#include <algorithm>

#include "mx.h"

namespace oprag {
namespace {

using namespace dev;

template <int BITS>
__device__ __forceinline__ unsigned code_at(const unsigned char* block, int i) {
  const int bit = i * BITS;
  unsigned v = block[bit / 8] >> (bit % 8);
  if (bit % 8 + BITS > 8) v |= (unsigned)block[bit / 8 + 1] << (8 - bit % 8);
  return v & ((1u << BITS) - 1);
}

// One thread per score.
template <int DT, int QBITS, int RBITS>
__global__ __launch_bounds__(256) void scores_kernel(MxRows q, MxRows r, void* __restrict__ out, long long ld) {
  const long long total = q.rows * r.rows, stride = (long long)gridDim.x * 256;
  for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < total; t += stride) {
    const long long iq = t / r.rows, ir = t - iq * r.rows;
    float sum = 0.f;
    for (int b = 0; b < q.nb; ++b) {
      const unsigned char* cq = q.codes + (iq * q.nb + b) * (4 * QBITS);
      const unsigned char* cr = r.codes + (ir * r.nb + b) * (4 * RBITS);
      float s = 0.f;
      for (int i = 0; i < 32; ++i) s = fmaf(mx_decode<QBITS>(code_at<QBITS>(cq, i)), mx_decode<RBITS>(code_at<RBITS>(cr, i)), s);
      sum += s * mx_scale(q.scales[iq * q.nb + b]) * mx_scale(r.scales[ir * r.nb + b]);
    }
    store_from_f32<DT>(out, iq * ld + ir, sum);
  }
}

}  // namespace

hipError_t launch_mx_scores(const MxRows& q, const MxRows& rows, void* out, int dtype, long long ld, hipStream_t s) {
  const unsigned grid = (unsigned)std::min<long long>((q.rows * rows.rows + 255) / 256, 1 << 16);
  return with_dtype(dtype, [&](auto dt) {
    return with_bits(q.bits, [&](auto qb) {
      return with_bits(rows.bits, [&](auto rb) {
        scores_kernel<dt(), qb(), rb()><<<grid, 256, 0, s>>>(q, rows, out, ld);
        return hipGetLastError();
      });
    });
  });
}

}  // namespace oprag
