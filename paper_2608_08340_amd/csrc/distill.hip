// Distillation of scores towards ranked lists (oprag_distill_loss, _grad, _step).
//
// With z = s / tau over the n rows of a query and p the softmax of the list's scores over t_tau:
//   lse = max + log sum exp(z - max),   loss = sum_e p_e (log p_e - z_id(e)) + lse,
//   grad_i = w / tau (exp(z_i - lse) - sum of p_e with id(e) = i).
#include <algorithm>

#include "mx.h"

namespace oprag {
namespace {

using namespace dev;

constexpr int kThreads = 256;
constexpr float kNegInfF = -__builtin_inff();

// s / tau rounded as a division is (r = 1 / tau): the remainder of the first guess corrects it.
// Infinite and NaN values pass through.
__device__ __forceinline__ float div_tau(float s, float tau, float r) {
  const float q = s * r, e = fmaf(-q, tau, s);
  return fabsf(q) < 0x1p120f ? fmaf(e, r, q) : q;
}

template <typename T>
__device__ __forceinline__ T block_sum(T v, T* part) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  T s = 0;
  for (int i = 0; i < kThreads / 64; ++i) s += part[i];
  return s;
}
// The larger, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) { return a != a ? a : b != b ? b : fmaxf(a, b); }
__device__ __forceinline__ float block_max(float v, float* part) {
  for (int o = 32; o > 0; o >>= 1) v = max_nan(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = part[0];
  for (int i = 1; i < kThreads / 64; ++i) m = max_nan(m, part[i]);
  return m;
}

// One workgroup per query.
template <int DT>
__global__ __launch_bounds__(kThreads) void distill_kernel(DistillArgs a) {
  __shared__ float pf[kThreads / 64];
  __shared__ double pd[kThreads / 64];
  __shared__ float sp[kMaxK];
  __shared__ long long sid[kMaxK];
  const float r = 1.f / a.tau;
  for (long long q = blockIdx.x; q < a.nq; q += gridDim.x) {
    const int tid = threadIdx.x;
    // The teacher: thread e holds entry e.
    const long long id = tid < a.k ? a.ids[q * a.k + tid] : -1;
    const float t = tid < a.k ? a.t[q * a.k + tid] : kNegInfF;
    const bool entry = id >= 0 && id < a.n && t > kNegInfF;
    const float u = entry ? t / a.t_tau : kNegInfF;
    const float umax = block_max(u, pf);
    const float eu = entry ? expf(u - umax) : 0.f;
    const float mass = block_sum(eu, pf);
    const bool some = umax != kNegInfF;
    const float p = some ? eu / mass : 0.f;
    const float z_id = entry ? div_tau(load_as_f32<DT>(a.logits, q * a.ld + id), a.tau, r) : 0.f;
    float zmax, total;
    if (a.lse_in) {
      zmax = a.lse_in[q];
      total = 1.f;
    } else {
      float m = kNegInfF;
      for (long long i = tid; i < a.n; i += kThreads) m = max_nan(m, div_tau(load_as_f32<DT>(a.logits, q * a.ld + i), a.tau, r));
      zmax = block_max(m, pf);
      float s = 0.f;
      for (long long i = tid; i < a.n; i += kThreads) {
        const float z = div_tau(load_as_f32<DT>(a.logits, q * a.ld + i), a.tau, r);
        s += z == kNegInfF ? 0.f : expf(z - zmax);
      }
      total = block_sum(s, pf);
    }
    if (a.loss) {
      const double lse = (double)zmax + log((double)total);
      double term = 0.0;
      if (p > 0.f && z_id == kNegInfF)
        term = __builtin_inf();  // a row that the student rules out
      else if (p > 0.f || p != p)
        term = (double)p * ((double)(u - umax) - log((double)mass) - (double)z_id + lse);
      const double loss = block_sum(term, pd);
      if (tid == 0) {
        a.loss[q] = some ? (float)loss : 0.f;
        if (a.lse) a.lse[q] = (float)lse;
      }
    }
    if (a.grad) {
      const float w = mass == mass ? a.weight[q] / a.tau : mass;  // a NaN teacher: a NaN gradient
      if (tid < a.k) {
        sp[tid] = p;
        sid[tid] = entry ? id : -1;
      }
      __syncthreads();
      for (long long i = tid; i < a.n; i += kThreads) {
        const float z = div_tau(load_as_f32<DT>(a.logits, q * a.ld + i), a.tau, r);
        const float e = z == kNegInfF ? 0.f : expf(z - zmax) / total;
        store_from_f32<DT>(a.grad, q * a.grad_ld + i, some ? w * e : 0.f);
      }
      __syncthreads();
      if (entry) {
        float mine = 0.f;
        bool first = true;
        for (int e = 0; e < a.k; ++e)
          if (sid[e] == id) {
            if (e < tid) first = false;
            mine += sp[e];
          }
        const float e = z_id == kNegInfF ? 0.f : expf(z_id - zmax) / total;
        if (first) store_from_f32<DT>(a.grad, q * a.grad_ld + id, w * (e - mine));
      }
      __syncthreads();
    }
  }
}

}  // namespace

size_t distill_workspace_bytes(long long, long long) { return 0; }

hipError_t launch_distill(const DistillArgs& a, void*, hipStream_t s) {
  return with_dtype(a.dtype, [&](auto dt) {
    distill_kernel<dt()><<<(unsigned)std::min<long long>(a.nq, 1 << 16), kThreads, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace oprag
