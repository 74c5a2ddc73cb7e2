// Distillation of scores towards ranked lists (oprag_distill_loss, _grad, _step).
//
// With z = s / tau over the n rows of a query and p the softmax of the list's scores over t_tau:
//   lse = z_max + log S,  S = sum exp(z - z_max),   loss = sum_e p_e (log p_e - z_id(e)) + lse,
//   grad_i = w / tau (exp(z_i - lse) - sum of p_e with id(e) = i).
// exp(z_i - z_max) is 2^((s_i - s_max) c) with c = log2(e) / tau as two floats: the difference comes first, so
// the error is small against the exponent, not against z.  The few numbers per query (lse, the loss) are
// made in fp64.
//
// The logits are read once where they fit the registers of a workgroup (rows of up to 32,768: loss, or
// loss and gradient, in one launch, bound by the bytes read and written).  Longer rows go in
// pieces of 8,192 over workgroups, each held in registers alike: one launch leaves every piece's
// maximum, sum and share of sum p z in the workspace, a second joins them and, for the gradient,
// reads the piece again.  A piece's gradient is stored densely; the list's entries on it are then
// stored again by the threads that hold them, with their p taken off.
#include <algorithm>
#include <cmath>

#include "mx.h"

namespace oprag {
namespace {

using namespace dev;

constexpr float kMinusInf = -__builtin_inff();
constexpr int kPiece = 8192;      // rows of a piece
constexpr int kJoinHere = 256;    // pieces of a query that every workgroup of the gradient joins by itself

struct Piece {      // what the first launch leaves of a piece
  float max, sum;   // s_max and sum 2^((s - s_max) c) of the piece
  double pz;        // sum of p z over the entries on it
};

struct Args {
  DistillArgs a;
  float c_hi, c_lo;   // log2(e) / tau, rounded towards zero, and the rest
  Piece* pieces;      // [nq x n_pieces]
  Piece* joined;      // [nq]: of whole queries, or null
  int n_pieces;
  long long q0;       // the launch's first query: a workgroup per query (and piece), 2^15 queries a launch (a loop over
                      // queries in the kernel keeps the constants of the fp64 logarithms in registers, and spills)
};

// Maxima leave NaN out; the sums that follow do not, and all that is made of a sum is NaN then.

// 2^(d c) for d <= 0 (both parts of c are >= 0, so d = -inf gives 0).
__device__ __forceinline__ float exp_diff(float d, const Args& p) {
  return __builtin_amdgcn_exp2f(fmaf(d, p.c_hi, d * p.c_lo));
}

// v becomes 2^((v - s_max) c); returns the sum.
template <int N>
__device__ __forceinline__ float exp_all(float (&v)[N], float s_max, const Args& p) {
  float s = 0.f;
  if (s_max == kMinusInf) {  // nothing but -inf and NaN
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = v[i] != v[i] ? v[i] : 0.f;
      s += v[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = exp_diff(v[i] - s_max, p);
      s += v[i];
    }
  }
  return s;
}
__device__ __forceinline__ float inverse(float s_max, float sum) { return s_max == kMinusInf && sum == sum ? 0.f : 1.f / sum; }

// Reductions over a workgroup of T threads.  The caller leaves a barrier between two uses of `part`.
template <int T>
__device__ __forceinline__ float group_max(float v, float* part) {
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < T / 64; ++i) v = fmaxf(v, part[i]);
  return v;
}
template <int T>
__device__ __forceinline__ float group_sum(float v, float* part) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
#pragma unroll
  for (int i = 1; i < T / 64; ++i) v += part[i];
  return v;
}
template <typename X>
__device__ __forceinline__ X wave_sum(X v) {
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// A query's teacher, in LDS.
struct Teacher {
  double plogp;             // sum of p log p
  double pz;                // sum of p z over the entries on the rows at hand (-inf: one of them is masked)
  float weight;             // weight / tau (NaN: the scores are not numbers)
  int some;                 // there are entries
  long long id[kMaxK];      // -1: no entry, or not on the rows at hand
  float p[kMaxK], s[kMaxK]; // probability and logit of such an entry
};

// Made by one wave, for rows [i0, i1): lane l has entries l and l + 64.
template <int DT>
__device__ __forceinline__ void make_teacher(const DistillArgs& a, long long q, long long i0, long long i1, Teacher& w) {
  const int lane = threadIdx.x & 63;
  long long id[2];
  float u[2], top = kMinusInf;
  int some = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int e = lane + 64 * j;
    id[j] = -1;
    u[j] = kMinusInf;
    if (e < a.k) {
      const long long at = a.ids[q * a.k + e];
      const float t = a.t[q * a.k + e];
      if (at >= 0 && at < a.n && t > kMinusInf) {
        id[j] = at;
        u[j] = t / a.t_tau;
        some = 1;  // (one whose quotient is -inf has p = 0, but is an entry)
      }
    }
    top = fmaxf(top, u[j]);
  }
  for (int o = 32; o > 0; o >>= 1) {
    top = fmaxf(top, __shfl_xor(top, o));
    some |= __shfl_xor(some, o);
  }
  float x[2];
#pragma unroll
  for (int j = 0; j < 2; ++j)  // (all quotients -inf: the entries are equal; an infinite one: NaN)
    x[j] = id[j] < 0 ? 0.f : u[j] == top ? (top == kMinusInf ? 1.f : top - top + 1.f) : expf(u[j] - top);
  const float mass = wave_sum(x[0] + x[1]);
  double plogp = 0.0, pz = 0.0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float p = id[j] < 0 ? 0.f : x[j] / mass;
    if (p > 0.f) plogp += (double)p * ((u[j] == top ? 0.0 : (double)(u[j] - top)) - log((double)mass));
    if (lane + 64 * j < a.k) {
      const bool here = id[j] >= i0 && id[j] < i1;
      const float s = here ? load_as_f32<DT>(a.logits, q * a.ld + id[j]) : 0.f;
      if (here && p > 0.f) pz += (double)p * ((double)s / (double)a.tau);
      w.id[lane + 64 * j] = here ? id[j] : -1;
      w.p[lane + 64 * j] = p;
      w.s[lane + 64 * j] = s;
    }
  }
  plogp = wave_sum(plogp);
  pz = wave_sum(pz);
  if (lane == 0) {
    w.plogp = plogp;
    w.pz = pz;
    w.some = some;
    w.weight = mass != mass ? mass : a.weight ? a.weight[q] / a.tau : 0.f;
  }
}

__device__ __forceinline__ double lse_of(float s_max, float sum, const DistillArgs& a) {
  return s_max == kMinusInf && sum == sum ? -__builtin_inf() : (double)s_max / (double)a.tau + log((double)sum);
}
__device__ __forceinline__ float loss_of(const Teacher& w, double pz, double lse) {
  if (!w.some) return 0.f;
  if (w.weight != w.weight || lse != lse || pz != pz) return __builtin_nanf("");
  if (pz == -__builtin_inf()) return __builtin_inff();
  return (float)(w.plogp - pz + lse);
}

// The elements of a piece that thread t of T holds: V in 16-byte vectors, vector i at (i T + t) EV, and of what is left
// after the last whole vector one, for t < EV.  Where there is none: -inf.
template <int DT>
constexpr int vec_of() {
  return DT == kDtypeF32 ? 4 : 8;
}
template <int DT>
struct Raw;
template <>
struct Raw<kDtypeF32> { typedef float T; };
template <>
struct Raw<kDtypeBF16> { typedef unsigned short T; };
template <>
struct Raw<kDtypeF16> { typedef _Float16 T; };
template <int DT>
constexpr long long size_of() {
  return DT == kDtypeF32 ? 4 : 2;
}

// The thread's index, not known to be the same as before: offsets made of it are made where they are used
// instead of being kept, and spilled, for a whole loop.
__device__ __forceinline__ int fresh_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

template <int DT, int T, int V>
__device__ __forceinline__ void load_piece(const void* row, int n, float (&v)[V + 1]) {
  constexpr int EV = vec_of<DT>(), NV = V / EV;
  typedef typename Raw<DT>::T E;
  typedef E Vec __attribute__((ext_vector_type(EV), aligned(sizeof(E))));
  const E* p = static_cast<const E*>(row);
  const int whole = n / EV, t = fresh_thread();
  v[V] = whole * EV + t < n && t < EV ? load_as_f32<DT>(p, whole * EV + t) : kMinusInf;
  if (whole == 0) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = kMinusInf;
    return;
  }
  Vec x[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i)  // past the end: the last vector, not used
    x[i] = *reinterpret_cast<const Vec*>(p + (unsigned)min(i * T + t, whole - 1) * EV);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < EV; ++e) {
      const E one = x[i][e];
      v[i * EV + e] = i * T + t < whole ? load_as_f32<DT>(&one, 0) : kMinusInf;
    }
}

// out[..] = scale v, or zeros, whatever v is
template <int DT, int T, int V>
__device__ __forceinline__ void store_piece(void* row, int n, const float (&v)[V + 1], bool some, float scale) {
  constexpr int EV = vec_of<DT>(), NV = V / EV;
  typedef typename std::conditional<DT == kDtypeBF16, __bf16, typename Raw<DT>::T>::type E;
  typedef E Vec __attribute__((ext_vector_type(EV), aligned(sizeof(E))));
  E* p = static_cast<E*>(row);
  const int whole = n / EV, t = fresh_thread();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    Vec x;
#pragma unroll
    for (int e = 0; e < EV; ++e) x[e] = (E)(some ? v[i * EV + e] * scale : 0.f);
    if (i * T + t < whole) *reinterpret_cast<Vec*>(p + (unsigned)(i * T + t) * EV) = x;
    __builtin_amdgcn_sched_barrier(0);  // one vector after the other: all products at once would not fit
  }
  if (whole * EV + t < n && t < EV) p[whole * EV + t] = (E)(some ? v[V] * scale : 0.f);
}

// The entries, once the piece's own stores have arrived: the probability there, less all p of its row (a row that is
// listed twice is stored once).
template <int DT, typename F>
__device__ __forceinline__ void store_entries(const DistillArgs& a, long long q, const Teacher& w, F&& prob) {
  for (int e = threadIdx.x; e < a.k; e += 64) {
    const long long id = w.id[e];
    float all = 0.f;
    bool first = id >= 0;
    for (int f = 0; f < a.k; ++f)
      if (w.id[f] == id) {
        all += w.p[f];
        first = first && f >= e;
      }
    if (first) store_from_f32<DT>(a.grad, q * a.grad_ld + id, w.weight * (prob(w.s[e]) - all));
  }
}

// Whole rows of up to T V elements, one workgroup each: the loss, and with GRAD the gradient.
template <int DT, int T, int V, bool GRAD>
__global__ __launch_bounds__(T, 4) void row_kernel(Args p) {
  const DistillArgs& a = p.a;
  __shared__ float part[2][T / 64];
  __shared__ Teacher w;
  const int wave = threadIdx.x >> 6;
  const long long q = p.q0 + blockIdx.x;
  if (wave == 0) make_teacher<DT>(a, q, 0, a.n, w);  // (fp64: before and after the row takes the registers)
  float v[V + 1];
  load_piece<DT, T, V>(static_cast<const char*>(a.logits) + q * a.ld * size_of<DT>(), (int)a.n, v);
  float m = v[0];
#pragma unroll
  for (int i = 1; i <= V; ++i) m = fmaxf(m, v[i]);
  const float s_max = group_max<T>(m, part[0]);
  const float sum = group_sum<T>(exp_all<V + 1>(v, s_max, p), part[1]);
  const float unit = inverse(s_max, sum);
  if constexpr (GRAD) {
    store_piece<DT, T, V>(static_cast<char*>(a.grad) + q * a.grad_ld * size_of<DT>(), (int)a.n, v, w.some, w.weight * unit);
    // Every store of the row has arrived before the entries on it are stored again.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (wave == 0 && w.some)
      store_entries<DT>(a, q, w, [&](float s1) { return s_max == kMinusInf ? 0.f : exp_diff(s1 - s_max, p) * unit; });
  }
  if (threadIdx.x == 0) {
    const double lse = lse_of(s_max, sum, a);
    a.loss[q] = loss_of(w, w.pz, lse);
    if (a.lse) a.lse[q] = (float)lse;
  }
}

// A piece's maximum, sum and sum of p z.
template <int DT>
__global__ __launch_bounds__(256, 4) void piece_kernel(Args p) {
  const DistillArgs& a = p.a;
  __shared__ float part[2][4];
  __shared__ Teacher w;
  const long long q = p.q0 + blockIdx.y, i0 = (long long)blockIdx.x * kPiece, i1 = min(i0 + kPiece, a.n);
  float v[33];
  load_piece<DT, 256, 32>(static_cast<const char*>(a.logits) + (q * a.ld + i0) * size_of<DT>(), (int)(i1 - i0), v);
  if (threadIdx.x < 64) make_teacher<DT>(a, q, i0, i1, w);
  float m = v[0];
#pragma unroll
  for (int i = 1; i <= 32; ++i) m = fmaxf(m, v[i]);
  const float s_max = group_max<256>(m, part[0]);
  const float sum = group_sum<256>(exp_all<33>(v, s_max, p), part[1]);
  if (threadIdx.x == 0) p.pieces[q * p.n_pieces + blockIdx.x] = Piece{s_max, sum, w.pz};
}

// A query's pieces as one, in every thread of a workgroup of 256.
__device__ __forceinline__ Piece join(const Args& p, long long q, float* part, double* part64) {
  const Piece* from = p.pieces + q * p.n_pieces;
  float m = kMinusInf;
  for (int i = threadIdx.x; i < p.n_pieces; i += 256) m = fmaxf(m, from[i].max);
  m = group_max<256>(m, part);
  double sum = 0.0, pz = 0.0;
  for (int i = threadIdx.x; i < p.n_pieces; i += 256) {
    const Piece x = from[i];
    sum += (double)x.sum * (m == kMinusInf ? 1.0 : (double)exp_diff(x.max - m, p));
    pz += x.pz;
  }
  sum = wave_sum(sum);
  pz = wave_sum(pz);
  if ((threadIdx.x & 63) == 0) {
    part64[threadIdx.x >> 6] = sum;
    part64[4 + (threadIdx.x >> 6)] = pz;
  }
  __syncthreads();
  return Piece{m, (float)(part64[0] + part64[1] + part64[2] + part64[3]), part64[4] + part64[5] + part64[6] + part64[7]};
}

// Whole queries from their pieces: loss and lse, and what the gradient of very long rows needs.
template <int DT>
__global__ __launch_bounds__(256) void join_kernel(Args p) {
  __shared__ float part[4];
  __shared__ double part64[8];
  __shared__ Teacher w;
  const DistillArgs& a = p.a;
  const long long q = p.q0 + blockIdx.x;
  if (threadIdx.x < 64) make_teacher<DT>(a, q, 0, 0, w);
  const Piece x = join(p, q, part, part64);
  if (threadIdx.x == 0) {
    const double lse = lse_of(x.max, x.sum, a);
    a.loss[q] = loss_of(w, x.pz, lse);
    if (a.lse) a.lse[q] = (float)lse;
    if (p.joined) p.joined[q] = x;
  }
}

// The gradient of a piece: from lse (LSE), or from the query's pieces, with the loss by its first workgroup.
template <int DT, bool LSE>
__global__ __launch_bounds__(256, 4) void grad_kernel(Args p) {
  const DistillArgs& a = p.a;
  __shared__ float part[4];
  __shared__ double part64[8];
  __shared__ Teacher w;
  const long long q = p.q0 + blockIdx.y, i0 = (long long)blockIdx.x * kPiece, i1 = min(i0 + kPiece, a.n);
  float v[33];
  load_piece<DT, 256, 32>(static_cast<const char*>(a.logits) + (q * a.ld + i0) * size_of<DT>(), (int)(i1 - i0), v);
  if (threadIdx.x < 64) make_teacher<DT>(a, q, i0, i1, w);
  Piece x{};
  float l_hi = 0.f, l_lo = 0.f, unit = 1.f;
  if constexpr (LSE) {
    // lse log2(e) in two parts; z_i - lse is formed from the exact product s c.
    const double l = (double)a.lse_in[q] * 1.4426950408889634074;
    l_hi = (float)l;
    l_lo = fabsf(l_hi) < __builtin_inff() ? (float)(l - (double)l_hi) : 0.f;
    __syncthreads();
  } else {
    if (p.joined) {
      x = p.joined[q];
      __syncthreads();
    } else {
      x = join(p, q, part, part64);
      if (threadIdx.x == 0 && i0 == 0) a.loss[q] = loss_of(w, x.pz, lse_of(x.max, x.sum, a));
    }
    unit = inverse(x.max, x.sum);
  }
  const float x_max = x.max == kMinusInf ? 0.f : x.max;
  auto prob = [&](float s) {
    if constexpr (LSE) {
      const float hi = s * p.c_hi, lo = fmaf(s, p.c_hi, -hi) + s * p.c_lo;
      return hi == kMinusInf ? (l_hi != l_hi ? l_hi : 0.f) : __builtin_amdgcn_exp2f((hi - l_hi) + (lo - l_lo));
    } else {
      return exp_diff(s - x_max, p);  // (every logit -inf: 0 and unit 0)
    }
  };
#pragma unroll
  for (int i = 0; i <= 32; ++i) v[i] = prob(v[i]);
  store_piece<DT, 256, 32>(static_cast<char*>(a.grad) + (q * a.grad_ld + i0) * size_of<DT>(), (int)(i1 - i0), v, w.some,
                           w.weight * unit);
  // Every store of the piece has arrived before the entries on it are stored again.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x < 64 && w.some) store_entries<DT>(a, q, w, [&](float s1) { return prob(s1) * unit; });
}

int pieces_of(long long n) { return (int)((n + kPiece - 1) / kPiece); }
constexpr long long kRow = 32768;  // longest rows that one workgroup takes
constexpr long long kSlab = 32768; // queries of a launch

}  // namespace

size_t distill_workspace_bytes(long long nq, long long n) {
  if (n <= kRow) return 0;
  return ((size_t)nq * (size_t)pieces_of(n) + (size_t)nq) * sizeof(Piece);
}

hipError_t launch_distill(const DistillArgs& a, void* ws, hipStream_t s) {
  Args p;
  p.a = a;
  const double c = 1.4426950408889634074 / (double)a.tau;
  p.c_hi = (float)c;
  if ((double)p.c_hi > c) p.c_hi = std::nextafterf(p.c_hi, 0.f);
  p.c_lo = (float)(c - (double)p.c_hi);
  p.n_pieces = std::max(1, pieces_of(a.n));
  p.pieces = static_cast<Piece*>(ws);
  return with_dtype(a.dtype, [&](auto dt) {
    for (p.q0 = 0; p.q0 < a.nq; p.q0 += kSlab) {
      const unsigned nq = (unsigned)std::min(kSlab, a.nq - p.q0);
      const dim3 grid((unsigned)p.n_pieces, nq);
      if (!a.loss) {
        grad_kernel<dt(), true><<<grid, 256, 0, s>>>(p);
      } else if (a.n <= kRow) {
        auto rows = [&](auto grad) {
          if (a.n <= 256 * 16)
            row_kernel<dt(), 256, 16, grad()><<<nq, 256, 0, s>>>(p);
          else if (a.n <= 512 * 32)
            row_kernel<dt(), 512, 32, grad()><<<nq, 512, 0, s>>>(p);
          else
            row_kernel<dt(), 512, 64, grad()><<<nq, 512, 0, s>>>(p);
        };
        if (a.grad)
          rows(std::true_type{});
        else
          rows(std::false_type{});
      } else {
        p.joined = a.grad && p.n_pieces > kJoinHere ? p.pieces + a.nq * p.n_pieces : nullptr;
        piece_kernel<dt()><<<grid, 256, 0, s>>>(p);
        if (!a.grad || p.joined) join_kernel<dt()><<<nq, 256, 0, s>>>(p);
        if (a.grad) grad_kernel<dt(), false><<<grid, 256, 0, s>>>(p);
      }
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

}  // namespace oprag
