// Inner products of rows in the microscaled format (oprag_mx_scores).
//
// S[q, i] = sum over blocks b of 2^(cq + ci - 254) sum_j q[b, j] x[b, j].  One scaled matrix instruction takes 16 rows
// and 16 queries over 128 elements (four blocks), in 4 or 6 bits, and applies both scale bytes of
// every block itself; its sums are fp32.
//
// A workgroup of four waves keeps a block of QT x 16 queries in LDS and passes over a run of row
// tiles.  A wave owns RT x 16 rows of a tile: it loads their codes and scales straight into
// registers (no other wave needs them), sixteen blocks ahead of the product that uses them, and
// reads the queries' fragments from LDS, where they lie in the order of the lanes.  The rows that a
// lane loads are permuted so that its sums are of RT x 4 consecutive rows, which it stores as one piece.
#include <algorithm>

#include "mfma.h"
#include "mx.h"

namespace oprag {
namespace {

using namespace dev;

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ScoresArgs {
  MxRows q, r;
  void* out;
  long long ld;
  int dtype;
  int n_qblocks, n_chunks;  // chunk c takes row tiles [c tiles / n_chunks, (c + 1) tiles / n_chunks)
  long long tiles;
};

// One lane's share of a block: 16 or 24 bytes.
template <int BITS>
struct Codes {
  static constexpr int kWords = BITS;
  unsigned w[BITS];
  __device__ __forceinline__ void load(const unsigned char* p) {
    const uint4 a = *reinterpret_cast<const uint4*>(__builtin_assume_aligned(p, BITS == 4 ? 16 : 8));
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    if constexpr (BITS == 6) {
      const uint2 b = *reinterpret_cast<const uint2*>(p + 16);
      w[4] = b.x, w[5] = b.y;
    }
  }
  __device__ __forceinline__ i32x8 operand() const {
    i32x8 v = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    if constexpr (BITS == 6) v[4] = (int)w[4], v[5] = (int)w[5];
    return v;
  }
};

template <int RB, int QB, int STEP>
__device__ __forceinline__ f32x4 mfma_mx(const Codes<RB>& a, unsigned sa, const Codes<QB>& b, unsigned sb, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.operand(), b.operand(), c, RB == 4 ? 4 : 2, QB == 4 ? 4 : 2,
                                                          0, (int)sa, STEP, (int)sb);
}

// Four steps of 128 elements of a wave's rows.
template <int RB, int RT>
struct RowSet {
  Codes<RB> c[RT][4];
  unsigned s[RT][4];
};

template <int QT>
constexpr int lds_steps() {
  return QT == 8 ? 8 : QT == 4 ? 16 : 32;  // steps of 128 elements of the queries that LDS holds
}

// N consecutive rows' sums to out[row ..], as many as there are.
template <typename T, int N>
__device__ __forceinline__ void store_rows(T* p, const float (&v)[N], long long left) {
  typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  if (left >= N) {
    V o;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = (T)v[i];
    *reinterpret_cast<V*>(p) = o;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) p[i] = (T)v[i];
  }
}

template <int QB, int RB, int RT, int QT>
__global__ __launch_bounds__(256, 2) void scores_kernel(ScoresArgs p) {
  constexpr int KC = lds_steps<QT>();
  // [kc / 4][QT][64] scale bytes of four steps, [kc][QT][64] codes: their first 16 bytes, and the other 8
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int kc = min(KC, (p.r.nb + 15) / 16 * 4);
  unsigned* lds_s = reinterpret_cast<unsigned*>(lds);
  uint4* lds_lo = reinterpret_cast<uint4*>(lds_s + kc / 4 * QT * 64);
  uint2* lds_hi = reinterpret_cast<uint2*>(lds_lo + kc * QT * 64);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, g = lane >> 4;
  const int nb = p.r.nb, steps = (nb + 3) / 4, sets = (steps + 3) / 4;
  const long long row_bytes = (long long)nb * (4 * RB);
  const long long items = (long long)p.n_qblocks * p.n_chunks;
  for (long long item = logical_block(); item < items; item += gridDim.x) {
    const long long chunk = item / p.n_qblocks, q0 = (item - chunk * p.n_qblocks) * (QT * 16);
    const long long t0 = chunk * p.tiles / p.n_chunks, t1 = (chunk + 1) * p.tiles / p.n_chunks;

    // Queries' steps [first, first + KC) to LDS: zeros, with a scale of one, past the last block and the last query.
    auto stage = [&](int first) {
      __syncthreads();
      const int have = min(KC, (steps - first + 3) & ~3);
      for (int f = wave; f < have * QT; f += 4) {
        const int st = f / QT, qt = f - st * QT, b = (first + st) * 4 + g;
        const long long q = q0 + qt * 16 + r16;
        Codes<QB> c = {};
        if (b < nb && q < p.q.rows) c.load(p.q.codes + (q * nb + b) * (4 * QB));
        lds_lo[f * 64 + lane] = make_uint4(c.w[0], c.w[1], c.w[2], c.w[3]);
        if constexpr (QB == 6) lds_hi[f * 64 + lane] = make_uint2(c.w[4], c.w[5]);
      }
      for (int f = wave; f < have / 4 * QT; f += 4) {
        const int st = f / QT * 4, qt = f % QT;
        const long long q = q0 + qt * 16 + r16;
        unsigned v = 0x7f7f7f7fu;
        if (q < p.q.rows) {
          v = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int b = (first + st + j) * 4 + g;
            v |= (b < nb ? p.q.scales[q * nb + b] : 127u) << (8 * j);
          }
        }
        lds_s[f * 64 + lane] = v;
      }
      __syncthreads();
    };

    // The row of subtile t that this lane loads, within the tile.
    auto load = [&](RowSet<RB, RT>& a, long long tile, int set) {
      const long long base = tile * (64 * RT);
      const unsigned char* codes = p.r.codes + base * row_bytes;
      const unsigned char* scales = p.r.scales + base * nb;
      const int last = (int)min(p.r.rows - base, 64ll * RT) - 1;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int row = min(wave * 16 * RT + 4 * RT * (r16 >> 2) + 4 * t + (r16 & 3), last);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int step = set * 4 + j, b = step * 4 + g;
          if (step < steps) {
            const int bc = min(b, nb - 1);
            a.c[t][j].load(codes + (unsigned)row * (unsigned)row_bytes + (unsigned)bc * (4 * RB));
            const unsigned s = scales[(unsigned)row * (unsigned)nb + (unsigned)bc];
            a.s[t][j] = b < nb ? s : 127u;  // the queries are zero there
          }
        }
      }
    };

    f32x4 acc[RT][QT];
    auto clear = [&] {
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int j = 0; j < QT; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    auto product = [&](const RowSet<RB, RT>& a, int set) {
      const int at = set % (KC / 4);
      unsigned sb[QT];
#pragma unroll
      for (int j = 0; j < QT; ++j) sb[j] = lds_s[(at * QT + j) * 64 + lane];
      auto one = [&](auto st) {
        constexpr int s = decltype(st)::value;
        if (set * 4 + s >= steps) return;
#pragma unroll
        for (int j = 0; j < QT; ++j) {
          Codes<QB> b;
          const int f = ((at * 4 + s) * QT + j) * 64 + lane;
          const uint4 lo = lds_lo[f];
          b.w[0] = lo.x, b.w[1] = lo.y, b.w[2] = lo.z, b.w[3] = lo.w;
          if constexpr (QB == 6) {
            const uint2 hi = lds_hi[f];
            b.w[4] = hi.x, b.w[5] = hi.y;
          }
#pragma unroll
          for (int t = 0; t < RT; ++t) acc[t][j] = mfma_mx<RB, QB, s>(a.c[t][s], a.s[t][s], b, sb[j], acc[t][j]);
        }
      };
      one(std::integral_constant<int, 0>{});
      one(std::integral_constant<int, 1>{});
      one(std::integral_constant<int, 2>{});
      one(std::integral_constant<int, 3>{});
    };
    auto store = [&](long long tile) {
      const long long row = tile * (64 * RT) + wave * 16 * RT + 4 * RT * g;
      const long long left = p.r.rows - row;
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        const long long q = q0 + j * 16 + r16;
        if (q >= p.q.rows) continue;
        float v[4 * RT];
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * t + i] = acc[t][j][i];
        const long long at = q * p.ld + row;
        if (p.dtype == kDtypeF32)
          store_rows(static_cast<float*>(p.out) + at, v, left);
        else if (p.dtype == kDtypeBF16)
          store_rows(static_cast<__bf16*>(p.out) + at, v, left);
        else
          store_rows(static_cast<_Float16*>(p.out) + at, v, left);
      }
    };

    const bool resident = steps <= KC;
    long long tile = t0, next_tile = t0;
    int set = 0, next_set = 0;
    RowSet<RB, RT> a, b;
    auto advance = [&] {
      if (++next_set == sets) next_set = 0, ++next_tile;
    };
    auto turn = [&](RowSet<RB, RT>& cur, RowSet<RB, RT>& next) {
      if (set == 0) clear();
      if (!resident && set % (KC / 4) == 0) stage(set * 4);
      advance();
      if (next_tile < t1) load(next, next_tile, next_set);
      product(cur, set);
      if (set == sets - 1) store(tile);
      tile = next_tile, set = next_set;
    };
    if (tile < t1) load(a, tile, 0);
    if (resident) stage(0);
    while (tile < t1) {
      turn(a, b);
      if (tile >= t1) break;
      turn(b, a);
    }
  }
}

template <int QB, int RB, int RT, int QT>
hipError_t launch(ScoresArgs p, hipStream_t s) {
  p.n_qblocks = (int)((p.q.rows + 16 * QT - 1) / (16 * QT));
  p.tiles = (p.r.rows + 64 * RT - 1) / (64 * RT);
  p.n_chunks = (int)std::max<long long>(1, std::min<long long>(p.tiles, 512 / std::min(p.n_qblocks, 512)));
  const long long items = (long long)p.n_qblocks * p.n_chunks;
  const int kc = std::min(lds_steps<QT>(), (p.r.nb + 15) / 16 * 4);
  const unsigned lds = (unsigned)(kc * QT * 64 * (4 * QB + 1));
  scores_kernel<QB, RB, RT, QT><<<(unsigned)std::min<long long>(items, 1 << 20), 256, lds, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_scores(const MxRows& q, const MxRows& rows, void* out, int dtype, long long ld, hipStream_t s) {
  ScoresArgs p = {};
  p.q = q;
  p.r = rows;
  p.out = out;
  p.ld = ld;
  p.dtype = dtype;
  return with_bits(q.bits, [&](auto qb) {
    return with_bits(rows.bits, [&](auto rb) {
      if (q.rows <= 16) return launch<qb(), rb(), 1, 1>(p, s);
      if (q.rows <= 64) return launch<qb(), rb(), 1, 4>(p, s);
      return launch<qb(), rb(), 2, 8>(p, s);
    });
  });
}

}  // namespace oprag
