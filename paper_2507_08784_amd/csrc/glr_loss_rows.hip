// The rows of the losses that need a row's softmax and its target's
// log-probability: token log-probabilities, the preference and the policy loss.
#include <type_traits>

#include "glr_loss.hpp"

namespace glr {
namespace {

__device__ __forceinline__ double row_logp(const Rows& r, float zy, float m, float s) {
  return ((double)zy - (double)m) * r.inv_t - log((double)s);
}

// stores the row's terms and returns g = d loss / d lp times grad_scale / T
__device__ __forceinline__ double row_terms(const Rows& r, const Terms& a, const RowPos& p, int seq, double lp,
                                            float m, float s) {
  if (a.op == OP_LOGP) {
    a.logps[p.t] = (float)lp;
    if (a.stats) {
      a.stats[2 * (int64_t)p.t] = m;
      a.stats[2 * (int64_t)p.t + 1] = s;
    }
    return a.coef.p ? (double)ld_f(a.coef, p) * r.gscale : 0.0;
  } else if (a.op == OP_COEF) {
    return (double)(a.seq_coef ? a.seq_coef[seq] : ld_f(a.coef, p)) * r.gscale;
  } else {
    double w;
    if (a.by_seq) {
      const int n = a.count[seq];
      w = 1.0 / ((double)a.seqs.n * (n > 0 ? n : 1));
    } else {
      w = 1.0 / (a.denom > 0.0 ? a.denom : (double)(*a.count > 0 ? *a.count : 1));
    }
    const double A = ld_f(a.adv, p);
    const double ratio = exp(lp - (double)ld_f(a.old, p));
    const double in = ratio < a.low ? a.low : ratio > a.high ? a.high : ratio;   // NaN stays
    const double u = ratio * A, v = in * A;
    const bool cut = u > v;
    double term = cut ? -v : -u, slope = cut ? 0.0 : -u, k = 0.0;
    if (a.ref.p) {
      const double d = (double)ld_f(a.ref, p) - lp, x = expm1(d);
      k = x - d;
      term += a.kl * k;
      slope -= a.kl * x;
    }
    a.logps[p.t] = (float)lp;
    a.part[p.t] = (float)(w * term);
    a.part[(int64_t)r.rows + p.t] = (float)(w * k);
    a.part[2 * (int64_t)r.rows + p.t] = cut ? (float)w : 0.f;
    return w * slope * r.gscale;
  }
}
// what a masked row leaves
__device__ __forceinline__ void row_masked(const Rows& r, const Terms& a, const RowPos& p) {
  if (a.op == OP_LOGP) {
    a.logps[p.t] = 0.f;
    if (a.stats) {
      a.stats[2 * (int64_t)p.t] = 0.f;
      a.stats[2 * (int64_t)p.t + 1] = 1.f;
    }
  } else if (a.op == OP_POLICY) {
    a.logps[p.t] = 0.f;
    for (int k = 0; k < 3; ++k) a.part[k * (int64_t)r.rows + p.t] = 0.f;
  }
}


// A workgroup a row.  Each thread keeps its own running maximum and sum over
// the pieces it has (one exchange then makes the row's), and the row's terms
// are one thread's work.  GRAD without a softmax (OP_COEF) has the row's m and
// s from an earlier call.
template <class T, bool COEF, int NT, int NV, bool KEEP>
__global__ void __launch_bounds__(NT) k_loss_row(Rows r, Terms a) {
  constexpr int N = Piece<T>::N;
  __shared__ float sh[NT / 64];
  __shared__ float coef[2];
  const RowPos p = row_pos(r, blockIdx.x);
  int y;
  bool live = row_target(r, p, y);
  int seq = (int)p.b;
  if (live && a.seqs.cu) {
    seq = seq_of(a.seqs, p.t, r.rows);
    live = seq >= 0;
  }
  T* dz = r.dz.p ? static_cast<T*>(const_cast<void*>(r.dz.p)) + p.of(r.dz) : nullptr;
  if (!live) {
    if (threadIdx.x == 0) row_masked(r, a, p);
    if (dz) row_zero<T, NT>(dz, r.V);
    return;
  }
  RowRegs<T, NT, NV, KEEP> row;
  row.open(static_cast<const T*>(r.z.p) + p.of(r.z), r.V, threadIdx.x);
  const float zy = y >= 0 ? load_z(row.z + y) : __builtin_nanf("");
  float m, s;
  if constexpr (COEF) {
    m = a.stats[2 * (int64_t)p.t];
    s = a.stats[2 * (int64_t)p.t + 1];
  } else {
    float mt = row.tail, st = row.tail > -INFINITY || row.tail != row.tail ? exp2_of((row.tail - row.tail) * r.c) : 0.f;
    row.chunks([&](int) {
      float top = mt;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float x[N];
        unpack<T>(row.raw[v], x);
#pragma unroll
        for (int k = 0; k < N; ++k) top = fmaxf(top, x[k]);
        piece_end(top);
      }
      const float base = top == -INFINITY ? 0.f : top;
      st *= exp2_of((mt - base) * r.c);     // (mt = -inf: st is 0, and stays)
      mt = top;
      row.repack();
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float x[N];
        unpack<T>(row.raw[v], x);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = exp2_of((x[k] - base) * r.c);
        st += sum_of(x);
        piece_end(st);
      }
    });
    m = block_max<NT>(mt, sh);
    s = block_sum<NT>(st * exp2_of((mt - m) * r.c), sh);
  }
  if (threadIdx.x == 0) {
    const double lp = row_logp(r, zy, m, s);
    const double g = row_terms(r, a, p, seq, lp, m, s);
    coef[0] = y >= 0 ? (float)(g / (double)s) : __builtin_nanf("");
    coef[1] = (float)g;
  }
  if (!dz) return;
  __syncthreads();
  const float f = -coef[0], g = coef[1];
  const int iy = y / N, ky = y % N;
  row.chunks([&](int first) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int i = first + v * NT;
      float x[N];
      unpack<T>(row.raw[v], x);
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = f * exp2_of((x[k] - m) * r.c);
      if (i == iy) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] += k == ky ? g : 0.f;
      }
      if (i < row.whole) st_piece(dz + (int64_t)i * N, pack<T>(x));
      piece_end();
    }
  });
  const int at = row.whole * N + (int)threadIdx.x;
  if (at < r.V) store_z(dz + at, f * exp2_of((row.tail - m) * r.c) + (at == y ? g : 0.f));
}

template <class T, bool COEF, int NT, int NV, bool KEEP>
void go(const Rows& r, const Terms& a, void* stream) {
  launch("loss rows", k_loss_row<T, COEF, NT, NV, KEEP>, r.rows, NT, 0, stream, r, a);
}

template <class T>
void rows_of(const Rows& r, const Terms& a, void* stream) {
  const int n = r.V / Piece<T>::N;          // pieces of a row
  if (a.op == OP_COEF) {
    if (n <= 256) return go<T, true, 64, 4, false>(r, a, stream);
    if (n <= 2048) return go<T, true, 256, 4, false>(r, a, stream);
    return go<T, true, 1024, 4, false>(r, a, stream);
  }
  if (!r.dz.p) {
    if (n <= 256) return go<T, false, 64, 4, false>(r, a, stream);
    if (n <= 2048) return go<T, false, 256, 4, false>(r, a, stream);
    return go<T, false, 1024, 4, false>(r, a, stream);
  }
  if (n <= 64) return go<T, false, 64, 1, true>(r, a, stream);
  if (n <= 128) return go<T, false, 64, 2, true>(r, a, stream);
  if (n <= 256) return go<T, false, 64, 4, true>(r, a, stream);
  if (n <= 512) return go<T, false, 256, 2, true>(r, a, stream);
  if (n <= 1024) return go<T, false, 256, 4, true>(r, a, stream);
  if (n <= 2048) return go<T, false, 512, 4, true>(r, a, stream);
  if (n <= 4096) return go<T, false, 512, 8, true>(r, a, stream);
  if (n <= 6144) return go<T, false, 1024, 6, true>(r, a, stream);
  if (n <= 7168) return go<T, false, 1024, 7, true>(r, a, stream);
  if (n <= 8192) return go<T, false, 1024, 8, true>(r, a, stream);
  if (n <= 10240) return go<T, false, 1024, 10, true>(r, a, stream);
  if (n <= 13312) return go<T, false, 1024, 13, true>(r, a, stream);
  if (n <= 16384) return go<T, false, 1024, 16, true>(r, a, stream);
  if (n <= 20480) return go<T, false, 1024, 20, true>(r, a, stream);
  return go<T, false, 1024, 8, false>(r, a, stream);
}

}  // namespace

void loss_rows(int dtype, const Rows& r, const Terms& a, void* stream) {
  if (dtype == GLR_F32) rows_of<float>(r, a, stream);
  else if (dtype == GLR_BF16) rows_of<bf16_t>(r, a, stream);
  else rows_of<f16_t>(r, a, stream);
}

}  // namespace glr
