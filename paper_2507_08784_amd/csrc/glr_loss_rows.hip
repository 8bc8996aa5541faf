// The rows of the losses that need a row's softmax and its target's
// log-probability: token log-probabilities, the preference and the policy loss.
#include <type_traits>

#include "glr_loss.hpp"

namespace glr {
namespace {

// What a row's terms need beside its sums, loaded while the row is on its way.
struct RowIn {
  float zy, coef, old, adv, ref;
  double weight;      // policy: of the row
};
__device__ __forceinline__ RowIn row_in(const Rows& r, const Terms& a, const RowPos& p, int seq, float zy) {
  RowIn x = {};
  x.zy = zy;
  if (a.op == OP_LOGP) {
    if (a.coef.p) x.coef = ld_f(a.coef, p);
    return x;
  }
  x.old = ld_f(a.old, p);
  x.adv = ld_f(a.adv, p);
  if (a.ref.p) x.ref = ld_f(a.ref, p);
  double n = a.denom;
  if (a.by_seq) n = (double)a.seqs.n * max(a.count[seq], 1);
  else if (n == 0.0) n = max(a.count ? *a.count : count_rows(r, a.seqs), 1);
  x.weight = 1.0 / n;
  return x;
}

// stores the row's terms and returns g = d loss / d lp times grad_scale / T
__device__ __forceinline__ double row_terms(const Rows& r, const Terms& a, const RowPos& p, const RowIn& x, float m,
                                            float s) {
  const double lp = ((double)x.zy - (double)m) * r.inv_t - log((double)s);
  a.logps[p.t] = (float)lp;
  if (a.op == OP_LOGP) {
    if (a.stats) {
      a.stats[2 * (int64_t)p.t] = m;
      a.stats[2 * (int64_t)p.t + 1] = s;
    }
    return (double)x.coef * r.gscale;
  }
  const double ratio = exp(lp - (double)x.old);
  const double in = ratio < a.low ? a.low : ratio > a.high ? a.high : ratio;   // NaN stays
  const double u = ratio * (double)x.adv, v = in * (double)x.adv;
  const bool cut = u > v;
  double term = cut ? -v : -u, slope = cut ? 0.0 : -u, k = 0.0;
  if (a.ref.p) {
    const double d = (double)x.ref - lp, y = expm1(d);
    k = y - d;
    term += a.kl * k;
    slope -= a.kl * y;
  }
  a.part[p.t] = (float)(x.weight * term);
  a.part[(int64_t)r.rows + p.t] = (float)(x.weight * k);
  a.part[2 * (int64_t)r.rows + p.t] = cut ? (float)x.weight : 0.f;
  return x.weight * slope * r.gscale;
}
// what a masked row leaves
__device__ __forceinline__ void row_masked(const Rows& r, const Terms& a, const RowPos& p) {
  a.logps[p.t] = 0.f;
  if (a.op == OP_LOGP) {
    if (a.stats) {
      a.stats[2 * (int64_t)p.t] = 0.f;
      a.stats[2 * (int64_t)p.t + 1] = 1.f;
    }
    return;
  }
  for (int k = 0; k < 3; ++k) a.part[k * (int64_t)r.rows + p.t] = 0.f;
}

// whether a row is trained on; its target and its sequence
__device__ __forceinline__ bool row_live(const Rows& r, const Seqs& q, const RowPos& p, int& y, int& seq) {
  seq = (int)p.b;
  if (!row_target(r, p, y)) return false;
  if (q.cu) seq = seq_of(q, p.t, r.rows);
  return seq >= 0;
}

// a sweep of gradient elements: f e_j, and g more at the target
template <class T, int NT, int NV, bool KEEP>
__device__ __forceinline__ void write_grad(RowRegs<T, NT, NV, KEEP>& row, T* dz, float c, float m, float f, float g, int y) {
  constexpr int N = Piece<T>::N;
  const int iy = y / N, ky = y % N;
  row.chunks([&](int first) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int i = first + v * NT;
      float x[N];
      unpack<T>(row.raw[v], x);
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = f * exp2_of((x[k] - m) * c);
      if (i == iy) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] += k == ky ? g : 0.f;
      }
      if (i < row.whole) st_piece(dz + (int64_t)i * N, pack<T>(x));
      piece_end();
    }
  });
  const int at = row.whole * N + row.tid;
  if (at < row.V) store_z(dz + at, f * exp2_of((row.tail - m) * c) + (at == y ? g : 0.f));
}

// A workgroup a row: the first waves have the row, the last its terms (what they
// need is loaded while the row is on its way, and their fp64 takes no
// registers beside a row's).  Each thread keeps its own running maximum and
// sum over the pieces it has; one exchange makes the row's.
template <class T, int NT, int NV, bool KEEP>
__global__ void __launch_bounds__(NT + 64) k_loss_row(Rows r, Terms a) {
  constexpr int N = Piece<T>::N, NW = NT / 64;
  __shared__ float m_s[NW], s_s[NW];
  __shared__ float f_s[3];
  const RowPos p = row_pos(r, blockIdx.x);
  int y, seq;
  const bool live = row_live(r, a.seqs, p, y, seq);
  T* dz = r.dz.p ? static_cast<T*>(const_cast<void*>(r.dz.p)) + p.of(r.dz) : nullptr;
  if (!live) {
    if (threadIdx.x == 0) row_masked(r, a, p);
    if (dz) row_zero<T, NT + 64>(dz, r.V);
    return;
  }
  const T* z = static_cast<const T*>(r.z.p) + p.of(r.z);
  // (a scalar: the two parts meet at the same number of barriers, wave by wave)
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if (wave < NW) {
    RowRegs<T, NT, NV, KEEP> row;
    row.open(z, r.V, threadIdx.x);
    float mt = row.tail, st = mt == -INFINITY ? 0.f : exp2_of((row.tail - mt) * r.c);
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
    const float mw = wave_max(mt);
    const float sw = wave_sum(mt == -INFINITY ? st : st * exp2_of((mt - mw) * r.c));
    if ((threadIdx.x & 63) == 0) {
      m_s[wave] = mw;
      s_s[wave] = sw;
    }
    __syncthreads();
    if (!dz) return;
    __syncthreads();
    write_grad(row, dz, r.c, f_s[0], f_s[1], f_s[2], y);
    return;
  }
  const float nan = __builtin_nanf("");
  const RowIn x = row_in(r, a, p, seq, y >= 0 ? load_z(z + y) : nan);
  __syncthreads();
  const int lane = threadIdx.x & 63;
  const float mw = lane < NW ? m_s[lane] : -INFINITY;
  const float m = wave_max(mw);
  const float s = wave_sum(lane < NW ? s_s[lane] * exp2_of((mw - m) * r.c) : 0.f);     // (all -inf: NaN)
  if (lane == 0) {
    const double g = row_terms(r, a, p, x, m, s);
    f_s[0] = m;
    f_s[1] = y >= 0 ? (float)(-g / (double)s) : nan;
    f_s[2] = (float)g;
  }
  if (dz) __syncthreads();
}

// The gradient from the row's m and s of an earlier call: one sweep.
template <class T, int NT, int NV>
__global__ void __launch_bounds__(NT) k_loss_grad(Rows r, Terms a) {
  const RowPos p = row_pos(r, blockIdx.x);
  int y, seq;
  const bool live = row_live(r, a.seqs, p, y, seq);
  T* dz = static_cast<T*>(const_cast<void*>(r.dz.p)) + p.of(r.dz);
  if (!live) return row_zero<T, NT>(dz, r.V);
  const float m = a.stats[2 * (int64_t)p.t], s = a.stats[2 * (int64_t)p.t + 1];
  const double g = (double)(a.seq_coef ? a.seq_coef[seq] : ld_f(a.coef, p)) * r.gscale;
  RowRegs<T, NT, NV, false> row;
  row.open(static_cast<const T*>(r.z.p) + p.of(r.z), r.V, threadIdx.x);
  write_grad(row, dz, r.c, m, y >= 0 ? (float)(-g / (double)s) : __builtin_nanf(""), (float)g, y);
}

template <class T, int NT, int NV, bool KEEP>
void row(const Rows& r, const Terms& a, void* stream) {
  launch("loss rows", k_loss_row<T, NT, NV, KEEP>, r.rows, NT + 64, 0, stream, r, a);
}
template <class T, int NT, int NV>
void grad(const Rows& r, const Terms& a, void* stream) {
  launch("loss gradient rows", k_loss_grad<T, NT, NV>, r.rows, NT, 0, stream, r, a);
}

template <class T>
void rows_of(const Rows& r, const Terms& a, void* stream) {
  const int n = r.V / Piece<T>::N;          // pieces of a row
  if (a.op == OP_COEF) {
    if (n <= 256) return grad<T, 64, 4>(r, a, stream);
    if (n <= 2048) return grad<T, 256, 4>(r, a, stream);
    return grad<T, 1024, 4>(r, a, stream);
  }
  if (!r.dz.p) {
    if (n <= 256) return row<T, 64, 4, false>(r, a, stream);
    if (n <= 1024 || r.rows >= 1024) return row<T, 192, 4, false>(r, a, stream);
    return row<T, 960, 4, false>(r, a, stream);
  }
  if (n <= 128) return row<T, 64, 2, true>(r, a, stream);
  if (n <= 256) return row<T, 64, 4, true>(r, a, stream);
  if (n <= 768) return row<T, 192, 4, true>(r, a, stream);
  if (n <= 1792) return row<T, 448, 4, true>(r, a, stream);
  if (n <= 4032) return row<T, 448, 9, true>(r, a, stream);
  if (n <= 6720) return row<T, 960, 7, true>(r, a, stream);
  if (n <= 9600) return row<T, 960, 10, true>(r, a, stream);
  if (n <= 13440) return row<T, 960, 14, true>(r, a, stream);
  if (n <= 16320) return row<T, 960, 17, true>(r, a, stream);
  if (n <= 20160) return row<T, 960, 21, true>(r, a, stream);
  return row<T, 960, 8, false>(r, a, stream);
}

}  // namespace

void loss_rows(int dtype, const Rows& r, const Terms& a, void* stream) {
  if (dtype == GLR_F32) rows_of<float>(r, a, stream);
  else if (dtype == GLR_BF16) rows_of<bf16_t>(r, a, stream);
  else rows_of<f16_t>(r, a, stream);
}

}  // namespace glr
