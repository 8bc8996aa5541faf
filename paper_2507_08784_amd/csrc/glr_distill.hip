// Distillation from a teacher's top logits: the rows.
#include <type_traits>

#include "glr_loss.hpp"

namespace glr {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float ld_teacher(const Teach& q, int64_t at, int k) {
  if (q.ttype == GLR_F32) return static_cast<const float*>(q.t.p)[at + k];
  if (q.ttype == GLR_BF16) return load_z(static_cast<const bf16_t*>(q.t.p) + at + k);
  return load_z(static_cast<const f16_t*>(q.t.p) + at + k);
}

// whether element k of piece i is outside the teacher's list
template <int N>
__device__ __forceinline__ uint32_t listed_bits(const uint32_t* bits, int i) {
  return bits[i * N >> 5] >> (i * N & 31);
}

// A workgroup a row.  The list's tokens are marked in a bitmap over the
// vocabulary in LDS: the mass outside the list is summed as such (the total
// less the list's would cancel where the list holds nearly all of it), and a
// repeated token is seen.  REST: there is such a mass; TWO: hard labels at a
// temperature other than the list's, which need a second sum.  The list's own
// gradient elements are written over the dense ones behind a barrier.
template <class T, bool REST, bool TWO, int NT, int NV, bool KEEP>
__global__ void __launch_bounds__(NT) k_distill_row(Rows r, Teach q) {
  constexpr int N = Piece<T>::N;
  extern __shared__ uint32_t bits[];
  const int words = (r.V + 31) / 32;
  int* id_s = reinterpret_cast<int*>(bits + words);
  float* zk_s = reinterpret_cast<float*>(id_s + q.top);
  float* p_s = zk_s + q.top;
  __shared__ float shf[NT / 64];
  __shared__ double shd[NT / 64];
  __shared__ int bad_s, again_s;
  const RowPos p = row_pos(r, blockIdx.x);
  int y;
  const bool live = row_target(r, p, y);
  T* dz = r.dz.p ? static_cast<T*>(const_cast<void*>(r.dz.p)) + p.of(r.dz) : nullptr;
  if (!live) {
    if (threadIdx.x == 0) q.losses[p.t] = 0.f;
    if (dz) row_zero<T, NT>(dz, r.V);
    return;
  }
  RowRegs<T, NT, NV, KEEP> row;
  row.open(static_cast<const T*>(r.z.p) + p.of(r.z), r.V);
  const T* z = row.z;
  for (int j = threadIdx.x; j < words; j += NT) bits[j] = 0u;
  if (threadIdx.x == 0) bad_s = again_s = 0;
  __syncthreads();
  const int64_t ido = p.of(q.ids), to = p.of(q.t);
  int have = 0;                       // entries, and (above 16 bits) distinct tokens
  float high = -INFINITY;
  for (int k = threadIdx.x; k < q.top; k += NT) {
    const int64_t id = ld_int(q.ids.p, ido + k, q.id64);
    const float t = ld_teacher(q, to, k);
    int at = -1;
    if (id >= r.V) {
      bad_s = 1;
    } else if (id >= 0 && t != -INFINITY) {
      at = (int)id;
      const uint32_t bit = 1u << (at & 31);
      if (atomicOr(&bits[at >> 5], bit) & bit) again_s = 1;
      else have += 1 << 16;
      ++have;
      high = fmaxf(high, t);
    }
    id_s[k] = at;
    p_s[k] = t;
    zk_s[k] = at >= 0 ? load_z(z + at) : 0.f;
  }
  have = block_sum<NT, int>(have, reinterpret_cast<int*>(shf));
  high = block_max<NT>(high, shf);    // (its barriers also end the marking)
  const bool rest = REST && (have & 0xFFFF) > 0 && (have >> 16) < r.V;

  // sums of the row: all tokens, those outside the list, all at temperature 1
  float mt = row.tail, st = 0.f, ot = 0.f, ut = 0.f;
  const int tail_at = row.whole * N + (int)threadIdx.x;
  if (tail_at < r.V) {
    st = exp2_of((row.tail - mt) * r.c);
    if (mt == -INFINITY) st = 0.f;
    ut = st;
    if (REST) ot = bits[tail_at >> 5] >> (tail_at & 31) & 1u ? 0.f : st;
  }
  row.chunks([&](int first) {
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
    const float by = exp2_of((mt - base) * r.c);
    st *= by;
    if (REST) ot *= by;
    if (TWO) ut *= exp2_of((mt - base) * kLog2e);
    mt = top;
    row.repack();
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float x[N];
      unpack<T>(row.raw[v], x);
      const int i = first + v * NT;
      const uint32_t in = REST && i < row.whole ? listed_bits<N>(bits, i) : 0u;
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] -= base;
      if (TWO) {
        float u[N];
#pragma unroll
        for (int k = 0; k < N; ++k) u[k] = exp2_of(x[k] * kLog2e);
        ut += sum_of(u);
        piece_end(ut);
      }
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = exp2_of(x[k] * r.c);
      st += sum_of(x);
      piece_end(st);
      if (REST) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = in >> k & 1u ? 0.f : x[k];
        ot += sum_of(x);
        piece_end(ot);
      }
    }
  });
  const float m = block_max<NT>(mt, shf);
  const float by = exp2_of((mt - m) * r.c);
  const float s = block_sum<NT>(st * by, shf);
  const float so = REST ? block_sum<NT>(ot * by, shf) : 0.f;
  const float s1 = TWO ? block_sum<NT>(ut * exp2_of((mt - m) * kLog2e), shf) : s;

  // the teacher's masses and their divergence
  const double logs = log((double)s);
  double norm;
  if (q.lse.p) {
    norm = ld_f(q.lse, p);
  } else {
    double sum = 0.0;
    for (int k = threadIdx.x; k < q.top; k += NT)
      if (id_s[k] >= 0) sum += exp(((double)p_s[k] - (double)high) * r.inv_t);
    norm = (double)high * r.inv_t + log(block_sum<NT, double>(sum, shd));
  }
  double kl = 0.0, mass = 0.0;
  for (int k = threadIdx.x; k < q.top; k += NT) {
    double pk = 0.0;
    if (id_s[k] >= 0) {
      const double lpk = (double)p_s[k] * r.inv_t - norm;
      pk = exp(lpk);
      if (pk > 0.0) kl += pk * (lpk - (((double)zk_s[k] - (double)m) * r.inv_t - logs));
      else kl += pk;        // (NaN stays)
    }
    p_s[k] = (float)pk;
    mass += pk;
  }
  kl = block_sum<NT, double>(kl, shd);
  mass = block_sum<NT, double>(mass, shd);
  double left = 0.0;
  if (rest) {
    left = 1.0 - mass;
    if (left < kRestFloor) left = 0.0;
    if (left != 0.0) kl += left * (log(left) - (log((double)so) - logs));
  }
  const float nan = __builtin_nanf("");
  const bool bad = bad_s != 0 || y < 0;
  if (threadIdx.x == 0) {
    double loss = (1.0 - q.hard) * kl / (r.inv_t * r.inv_t);
    if (q.hard > 0.0) loss -= q.hard * ((double)(y >= 0 ? load_z(z + y) : nan) - (double)m - log((double)s1));
    q.losses[p.t] = bad ? nan : (float)loss;
  }
  if (!dz) return;
  const double n = q.denom > 0.0 ? q.denom : (double)(q.count ? (*q.count > 0 ? *q.count : 1) : r.rows);
  const double scale = r.gscale / r.inv_t / n;     // grad_scale / n
  const double soft = (1.0 - q.hard) / r.inv_t * scale;
  float f_out = bad ? nan : (float)(soft * ((mass + left) / (double)s - (left != 0.0 ? left / (double)so : 0.0)));
  float f_in = (float)(soft * (mass + left) / (double)s);
  const float f1 = (float)(q.hard * scale / (double)s1), h = (float)(q.hard * scale), sf = (float)soft;
  if (!TWO) {                 // one exponential serves both terms
    f_out += f1;
    f_in += f1;
  }
  // (every thread has read what it needs of the row: a gradient may replace it)
  const int iy = q.hard > 0.0 ? y / N : -1, ky = y % N;
  row.chunks([&](int first) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int i = first + v * NT;
      float x[N];
      unpack<T>(row.raw[v], x);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float d = x[k] - m;
        x[k] = f_out * exp2_of(d * r.c);
        if (TWO) x[k] = fmaf(f1, exp2_of(d * kLog2e), x[k]);
      }
      if (i == iy) {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] -= k == ky ? h : 0.f;
      }
      if (i < row.whole) st_piece(dz + (int64_t)i * N, pack<T>(x));
      piece_end();
    }
  });
  if (tail_at < r.V) {
    const float d = row.tail - m;
    float x = f_out * exp2_of(d * r.c);
    if (TWO) x = fmaf(f1, exp2_of(d * kLog2e), x);
    store_z(dz + tail_at, x - (tail_at == y ? h : 0.f));
  }
  __threadfence_block();
  __syncthreads();
  for (int k = threadIdx.x; k < q.top; k += NT) {
    const int j = id_s[k];
    if (j < 0) continue;
    float mine = p_s[k];
    if (again_s) {             // a repeated token: its first entry has the sum of its masses
      bool first = true;
      for (int i = 0; i < k; ++i) first = first && id_s[i] != j;
      if (!first) continue;
      for (int i = k + 1; i < q.top; ++i)
        if (id_s[i] == j) mine += p_s[i];
    }
    const float d = zk_s[k] - m;
    float x = fmaf(f_in, exp2_of(d * r.c), -sf * mine);
    if (TWO) x = fmaf(f1, exp2_of(d * kLog2e), x);
    if (j == y) x -= h;
    store_z(dz + j, bad ? nan : x);
  }
}

template <class T, bool REST, bool TWO, int NT, int NV, bool KEEP>
void go(const Rows& r, const Teach& q, void* stream) {
  launch("distillation rows", k_distill_row<T, REST, TWO, NT, NV, KEEP>, r.rows, NT,
         (((size_t)r.V + 31) / 32 + 3 * (size_t)q.top) * 4, stream, r, q);
}

template <class T, bool REST, bool TWO>
void rows_of(const Rows& r, const Teach& q, void* stream) {
  const int n = r.V / Piece<T>::N;          // pieces of a row
  if (n <= 128) return go<T, REST, TWO, 64, 2, true>(r, q, stream);
  if (n <= 256) return go<T, REST, TWO, 64, 4, true>(r, q, stream);
  if (n <= 1024) return go<T, REST, TWO, 256, 4, true>(r, q, stream);
  if (n <= 2048) return go<T, REST, TWO, 512, 4, true>(r, q, stream);
  if (n <= 4096) return go<T, REST, TWO, 512, 8, true>(r, q, stream);
  if (n <= 8192) return go<T, REST, TWO, 1024, 8, true>(r, q, stream);
  if (n <= 13312) return go<T, REST, TWO, 1024, 13, true>(r, q, stream);
  if (n <= 16384) return go<T, REST, TWO, 1024, 16, true>(r, q, stream);
  return go<T, REST, TWO, 1024, 8, false>(r, q, stream);
}

template <class T>
void variants(const Rows& r, const Teach& q, void* stream) {
  const bool rest = q.lse.p != nullptr, two = q.hard > 0.0 && r.inv_t != 1.0;
  if (rest) return two ? rows_of<T, true, true>(r, q, stream) : rows_of<T, true, false>(r, q, stream);
  return two ? rows_of<T, false, true>(r, q, stream) : rows_of<T, false, false>(r, q, stream);
}

}  // namespace

void distill_rows(int dtype, const Rows& r, const Teach& q, void* stream) {
  if (dtype == GLR_F32) variants<float>(r, q, stream);
  else if (dtype == GLR_BF16) variants<bf16_t>(r, q, stream);
  else variants<f16_t>(r, q, stream);
}

}  // namespace glr
