// Orthogonalisation of matrices whose shorter side has at most ORTH_SMALL values,
// in fp64 and three launches.
//
// The quintic's steps are functions of the Gram matrix: with A = X X^T and Q = a + b A
// + c A^2, X' = Q X and A' = Q A Q, and all of these commute, so the result is
// P U with P = the product of the steps' Q, and U is read twice instead of eleven
// times: for A (with the momentum's update), and for P U.  Between them one
// workgroup forms P from matrices of m x m in LDS.
//
// In fp32 that would lose the small singular values, which A holds squared and
// the steps let grow by a^2 = 12 each; in fp64 they stay, with more of their bits
// than steps on X itself keep in fp32.
//
// What bounds it: three launches, and for 64 rows the 17 products of 64 x 64 on one CU
// (its fp64 matrix instructions, half of each product spared by symmetry).
#pragma once

#include "ops_common.h"

namespace nf {

// A stack of matrices in memory, in elements.
template <class T>
struct Stack {
  T* p;
  int64_t ld, stride;
};

// U of a gradient and the momentum after the step
__device__ __forceinline__ float direction(float g, float m, float momentum, bool nesterov) {
  return nesterov ? fmaf(momentum, m, g) : m;
}

constexpr int ORTH_SMALL = 64;
constexpr int SMALL_COLS = 64;         // columns that a workgroup of the Gram matrix holds at a time
constexpr int SMALL_PARTS = 16;         // at most; partial Gram matrices
constexpr int SMALL_OUT = 64;           // columns that a workgroup of the result has

typedef double doublex4 __attribute__((ext_vector_type(4)));

// MB blocks of 16 in a row; their places on and below the diagonal
template <int MB>
struct SmallShape {
  static constexpr int M = 16 * MB, BLOCKS = MB * (MB + 1) / 2, PITCH = M + 4;
};
// block k's row and column of blocks
__device__ constexpr int small_row(int k) { return k < 1 ? 0 : k < 3 ? 1 : k < 6 ? 2 : 3; }
__device__ constexpr int small_col(int k) { return k - small_row(k) * (small_row(k) + 1) / 2; }

struct SmallPlan {
  int m, n, mb, parts;
  int64_t sums, p, bytes;               // offsets in a matrix's share of the workspace
};

inline SmallPlan small_plan(int64_t rows, int64_t cols) {
  SmallPlan s{};
  s.m = (int)(rows < cols ? rows : cols);
  s.n = (int)(rows < cols ? cols : rows);
  s.mb = (s.m + 15) / 16;
  const int64_t pieces = (s.n + SMALL_COLS - 1) / SMALL_COLS;
  s.parts = (int)(pieces < SMALL_PARTS ? pieces : SMALL_PARTS);
  s.sums = 0;
  s.p = (int64_t)s.parts * (s.mb * (s.mb + 1) / 2) * 256 * 8;
  s.bytes = s.p + (int64_t)s.mb * s.mb * 256 * 8;
  return s;
}

template <class T>
struct SmallArgs {
  Stack<const T> g;
  Stack<const float> m;                 // momentum before the step, or null
  Stack<float> m_out;
  float momentum;
  bool nesterov, turned;
  char* work;
  SmallPlan p;
  int out_type;
  void* out;
  int64_t ldo, stride_o;
  const void* w;                        // or null
  int64_t ldw, stride_w;
  float keep, rate;
};

// U's values of columns j0 .. j0 + COLS - 1 (of the longer side) into LDS, zeros past
// the matrix.  FIRST: the momentum is updated on the way.  The loads of N values are
// under way together (places past the matrix read its first value instead).
template <class T, int MB, int COLS, int PITCH, bool FIRST>
__device__ __forceinline__ void small_load(const SmallArgs<T>& a, int z, int j0, float (*xs)[PITCH]) {
  constexpr int M = 16 * MB, N = M * COLS / 256 % 8 == 0 ? 8 : 4;
  static_assert(M * COLS % (N * 256) == 0, "whole rounds");
  const T* const g = a.g.p + z * a.g.stride;
  const float* const mo = a.m.p ? (FIRST ? a.m.p + z * a.m.stride : a.m_out.p + z * a.m_out.stride) : nullptr;
#pragma unroll 1
  for (int e0 = threadIdx.x; e0 < M * COLS; e0 += N * 256) {
    float u[N], m[N];
    int64_t at[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = e0 + n * 256;
      const int i = a.turned ? e % M : e / COLS, j = j0 + (a.turned ? e / M : e % COLS);
      const bool in = i < a.p.m && j < a.p.n;
      const int64_t r = in ? a.turned ? j : i : 0, k = in ? a.turned ? i : j : 0;
      u[n] = to_float(g[r * a.g.ld + k]);
      at[n] = in ? r * a.m.ld + k : -1;
      if (mo) m[n] = mo[r * a.m.ld + k];
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = e0 + n * 256;
      if (mo) {
        if constexpr (FIRST) {
          m[n] = fmaf(a.momentum, m[n], u[n]);
          if (at[n] >= 0) a.m_out.p[z * a.m_out.stride + at[n]] = m[n];
        }
        u[n] = direction(u[n], m[n], a.momentum, a.nesterov);
      }
      xs[a.turned ? e % M : e / COLS][a.turned ? e / M : e % COLS] = at[n] >= 0 ? u[n] : 0.f;
    }
  }
}

template <class T, int MB>
__global__ void __launch_bounds__(256) small_gram_kernel(const SmallArgs<T> a) {
  typedef SmallShape<MB> S;
  __shared__ float xs[S::M][SMALL_COLS + 4];
  __shared__ double red[4][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, z = blockIdx.y;
  doublex4 acc[S::BLOCKS] = {};
  for (int j0 = blockIdx.x * SMALL_COLS; j0 < a.p.n; j0 += gridDim.x * SMALL_COLS) {
    small_load<T, MB, SMALL_COLS, SMALL_COLS + 4, true>(a, z, j0, xs);
    __syncthreads();
    for (int s = wave; s < SMALL_COLS / 4; s += 4) {
      double f[MB];
#pragma unroll
      for (int b = 0; b < MB; ++b) f[b] = (double)xs[16 * b + (lane & 15)][4 * s + (lane >> 4)];
#pragma unroll
      for (int k = 0; k < S::BLOCKS; ++k)
        acc[k] = __builtin_amdgcn_mfma_f64_16x16x4f64(f[small_row(k)], f[small_col(k)], acc[k], 0, 0, 0);
    }
    __syncthreads();
  }
  double* const sums = reinterpret_cast<double*>(a.work + z * a.p.bytes + a.p.sums) + (int64_t)blockIdx.x * S::BLOCKS * 256;
#pragma unroll
  for (int k = 0; k < S::BLOCKS; ++k) {
#pragma unroll
    for (int v = 0; v < 4; ++v) red[wave][v * 64 + lane] = acc[k][v];
    __syncthreads();
    const int t = threadIdx.x;
    sums[k * 256 + t] = (red[0][t] + red[1][t]) + (red[2][t] + red[3][t]);
    __syncthreads();
  }
}

constexpr int CHAIN_WAVES = 8;

template <int MB>
__global__ void __launch_bounds__(64 * CHAIN_WAVES) small_chain_kernel(char* work, const SmallPlan p, float qa, float qb, float qc,
                                                                       int steps) {
  typedef SmallShape<MB> S;
  constexpr int SIZE = S::M * S::PITCH;
  __shared__ double lds[4 * SIZE];
  // matrices by their place in LDS
  int A = 0, Q = SIZE, R = 2 * SIZE, P = 3 * SIZE;
  __shared__ double shared_sum;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  char* const w = work + blockIdx.x * p.bytes;
  const double* const sums = reinterpret_cast<const double*>(w + p.sums);
  for (int e = tid; e < S::BLOCKS * 256; e += 64 * CHAIN_WAVES) {
    // all parts' loads under way together
    double part[SMALL_PARTS], s = 0.0;
#pragma unroll
    for (int q = 0; q < SMALL_PARTS; ++q) part[q] = q < p.parts ? sums[(int64_t)q * S::BLOCKS * 256 + e] : 0.0;
#pragma unroll
    for (int q = 0; q < SMALL_PARTS; ++q) s += part[q];
    const int k = e >> 8, l = e & 63, v = (e >> 6) & 3;
    const int i = 16 * small_row(k) + 4 * v + (l >> 4), j = 16 * small_col(k) + (l & 15);
    lds[A + i * S::PITCH + j] = s;
    lds[A + j * S::PITCH + i] = s;
  }
  __syncthreads();
  if (wave == 0) {
    const double s = wave_sum(lane < S::M ? lds[A + lane * S::PITCH + lane] : 0.0);
    if (lane == 0) shared_sum = s;
  }
  __syncthreads();
  const double trace = shared_sum;
  const double inv = trace == 0.0 ? 0.0 : trace < __builtin_inf() ? 1.0 / trace : __builtin_nan("");
  auto each = [&](auto&& f) {
#pragma unroll
    for (int e = tid; e < S::M * S::M; e += 64 * CHAIN_WAVES) f(e / S::M, e % S::M, e / S::M * S::PITCH + e % S::M);
    __syncthreads();
  };
  each([&](int, int, int o) { lds[A + o] *= inv; });
  // Products of matrices that commute and are symmetric: rows by rows, half the
  // blocks.  A block's operands are read before its first instruction, which would
  // wait for each pair otherwise; r[v] is element (4 v + lane / 16, lane % 16) of block k.
  auto form = [&](int X, int Y, int k, double (&r)[4]) {
    const double* const px = lds + X + (16 * small_row(k) + (lane & 15)) * S::PITCH + (lane >> 4);
    const double* const py = lds + Y + (16 * small_col(k) + (lane & 15)) * S::PITCH + (lane >> 4);
    double x[S::M / 4], y[S::M / 4];
#pragma unroll
    for (int s = 0; s < S::M / 4; ++s) {
      x[s] = px[4 * s];
      y[s] = py[4 * s];
    }
    __builtin_amdgcn_sched_barrier(0);
    // two sums, so that the instructions do not all wait for one another
    doublex4 c0 = {}, c1 = {};
#pragma unroll
    for (int s = 0; s < S::M / 4; s += 2) {
      c0 = __builtin_amdgcn_mfma_f64_16x16x4f64(x[s], y[s], c0, 0, 0, 0);
      c1 = __builtin_amdgcn_mfma_f64_16x16x4f64(x[s + 1], y[s + 1], c1, 0, 0, 0);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) r[v] = c0[v] + c1[v];
  };
  auto place = [&](int k, int v, int& i, int& j) {
    i = 16 * small_row(k) + 4 * v + (lane >> 4);
    j = 16 * small_col(k) + (lane & 15);
    return i * S::PITCH + j;
  };
  auto keep = [&](int C, int k, const double (&r)[4]) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      int i, j;
      lds[C + place(k, v, i, j)] = r[v];
      if (small_row(k) != small_col(k)) lds[C + j * S::PITCH + i] = r[v];
    }
  };
  constexpr int MINE = (S::BLOCKS + CHAIN_WAVES - 1) / CHAIN_WAVES;     // of P's blocks, at most
  for (int step = 0; step < steps; ++step) {
    const bool last = step + 1 == steps;
    // Q = a + b A + c A^2
    for (int k = wave; k < S::BLOCKS; k += CHAIN_WAVES) {
      double r[4];
      form(A, A, k, r);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        int i, j;
        const int o = place(k, v, i, j);
        r[v] = (double)qc * r[v] + (double)qb * lds[A + o] + (i == j ? (double)qa : 0.0);
      }
      keep(Q, k, r);
    }
    __syncthreads();
    // R = A Q and, from the second step on, P = Q P, whose old values are read until all are formed
    double mine[MINE][4];
#pragma unroll
    for (int n = 0; n < MINE; ++n) {
      const int k = CHAIN_WAVES - 1 - wave + n * CHAIN_WAVES;           // (the waves that R leaves idle first)
      if (step > 0 && k < S::BLOCKS) form(Q, P, k, mine[n]);
    }
    if (!last)
      for (int k = wave; k < S::BLOCKS; k += CHAIN_WAVES) {
        double r[4];
        form(A, Q, k, r);
        keep(R, k, r);
      }
    __syncthreads();
    if (step > 0) {
#pragma unroll
      for (int n = 0; n < MINE; ++n) {
        const int k = CHAIN_WAVES - 1 - wave + n * CHAIN_WAVES;
        if (k < S::BLOCKS) keep(P, k, mine[n]);
      }
    }
    // A = R Q
    if (!last)
      for (int k = wave; k < S::BLOCKS; k += CHAIN_WAVES) {
        double r[4];
        form(R, Q, k, r);
        keep(A, k, r);
      }
    if (step == 0) {                     // P = Q: its place takes the next step's Q
      __syncthreads();
      const int old = P;
      P = Q;
      Q = old;
    }
    __syncthreads();
  }
  const double size = sqrt(inv);
  double* const out = reinterpret_cast<double*>(w + p.p);
  each([&](int i, int j, int o) { out[i * S::M + j] = lds[P + o] * size; });
}

template <class T, int MB>
__global__ void __launch_bounds__(256) small_apply_kernel(const SmallArgs<T> a) {
  typedef SmallShape<MB> S;
  __shared__ float xs[S::M][SMALL_OUT + 16];
  __shared__ double ps[S::M * S::PITCH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, z = blockIdx.y, j0 = blockIdx.x * SMALL_OUT;
  const double* const p = reinterpret_cast<const double*>(a.work + z * a.p.bytes + a.p.p);
  // the weights before the step, on their way while the products are formed
  float w[MB][4] = {};
  auto where = [&](int b, int v, int64_t& r, int64_t& k) {
    const int down = 4 * v + (lane >> 4), across = lane & 15;
    const int i = 16 * b + (a.turned ? across : down), j = j0 + 16 * wave + (a.turned ? down : across);
    r = a.turned ? j : i;
    k = a.turned ? i : j;
    return i < a.p.m && j < a.p.n;
  };
  if (a.w) {
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        int64_t r, k;
        const int64_t at = where(b, v, r, k) ? z * a.stride_w + r * a.ldw + k : 0;
        w[b][v] = a.out_type == NF_F32 ? static_cast<const float*>(a.w)[at]
                                       : to_float(static_cast<const bf16_t*>(a.w)[at]);
      }
  }
#pragma unroll
  for (int e = threadIdx.x; e < S::M * S::M; e += 256) ps[e / S::M * S::PITCH + e % S::M] = p[e];
  small_load<T, MB, SMALL_OUT, SMALL_OUT + 16, false>(a, z, j0, xs);
  __syncthreads();
  // a wave has 16 columns; the user's rows lie along the lanes
  doublex4 acc[MB] = {};
  const int c = 16 * wave + (lane & 15), kk = lane >> 4;
#pragma unroll
  for (int s = 0; s < S::M / 4; ++s) {
    const double x = (double)xs[4 * s + kk][c];
#pragma unroll
    for (int b = 0; b < MB; ++b) {
      const double q = ps[(16 * b + (lane & 15)) * S::PITCH + 4 * s + kk];
      acc[b] = a.turned ? __builtin_amdgcn_mfma_f64_16x16x4f64(x, q, acc[b], 0, 0, 0)
                        : __builtin_amdgcn_mfma_f64_16x16x4f64(q, x, acc[b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      int64_t r, k;
      if (!where(b, v, r, k)) continue;
      float y = (float)acc[b][v];
      if (a.w) y = fmaf(-a.rate, y, a.keep * w[b][v]);
      const int64_t o = z * a.stride_o + r * a.ldo + k;
      if (a.out_type == NF_F32) static_cast<float*>(a.out)[o] = y;
      else static_cast<bf16_t*>(a.out)[o] = from_float<bf16_t>(y);
    }
}

template <class T, int MB>
hipError_t launch_small(const SmallArgs<T>& a, int64_t count, float qa, float qb, float qc, int steps, hipStream_t s) {
  hipError_t e = op_launch(small_gram_kernel<T, MB>, dim3((unsigned)a.p.parts, (unsigned)count), dim3(256), s, a);
  if (e != hipSuccess) return e;
  e = op_launch(small_chain_kernel<MB>, dim3((unsigned)count), dim3(64 * CHAIN_WAVES), s, a.work, a.p, qa, qb, qc, steps);
  if (e != hipSuccess) return e;
  return op_launch(small_apply_kernel<T, MB>, dim3((unsigned)((a.p.n + SMALL_OUT - 1) / SMALL_OUT), (unsigned)count), dim3(256), s, a);
}

}  // namespace nf
