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
// What bounds it: three launches of 3.5 us and more, and the 17 products of m x m on one
// CU.  Measured, launches included (us; Gram matrix, chain, result):
//   12 x 784 fp32   3.5   6.7  3.6      4096 x 12 bf16, two    4.1   9.0  3.7
//   30 x 784        5.2  10.5  4.0      4096 x 30              6.8  12.6  4.3
//   64 x 784        7.1  38.8  4.7      4096 x 64             10.8  44.2  6.0
// (20 us of the 38.8 are what its fp64 matrix instructions take, half of each product
// spared by symmetry.)  16 partial Gram matrices at most: 16.9 and 39.5 for the last, 64: 8.8 and
// 53.1.  A result of 64 columns a workgroup, with P in LDS: 12.9 instead of 4.7.
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
constexpr int SMALL_PARTS = 32;         // at most; partial Gram matrices
constexpr int SMALL_OUT = 16;           // columns of the result that a workgroup forms at a time

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
template <class T, int MB, int COLS, int PITCH, int THREADS, bool FIRST>
__device__ __forceinline__ void small_load(const SmallArgs<T>& a, int z, int j0, float (*xs)[PITCH]) {
  constexpr int M = 16 * MB, N = M * COLS / THREADS % 8 == 0 ? 8 : 4;
  static_assert(M * COLS % (N * THREADS) == 0, "whole rounds");
  const T* const g = a.g.p + z * a.g.stride;
  const float* const mo = a.m.p ? (FIRST ? a.m.p + z * a.m.stride : a.m_out.p + z * a.m_out.stride) : nullptr;
#pragma unroll 1
  for (int e0 = threadIdx.x; e0 < M * COLS; e0 += N * THREADS) {
    float u[N], m[N];
    int64_t at[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = e0 + n * THREADS;
      const int i = a.turned ? e % M : e / COLS, j = j0 + (a.turned ? e / M : e % COLS);
      const bool in = i < a.p.m && j < a.p.n;
      const int64_t r = in ? a.turned ? j : i : 0, k = in ? a.turned ? i : j : 0;
      u[n] = to_float(g[r * a.g.ld + k]);
      at[n] = in ? r * a.m.ld + k : -1;
      if (mo) m[n] = mo[r * a.m.ld + k];
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int e = e0 + n * THREADS;
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
  __shared__ double red[4][S::BLOCKS * 256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, z = blockIdx.y;
  doublex4 acc[S::BLOCKS] = {};
  for (int j0 = blockIdx.x * SMALL_COLS; j0 < a.p.n; j0 += gridDim.x * SMALL_COLS) {
    small_load<T, MB, SMALL_COLS, SMALL_COLS + 4, 256, true>(a, z, j0, xs);
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
  for (int k = 0; k < S::BLOCKS; ++k)
#pragma unroll
    for (int v = 0; v < 4; ++v) red[wave][k * 256 + v * 64 + lane] = acc[k][v];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < S::BLOCKS; ++k) {
    const int t = k * 256 + threadIdx.x;
    sums[t] = (red[0][t] + red[1][t]) + (red[2][t] + red[3][t]);
  }
}

// A symmetric matrix in LDS, by blocks of 16 x 16 as a product's registers have them:
// register v of lane l is element (4 v + l / 16, l % 16) of the block.  Read with its rows
// and columns exchanged, that is also what a lane holds of either operand of a matrix
// instruction, so a product's blocks are the next one's operands as they stand: two
// 16-byte reads a block, four values of k.  (A lane's pairs of registers are neighbours;
// the lanes' quarters lie 64 bytes apart, so that a transposed block's writes too go to all banks.)
constexpr int BLOCK_PLANE = 4 * (16 * 2 + 8), BLOCK_LDS = 2 * BLOCK_PLANE;      // doubles
__device__ __forceinline__ int block_at(int v, int l) {
  return (v >> 1) * BLOCK_PLANE + (l >> 4) * (16 * 2 + 8) + (l & 15) * 2 + (v & 1);
}

constexpr int chain_waves(int mb) { return mb == 1 ? 2 : 8; }

template <int MB>
__global__ void __launch_bounds__(64 * chain_waves(MB)) small_chain_kernel(char* work, const SmallPlan p, float qa, float qb,
                                                                           float qc, int steps) {
  typedef SmallShape<MB> S;
  constexpr int NW = chain_waves(MB), SIZE = MB * MB * BLOCK_LDS;
  // Products of matrices that commute are symmetric: the blocks on and below the
  // diagonal are formed and stored twice, or up to 32 rows, where waves would idle, all.
  constexpr bool HALF = MB > 2;
  constexpr int BLOCKS = HALF ? S::BLOCKS : MB * MB;
  __shared__ __align__(16) double lds[4 * SIZE];
  double *A = lds, *Q = lds + SIZE, *R = lds + 2 * SIZE, *P = lds + 3 * SIZE;
  double* const diagonal = R;           // before the first product
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  char* const w = work + blockIdx.x * p.bytes;
  const double* const sums = reinterpret_cast<const double*>(w + p.sums);
  auto block_row = [](int k) { return HALF ? small_row(k) : k / MB; };
  auto block_col = [](int k) { return HALF ? small_col(k) : k % MB; };
  // element (v, lane) of the block (i, j) with j <= i, and of its transposed
  auto place = [&](double* X, int i, int j, int v, double x) {
    X[(i * MB + j) * BLOCK_LDS + block_at(v, lane)] = x;
    if (i != j) X[(j * MB + i) * BLOCK_LDS + block_at((lane & 15) >> 2, (lane & 3) * 16 + 4 * v + (lane >> 4))] = x;
  };

  constexpr int ROUNDS = (S::BLOCKS * 4 + NW - 1) / NW;
  double part[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int e = tid + r * 64 * NW;
    double s = 0.0;
    // the loads of 16 parts are under way together
    for (int q0 = 0; q0 < p.parts; q0 += 16) {
      double x[16];
#pragma unroll
      for (int q = 0; q < 16; ++q)
        x[q] = q0 + q < p.parts && e < S::BLOCKS * 256 ? sums[(int64_t)(q0 + q) * S::BLOCKS * 256 + e] : 0.0;
#pragma unroll
      for (int q = 0; q < 16; ++q) s += x[q];
    }
    part[r] = s;
    const int k = e >> 8, v = (e >> 6) & 3, i = 4 * v + (lane >> 4);
    if (e < S::BLOCKS * 256 && small_row(k) == small_col(k) && i == (lane & 15)) diagonal[16 * small_row(k) + i] = s;
  }
  __syncthreads();
  const double trace = wave_sum(lane < S::M ? diagonal[lane] : 0.0);
  const double inv = trace == 0.0 ? 0.0 : trace < __builtin_inf() ? 1.0 / trace : __builtin_nan("");
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int e = tid + r * 64 * NW, k = e >> 8;
    if (e < S::BLOCKS * 256) place(A, small_row(k), small_col(k), (e >> 6) & 3, part[r] * inv);
  }
  __syncthreads();

  // r[v]: register v of block k of X Y
  auto form = [&](const double* X, const double* Y, int k, double (&r)[4]) {
    const double* const px = X + block_row(k) * BLOCK_LDS;
    const double* const py = Y + block_col(k) * BLOCK_LDS;
    double x[MB][4], y[MB][4];
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        x[b][v] = px[b * MB * BLOCK_LDS + block_at(v, lane)];
        y[b][v] = py[b * MB * BLOCK_LDS + block_at(v, lane)];
      }
    // two sums, so that the instructions do not all wait for one another
    doublex4 c0 = {}, c1 = {};
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
      for (int v = 0; v < 4; v += 2) {
        c0 = __builtin_amdgcn_mfma_f64_16x16x4f64(x[b][v], y[b][v], c0, 0, 0, 0);
        c1 = __builtin_amdgcn_mfma_f64_16x16x4f64(x[b][v + 1], y[b][v + 1], c1, 0, 0, 0);
      }
#pragma unroll
    for (int v = 0; v < 4; ++v) r[v] = c0[v] + c1[v];
  };
  auto keep = [&](double* C, int k, const double (&r)[4]) {
    if constexpr (HALF) {
#pragma unroll
      for (int v = 0; v < 4; ++v) place(C, block_row(k), block_col(k), v, r[v]);
    } else {
#pragma unroll
      for (int v = 0; v < 4; ++v) C[k * BLOCK_LDS + block_at(v, lane)] = r[v];
    }
  };
  constexpr int MINE = (BLOCKS + NW - 1) / NW;            // of P's blocks, at most
  for (int step = 0; step < steps; ++step) {
    const bool last = step + 1 == steps;
    // Q = a + b A + c A^2
    for (int k = wave; k < BLOCKS; k += NW) {
      double r[4];
      form(A, A, k, r);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const bool on = block_row(k) == block_col(k) && 4 * v + (lane >> 4) == (lane & 15);
        r[v] = (double)qc * r[v] + (double)qb * A[(block_row(k) * MB + block_col(k)) * BLOCK_LDS + block_at(v, lane)] +
               (on ? (double)qa : 0.0);
      }
      keep(Q, k, r);
    }
    __syncthreads();
    // R = A Q and, from the second step on, P = Q P, whose old values are read until all are formed
    double mine[MINE][4];
#pragma unroll
    for (int n = 0; n < MINE; ++n) {
      const int k = NW - 1 - wave + n * NW;               // (the waves that R leaves idle first)
      if (step > 0 && k < BLOCKS) form(Q, P, k, mine[n]);
    }
    if (!last)
      for (int k = wave; k < BLOCKS; k += NW) {
        double r[4];
        form(A, Q, k, r);
        keep(R, k, r);
      }
    __syncthreads();
    if (step > 0) {
#pragma unroll
      for (int n = 0; n < MINE; ++n) {
        const int k = NW - 1 - wave + n * NW;
        if (k < BLOCKS) keep(P, k, mine[n]);
      }
    }
    // A = R Q
    if (!last)
      for (int k = wave; k < BLOCKS; k += NW) {
        double r[4];
        form(R, Q, k, r);
        keep(A, k, r);
      }
    __syncthreads();
    if (step == 0) {                     // P = Q: its place takes the next step's Q
      double* const old = P;
      P = Q;
      Q = old;
    }
  }
  // P's blocks as they lie in LDS, without the gaps
  const double size = sqrt(inv);
  double* const out = reinterpret_cast<double*>(w + p.p);
#pragma unroll
  for (int e = tid; e < MB * MB * 256; e += 64 * NW) {
    const int k = e >> 8, h = (e >> 7) & 1, l = (e >> 1) & 63;
    out[e] = P[k * BLOCK_LDS + block_at(2 * h + (e & 1), l)] * size;
  }
}

constexpr int APPLY_BLOCKS = 1024;       // at most, of a matrix

// 16 columns a time and a block of 16 rows of the result a wave, which holds P's rows.
template <class T, int MB>
__global__ void __launch_bounds__(64 * MB) small_apply_kernel(const SmallArgs<T> a) {
  typedef SmallShape<MB> S;
  __shared__ float xs[S::M][SMALL_OUT + 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, z = blockIdx.y;
  const double* const p = reinterpret_cast<const double*>(a.work + z * a.p.bytes + a.p.p);
  double q[MB][4];                      // (k, row) of block (b, wave)
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int v = 0; v < 4; ++v) q[b][v] = p[(b * MB + wave) * 256 + (v >> 1) * 128 + lane * 2 + (v & 1)];
#pragma unroll 1
  for (int j0 = blockIdx.x * SMALL_OUT; j0 < a.p.n; j0 += gridDim.x * SMALL_OUT) {
    // the user's rows lie along the lanes
    int64_t at[4], from[4];
    bool in[4];
    float w[4] = {};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int down = 4 * v + (lane >> 4), across = lane & 15;
      const int i = 16 * wave + (a.turned ? across : down), j = j0 + (a.turned ? down : across);
      const int64_t r = a.turned ? j : i, k = a.turned ? i : j;
      in[v] = i < a.p.m && j < a.p.n;
      at[v] = r * a.ldo + k;
      from[v] = in[v] ? z * a.stride_w + r * a.ldw + k : 0;
    }
    // the weights before the step, on their way while the products are formed
    auto weights = [&](const auto* x) {
#pragma unroll
      for (int v = 0; v < 4; ++v) w[v] = to_float(x[from[v]]);
    };
    if (a.w) {
      if (a.out_type == NF_F32) weights(static_cast<const float*>(a.w));
      else weights(static_cast<const bf16_t*>(a.w));
    }
    small_load<T, MB, SMALL_OUT, SMALL_OUT + 2, 64 * MB, false>(a, z, j0, xs);
    __syncthreads();
    doublex4 c0 = {}, c1 = {};
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const double x = (double)xs[16 * b + 4 * v + (lane >> 4)][lane & 15];
        doublex4& c = v & 1 ? c1 : c0;
        c = a.turned ? __builtin_amdgcn_mfma_f64_16x16x4f64(x, q[b][v], c, 0, 0, 0)
                     : __builtin_amdgcn_mfma_f64_16x16x4f64(q[b][v], x, c, 0, 0, 0);
      }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      if (!in[v]) continue;
      float y = (float)(c0[v] + c1[v]);
      if (a.w) y = fmaf(-a.rate, y, a.keep * w[v]);
      const int64_t o = z * a.stride_o + at[v];
      if (a.out_type == NF_F32) static_cast<float*>(a.out)[o] = y;
      else static_cast<bf16_t*>(a.out)[o] = from_float<bf16_t>(y);
    }
  }
}

template <class T, int MB>
hipError_t launch_small(const SmallArgs<T>& a, int64_t count, float qa, float qb, float qc, int steps, hipStream_t s) {
  hipError_t e = op_launch(small_gram_kernel<T, MB>, dim3((unsigned)a.p.parts, (unsigned)count), dim3(256), s, a);
  if (e != hipSuccess) return e;
  e = op_launch(small_chain_kernel<MB>, dim3((unsigned)count), dim3(64 * chain_waves(MB)), s, a.work, a.p, qa, qb, qc, steps);
  if (e != hipSuccess) return e;
  const int pieces = (a.p.n + SMALL_OUT - 1) / SMALL_OUT;
  return op_launch(small_apply_kernel<T, MB>, dim3((unsigned)(pieces < APPLY_BLOCKS ? pieces : APPLY_BLOCKS), (unsigned)count),
                   dim3(64 * MB), s, a);
}

}  // namespace nf
