// Orthogonalised updates of weight matrices by Newton-Schulz products.
//
// X = U / |U|_F (transposed where it has more rows than columns, so that m <= n),
// then NF_ORTH_STEPS times
//   A = X X^T,  B = b A + c A^2,  X = a X + B X,  (a, b, c) = (3.4445, -4.7750, 2.0315),
// a quintic in the singular values that takes those above about 1e-3 near 1.
// They stay below 1.21, so the entries of X, A and B stay below 1.21, 1.47 and
// 2.81, and all are held in f16 times 2^14: no value is out of range, and what is
// below f16's normal range is below 2^-28.
//
// fp32 weights: every matrix is kept in pairs of f16 parts (22 bits) and a product
// formed of three (rows_mm.h).  Singular values below the largest's 1e-3 grow by
// a^5 = 485 with all noise beside them, so fewer bits than fp32's show there:
// relative errors of the result against 64 bits, sums of 64 outer products of 512,
// 5e-6 in pairs, 9e-6 in fp32, 2e-2 in one f16.
//
// bf16 weights: one f16 a value in the products, X itself in fp32 (aX, the only
// part that noise beside small singular values is carried on by).  The diagonals
// of A and B are kept in fp32 and left out of the products: near the end A is
// nearly diagonal, and its rounding would be most of the error (1.0 - 1.3e-3 for
// 1.4 - 2.8e-3 with them, where bf16's own rounding is 1.7e-3).
//
// A and B are symmetric: their tiles on and below the diagonal are formed and
// stored twice.  Both X and X^T are kept, so that all products are of rows by
// rows.
#include <cmath>

#include "rows_mm.h"

namespace nf {
namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float UNIT = 16384.f, PER_UNIT = 1.f / UNIT;
constexpr int SUM_BLOCKS = 256;        // at most; partial sums of a matrix

// where element (r, c) of an operand lies; its second part 64 bytes on
template <int KIND>
__device__ __forceinline__ int64_t place(int64_t r, int c, int64_t pitch) {
  return KIND == MM_PARTS2 ? r * pitch + (c / PARTS2_GROUP) * 128 + (c % PARTS2_GROUP) * 2 : r * pitch + c * 2;
}
template <int KIND>
__device__ __forceinline__ void put_value(char* p, int64_t at, float x) {
  const _Float16 h = (_Float16)x;
  *reinterpret_cast<_Float16*>(p + at) = h;
  if constexpr (KIND == MM_PARTS2) *reinterpret_cast<_Float16*>(p + at + 64) = (_Float16)(x - (float)h);
}
template <int KIND>
__device__ __forceinline__ void put_four(char* p, int64_t at, const float (&x)[4]) {
  f16x4 h, l;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = (_Float16)x[i];
    l[i] = (_Float16)(x[i] - (float)h[i]);
  }
  *reinterpret_cast<f16x4*>(p + at) = h;
  if constexpr (KIND == MM_PARTS2) *reinterpret_cast<f16x4*>(p + at + 64) = l;
}
template <int KIND>
__device__ __forceinline__ float get_value(const char* p, int64_t at) {
  float x = (float)*reinterpret_cast<const _Float16*>(p + at);
  if constexpr (KIND == MM_PARTS2) x += (float)*reinterpret_cast<const _Float16*>(p + at + 64);
  return x;
}

// The buffers of one matrix (offsets in its share of the workspace; pitches in
// bytes, whole stages).
struct OrthPlan {
  int m, n;                   // shorter and longer side
  int64_t px, pt, pm;         // pitches of rows of n, of rows of m, of the fp32 X
  int64_t x, xt[2], a, b, xm, da, db, sums;
  int64_t bytes;              // of one matrix
};

int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

OrthPlan orth_plan(bool parts, int64_t rows, int64_t cols) {
  OrthPlan p{};
  p.m = (int)(rows < cols ? rows : cols);
  p.n = (int)(rows < cols ? cols : rows);
  p.px = parts ? up(p.n, 32) * 4 : up(p.n, 64) * 2;
  p.pt = parts ? up(p.m, 32) * 4 : up(p.m, 64) * 2;
  p.pm = parts ? 0 : up(p.n, 64) * 4;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t r = at;
    at += up(bytes, 256);
    return r;
  };
  p.sums = take(SUM_BLOCKS * 8);
  p.x = take(p.m * p.px);
  p.xt[0] = take(p.n * p.pt);
  p.xt[1] = take(p.n * p.pt);
  p.a = take(p.m * p.pt);
  p.b = take(p.m * p.pt);
  p.xm = take(p.m * p.pm);
  p.da = take(parts ? 0 : p.m * 4);
  p.db = take(parts ? 0 : p.m * 4);
  p.bytes = at;
  return p;
}

// A stack of matrices in memory, in elements.
template <class T>
struct Stack {
  T* p;
  int64_t ld, stride;
};

// ---- U, its momentum and the sum of its squares ------------------------------
template <class T>
struct SumArgs {
  Stack<const T> g;
  Stack<const float> m;       // momentum before the step, or null
  Stack<float> m_out;
  float momentum;
  bool nesterov;
  int64_t rows, cols;
  char* work;
  int64_t share, sums;        // bytes of a matrix's share, offset of its sums
};

__device__ __forceinline__ float direction(float g, float m, float momentum, bool nesterov) {
  return nesterov ? fmaf(momentum, m, g) : m;
}

template <class T>
__global__ void __launch_bounds__(256) orth_sum_kernel(const SumArgs<T> a) {
  constexpr int E = Vec16<T>::N;
  const int z = blockIdx.y;
  const T* const g = a.g.p + (int64_t)z * a.g.stride;
  const float* const m = a.m.p ? a.m.p + (int64_t)z * a.m.stride : nullptr;
  float* const mo = a.m.p ? a.m_out.p + (int64_t)z * a.m_out.stride : nullptr;
  const int64_t vecs = (a.cols + E - 1) / E, total = a.rows * vecs;
  double sum = 0.0;
  auto add = [&](float u) { sum = fma((double)u, (double)u, sum); };
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = a.rows == 1 ? 0 : i / vecs;
    const int64_t c = (i - r * vecs) * E;
    if (c + E <= a.cols) {
      const Vec16<T> v = load16(g + r * a.g.ld + c);
      if (m) {
        float x[E];
        __builtin_memcpy(x, m + r * a.m.ld + c, E * 4);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float gv = to_float(v.v[e]);
          x[e] = fmaf(a.momentum, x[e], gv);
          add(direction(gv, x[e], a.momentum, a.nesterov));
        }
        __builtin_memcpy(mo + r * a.m_out.ld + c, x, E * 4);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) add(to_float(v.v[e]));
      }
    } else {
      for (int64_t k = c; k < a.cols; ++k) {
        const float gv = to_float(g[r * a.g.ld + k]);
        if (m) {
          const float x = fmaf(a.momentum, m[r * a.m.ld + k], gv);
          mo[r * a.m_out.ld + k] = x;
          add(direction(gv, x, a.momentum, a.nesterov));
        } else {
          add(gv);
        }
      }
    }
  }
  __shared__ double part[4];
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0)
    reinterpret_cast<double*>(a.work + z * a.share + a.sums)[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// ---- X and X^T ---------------------------------------------------------------
template <class T>
struct FillArgs {
  Stack<const T> g;
  Stack<const float> m;       // momentum after the step, or null
  float momentum;
  bool nesterov;
  bool turned;                // the user's matrix is X^T
  int blocks;                 // partial sums
  char* work;
  OrthPlan p;
};

// a tile of 64 x 64 of X a workgroup
template <class T, int KIND>
__global__ void __launch_bounds__(256) orth_fill_kernel(const FillArgs<T> a) {
  const OrthPlan& p = a.p;
  char* const w = a.work + blockIdx.z * p.bytes;
  __shared__ float tile[64][65];
  __shared__ double part[4];
  const int tid = threadIdx.x;
  double s = tid < a.blocks ? reinterpret_cast<const double*>(w + p.sums)[tid] : 0.0;
  s = wave_sum(s);
  if ((tid & 63) == 0) part[tid >> 6] = s;
  __syncthreads();
  const double sum = (part[0] + part[1]) + (part[2] + part[3]);
  // a matrix of zeros stays one; one that is not finite becomes NaN throughout
  const double inv = sum == 0.0 ? 0.0 : sum < __builtin_inf() ? (double)UNIT / sqrt(sum) : __builtin_nan("");
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
  const T* const g = a.g.p + (int64_t)blockIdx.z * a.g.stride;
  const float* const mom = a.m.p ? a.m.p + (int64_t)blockIdx.z * a.m.stride : nullptr;
  for (int e = tid; e < 64 * 64; e += 256) {
    // lanes along the user's rows
    const int c = e & 63, r = e >> 6;
    const int i = i0 + (a.turned ? c : r), j = j0 + (a.turned ? r : c);
    float v = 0.f;
    if (i < p.m && j < p.n) {
      const int64_t ur = a.turned ? j : i, uc = a.turned ? i : j;
      float u = to_float(g[ur * a.g.ld + uc]);
      if (mom) u = direction(u, mom[ur * a.m.ld + uc], a.momentum, a.nesterov);
      v = (float)((double)u * inv);
      if (inv != inv) v = __builtin_nanf("");
    }
    if (a.turned) tile[c][r] = v;
    else tile[r][c] = v;
  }
  __syncthreads();
  const int nx = (int)(p.px / (KIND == MM_PARTS2 ? 4 : 2)), nt = (int)(p.pt / (KIND == MM_PARTS2 ? 4 : 2));
  for (int e = tid; e < 64 * 16; e += 256) {
    const int r = e >> 4, c = (e & 15) * 4;
    if (i0 + r < p.m && j0 + c < nx) {
      const float x[4] = {tile[r][c], tile[r][c + 1], tile[r][c + 2], tile[r][c + 3]};
      put_four<KIND>(w + p.x, place<KIND>(i0 + r, j0 + c, p.px), x);
      if constexpr (KIND == MM_F16)
        *reinterpret_cast<float4*>(w + p.xm + (i0 + r) * p.pm + (j0 + c) * 4) = make_float4(x[0], x[1], x[2], x[3]);
    }
    if (j0 + r < p.n && i0 + c < nt) {
      const float x[4] = {tile[c][r], tile[c + 1][r], tile[c + 2][r], tile[c + 3][r]};
      put_four<KIND>(w + p.xt[0], place<KIND>(j0 + r, i0 + c, p.pt), x);
    }
  }
}

// ---- the products -------------------------------------------------------------
enum OrthProduct { PROD_GRAM, PROD_POLY, PROD_STEP, PROD_LAST };

struct MmArgs {
  OrthPlan p;
  char* work;
  int from;                   // which X^T this step reads
  int total, mt, nt;          // tiles
  // PROD_LAST: the user's result and, for an update, the weights before it
  bool turned;
  int out_type;               // an nf_dtype
  void* out;
  int64_t ldo, stride_o;
  const void* w;              // or null
  int64_t ldw, stride_w;
  float keep, rate;           // w' = keep w - rate X
};

__device__ __forceinline__ void put_result(const MmArgs& a, int z, int64_t r, int64_t c, float x) {
  const int64_t o = z * a.stride_o + r * a.ldo + c;
  if (a.w) {
    const int64_t i = z * a.stride_w + r * a.ldw + c;
    const float w = a.out_type == NF_F32 ? static_cast<const float*>(a.w)[i]
                                         : to_float(static_cast<const bf16_t*>(a.w)[i]);
    x = fmaf(-a.rate, x, a.keep * w);
  }
  if (a.out_type == NF_F32)
    static_cast<float*>(a.out)[o] = x;
  else
    static_cast<bf16_t*>(a.out)[o] = from_float<bf16_t>(x);
}

template <int KIND, int PROD, int BM, int BN, int WM, int WN, int NS, int OCC>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64, OCC) orth_mm_kernel(const MmArgs a) {
  typedef MmTile<KIND, BM, BN, WM, WN, NS> Tile;
  __shared__ __attribute__((aligned(1024))) char lds[Tile::LDS];
  const OrthPlan& p = a.p;
  const int z = blockIdx.y;
  char* const w = a.work + z * p.bytes;
  int bx, by;
  if constexpr (PROD == PROD_GRAM || PROD == PROD_POLY) {
    static_assert(BM == BN, "square tiles");
    if (!mm_place_lower(a.total, bx, by)) return;
  } else {
    if (!mm_place(a.total, a.mt, a.nt, bx, by)) return;
  }
  const int m0 = __builtin_amdgcn_readfirstlane(bx * BM), n0 = __builtin_amdgcn_readfirstlane(by * BN);
  const MmRows X{w + p.x, p.px, p.m}, XT{w + p.xt[a.from], p.pt, p.n}, A{w + p.a, p.pt, p.m}, B{w + p.b, p.pt, p.m};
  typename Tile::Acc acc[Tile::TM][Tile::TN];
  if constexpr (PROD == PROD_GRAM)
    Tile::run(X, X, (int)p.px, m0, n0, lds, acc);
  else if constexpr (PROD == PROD_POLY)
    Tile::run(A, A, (int)p.pt, m0, n0, lds, acc);
  else if (PROD == PROD_LAST && a.turned)
    Tile::run(XT, B, (int)p.pt, m0, n0, lds, acc);
  else
    Tile::run(B, XT, (int)p.pt, m0, n0, lds, acc);

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
  const int per = KIND == MM_PARTS2 ? 4 : 2;
  const int wide_m = (int)(p.pt / per), wide_n = (int)(p.px / per);   // with the zeros up to the pitch
  float* const da = reinterpret_cast<float*>(w + p.da);
  float* const db = reinterpret_cast<float*>(w + p.db);
#pragma unroll
  for (int ti = 0; ti < Tile::TM; ++ti)
#pragma unroll
    for (int tj = 0; tj < Tile::TN; ++tj) {
      const int j = n0 + wn + tj * 32 + (lane & 31);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int i = m0 + wm + ti * 32 + 8 * q + 4 * (lane >> 5);    // the first of four rows
        float v[4];
        if constexpr (PROD == PROD_GRAM || PROD == PROD_POLY) {
          char* const C = w + (PROD == PROD_GRAM ? p.a : p.b);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float x = acc[ti][tj][4 * q + c] * PER_UNIT;
            const bool in = i + c < p.m && j < p.m;
            if constexpr (PROD == PROD_POLY) {
              const float e = in ? get_value<KIND>(w + p.a, place<KIND>(i + c, j, p.pt)) : 0.f;
              if constexpr (KIND == MM_F16) {
                const float di = in ? da[i + c] : 0.f, dj = in ? da[j] : 0.f;
                // (D + F)^2, F without a diagonal
                x = i + c == j ? fmaf(di * PER_UNIT, di, x) : fmaf((di + dj) * PER_UNIT, e, x);
                x = fmaf(NS_C, x, NS_B * (i + c == j ? di : e));
              } else {
                x = fmaf(NS_C, x, NS_B * e);
              }
            }
            if constexpr (KIND == MM_F16) {
              if (i + c == j) {
                if (in) (PROD == PROD_GRAM ? da : db)[j] = x;
                x = 0.f;
              }
            }
            v[c] = in ? x : 0.f;
            if (i + c < p.m && j < wide_m) put_value<KIND>(C, place<KIND>(i + c, j, p.pt), v[c]);
          }
          if (bx != by && j < p.m && i < wide_m) put_four<KIND>(C, place<KIND>(j, i, p.pt), v);
        } else if (PROD == PROD_LAST && a.turned) {
          // rows of X^T down, rows of B across
          float4 four = make_float4(0.f, 0.f, 0.f, 0.f);
          if constexpr (KIND == MM_F16)
            if (j < p.m && i < wide_n) four = *reinterpret_cast<const float4*>(w + p.xm + j * p.pm + (int64_t)i * 4);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (i + c >= p.n || j >= p.m) continue;
            float x;
            if constexpr (KIND == MM_PARTS2) {
              const float e = get_value<KIND>(w + p.xt[a.from], place<KIND>(i + c, j, p.pt));
              x = fmaf(NS_A, e, acc[ti][tj][4 * q + c] * PER_UNIT);
            } else {
              const float e = c == 0 ? four.x : c == 1 ? four.y : c == 2 ? four.z : four.w;
              x = fmaf(NS_A, e, fmaf(db[j] * PER_UNIT, (float)(_Float16)e, acc[ti][tj][4 * q + c] * PER_UNIT));
            }
            put_result(a, z, i + c, j, x * PER_UNIT);
          }
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const bool in = i + c < p.m && j < p.n;
            float x = 0.f;
            if (in) {
              if constexpr (KIND == MM_PARTS2) {
                const float e = get_value<KIND>(w + p.x, place<KIND>(i + c, j, p.px));
                x = fmaf(NS_A, e, acc[ti][tj][4 * q + c] * PER_UNIT);
              } else {
                float* const xm = reinterpret_cast<float*>(w + p.xm + (i + c) * p.pm) + j;
                const float e = *xm;
                x = fmaf(NS_A, e, fmaf(db[i + c] * PER_UNIT, (float)(_Float16)e, acc[ti][tj][4 * q + c] * PER_UNIT));
                if constexpr (PROD == PROD_STEP) *xm = x;
              }
              if constexpr (PROD == PROD_STEP)
                put_value<KIND>(w + p.x, place<KIND>(i + c, j, p.px), x);
              else
                put_result(a, z, i + c, j, x * PER_UNIT);
            }
            v[c] = x;
          }
          if constexpr (PROD == PROD_STEP)
            if (j < p.n && i < wide_m) put_four<KIND>(w + p.xt[a.from ^ 1], place<KIND>(j, i, p.pt), v);
        }
      }
    }
}

template <int KIND, int PROD, int BM, int WM, int WN, int NS, int OCC>
hipError_t launch_tile(MmArgs a, int64_t count, hipStream_t s) {
  const int rows = PROD == PROD_LAST && a.turned ? a.p.n : a.p.m;
  const int cols = PROD == PROD_LAST && a.turned ? a.p.m : PROD == PROD_STEP || PROD == PROD_LAST ? a.p.n : a.p.m;
  a.mt = (rows + BM - 1) / BM;
  a.nt = (cols + BM - 1) / BM;
  a.total = PROD == PROD_GRAM || PROD == PROD_POLY ? a.mt * (a.mt + 1) / 2 : a.mt * a.nt;
  return launch_k(orth_mm_kernel<KIND, PROD, BM, BM, WM, WN, NS, OCC>, dim3(mm_grid(a.total), (unsigned)count),
                  dim3((BM / WM) * (BM / WN) * 64), 0, s, a);
}

template <int KIND, int PROD>
hipError_t launch_product(const MmArgs& a, int64_t count, int units, hipStream_t s) {
  const int64_t m = a.p.m, n = PROD == PROD_GRAM || PROD == PROD_POLY ? a.p.m : a.p.n;
  auto tiles = [&](int64_t b) { return count * ((m + b - 1) / b) * ((n + b - 1) / b); };
  if (tiles(256) >= units) return launch_tile<KIND, PROD, 256, 128, 64, 2, 2>(a, count, s);
  if (tiles(128) >= units) return launch_tile<KIND, PROD, 128, 64, 64, 2, 2>(a, count, s);
  return launch_tile<KIND, PROD, 64, 32, 32, 3, 2>(a, count, s);
}

struct OrthCall {
  int64_t count, rows, cols;
  int g_type, out_type;
  const void* g;
  int64_t ldg, stride_g;
  const float* m;             // or null: no momentum, no weights
  float* m_out;
  float momentum;
  bool nesterov;
  const void* w;
  float keep, rate;
  void* out;
  int64_t ldo, stride_o;
  void* work;
};

template <class T, int KIND>
hipError_t orth_run(const OrthCall& c, int units, hipStream_t s) {
  const OrthPlan p = orth_plan(KIND == MM_PARTS2, c.rows, c.cols);
  char* const work = static_cast<char*>(c.work);
  const int64_t ldm = c.cols, stride_m = c.rows * c.cols;
  SumArgs<T> u{};
  u.g = {static_cast<const T*>(c.g), c.ldg, c.stride_g};
  u.m = {c.m, ldm, stride_m};
  u.m_out = {c.m_out, ldm, stride_m};
  u.momentum = c.momentum;
  u.nesterov = c.nesterov;
  u.rows = c.rows;
  u.cols = c.cols;
  if (c.ldg == c.cols) {       // rows without gaps are one long row
    u.rows = 1;
    u.cols = c.rows * c.cols;
  }
  u.work = work;
  u.share = p.bytes;
  u.sums = p.sums;
  // 2048 values a workgroup and more, and enough workgroups for the card
  const int64_t want = (c.rows * c.cols + 2047) / 2048;
  const int blocks = (int)(want < SUM_BLOCKS ? want : SUM_BLOCKS);
  hipError_t e = launch_k(orth_sum_kernel<T>, dim3((unsigned)blocks, (unsigned)c.count), dim3(256), 0, s, u);
  if (e != hipSuccess) return e;
  FillArgs<T> f{};
  f.g = u.g;
  f.m = {c.m_out, ldm, stride_m};
  f.momentum = c.momentum;
  f.nesterov = c.nesterov;
  f.turned = c.rows > c.cols;
  f.blocks = blocks;
  f.work = work;
  f.p = p;
  e = launch_k(orth_fill_kernel<T, KIND>, dim3((unsigned)((p.n + 63) / 64), (unsigned)((p.m + 63) / 64), (unsigned)c.count),
               dim3(256), 0, s, f);
  if (e != hipSuccess) return e;
  MmArgs a{};
  a.p = p;
  a.work = work;
  a.turned = f.turned;
  a.out_type = c.out_type;
  a.out = c.out;
  a.ldo = c.ldo;
  a.stride_o = c.stride_o;
  a.w = c.w;
  a.ldw = ldm;
  a.stride_w = stride_m;
  a.keep = c.keep;
  a.rate = c.rate;
  for (int k = 0; k < NF_ORTH_STEPS; ++k) {
    a.from = k & 1;
    if ((e = launch_product<KIND, PROD_GRAM>(a, c.count, units, s)) != hipSuccess) return e;
    if ((e = launch_product<KIND, PROD_POLY>(a, c.count, units, s)) != hipSuccess) return e;
    e = k + 1 < NF_ORTH_STEPS ? launch_product<KIND, PROD_STEP>(a, c.count, units, s)
                              : launch_product<KIND, PROD_LAST>(a, c.count, units, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

nf_status check_stack(const char* what, const void* p, int64_t elem, int64_t rows, int64_t cols, int64_t ld) {
  if (!p) return op_fail(NF_EINVAL, "NULL %s", what);
  if (!op_aligned(p, (uintptr_t)elem)) return op_fail(NF_EINVAL, "%s is not aligned to its elements", what);
  if (ld < cols) return op_fail(NF_ESHAPE, "%s: the row pitch is smaller than the columns", what);
  (void)rows;
  return NF_OK;
}

nf_status check_sizes(int64_t count, int64_t rows, int64_t cols) {
  if (count < 0 || rows < 1 || cols < 1) return op_fail(NF_EINVAL, "count must be at least 0, rows and columns at least 1");
  if (rows > NF_ORTH_MAX || cols > NF_ORTH_MAX || count > 65535)
    return op_fail(NF_ESHAPE, "at most 65535 matrices of %d rows and columns", NF_ORTH_MAX);
  return NF_OK;
}

nf_status check_work(const void* work, int64_t have, int64_t need) {
  if (!work) return op_fail(NF_EINVAL, "NULL workspace");
  if (!op_aligned(work, 256)) return op_fail(NF_EINVAL, "the workspace is not aligned to 256 bytes");
  if (have < need) return op_fail(NF_ESHAPE, "the workspace has %lld bytes, %lld are needed", (long long)have, (long long)need);
  return NF_OK;
}

nf_status orth_call(const OrthCall& c, void* stream) {
  const int units = op_compute_units();
  if (units <= 0) return op_fail(NF_EDEVICE, "no usable HIP device");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool parts = c.out_type == NF_F32;
  hipError_t e;
  if (c.g_type == NF_F32)
    e = orth_run<float, MM_PARTS2>(c, units, s);
  else
    e = parts ? orth_run<bf16_t, MM_PARTS2>(c, units, s) : orth_run<bf16_t, MM_F16>(c, units, s);
  return op_result(e, "orthogonalisation");
}

}  // namespace
}  // namespace nf

using namespace nf;

extern "C" {

int64_t nf_orthogonalize_work(int32_t dtype, int64_t count, int64_t rows, int64_t cols) {
  op_begin();
  if (dtype != NF_F32 && dtype != NF_BF16) {
    op_fail(NF_EINVAL, "matrices must be fp32 or bf16 (dtype %d)", dtype);
    return -1;
  }
  if (check_sizes(count, rows, cols) != NF_OK) return -1;
  const OrthPlan p = orth_plan(dtype == NF_F32, rows, cols);
  if (count > 0 && p.bytes > INT64_MAX / count) {
    op_fail(NF_ESHAPE, "the workspace's size does not fit");
    return -1;
  }
  return p.bytes * count;
}

nf_status nf_orthogonalize(const void* d_x, int32_t dtype, int64_t count, int64_t rows, int64_t cols, int64_t ld,
                           int64_t stride, void* d_out, int64_t ld_out, int64_t stride_out, void* d_work,
                           int64_t work_bytes, void* stream) {
  op_begin();
  const int64_t need = nf_orthogonalize_work(dtype, count, rows, cols);
  if (need < 0) return op_float_type(dtype) && dtype != NF_F16 ? (count < 0 || rows < 1 || cols < 1 ? NF_EINVAL : NF_ESHAPE) : NF_EINVAL;
  if (count == 0) return NF_OK;
  const int64_t e = op_size(dtype);
  nf_status st = check_stack("the matrices", d_x, e, rows, cols, ld);
  if (st == NF_OK) st = check_stack("the result", d_out, e, rows, cols, ld_out);
  if (st == NF_OK) st = check_work(d_work, work_bytes, need);
  if (st != NF_OK) return st;
  if (count > 1 && (stride < 0 || stride_out < (rows - 1) * ld_out + cols))
    return op_fail(NF_ESHAPE, "the results overlap one another");
  OrthCall c{};
  c.count = count;
  c.rows = rows;
  c.cols = cols;
  c.g_type = c.out_type = dtype;
  c.g = d_x;
  c.ldg = ld;
  c.stride_g = stride;
  c.out = d_out;
  c.ldo = ld_out;
  c.stride_o = stride_out;
  c.work = d_work;
  return orth_call(c, stream);
}

nf_status nf_muon_step(const void* d_w, int32_t w_dtype, const float* d_m, const void* d_g, int32_t g_dtype,
                       int64_t count, int64_t rows, int64_t cols, float eta, float momentum, int32_t nesterov,
                       float decay, void* d_w_out, float* d_m_out, void* d_work, int64_t work_bytes, void* stream) {
  op_begin();
  if ((w_dtype != NF_F32 && w_dtype != NF_BF16) || (g_dtype != NF_F32 && g_dtype != NF_BF16))
    return op_fail(NF_EINVAL, "weights and gradients must be fp32 or bf16 (dtypes %d, %d)", w_dtype, g_dtype);
  if (w_dtype == NF_BF16 && g_dtype == NF_F32)
    return op_fail(NF_EINVAL, "fp32 gradients go with fp32 weights");
  if (nesterov != 0 && nesterov != 1) return op_fail(NF_EINVAL, "nesterov must be 0 or 1");
  if (!(eta >= 0.f && eta < __builtin_inff()) || !(decay >= 0.f && decay < __builtin_inff()) ||
      !(momentum >= 0.f && momentum < 1.f))
    return op_fail(NF_EINVAL, "eta and decay must be at least 0 and finite, momentum in [0, 1)");
  nf_status st = check_sizes(count, rows, cols);
  if (st != NF_OK) return st;
  const int64_t need = nf_orthogonalize_work(w_dtype, count, rows, cols);
  if (need < 0) return NF_ESHAPE;
  if (count == 0) return NF_OK;
  st = check_stack("the weights", d_w, op_size(w_dtype), rows, cols, cols);
  if (st == NF_OK) st = check_stack("the momentum", d_m, 4, rows, cols, cols);
  if (st == NF_OK) st = check_stack("the gradient", d_g, op_size(g_dtype), rows, cols, cols);
  if (st == NF_OK) st = check_stack("the new weights", d_w_out, op_size(w_dtype), rows, cols, cols);
  if (st == NF_OK) st = check_stack("the new momentum", d_m_out, 4, rows, cols, cols);
  if (st == NF_OK) st = check_work(d_work, work_bytes, need);
  if (st != NF_OK) return st;
  const int64_t all = count * rows * cols;
  if (d_w != d_w_out && op_overlap(d_w, all * op_size(w_dtype), d_w_out, all * op_size(w_dtype)))
    return op_fail(NF_EINVAL, "the new weights overlap the old without being them");
  if (d_m != d_m_out && op_overlap(d_m, all * 4, d_m_out, all * 4))
    return op_fail(NF_EINVAL, "the new momentum overlaps the old without being it");
  if (op_overlap(d_g, all * op_size(g_dtype), d_m_out, all * 4) ||
      op_overlap(d_w, all * op_size(w_dtype), d_m_out, all * 4) ||
      op_overlap(d_w_out, all * op_size(w_dtype), d_m_out, all * 4))
    return op_fail(NF_EINVAL, "the new momentum overlaps weights or gradient");
  OrthCall c{};
  c.count = count;
  c.rows = rows;
  c.cols = cols;
  c.g_type = g_dtype;
  c.out_type = w_dtype;
  c.g = d_g;
  c.ldg = cols;
  c.stride_g = rows * cols;
  c.m = d_m;
  c.m_out = d_m_out;
  c.momentum = momentum;
  c.nesterov = nesterov != 0;
  c.w = d_w;
  c.keep = 1.f - eta * decay;
  c.rate = eta * std::sqrt(rows > cols ? (float)rows / (float)cols : 1.f);
  c.out = d_w_out;
  c.ldo = cols;
  c.stride_o = rows * cols;
  c.work = d_work;
  return orth_call(c, stream);
}

}  // extern "C"
