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
//
// What bounds it, measured with all launches (us): the matrix cores at the card's power for
// a step of 4096 x 4096 fp32, 3850 - 3890 (1.07 PFLOP/s of f16 products, as a plain one of 4096
// reaches); for one of bf16, 1780 where its products at that rate take 1250, also the fp32 X's
// bytes (0.93 PFLOP/s in the steps, 0.75 in X X^T, 77 of fill and sums); 17 launches of 7 - 14
// for 1024 x 784 fp32, 167, and four of 517 x 1001 bf16, 157, of which 3.5 each are the launch
// and most of the rest the way of a tile's operands into a few compute units.  The last
// product of bf16 matrices in tiles of 128 does not fit its 128 registers and keeps 35 in scratch:
// 48 for 3000 x 1500 where the steps before take 35.
#include <cmath>

#include "orth_small.h"
#include "rows_mm.h"

namespace nf {
namespace {

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float UNIT = 16384.f, PER_UNIT = 1.f / UNIT;
constexpr int SUM_BLOCKS = 1024;       // at most; partial sums of a matrix

// where element (r, c) of an operand lies; its second part 64 bytes on
template <int KIND>
__device__ __forceinline__ int64_t place(int64_t r, int c, int64_t pitch) {
  return KIND == MM_PARTS2 ? r * pitch + (c / PARTS2_GROUP) * 128 + (c % PARTS2_GROUP) * 2 : r * pitch + c * 2;
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

// The buffers of one matrix (offsets in its share of the workspace; pitches in
// bytes).
struct OrthPlan {
  int m, n;                   // shorter and longer side
  int kx, kt;                 // bytes of a row of n, in whole stages, and of m, in whole tiles of 32; zeros past the last
  int64_t px, pt, pm;         // pitches of rows of n, of rows of m, of the fp32 X
  int64_t x, xt[2], a, b, xm, da, db, sums;
  int64_t bytes;              // of one matrix
};

int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

// A pitch of at least `bytes` that is an odd number of stages: rows whose pitch is
// a multiple of 4096 bytes begin in the same one of a cache's channels, and a tile's
// rows would all be read from it at one time.
int64_t odd_pitch(int64_t bytes) { return (up(bytes, 128) / 128 | 1) * 128; }

OrthPlan orth_plan(bool parts, int64_t rows, int64_t cols) {
  OrthPlan p{};
  p.m = (int)(rows < cols ? rows : cols);
  p.n = (int)(rows < cols ? cols : rows);
  p.kx = (int)orth_wide(parts, p.n);
  p.kt = (int)orth_narrow(parts, p.m);
  p.px = odd_pitch(p.kx);
  p.pt = odd_pitch(p.kt);
  p.pm = parts ? 0 : odd_pitch(2 * (int64_t)p.kx);
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
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
  const T* const g = a.g.p + (int64_t)blockIdx.z * a.g.stride;
  const float* const mom = a.m.p ? a.m.p + (int64_t)blockIdx.z * a.m.stride : nullptr;
  // The loads of a thread's values are under way together, and with those of the sums
  // (lanes along the user's rows; places past the matrix read its first value instead).
  constexpr int N = 64 * 64 / 256;
  T u[N];
  float m[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int e = k * 256 + tid, c = e & 63, r = e >> 6;
    const int i = i0 + (a.turned ? c : r), j = j0 + (a.turned ? r : c);
    const bool in = i < p.m && j < p.n;
    const int64_t ur = in ? a.turned ? j : i : 0, uc = in ? a.turned ? i : j : 0;
    u[k] = g[ur * a.g.ld + uc];
    m[k] = mom ? mom[ur * a.m.ld + uc] : 0.f;
  }
  double s = 0.0;
  for (int i = tid; i < a.blocks; i += 256) s += reinterpret_cast<const double*>(w + p.sums)[i];
  s = wave_sum(s);
  if ((tid & 63) == 0) part[tid >> 6] = s;
  __syncthreads();
  const double sum = (part[0] + part[1]) + (part[2] + part[3]);
  // a matrix of zeros stays one; one that is not finite becomes NaN throughout
  const double inv = sum == 0.0 ? 0.0 : sum < __builtin_inf() ? (double)UNIT / sqrt(sum) : __builtin_nan("");
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int e = k * 256 + tid, c = e & 63, r = e >> 6;
    const int i = i0 + (a.turned ? c : r), j = j0 + (a.turned ? r : c);
    float x = to_float(u[k]);
    if (mom) x = direction(x, m[k], a.momentum, a.nesterov);
    const float v = !(i < p.m && j < p.n) ? 0.f : inv != inv ? __builtin_nanf("") : (float)((double)x * inv);
    if (a.turned) tile[c][r] = v;
    else tile[r][c] = v;
  }
  __syncthreads();
  const int nx = p.kx / (KIND == MM_PARTS2 ? 4 : 2), nt = p.kt / (KIND == MM_PARTS2 ? 4 : 2);
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

typedef unsigned mm_u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned mm_u32x4 __attribute__((ext_vector_type(4)));
typedef float mm_f32x4 __attribute__((ext_vector_type(4)));

// The rows of a matrix from row r0 on as a buffer: what lies at TILE_OOB reads as
// zero and is not stored, so that an epilogue needs no branches and its loads do
// not wait for one another.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(void* p, int64_t r0, int64_t pitch) {
  return __builtin_amdgcn_make_buffer_rsrc(static_cast<char*>(p) + r0 * pitch, (short)0, (int)TILE_OOB, 0x00020000);
}
__device__ __forceinline__ float load_f32(const __amdgpu_buffer_rsrc_t& r, unsigned off) {
  return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0));
}
__device__ __forceinline__ void store_f32(const __amdgpu_buffer_rsrc_t& r, unsigned off, float x) {
  __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, x), r, off, 0, 0);
}
template <int KIND>
__device__ __forceinline__ unsigned across(int c) {       // bytes from a row's beginning to its element c
  return KIND == MM_PARTS2 ? (unsigned)((c / PARTS2_GROUP) * 128 + (c % PARTS2_GROUP) * 2) : (unsigned)(c * 2);
}
template <int KIND>
struct Four {                                             // four elements of a row, as they are loaded
  f16x4 h, l;
  __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t& r, unsigned off) {
    h = __builtin_bit_cast(f16x4, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0));
    if constexpr (KIND == MM_PARTS2) l = __builtin_bit_cast(f16x4, __builtin_amdgcn_raw_buffer_load_b64(r, off + 64u, 0, 0));
  }
  __device__ __forceinline__ float operator[](int c) const {
    return KIND == MM_PARTS2 ? (float)h[c] + (float)l[c] : (float)h[c];
  }
};
template <int KIND>
__device__ __forceinline__ void store_four(const __amdgpu_buffer_rsrc_t& r, unsigned off, const float (&x)[4]) {
  f16x4 h, l;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    h[c] = (_Float16)x[c];
    l[c] = (_Float16)(x[c] - (float)h[c]);
  }
  __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(mm_u32x2, h), r, off, 0, 0);
  if constexpr (KIND == MM_PARTS2) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(mm_u32x2, l), r, off + 64u, 0, 0);
}

// four neighbours of a row of the user's matrix; `n` of them are inside it
__device__ __forceinline__ void load_user(const void* p, int type, int64_t at, int n, float (&x)[4]) {
  auto go = [&](auto e) {
    typedef decltype(e) T;
    const T* const q = static_cast<const T*>(p) + at;
    T v[4] = {};
    if (n >= 4) {
      __builtin_memcpy(v, q, sizeof v);
    } else {
#pragma unroll
      for (int c = 0; c < 3; ++c)
        if (c < n) v[c] = q[c];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) x[c] = to_float(v[c]);
  };
  if (type == NF_F32) go(float());
  else go(bf16_t());
}
__device__ __forceinline__ void store_user(void* p, int type, int64_t at, int n, const float (&x)[4]) {
  auto go = [&](auto e) {
    typedef decltype(e) T;
    T* const q = static_cast<T*>(p) + at;
    T v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = from_float<T>(x[c]);
    if (n >= 4) {
      __builtin_memcpy(q, v, sizeof v);
    } else {
#pragma unroll
      for (int c = 0; c < 3; ++c)
        if (c < n) q[c] = v[c];
    }
  };
  if (type == NF_F32) go(float());
  else go(bf16_t());
}

template <int KIND, int PROD, int BM, int BN, int WM, int WN, int NS, int G, int OCC>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * G * 64, OCC) orth_mm_kernel(const MmArgs a) {
  typedef MmTile<KIND, BM, BN, WM, WN, NS, G> Tile;
  __shared__ __attribute__((aligned(1024))) char lds[Tile::LDS];
  constexpr bool SQUARE = PROD == PROD_GRAM || PROD == PROD_POLY;
  const OrthPlan& p = a.p;
  const int z = blockIdx.y;
  char* const w = a.work + z * p.bytes;
  int bx, by;
  if constexpr (SQUARE) {
    static_assert(BM == BN, "square tiles");
    if (!mm_place_lower(a.total, bx, by)) return;
  } else {
    if (!mm_place(a.total, a.mt, a.nt, bx, by)) return;
  }
  const int m0 = __builtin_amdgcn_readfirstlane(bx * BM), n0 = __builtin_amdgcn_readfirstlane(by * BN);
  const MmRows X{w + p.x, p.px, p.m}, XT{w + p.xt[a.from], p.pt, p.n}, A{w + p.a, p.pt, p.m}, B{w + p.b, p.pt, p.m};
  const bool turned = PROD == PROD_LAST && a.turned;     // rows of X^T down, rows of B across
  Tile tile;
  if constexpr (PROD == PROD_GRAM)
    tile.run(X, X, p.kx, m0, n0, lds);
  else if constexpr (PROD == PROD_POLY)
    tile.run(A, A, p.kt, m0, n0, lds);
  else
    tile.run(turned ? XT : B, turned ? B : XT, p.kt, m0, n0, lds);

  constexpr int per = KIND == MM_PARTS2 ? 4 : 2;
  const int wide_m = p.kt / per;                          // columns of m, with the zeros behind them
  const int rows = turned ? p.n : p.m, cols = turned || SQUARE ? p.m : p.n;
  const int pt = (int)p.pt, px = (int)p.px, pm = (int)p.pm;

  // Buffers that begin at the tile's first row (`back`: at its first column's row)
  const int pd = SQUARE || turned ? pt : px;
  const auto to = rows_from(w + (PROD == PROD_GRAM ? p.a : PROD == PROD_POLY ? p.b : p.x), m0, pd);
  const auto back = rows_from(w + (PROD == PROD_GRAM ? p.a : PROD == PROD_POLY ? p.b : p.xt[a.from ^ 1]), n0, pt);
  const auto in = rows_from(w + (PROD == PROD_POLY ? p.a : turned ? p.xt[a.from] : p.x), m0, pd);
  const auto xm = rows_from(w + p.xm, turned ? n0 : m0, pm);
  const auto da = rows_from(w + p.da, 0, 0), db = rows_from(w + p.db, 0, 0);

  constexpr bool STEPPING = PROD == PROD_STEP || PROD == PROD_LAST;
  struct Inputs {               // of a round: four neighbours
    Four<KIND> e;               // of A or X
    mm_f32x4 x;                 // of the fp32 X
    mm_f32x4 dj;                // of the diagonal, at the columns
    float di;                   // and at the row
    float w[4];
  };
  auto load = [&](int b, Inputs (&q)[Tile::ROUNDS]) {
    const int lj = tile.wn + (b % Tile::TN) * 32 + tile.col(), j = n0 + lj;
#pragma unroll
    for (int r = 0; r < Tile::ROUNDS; ++r) {
      const int li = tile.wm + (b / Tile::TN) * 32 + tile.row(r), i = m0 + li;
      // (four that begin inside may pass the last: zeros)
      const bool ok = i < rows && j < cols;
      if constexpr (PROD == PROD_POLY || (STEPPING && KIND == MM_PARTS2))
        q[r].e.load(in, ok ? (unsigned)(li * pd) + across<KIND>(j) : TILE_OOB);
      if constexpr (KIND == MM_F16 && PROD != PROD_GRAM) {
        const auto& d = PROD == PROD_POLY ? da : db;
        if (PROD == PROD_POLY || !turned) q[r].di = load_f32(d, ok ? (unsigned)i * 4u : TILE_OOB);
        if (PROD == PROD_POLY || turned)
          q[r].dj = __builtin_bit_cast(mm_f32x4, __builtin_amdgcn_raw_buffer_load_b128(d, ok ? (unsigned)j * 4u : TILE_OOB, 0, 0));
      }
      if constexpr (KIND == MM_F16 && STEPPING) {
        if (turned) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            q[r].x[c] = load_f32(xm, ok && j + c < cols ? (unsigned)((lj + c) * pm + i * 4) : TILE_OOB);
        } else {
          q[r].x = __builtin_bit_cast(
              mm_f32x4, __builtin_amdgcn_raw_buffer_load_b128(xm, ok ? (unsigned)(li * pm + j * 4) : TILE_OOB, 0, 0));
        }
      }
      if constexpr (PROD == PROD_LAST)
        if (a.w && ok) load_user(a.w, a.out_type, z * a.stride_w + i * a.ldw + j, cols - j, q[r].w);
    }
  };
  auto finish = [&](int b, const Inputs (&q)[Tile::ROUNDS]) {
    const int bi = tile.wm + (b / Tile::TN) * 32, bj = tile.wn + (b % Tile::TN) * 32;
    const int lj = bj + tile.col(), j = n0 + lj;
    tile.spread(b);
    float v[Tile::ROUNDS][4];
#pragma unroll
    for (int r = 0; r < Tile::ROUNDS; ++r) {
      tile.template sums<float>(r, v[r]);
      const int li = bi + tile.row(r), i = m0 + li;
      const bool ok = i < rows && j < cols;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float x = v[r][c] * PER_UNIT;
        if constexpr (PROD == PROD_POLY) {
          const float e = q[r].e[c];
          if constexpr (KIND == MM_F16) {
            const float di = q[r].di;                     // (D + F)^2, F without a diagonal
            x = i == j + c ? fmaf(di * PER_UNIT, di, x) : fmaf((di + q[r].dj[c]) * PER_UNIT, e, x);
            x = fmaf(NS_C, x, NS_B * (i == j + c ? di : e));
          } else {
            x = fmaf(NS_C, x, NS_B * e);
          }
        }
        if constexpr (SQUARE && KIND == MM_F16) {
          store_f32(PROD == PROD_GRAM ? da : db, ok && i == j + c ? (unsigned)i * 4u : TILE_OOB, x);
          if (i == j + c) x = 0.f;
        }
        if constexpr (STEPPING) {
          if constexpr (KIND == MM_PARTS2) {
            x = fmaf(NS_A, q[r].e[c], x);
          } else {
            const float e = q[r].x[c];
            x = fmaf(NS_A, e, fmaf((turned ? q[r].dj[c] : q[r].di) * PER_UNIT, (float)(_Float16)e, x));
          }
        }
        v[r][c] = ok && j + c < cols ? x : 0.f;           // zeros behind the last
      }
      if constexpr (PROD == PROD_LAST) {
        float y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          y[c] = v[r][c] * PER_UNIT;
          if (a.w) y[c] = fmaf(-a.rate, y[c], a.keep * q[r].w[c]);
        }
        if (ok) store_user(a.out, a.out_type, z * a.stride_o + i * a.ldo + j, cols - j, y);
      } else {
        // (of X the zeros lie there already, from the first)
        const bool kept = i < rows && j < (SQUARE ? wide_m : cols);
        store_four<KIND>(to, kept ? (unsigned)(li * pd) + across<KIND>(j) : TILE_OOB, v[r]);
        if constexpr (PROD == PROD_STEP && KIND == MM_F16) {
          const mm_f32x4 y = {v[r][0], v[r][1], v[r][2], v[r][3]};
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(mm_u32x4, y), xm, kept ? (unsigned)(li * pm + j * 4) : TILE_OOB, 0, 0);
        }
      }
    }
    if constexpr (PROD == PROD_LAST) return;
    if (SQUARE && bx == by) return;
    if constexpr (G > 1) Tile::meet();                    // a sum's places are other waves' too
#pragma unroll
    for (int r = 0; r < Tile::ROUNDS; ++r) tile.put_back(r, v[r]);
    Tile::meet();
#pragma unroll
    for (int r = 0; r < Tile::ROUNDS; ++r) {
      const int lr = bj + tile.row(r), lc = bi + tile.col();
      float x[4];
      tile.crossed(r, x);
      store_four<KIND>(back, n0 + lr < cols && m0 + lc < wide_m ? (unsigned)(lr * pt) + across<KIND>(m0 + lc) : TILE_OOB, x);
    }
  };
  // a block's inputs are on their way while the block before is finished
  Inputs q[2][Tile::ROUNDS];
  load(0, q[0]);
#pragma unroll
  for (int b = 0; b < Tile::BLOCKS; ++b) {
    if (b + 1 < Tile::BLOCKS) load(b + 1, q[(b + 1) & 1]);
    finish(b, q[b & 1]);
  }
}

template <int KIND, int PROD, int BM, int WM, int WN, int NS, int G, int OCC>
hipError_t launch_tile(MmArgs a, int64_t count, hipStream_t s) {
  constexpr bool SQUARE = PROD == PROD_GRAM || PROD == PROD_POLY;
  const bool turned = PROD == PROD_LAST && a.turned;
  const int rows = turned ? a.p.n : a.p.m, cols = turned || SQUARE ? a.p.m : a.p.n;
  a.mt = (rows + BM - 1) / BM;
  a.nt = (cols + BM - 1) / BM;
  a.total = SQUARE ? a.mt * (a.mt + 1) / 2 : a.mt * a.nt;
  return op_launch(orth_mm_kernel<KIND, PROD, BM, BM, WM, WN, NS, G, OCC>, dim3(mm_grid(a.total), (unsigned)count),
                  dim3((BM / WM) * (BM / WN) * G * 64), s, a);
}

template <int KIND, int PROD>
hipError_t launch_product(const MmArgs& a, int64_t count, int units, hipStream_t s) {
  switch (orth_shape((OrthProduct)PROD, KIND == MM_PARTS2, count, a.p.m, a.p.n, units)) {
    case MM_32_GROUPS: return launch_tile<KIND, PROD, 32, 32, 32, 3, 4, 1>(a, count, s);
    case MM_64_GROUPS: return launch_tile<KIND, PROD, 64, 32, 32, 3, 2, 2>(a, count, s);
    case MM_64: return launch_tile<KIND, PROD, 64, 32, 32, 3, 1, 3>(a, count, s);
    case MM_128: return launch_tile<KIND, PROD, 128, 64, 32, 2, 1, 4>(a, count, s);
    case MM_192: return launch_tile<KIND, PROD, 192, 96, 96, 3, 1, 1>(a, count, s);
    default: return launch_tile<KIND, PROD, 256, 128, 64, 2, 1, 2>(a, count, s);
  }
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
  if (c.rows <= ORTH_SMALL || c.cols <= ORTH_SMALL) {
    SmallArgs<T> q{};
    q.g = {static_cast<const T*>(c.g), c.ldg, c.stride_g};
    q.m = {c.m, ldm, stride_m};
    q.m_out = {c.m_out, ldm, stride_m};
    q.momentum = c.momentum;
    q.nesterov = c.nesterov;
    q.turned = c.rows > c.cols;
    q.work = work;
    q.p = small_plan(c.rows, c.cols);
    q.out_type = c.out_type;
    q.out = c.out;
    q.ldo = c.ldo;
    q.stride_o = c.stride_o;
    q.w = c.w;
    q.ldw = ldm;
    q.stride_w = stride_m;
    q.keep = c.keep;
    q.rate = c.rate;
    switch (q.p.mb) {
      case 1: return launch_small<T, 1>(q, c.count, NS_A, NS_B, NS_C, NF_ORTH_STEPS, s);
      case 2: return launch_small<T, 2>(q, c.count, NS_A, NS_B, NS_C, NF_ORTH_STEPS, s);
      case 3: return launch_small<T, 3>(q, c.count, NS_A, NS_B, NS_C, NF_ORTH_STEPS, s);
      default: return launch_small<T, 4>(q, c.count, NS_A, NS_B, NS_C, NF_ORTH_STEPS, s);
    }
  }
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
  hipError_t e = op_launch(orth_sum_kernel<T>, dim3((unsigned)blocks, (unsigned)c.count), dim3(256), s, u);
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
  e = op_launch(orth_fill_kernel<T, KIND>, dim3((unsigned)((p.n + 63) / 64), (unsigned)((p.m + 63) / 64), (unsigned)c.count),
               dim3(256), s, f);
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

nf_status check_stack(const char* what, const void* p, int64_t elem, int64_t cols, int64_t ld) {
  if (!p) return op_fail(NF_EINVAL, "NULL %s", what);
  if (!op_aligned(p, (uintptr_t)elem)) return op_fail(NF_EINVAL, "%s is not aligned to its elements", what);
  if (ld < cols || ld > NF_ORTH_MAX_LD)
    return op_fail(NF_ESHAPE, "%s: the row pitch must be at least the columns and at most %d", what, NF_ORTH_MAX_LD);
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
  const int64_t one = rows <= ORTH_SMALL || cols <= ORTH_SMALL ? small_plan(rows, cols).bytes
                                                               : orth_plan(dtype == NF_F32, rows, cols).bytes;
  if (count > 0 && one > INT64_MAX / count) {
    op_fail(NF_ESHAPE, "the workspace's size does not fit");
    return -1;
  }
  return one * count;
}

nf_status nf_orthogonalize(const void* d_x, int32_t dtype, int64_t count, int64_t rows, int64_t cols, int64_t ld,
                           int64_t stride, void* d_out, int64_t ld_out, int64_t stride_out, void* d_work,
                           int64_t work_bytes, void* stream) {
  op_begin();
  const int64_t need = nf_orthogonalize_work(dtype, count, rows, cols);
  if (need < 0) return op_float_type(dtype) && dtype != NF_F16 ? (count < 0 || rows < 1 || cols < 1 ? NF_EINVAL : NF_ESHAPE) : NF_EINVAL;
  if (count == 0) return NF_OK;
  const int64_t e = op_size(dtype);
  nf_status st = check_stack("the matrices", d_x, e, cols, ld);
  if (st == NF_OK) st = check_stack("the result", d_out, e, cols, ld_out);
  if (st == NF_OK) st = check_work(d_work, work_bytes, need);
  if (st != NF_OK) return st;
  // results one behind another, or side by side in the same rows
  if (count > 1 && (stride < 0 || (stride_out < (rows - 1) * ld_out + cols &&
                                   (stride_out < cols || stride_out > (ld_out - cols) / (count - 1)))))
    return op_fail(NF_ESHAPE, "the results overlap one another");
  if (count == 1) stride = stride_out = 0;
  if (stride > INT64_MAX / 8 / count || stride_out > INT64_MAX / 8 / count)
    return op_fail(NF_ESHAPE, "the matrices times their stride do not fit");
  // matrices of at most ORTH_SMALL rows or columns are read again while results are written
  const OpArray x{d_x, count, stride * e, rows, ld * e, cols * e};
  const OpArray out{d_out, count, stride_out * e, rows, ld_out * e, cols * e};
  if (op_share(x, out) && !op_same(x, out)) return op_fail(NF_EINVAL, "the result overlaps the matrices without being them");
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
  st = check_stack("the weights", d_w, op_size(w_dtype), cols, cols);
  if (st == NF_OK) st = check_stack("the momentum", d_m, 4, cols, cols);
  if (st == NF_OK) st = check_stack("the gradient", d_g, op_size(g_dtype), cols, cols);
  if (st == NF_OK) st = check_stack("the new weights", d_w_out, op_size(w_dtype), cols, cols);
  if (st == NF_OK) st = check_stack("the new momentum", d_m_out, 4, cols, cols);
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
  // gradients of at most ORTH_SMALL rows or columns are read again while weights are written
  if (op_overlap(d_g, all * op_size(g_dtype), d_w_out, all * op_size(w_dtype)) && !(d_g == d_w_out && g_dtype == w_dtype))
    return op_fail(NF_EINVAL, "the new weights overlap the gradient without being it");
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
