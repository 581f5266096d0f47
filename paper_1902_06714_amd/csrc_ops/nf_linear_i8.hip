// Linear layers in 8-bit integers: y = act(x_scale w_scale (x_q w_q^T) + b), a
// scale for each row of x (token) and each row of w (output channel), and the
// quantisation of rows, q = rint(x 127 / max|x|), scale = max|x| / 127.
//
// Sums are whole numbers in 32 bits and exact: NF_LINEAR_I8_MAX inputs times
// 128 x 128 stay below 2^31.
//
// What bounds it, measured with the quantisation (us): the matrix cores for 8192 rows, 4096
// inputs and outputs in bf16, 156 (the product alone 140, 1.96 POP/s); the outputs' and
// operands' bytes, one after the other, for 10000 x 784 to 1024 in fp32, 31; the weights' bytes
// for one row of 4096 to 4096, 7.3 (2.3 TB/s; 3.5 of it the launch).
#include "nf_act.h"
#include "rows_mm.h"

namespace nf {
namespace {

// ---- quantisation --------------------------------------------------------------
// One row's factor and scale.  A row of zeros has scale 0; one with a NaN or an
// infinity has scale NaN, which makes its whole result NaN.  Rows so small that
// 127 / max would overflow are multiplied by a power of two first.
struct RowScale {
  float pre, factor, scale;
  bool zero;
};
__device__ __forceinline__ RowScale row_scale(float most, bool nan) {
  RowScale r;
  r.pre = most < 0x1p-100f ? 0x1p100f : 1.f;
  const bool bad = nan || most == __builtin_inff();
  r.zero = bad || most == 0.f;
  r.factor = r.zero ? 0.f : 127.f / (most * r.pre);
  r.scale = bad ? __builtin_nanf("") : most / 127.f;
  return r;
}
__device__ __forceinline__ int quantised(const RowScale& r, float x) {
  return r.zero ? 0 : (int)fminf(fmaxf(rintf(x * r.pre * r.factor), -127.f), 127.f);
}

template <class T>
struct QuantArgs {
  const T* x;
  int64_t ldx, ldq, rows;
  int cols, wide;              // wide: cols up to a whole 16, the zeros that are written
  int8_t* q;
  float* scale;
};

// THREADS / TPR rows a workgroup; NV vectors of a row in a thread's registers, 0: read twice.
// Bound by the bytes (8192 x 4096 bf16 23 us, 4.4 TB/s).  16 threads a row against a wave (us):
// 16000 x 40 f16 4.3, 7.3; 16000 x 100 f32 4.2, 6.2.
template <class T, int THREADS, int TPR, int NV>
__global__ void __launch_bounds__(THREADS) quant_kernel(const QuantArgs<T> a) {
  constexpr int E = Vec16<T>::N, W = TPR / 64;
  const int tid = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
  const bool live = row < a.rows;
  const T* const x = a.x + (live ? row : a.rows - 1) * a.ldx;
  auto load = [&](int j) {
    if (j + E <= a.cols) return load16(x + j);
    Vec16<T> r;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      r.v[e] = from_float<T>(0.f);
      if (j + e < a.cols) r.v[e] = x[j + e];
    }
    return r;
  };
  Vec16<T> keep[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int v = 0; v < NV; ++v) keep[v] = load((v * TPR + tid) * E);
  }
  auto each = [&](auto&& f) {
    if constexpr (NV > 0) {
#pragma unroll
      for (int v = 0; v < NV; ++v) f((v * TPR + tid) * E, keep[v]);
    } else {
      for (int j = tid * E; j < a.wide; j += TPR * E) f(j, load(j));
    }
  };
  float most = 0.f;
  int nan = 0;
  each([&](int, const Vec16<T>& v) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float f = to_float(v.v[e]);
      most = fmaxf(most, fabsf(f));
      nan |= f != f;
    }
  });
  if constexpr (TPR < 64) {
#pragma unroll
    for (int d = 1; d < TPR; d *= 2) {
      most = fmaxf(most, __shfl_xor(most, d));
      nan |= __shfl_xor(nan, d);
    }
  } else {
    most = wave_max(most);
    nan = __any(nan);
  }
  if constexpr (W > 1) {
    __shared__ float sm[THREADS / 64];
    __shared__ int sn[THREADS / 64];
    if ((threadIdx.x & 63) == 0) {
      sm[threadIdx.x >> 6] = most;
      sn[threadIdx.x >> 6] = nan;
    }
    __syncthreads();
    const int w0 = threadIdx.x / TPR * W;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      most = fmaxf(most, sm[w0 + w]);
      nan |= sn[w0 + w];
    }
  }
  if (!live) return;
  const RowScale r = row_scale(most, nan != 0);
  if (tid == 0) a.scale[row] = r.scale;
  int8_t* const q = a.q + row * a.ldq;
  each([&](int j, const Vec16<T>& v) {
    unsigned w[E / 4];
#pragma unroll
    for (int c = 0; c < E / 4; ++c) {
      w[c] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[c] |= (unsigned)(quantised(r, to_float(v.v[4 * c + e])) & 255) << (8 * e);
    }
    if (j < a.wide) __builtin_memcpy(q + j, w, E);     // whole 16 columns are written, the last with zeros
  });
}

template <class T>
hipError_t launch_quant(const T* x, int64_t ldx, int64_t rows, int cols, int8_t* q, int64_t ldq, float* scale,
                        hipStream_t s) {
  const int wide = (cols + 15) / 16 * 16, vecs = wide / Vec16<T>::N;
  auto go = [&](auto threads, auto of_row, auto held) {
    constexpr int TH = decltype(threads)::value, TPR = decltype(of_row)::value, NV = decltype(held)::value;
    return op_each_launch(rows, TH, TH / TPR, 1, [&](int64_t first, int64_t n) {
      const QuantArgs<T> b{x + first * ldx, ldx, ldq, n, cols, wide, q + first * ldq, scale + first};
      return op_launch(quant_kernel<T, TH, TPR, NV>, dim3((unsigned)((n + TH / TPR - 1) / (TH / TPR))), dim3(TH), s, b);
    });
  };
#define NF_QUANT(TH, TPR, NV) \
  if (vecs <= (TPR) * (NV))   \
    return go(std::integral_constant<int, TH>(), std::integral_constant<int, TPR>(), std::integral_constant<int, NV>());
  NF_QUANT(256, 16, 2)
  NF_QUANT(256, 64, 1)
  NF_QUANT(256, 64, 4)
  NF_QUANT(256, 256, 2)
  NF_QUANT(256, 256, 8)
#undef NF_QUANT
  return go(std::integral_constant<int, 1024>(), std::integral_constant<int, 1024>(), std::integral_constant<int, 0>());
}

// ---- the product ---------------------------------------------------------------
struct LinearArgs {
  const int8_t* xq;
  const int8_t* wq;
  int64_t ldx, ldw, ldy;
  const float* x_scale;
  const float* w_scale;
  const float* bias;           // or null
  int act;                     // an nf_act, or -1
  int rows, outputs, bytes;    // bytes: inputs up to a whole 16
  int y_type;
  void* y;
  int total, mt, nt;
};

template <int ACT>
__device__ __forceinline__ float activated(float z) {
  if constexpr (ACT < 0) {
    return z;
  } else {
    float f, fp;
    act_eval<float>(ACT, z, f, fp);
    // no activation hides that a row could not be quantised
    return z != z ? z : f;
  }
}
// calls f with the activation as a constant
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
  switch (act) {
    case ACT_GAUSSIAN: f(std::integral_constant<int, ACT_GAUSSIAN>()); break;
    case ACT_RELU: f(std::integral_constant<int, ACT_RELU>()); break;
    case ACT_SIGMOID: f(std::integral_constant<int, ACT_SIGMOID>()); break;
    case ACT_STEP: f(std::integral_constant<int, ACT_STEP>()); break;
    case ACT_TANH: f(std::integral_constant<int, ACT_TANH>()); break;
    default: f(std::integral_constant<int, -1>()); break;
  }
}
// Four neighbours of a row of y, `n` of them inside it.  No activation hides that
// a row could not be quantised.
template <class T, int ACT>
__device__ __forceinline__ void put_y(T* y, int n, const float (&z)[4]) {
  T v[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = from_float<T>(activated<ACT>(z[c]));
  if (n >= 4) {
    __builtin_memcpy(y, v, sizeof v);
  } else {
#pragma unroll
    for (int c = 0; c < 3; ++c)
      if (c < n) y[c] = v[c];
  }
}

template <class T, int BM, int BN, int WM, int WN, int NS, int G, int OCC>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * G * 64, OCC) linear_kernel(const LinearArgs a) {
  typedef MmTile<MM_I8, BM, BN, WM, WN, NS, G> Tile;
  __shared__ __attribute__((aligned(1024))) char lds[Tile::LDS];
  int bx, by;
  if (!mm_place(a.total, a.mt, a.nt, bx, by)) return;
  const int m0 = __builtin_amdgcn_readfirstlane(bx * BM), n0 = __builtin_amdgcn_readfirstlane(by * BN);
  const MmRows X{reinterpret_cast<const char*>(a.xq), a.ldx, a.rows};
  const MmRows Wt{reinterpret_cast<const char*>(a.wq), a.ldw, a.outputs};
  Tile tile;
  tile.run(X, Wt, a.bytes, m0, n0, lds);
  // the scales and biases of the wave's rows and columns, zeros past the last
  const auto xs = __builtin_amdgcn_make_buffer_rsrc((void*)a.x_scale, (short)0, a.rows * 4, 0x00020000);
  const auto ws = __builtin_amdgcn_make_buffer_rsrc((void*)a.w_scale, (short)0, a.outputs * 4, 0x00020000);
  const auto bs = __builtin_amdgcn_make_buffer_rsrc((void*)a.bias, (short)0, a.bias ? a.outputs * 4 : 0, 0x00020000);
  float w4[Tile::TN][4], b4[Tile::TN][4], x1[Tile::TM][Tile::ROUNDS];
#pragma unroll
  for (int t = 0; t < Tile::TN; ++t)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const unsigned off = (unsigned)(n0 + tile.wn + t * 32 + tile.col() + c) * 4u;
      w4[t][c] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(ws, off, 0, 0));
      b4[t][c] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(bs, off, 0, 0));
    }
#pragma unroll
  for (int t = 0; t < Tile::TM; ++t)
#pragma unroll
    for (int r = 0; r < Tile::ROUNDS; ++r)
      x1[t][r] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(
                                               xs, (unsigned)(m0 + tile.wm + t * 32 + tile.row(r)) * 4u, 0, 0));
  T* const y = static_cast<T*>(a.y);
  with_act(a.act, [&](auto act) {
#pragma unroll
    for (int b = 0; b < Tile::BLOCKS; ++b) {
      const int ti = b / Tile::TN, tj = b % Tile::TN;
      const int j = n0 + tile.wn + tj * 32 + tile.col();
      tile.spread(b);
#pragma unroll
      for (int r = 0; r < Tile::ROUNDS; ++r) {
        int s[4];
        tile.template sums<int>(r, s);
        const int i = m0 + tile.wm + ti * 32 + tile.row(r);
        float z[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) z[c] = (float)s[c] * x1[ti][r] * w4[tj][c] + b4[tj][c];
        if (i < a.rows && j < a.outputs) put_y<T, act.value>(y + (int64_t)i * a.ldy + j, a.outputs - j, z);
      }
    }
  });
}

template <class T, int BM, int WM, int WN, int NS, int G, int OCC, int BN = BM>
hipError_t launch_linear_tile(LinearArgs a, hipStream_t s) {
  constexpr int THREADS = (BM / WM) * (BN / WN) * G * 64;
  a.nt = (a.outputs + BN - 1) / BN;
  const int64_t rows = a.rows;
  return op_each_launch((rows + BM - 1) / BM, THREADS, 1, a.nt, [&](int64_t first, int64_t n) {
    LinearArgs b = a;
    const int64_t row = first * BM;
    b.xq += row * a.ldx;
    b.x_scale += row;
    b.y = static_cast<T*>(a.y) + row * a.ldy;
    b.rows = (int)(rows - row < n * BM ? rows - row : n * BM);
    b.mt = (int)n;
    b.total = b.mt * b.nt;
    return op_launch(linear_kernel<T, BM, BN, WM, WN, NS, G, OCC>, dim3(mm_grid(b.total)), dim3(THREADS), s, b);
  });
}

// ---- few rows: the weights' bytes ----------------------------------------------
// A workgroup forms 16 outputs of up to 16 rows.  Its 8 waves take turns along k, 64
// bytes at a time, with operands straight from memory (16 rows of weights across the
// lanes, 16 bytes each): the weights are read once, and nothing waits in LDS but the
// sums of the waves.
//
// X not void: at most FEW_WAVES rows of X are quantised here, by every workgroup for itself, while its first
// weights are on their way.
constexpr int FEW_WAVES = 8;
constexpr int FEW_AHEAD = 8;           // loads of weights a lane has under way
constexpr int FEW_Q = 65536;           // bytes of quantised rows in LDS

template <class X>
struct FewArgs {
  LinearArgs a;
  const X* x;                          // [rows][ldf]
  int64_t ldf;
  int inputs;
};

template <class X, class T>
__global__ void __launch_bounds__(64 * FEW_WAVES) linear_few_kernel(const FewArgs<X> f) {
  constexpr bool QUANT = !std::is_void_v<X>;
  const LinearArgs& a = f.a;
  __shared__ int part[FEW_WAVES][256];
  __shared__ __attribute__((aligned(16))) char q[QUANT ? FEW_Q : 16];
  __shared__ float scales[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n0 = blockIdx.x * 16;
  const int piece = (lane >> 4) * 16;                  // of 64 bytes of k
  const int rows = a.rows;
  const char* const w = reinterpret_cast<const char*>(a.wq) + (int64_t)min(n0 + (lane & 15), a.outputs - 1) * a.ldw;
  const mm_i32x4 zero = {0, 0, 0, 0};
  const int steps = (a.bytes + 63) / 64;
  auto weights = [&](int s) {
    const int k = s * 64 + piece;
    return k < a.bytes ? *reinterpret_cast<const mm_i32x4*>(w + k) : zero;
  };
  mm_i32x4 wq[FEW_AHEAD];
#pragma unroll
  for (int u = 0; u < FEW_AHEAD; ++u) wq[u] = weights(wave + u * FEW_WAVES);
  const char* xr;
  if constexpr (QUANT) {
    // one, two, four or all eight waves quantise a row; in LDS rows lie a pitch of
    // steps 64-byte pieces and 16 bytes apart
    constexpr int E = Vec16<X>::N;
    const int pitch = steps * 64 + 16;
    const int share = rows <= 1 ? 8 : rows <= 2 ? 4 : rows <= 4 ? 2 : 1;
    const int r = wave / share, stride = share * 64 * E, j0 = ((wave % share) * 64 + lane) * E;
    const X* const x = f.x + (int64_t)min(r, rows - 1) * f.ldf;
    auto load = [&](int j) {
      if (j + E <= f.inputs) return load16(x + j);
      Vec16<X> v;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v.v[e] = from_float<X>(0.f);
        if (j + e < f.inputs) v.v[e] = x[j + e];
      }
      return v;
    };
    constexpr int KEEP = 2;              // vectors that need not be read again
    Vec16<X> keep[KEEP];
#pragma unroll
    for (int u = 0; u < KEEP; ++u) keep[u] = load(j0 + u * stride);
    float most = 0.f;
    int nan = 0;
    auto look = [&](const Vec16<X>& v) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float y = to_float(v.v[e]);
        most = fmaxf(most, fabsf(y));
        nan |= y != y;
      }
    };
#pragma unroll
    for (int u = 0; u < KEEP; ++u) look(keep[u]);
#pragma unroll 4
    for (int j = j0 + KEEP * stride; j < f.inputs; j += stride) look(load(j));
    most = wave_max(most);
    nan = __any(nan);
    if (lane == 0) {
      part[wave][0] = __builtin_bit_cast(int, most);
      part[wave][1] = nan;
    }
    __syncthreads();
    for (int g = r * share; g < (r + 1) * share; ++g) {
      most = fmaxf(most, __builtin_bit_cast(float, part[g][0]));
      nan |= part[g][1];
    }
    const RowScale rs = row_scale(most, nan);
    auto put = [&](int j, const Vec16<X>& v) {
      unsigned o[E / 4];
#pragma unroll
      for (int c = 0; c < E / 4; ++c) {
        o[c] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[c] |= (unsigned)(quantised(rs, to_float(v.v[4 * c + e])) & 255) << (8 * e);
      }
      if (j < steps * 64) __builtin_memcpy(q + r * pitch + j, o, E);
    };
    if (r < rows) {
      if (lane == 0 && wave % share == 0) scales[r] = rs.scale;
#pragma unroll
      for (int u = 0; u < KEEP; ++u) put(j0 + u * stride, keep[u]);
#pragma unroll 4
      for (int j = j0 + KEEP * stride; j < steps * 64; j += stride) put(j, load(j));
    }
    __syncthreads();
    xr = q + min(lane & 15, rows - 1) * pitch;
  } else {
    xr = reinterpret_cast<const char*>(a.xq) + (int64_t)min(lane & 15, rows - 1) * a.ldx;
  }
  mm_i32x4 acc = zero;
  for (int s0 = wave; s0 < steps; s0 += FEW_WAVES * FEW_AHEAD) {
#pragma unroll
    for (int u = 0; u < FEW_AHEAD; ++u) {
      const int s = s0 + u * FEW_WAVES, k = s * 64 + piece;
      const mm_i32x4 now = wq[u];
      wq[u] = weights(s + FEW_WAVES * FEW_AHEAD);
      const mm_i32x4 x = k < a.bytes ? *reinterpret_cast<const mm_i32x4*>(xr + k) : zero;
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, now, acc, 0, 0, 0);
    }
  }
  // register v of a lane: row 4 (lane / 16) + v of x, output lane % 16
#pragma unroll
  for (int v = 0; v < 4; ++v) part[wave][v * 64 + lane] = acc[v];
  __syncthreads();
  if (tid >= 256) return;
  const int r = 4 * ((tid & 63) >> 4) + (tid >> 6), n = n0 + (tid & 15);
  int sum = 0;
#pragma unroll
  for (int g = 0; g < FEW_WAVES; ++g) sum += part[g][tid];
  if (r >= rows || n >= a.outputs) return;
  const float z = (float)sum * (QUANT ? scales[r] : a.x_scale[r]) * a.w_scale[n] + (a.bias ? a.bias[n] : 0.f);
  with_act(a.act, [&](auto act) {
    static_cast<T*>(a.y)[(int64_t)r * a.ldy + n] = from_float<T>(activated<act.value>(z));
  });
}

template <class X, class T>
hipError_t launch_few(const FewArgs<X>& f, hipStream_t s) {
  return op_launch(linear_few_kernel<X, T>, dim3((unsigned)((f.a.outputs + 15) / 16)), dim3(64 * FEW_WAVES), s, f);
}

// 16 rows are one operand of the matrix instruction; beyond, tiles of 64 x 64 that
// share operands through LDS are faster (4096 x 4096, us: 16 rows 8.1, tiles 9.7; 32 rows,
// two operands, 10.8, tiles 9.8; 784 -> 1024, 16 rows: 3.8, 5.5).  Up to four rows are quantised in
// place, which saves a launch (4096 x 4096: 1 row 8.3, 10.2 with the launch; 4 rows 10.2, 11.1; 8 rows
// 14.0, 11.6).
bool few_rows(int64_t rows) { return rows <= 16; }
bool few_quantises(int64_t rows, int64_t inputs) {
  return rows <= 4 && rows * ((inputs + 63) / 64 * 64 + 16) <= FEW_Q;
}

template <class T>
hipError_t launch_linear_as(const LinearArgs& a, int units, hipStream_t s) {
  switch (linear_shape(a.rows, a.outputs, a.bytes, units)) {
    case MM_32_GROUPS: return launch_linear_tile<T, 32, 32, 32, 3, 4, 1>(a, s);
    case MM_64_GROUPS: return launch_linear_tile<T, 64, 32, 32, 3, 2, 2>(a, s);
    case MM_64: return launch_linear_tile<T, 64, 32, 32, 3, 1, 3>(a, s);
    case MM_128: return launch_linear_tile<T, 128, 64, 32, 2, 1, 4>(a, s);
    case MM_128_192: return launch_linear_tile<T, 128, 64, 96, 2, 1, 2, 192>(a, s);
    case MM_192: return launch_linear_tile<T, 192, 96, 96, 3, 1, 1>(a, s);
    default: return launch_linear_tile<T, 256, 128, 64, 2, 1, 2>(a, s);
  }
}
hipError_t launch_linear(const LinearArgs& a, int units, hipStream_t s) {
  return with_type(a.y_type, [&](auto e) {
    typedef decltype(e) T;
    if (few_rows(a.rows)) return launch_few<void, T>(FewArgs<void>{a, nullptr, 0, 0}, s);
    return launch_linear_as<T>(a, units, s);
  });
}

int64_t whole16(int64_t v) { return (v + 15) / 16 * 16; }
// pitch of rows in the workspace: not a multiple of 4096, at which a tile's rows would
// all lie in the same one of a cache's channels
int64_t row_pitch(int64_t inputs) { return ((inputs + 127) / 128 | 1) * 128; }

nf_status check_linear(const void* wq, int64_t ldw, const float* w_scale, int act, int64_t rows, int64_t inputs,
                       int64_t outputs, const void* y, int y_type, int64_t ldy) {
  if (!op_float_type(y_type)) return op_fail(NF_EINVAL, "results must be fp32, bf16 or fp16 (dtype %d)", y_type);
  if (act < -1 || act > NF_TANH) return op_fail(NF_EINVAL, "unknown activation %d", act);
  if (rows < 0 || inputs < 1 || outputs < 1) return op_fail(NF_EINVAL, "rows must be at least 0, inputs and outputs at least 1");
  if (inputs > NF_LINEAR_I8_MAX || outputs > NF_LINEAR_I8_MAX || rows > (1 << 24))
    return op_fail(NF_ESHAPE, "at most %d inputs and outputs and 2^24 rows", NF_LINEAR_I8_MAX);
  if (ldw < whole16(inputs) || ldw % 16 != 0 || ldw > (1 << 22))
    return op_fail(NF_ESHAPE, "the weights' row pitch must be a multiple of 16 that holds the inputs, at most 2^22");
  if (ldy < outputs || ldy > INT64_MAX / 4 / (rows + 1)) return op_fail(NF_ESHAPE, "the result's row pitch does not fit its columns");
  if (!wq || !w_scale) return op_fail(NF_EINVAL, "NULL weights or scales");
  if (!op_aligned(wq, 16)) return op_fail(NF_EINVAL, "the weights are not aligned to 16 bytes");
  if (rows > 0 && !y) return op_fail(NF_EINVAL, "NULL result");
  if (!op_aligned(y, (uintptr_t)op_size(y_type))) return op_fail(NF_EINVAL, "the result is not aligned to its elements");
  return NF_OK;
}

}  // namespace
}  // namespace nf

using namespace nf;

extern "C" {

nf_status nf_quantize_rows(const void* d_x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, int8_t* d_q,
                           int64_t ld_q, float* d_scale, void* stream) {
  op_begin();
  if (!op_float_type(dtype)) return op_fail(NF_EINVAL, "rows must be fp32, bf16 or fp16 (dtype %d)", dtype);
  if (rows < 0 || cols < 1) return op_fail(NF_EINVAL, "rows must be at least 0, columns at least 1");
  if (cols > NF_LINEAR_I8_MAX || rows > (1 << 24))
    return op_fail(NF_ESHAPE, "at most %d columns and 2^24 rows", NF_LINEAR_I8_MAX);
  if (ld < cols || ld > INT64_MAX / 4 / (rows + 1)) return op_fail(NF_ESHAPE, "the row pitch does not fit the columns");
  if (ld_q < whole16(cols) || ld_q % 16 != 0 || ld_q > (1 << 22))
    return op_fail(NF_ESHAPE, "the quantised rows' pitch must be a multiple of 16 that holds the columns, at most 2^22");
  if (rows == 0) return NF_OK;
  if (!d_x || !d_q || !d_scale) return op_fail(NF_EINVAL, "NULL pointer");
  if (!op_aligned(d_x, (uintptr_t)op_size(dtype)) || !op_aligned(d_q, 16))
    return op_fail(NF_EINVAL, "rows must be aligned to their elements, quantised rows to 16 bytes");
  if (op_share({d_x, 1, 0, rows, ld * op_size(dtype), cols * op_size(dtype)}, {d_q, 1, 0, rows, ld_q, whole16(cols)}))
    return op_fail(NF_EINVAL, "the quantised rows overlap the rows");
  if (op_compute_units() <= 0) return op_fail(NF_EDEVICE, "no usable HIP device");
  return with_type(dtype, [&](auto e) {
    typedef decltype(e) T;
    return op_result(launch_quant<T>(static_cast<const T*>(d_x), ld, rows, (int)cols, d_q, ld_q, d_scale,
                                     static_cast<hipStream_t>(stream)),
                     "quantisation");
  });
}

nf_status nf_linear_i8(const int8_t* d_xq, int64_t ld_x, const float* d_x_scale, const int8_t* d_wq, int64_t ld_w,
                       const float* d_w_scale, const float* d_bias, int32_t act, int64_t rows, int64_t inputs,
                       int64_t outputs, void* d_y, int32_t y_dtype, int64_t ld_y, void* stream) {
  op_begin();
  const nf_status st = check_linear(d_wq, ld_w, d_w_scale, act, rows, inputs, outputs, d_y, y_dtype, ld_y);
  if (st != NF_OK) return st;
  if (ld_x < whole16(inputs) || ld_x % 16 != 0 || ld_x > (1 << 22))
    return op_fail(NF_ESHAPE, "the rows' pitch must be a multiple of 16 that holds the inputs, at most 2^22");
  if (rows == 0) return NF_OK;
  if (!d_xq || !d_x_scale) return op_fail(NF_EINVAL, "NULL rows or scales");
  if (!op_aligned(d_xq, 16)) return op_fail(NF_EINVAL, "the rows are not aligned to 16 bytes");
  const int64_t size = op_size(y_dtype);
  if (op_share({d_xq, 1, 0, rows, ld_x, whole16(inputs)}, {d_y, 1, 0, rows, ld_y * size, outputs * size}))
    return op_fail(NF_EINVAL, "the result overlaps the rows");
  const int units = op_compute_units();
  if (units <= 0) return op_fail(NF_EDEVICE, "no usable HIP device");
  const LinearArgs a{d_xq, d_wq, ld_x, ld_w, ld_y, d_x_scale, d_w_scale, d_bias, act, (int)rows, (int)outputs,
                     (int)whole16(inputs), y_dtype, d_y, 0, 0, 0};
  return op_result(launch_linear(a, units, static_cast<hipStream_t>(stream)), "8-bit linear layer");
}

int64_t nf_linear_i8_work(int64_t rows, int64_t inputs) {
  op_begin();
  if (rows < 0 || inputs < 1 || inputs > NF_LINEAR_I8_MAX || rows > (1 << 24)) {
    op_fail(NF_ESHAPE, "at most %d inputs and 2^24 rows", NF_LINEAR_I8_MAX);
    return -1;
  }
  return rows * row_pitch(inputs) + rows * 4;
}

nf_status nf_linear_i8_dynamic(const void* d_x, int32_t x_dtype, int64_t ld_x, const int8_t* d_wq, int64_t ld_w,
                               const float* d_w_scale, const float* d_bias, int32_t act, int64_t rows,
                               int64_t inputs, int64_t outputs, void* d_y, int32_t y_dtype, int64_t ld_y,
                               void* d_work, int64_t work_bytes, void* stream) {
  op_begin();
  if (!op_float_type(x_dtype)) return op_fail(NF_EINVAL, "rows must be fp32, bf16 or fp16 (dtype %d)", x_dtype);
  nf_status st = check_linear(d_wq, ld_w, d_w_scale, act, rows, inputs, outputs, d_y, y_dtype, ld_y);
  if (st != NF_OK) return st;
  if (ld_x < inputs || ld_x > INT64_MAX / 4 / (rows + 1)) return op_fail(NF_ESHAPE, "the rows' pitch does not fit the inputs");
  if (rows == 0) return NF_OK;
  if (!d_x) return op_fail(NF_EINVAL, "NULL rows");
  if (!op_aligned(d_x, (uintptr_t)op_size(x_dtype))) return op_fail(NF_EINVAL, "the rows are not aligned to their elements");
  const int64_t x_size = op_size(x_dtype), y_size = op_size(y_dtype);
  if (op_share({d_x, 1, 0, rows, ld_x * x_size, inputs * x_size}, {d_y, 1, 0, rows, ld_y * y_size, outputs * y_size}))
    return op_fail(NF_EINVAL, "the result overlaps the rows");
  if (!d_work || !op_aligned(d_work, 16)) return op_fail(NF_EINVAL, "the workspace is NULL or not aligned to 16 bytes");
  if (work_bytes < nf_linear_i8_work(rows, inputs))
    return op_fail(NF_ESHAPE, "the workspace has %lld bytes, %lld are needed", (long long)work_bytes,
                   (long long)nf_linear_i8_work(rows, inputs));
  const int units = op_compute_units();
  if (units <= 0) return op_fail(NF_EDEVICE, "no usable HIP device");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (few_quantises(rows, inputs))
    return with_type(x_dtype, [&](auto xe) {
      typedef decltype(xe) X;
      return with_type(y_dtype, [&](auto ye) {
        const LinearArgs a{nullptr, d_wq, 0, ld_w, ld_y, nullptr, d_w_scale, d_bias, act, (int)rows, (int)outputs,
                           (int)whole16(inputs), y_dtype, d_y, 0, 0, 0};
        const FewArgs<X> f{a, static_cast<const X*>(d_x), ld_x, (int)inputs};
        return op_result(launch_few<X, decltype(ye)>(f, s), "8-bit linear layer");
      });
    });
  const int64_t ldq = row_pitch(inputs);
  int8_t* const q = static_cast<int8_t*>(d_work);
  float* const scale = reinterpret_cast<float*>(q + rows * ldq);
  st = with_type(x_dtype, [&](auto e) {
    typedef decltype(e) T;
    return op_result(launch_quant<T>(static_cast<const T*>(d_x), ld_x, rows, (int)inputs, q, ldq, scale, s), "quantisation");
  });
  if (st != NF_OK) return st;
  const LinearArgs a{q, d_wq, ldq, ld_w, ld_y, scale, d_w_scale, d_bias, act, (int)rows, (int)outputs,
                     (int)whole16(inputs), y_dtype, d_y, 0, 0, 0};
  return op_result(launch_linear(a, units, s), "8-bit linear layer");
}

}  // extern "C"
