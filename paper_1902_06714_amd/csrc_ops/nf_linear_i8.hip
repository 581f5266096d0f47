// Linear layers in 8-bit integers: y = act(x_scale w_scale (x_q w_q^T) + b), a
// scale for each row of x (token) and each row of w (output channel), and the
// quantisation of rows, q = rint(x 127 / max|x|), scale = max|x| / 127.
//
// Sums are whole numbers in 32 bits and exact: NF_LINEAR_I8_MAX inputs times
// 128 x 128 stay below 2^31.
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

// THREADS / TPR rows a workgroup; NV vectors of a row in a thread's registers, 0: read twice
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
  most = wave_max(most);
  nan = __any(nan);
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
  const QuantArgs<T> a{x, ldx, ldq, rows, cols, (cols + 15) / 16 * 16, q, scale};
  const int vecs = a.wide / Vec16<T>::N;
#define NF_QUANT(TH, TPR, NV)     \
  if (vecs <= (TPR) * (NV))       \
    return launch_k(quant_kernel<T, TH, TPR, NV>, dim3((unsigned)((rows + (TH) / (TPR) - 1) / ((TH) / (TPR)))), \
                    dim3(TH), 0, s, a);
  NF_QUANT(256, 64, 1)
  NF_QUANT(256, 64, 4)
  NF_QUANT(256, 256, 2)
  NF_QUANT(256, 256, 8)
#undef NF_QUANT
  return launch_k(quant_kernel<T, 1024, 1024, 0>, dim3((unsigned)rows), dim3(1024), 0, s, a);
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
__device__ __forceinline__ void put_y(void* y, int type, int64_t at, float v) {
  if (type == NF_F32) static_cast<float*>(y)[at] = v;
  else if (type == NF_BF16) static_cast<bf16_t*>(y)[at] = from_float<bf16_t>(v);
  else static_cast<f16_t*>(y)[at] = from_float<f16_t>(v);
}

template <int BM, int BN, int WM, int WN, int NS, int OCC>
__global__ void __launch_bounds__((BM / WM) * (BN / WN) * 64, OCC) linear_kernel(const LinearArgs a) {
  typedef MmTile<MM_I8, BM, BN, WM, WN, NS> Tile;
  __shared__ __attribute__((aligned(1024))) char lds[Tile::LDS];
  int bx, by;
  if (!mm_place(a.total, a.mt, a.nt, bx, by)) return;
  const int m0 = __builtin_amdgcn_readfirstlane(bx * BM), n0 = __builtin_amdgcn_readfirstlane(by * BN);
  const MmRows X{reinterpret_cast<const char*>(a.xq), a.ldx, a.rows};
  const MmRows Wt{reinterpret_cast<const char*>(a.wq), a.ldw, a.outputs};
  typename Tile::Acc acc[Tile::TM][Tile::TN];
  Tile::run(X, Wt, a.bytes, m0, n0, lds, acc);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
  with_act(a.act, [&](auto act) {
#pragma unroll
    for (int tj = 0; tj < Tile::TN; ++tj) {
      const int j = n0 + wn + tj * 32 + (lane & 31);
      if (j >= a.outputs) continue;
      const float ws = a.w_scale[j], b = a.bias ? a.bias[j] : 0.f;
#pragma unroll
      for (int ti = 0; ti < Tile::TM; ++ti)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int i = m0 + wm + ti * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
          if (i >= a.rows) continue;
          const float z = (float)acc[ti][tj][v] * a.x_scale[i] * ws + b;
          put_y(a.y, a.y_type, (int64_t)i * a.ldy + j, activated<act.value>(z));
        }
    }
  });
}

template <int BM, int WM, int WN, int NS, int OCC>
hipError_t launch_linear_tile(LinearArgs a, hipStream_t s) {
  a.mt = (a.rows + BM - 1) / BM;
  a.nt = (a.outputs + BM - 1) / BM;
  a.total = a.mt * a.nt;
  return launch_k(linear_kernel<BM, BM, WM, WN, NS, OCC>, dim3(mm_grid(a.total)), dim3((BM / WM) * (BM / WN) * 64), 0, s, a);
}

hipError_t launch_linear(const LinearArgs& a, int units, hipStream_t s) {
  auto tiles = [&](int64_t b) { return ((a.rows + b - 1) / b) * ((a.outputs + b - 1) / b); };
  if (tiles(256) >= units) return launch_linear_tile<256, 128, 64, 2, 2>(a, s);
  if (tiles(128) >= units) return launch_linear_tile<128, 64, 64, 2, 2>(a, s);
  return launch_linear_tile<64, 32, 32, 3, 2>(a, s);
}

int64_t whole16(int64_t v) { return (v + 15) / 16 * 16; }

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
  if (op_overlap(d_x, ((rows - 1) * ld + cols) * op_size(dtype), d_q, (rows - 1) * ld_q + whole16(cols)))
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
  if (op_overlap(d_xq, (rows - 1) * ld_x + whole16(inputs), d_y, ((rows - 1) * ld_y + outputs) * op_size(y_dtype)))
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
  return rows * whole16(inputs) + rows * 4;
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
  if (op_overlap(d_x, ((rows - 1) * ld_x + inputs) * op_size(x_dtype), d_y,
                 ((rows - 1) * ld_y + outputs) * op_size(y_dtype)))
    return op_fail(NF_EINVAL, "the result overlaps the rows");
  if (!d_work || !op_aligned(d_work, 16)) return op_fail(NF_EINVAL, "the workspace is NULL or not aligned to 16 bytes");
  if (work_bytes < nf_linear_i8_work(rows, inputs))
    return op_fail(NF_ESHAPE, "the workspace has %lld bytes, %lld are needed", (long long)work_bytes,
                   (long long)nf_linear_i8_work(rows, inputs));
  const int units = op_compute_units();
  if (units <= 0) return op_fail(NF_EDEVICE, "no usable HIP device");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t ldq = whole16(inputs);
  int8_t* const q = static_cast<int8_t*>(d_work);
  float* const scale = reinterpret_cast<float*>(q + rows * ldq);
  st = with_type(x_dtype, [&](auto e) {
    typedef decltype(e) T;
    return op_result(launch_quant<T>(static_cast<const T*>(d_x), ld_x, rows, (int)inputs, q, ldq, scale, s), "quantisation");
  });
  if (st != NF_OK) return st;
  const LinearArgs a{q, d_wq, ldq, ld_w, ld_y, scale, d_w_scale, d_bias, act, (int)rows, (int)outputs,
                     (int)ldq, y_dtype, d_y, 0, 0, 0};
  return op_result(launch_linear(a, units, s), "8-bit linear layer");
}

}  // extern "C"
