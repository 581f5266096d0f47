// What the operators for the last layers of a language model share: element
// types, loads of rows at any alignment, reductions, and the checks that every
// entry point makes before it enqueues anything.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>
#include <type_traits>

#include "nf.h"
#include "nf_internal.h"

namespace nf {

struct bf16_t {
  uint16_t bits;
};
struct f16_t {
  _Float16 v;
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16_t x) {
  return __builtin_bit_cast(float, (unsigned)x.bits << 16);
}
__device__ __forceinline__ float to_float(f16_t x) { return (float)x.v; }

// rounded to nearest, ties to even (NaN stays NaN)
template <class T>
__device__ __forceinline__ T from_float(float x) {
  if constexpr (std::is_same_v<T, float>) {
    return x;
  } else if constexpr (std::is_same_v<T, bf16_t>) {
    return {__builtin_bit_cast(uint16_t, (__bf16)x)};
  } else {
    return {(_Float16)x};
  }
}

// 16 bytes of a row, at any address that its elements may have (the hardware
// takes wide loads and stores at any alignment)
template <class T>
struct Vec16 {
  static constexpr int N = 16 / sizeof(T);
  T v[N];
};
template <class T>
__device__ __forceinline__ Vec16<T> load16(const T* p) {
  Vec16<T> r;
  __builtin_memcpy(&r, p, 16);
  return r;
}
template <class T>
__device__ __forceinline__ void store16(T* p, const Vec16<T>& r) {
  __builtin_memcpy(p, &r, 16);
}

// Sums and maxima over a wave, in a fixed order; every lane gets the result.
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  return x;
}

// ---- entry points ----------------------------------------------------------
// The message is formatted into a fixed buffer; no exception leaves an entry.
template <class... A>
nf_status op_fail(nf_status st, const char* fmt, A... a) {
  char msg[256];
  std::snprintf(msg, sizeof msg, fmt, a...);
  try {
    set_error_message(msg);
  } catch (...) {
  }
  return st;
}
inline nf_status op_fail(nf_status st, const char* msg) {
  try {
    set_error_message(msg);
  } catch (...) {
  }
  return st;
}
inline void op_begin() {
  try {
    set_error_message("");
  } catch (...) {
  }
}
inline nf_status op_result(hipError_t e, const char* what) {
  if (e == hipSuccess) return NF_OK;
  (void)hipGetLastError();
  return op_fail(NF_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

// Launches a kernel of an operator (a plain launch: nothing times these one by one).
template <typename... P>
inline hipError_t op_launch(void (*kernel)(P...), dim3 grid, dim3 block, hipStream_t s,
                            const typename same_type<P>::type&... args) {
  void* argv[] = {const_cast<void*>(static_cast<const void*>(&args))..., nullptr};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, argv, 0, s);
}

// Rows in as many launches as they take: f(first, n) launches rows first .. first + n - 1 in
// workgroups of `block` threads, `per_block` rows each or `per_row` to a row.  (A grid
// holds fewer than 2^32 threads, and a grid of tiles up to 7 workgroups more.)
template <class F>
hipError_t op_each_launch(int64_t rows, int64_t block, int64_t per_block, int64_t per_row, F&& f) {
  const int64_t most = (0xffffffffll / block - 7) / per_row * per_block;
  for (int64_t first = 0; first < rows; first += most) {
    const hipError_t e = f(first, rows - first < most ? rows - first : most);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Compute units of the current device, or 0 where there is none (asked once
// for each device).
int op_compute_units();

inline bool op_float_type(int dtype) { return dtype == NF_F32 || dtype == NF_BF16 || dtype == NF_F16; }
inline int64_t op_size(int dtype) { return dtype == NF_F32 ? 4 : 2; }
inline bool op_aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Whether two ranges of bytes share any.
inline bool op_overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// An array of rows in memory, in bytes: `count` matrices of `rows` rows of `width`.
struct OpArray {
  const void* p;
  int64_t count, stride, rows, pitch, width;
  // one row a matrix is one matrix of such rows; what is never stepped over does not count
  OpArray plain() const {
    OpArray a = *this;
    if (a.rows == 1) a.rows = a.count, a.pitch = a.stride, a.count = 1;
    if (a.count == 1) a.stride = 0;
    if (a.rows == 1) a.pitch = a.width;
    return a;
  }
  int64_t matrix() const { return (rows - 1) * pitch + width; }
  int64_t span() const { return (count - 1) * stride + matrix(); }
  bool even() const { return pitch > 0 && stride % pitch == 0; }     // every row is whole pitches from the first
};

// Whether the rows of two arrays may share bytes.  Arrays that lie side by side in the
// rows of one buffer, or by turns in one stack, do not.
inline bool op_share(const OpArray& x, const OpArray& y) {
  const OpArray a = x.plain(), b = y.plain();
  if (!op_overlap(a.p, a.span(), b.p, b.span())) return false;
  const int64_t apart = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
  // pieces of na bytes and of nb bytes, all of them whole multiples of `step` apart
  auto by_turns = [](int64_t apart, int64_t step, int64_t na, int64_t nb) {
    const int64_t d = (apart % step + step) % step;
    return d >= na && step - d >= nb;
  };
  if (a.stride > 0 && a.stride == b.stride && by_turns(apart, a.stride, a.matrix(), b.matrix())) return false;
  if (a.even() && b.even() && a.pitch == b.pitch && by_turns(apart, a.pitch, a.width, b.width)) return false;
  // one that lies between two rows of the other
  if (a.even() && by_turns(apart, a.pitch, a.width, b.span())) return false;
  if (b.even() && by_turns(-apart, b.pitch, b.width, a.span())) return false;
  return true;
}
// Whether they are the same array.
inline bool op_same(const OpArray& x, const OpArray& y) {
  const OpArray a = x.plain(), b = y.plain();
  return a.p == b.p && a.count == b.count && a.stride == b.stride && a.rows == b.rows && a.pitch == b.pitch &&
         a.width == b.width;
}

// Calls f with a value of the element type `dtype` names.
template <class F>
auto with_type(int dtype, F&& f) {
  if (dtype == NF_BF16) return f(bf16_t());
  if (dtype == NF_F16) return f(f16_t());
  return f(float());
}

}  // namespace nf
