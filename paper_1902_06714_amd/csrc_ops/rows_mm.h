// Products of rows with rows, C(i, j) = sum over k of A(i, k) B(j, k), on the
// matrix cores, for operands that lie in memory as rows of bytes along k: i8,
// f16, or pairs of f16 parts.
//
// In all three a lane's operand of a matrix instruction is 16 consecutive bytes
// of a row (16 i8 of 32x32x32, 8 f16 of 32x32x16), so tiles of rows are moved to
// LDS the same way, 128 bytes of k a stage, by loads that write LDS themselves
// (16 bytes a lane, no registers).  Such a load writes a wave's 1024 bytes in
// lane order, so a row's eight 16-byte pieces are permuted by choosing which
// piece a lane loads: piece c of row r lies at place c ^ (r & 7), and the 8 rows
// that a quarter of a wave's read touches lie in all banks.
//
// Pairs of parts (PARTS2): x = h + l, h = f16(x), l = f16(x - h), kept in
// groups of 32 k as 64 bytes of h and then 64 bytes of l.  A product is formed as
// hl + lh + hh, each exact in the fp32 accumulators' inputs (11 x 11 bits); ll, below
// 2^-22 of it, is left out.
#pragma once

#include "ops_common.h"

namespace nf {

enum MmKind { MM_I8, MM_F16, MM_PARTS2 };

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float mm_f32x16 __attribute__((ext_vector_type(16)));
typedef int mm_i32x16 __attribute__((ext_vector_type(16)));
typedef int mm_i32x4 __attribute__((ext_vector_type(4)));

constexpr int MM_STAGE = 128;      // bytes of k of a stage
constexpr int PARTS2_GROUP = 32;   // k of a group of pairs of parts

template <int KIND>
struct MmAcc {
  typedef std::conditional_t<KIND == MM_I8, mm_i32x16, mm_f32x16> type;
};

// Rows of an operand: `rows` of them, `pitch` bytes apart (a multiple of 16, the
// base aligned to 16), of which the first `bytes` (a multiple of 16) count.
struct MmRows {
  const char* base;
  int64_t pitch;
  int rows;
};

// One wave's share of loading R rows of a stage by NW waves.
template <int R, int NW>
struct StageLoader {
  static constexpr int N = R / 8 / NW;          // loads of 8 rows
  static_assert(N * 8 * NW == R, "whole loads");
  __amdgpu_buffer_rsrc_t rsrc;
  unsigned off[N];

  // rows past the last are read as the last one: their sums are not stored
  __device__ __forceinline__ void init(const MmRows& m, int r0, int wave, int lane) {
    rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(m.base + (int64_t)r0 * m.pitch), (short)0, (int)TILE_OOB,
                                             0x00020000);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = (i * NW + wave) * 8 + (lane >> 3);
      const int at = min(r, m.rows - 1 - r0);
      off[i] = (unsigned)at * (unsigned)m.pitch + (unsigned)(((lane & 7) ^ (lane >> 3)) << 4);
    }
  }
  // stage at byte k0; `left` bytes of k from there (a lane whose piece lies past
  // them loads zeros: its offset lies past the buffer)
  template <bool TAIL>
  __device__ __forceinline__ void load(unsigned lds, int k0, int left, int wave, int lane) const {
    const bool in = !TAIL || (((lane & 7) ^ (lane >> 3)) << 4) < left;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const unsigned o = in ? off[i] + (unsigned)k0 : TILE_OOB;
      const unsigned to = __builtin_amdgcn_readfirstlane(lds + (i * NW + wave) * 1024);
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(o), "s"(rsrc)
                   : "memory", "m0");
    }
  }
};

template <int N>
__device__ __forceinline__ void wait_loads() {
  // and for the wave's own reads of LDS, which the next stage's loads may overwrite
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ void mm_product(mm_i32x16& c, const mm_i32x4& a, const mm_i32x4& b) {
  c = __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ void mm_product(mm_f32x16& c, const mm_i32x4& a, const mm_i32x4& b) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A tile of BM rows of A by BN rows of B, by waves of WM x WN; NS stages in LDS.
// Afterwards register v of acc[i][j] of a lane holds row
// wm + 32 i + 8 (v / 4) + 4 (lane / 32) + v % 4 and column wn + 32 j + lane % 32.
template <int KIND, int BM, int BN, int WM, int WN, int NS>
struct MmTile {
  static constexpr int NW = (BM / WM) * (BN / WN), THREADS = NW * 64;
  static constexpr int TM = WM / 32, TN = WN / 32;
  static constexpr int STAGE = (BM + BN) * MM_STAGE, LDS = NS * STAGE;
  typedef typename MmAcc<KIND>::type Acc;
  typedef StageLoader<BM, NW> LA;
  typedef StageLoader<BN, NW> LB;
  static constexpr int PER = LA::N + LB::N;     // a wave's loads of a stage

  __device__ __forceinline__ static void run(const MmRows& A, const MmRows& B, int bytes, int m0, int n0,
                                             char* lds, Acc (&acc)[TM][TN]) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
    LA la;
    LB lb;
    la.init(A, m0, wave, lane);
    lb.init(B, n0, wave, lane);
    const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const int stages = (bytes + MM_STAGE - 1) / MM_STAGE;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;

    auto request = [&](int t, int buf) {
      const int k0 = t * MM_STAGE, left = bytes - k0;
      const unsigned to = base + buf * STAGE;
      if (left >= MM_STAGE) {
        la.template load<false>(to, k0, left, wave, lane);
        lb.template load<false>(to + BM * MM_STAGE, k0, left, wave, lane);
      } else {
        la.template load<true>(to, k0, left, wave, lane);
        lb.template load<true>(to + BM * MM_STAGE, k0, left, wave, lane);
      }
    };
    int at[4];                                  // places of pieces 2 s + lane / 32 in a lane's row
#pragma unroll
    for (int s = 0; s < 4; ++s) at[s] = ((2 * s + (lane >> 5)) ^ (lane & 7)) << 4;
    const int ra = (wm + (lane & 31)) * MM_STAGE, rb = (BM + wn + (lane & 31)) * MM_STAGE;
    auto multiply = [&](int buf) {
      const char* const p = lds + buf * STAGE;
      auto frag = [&](int row, int s) {
        return *reinterpret_cast<const mm_i32x4*>(p + row + at[s]);
      };
      if constexpr (KIND == MM_PARTS2) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          mm_i32x4 a[TM][2], b[TN][2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
#pragma unroll
            for (int i = 0; i < TM; ++i) a[i][q] = frag(ra + i * 32 * MM_STAGE, s + 2 * q);
#pragma unroll
            for (int j = 0; j < TN; ++j) b[j][q] = frag(rb + j * 32 * MM_STAGE, s + 2 * q);
          }
#pragma unroll
          for (int x = 0; x < 3; ++x)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
              for (int j = 0; j < TN; ++j) mm_product(acc[i][j], a[i][x == 1], b[j][x == 0]);
        }
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          mm_i32x4 a[TM], b[TN];
#pragma unroll
          for (int i = 0; i < TM; ++i) a[i] = frag(ra + i * 32 * MM_STAGE, s);
#pragma unroll
          for (int j = 0; j < TN; ++j) b[j] = frag(rb + j * 32 * MM_STAGE, s);
#pragma unroll
          for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) mm_product(acc[i][j], a[i], b[j]);
        }
      }
    };

    // stage t lies in buffer t % NS; while it is multiplied, the next NS - 1 are on their way.
    // Behind the last stage each request is of no bytes: it loads zeros, and a
    // wait for the loads after a stage's own is a wait for the stage.
#pragma unroll
    for (int t = 0; t < NS - 1; ++t) request(t, t);
    int buf = 0;
    for (int t = 0; t < stages; ++t) {
      wait_loads<(NS - 2) * PER>();
      __builtin_amdgcn_s_barrier();             // everyone's loads of t are here, everyone's reads of t - 1 done
      asm volatile("" ::: "memory");
      request(t + NS - 1, (buf + NS - 1) % NS);
      multiply(buf);
      buf = buf + 1 == NS ? 0 : buf + 1;
    }
    wait_loads<0>();                            // nothing may write LDS after the tile
    __syncthreads();
  }
};

// The tile of workgroup b: consecutive tiles on an XCD (workgroup b runs on XCD
// b mod 8), in bands of 8 tile rows that share operands in its L2.
__device__ __forceinline__ bool mm_place(int total, int mt, int nt, int& bx, int& by) {
  const int per = (total + 7) / 8, b = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if (b >= total) return false;
  const int band = mt > 8 ? b / (8 * nt) : 0;
  const int in = b - band * (8 * nt), bh = min(8, mt - band * 8);
  by = in / bh;
  bx = band * 8 + in - by * bh;
  return true;
}
// The same for the tiles of a symmetric product on and below the diagonal (bx >= by).
__device__ __forceinline__ bool mm_place_lower(int total, int& bx, int& by) {
  const int per = (total + 7) / 8, b = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if (b >= total) return false;
  int r = (int)((sqrtf(8.f * (float)b + 1.f) - 1.f) * 0.5f);
  while (r * (r + 1) / 2 > b) --r;
  while ((r + 1) * (r + 2) / 2 <= b) ++r;
  bx = r;
  by = b - r * (r + 1) / 2;
  return true;
}
inline unsigned mm_grid(int64_t total) { return (unsigned)(8 * ((total + 7) / 8)); }

}  // namespace nf
