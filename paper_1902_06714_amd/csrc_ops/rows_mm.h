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

#include "mm_shape.h"
#include "ops_common.h"

namespace nf {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float mm_f32x16 __attribute__((ext_vector_type(16)));
typedef int mm_i32x16 __attribute__((ext_vector_type(16)));
typedef int mm_i32x4 __attribute__((ext_vector_type(4)));

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
  // load i of a stage at byte k0 (a multiple of 128); `in`: whether the lane's piece
  // lies inside the operand's bytes (else its offset lies past the buffer and it
  // loads zeros)
  __device__ __forceinline__ void load(int i, unsigned lds, int k0, bool in, int wave) const {
    const unsigned to = __builtin_amdgcn_readfirstlane(lds + (i * NW + wave) * 1024);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to),
                 "v"(in ? off[i] : TILE_OOB), "s"(rsrc), "s"(k0)
                 : "memory", "m0");
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

// A tile of BM rows of A by BN rows of B, by G groups of waves of WM x WN, each on
// its share of k; NS stages of each group in LDS.
//
// Stage t lies in buffer t % NS.  A step is 32 bytes of k of every row (64 of
// pairs of parts); its operands are read from LDS while the step before is
// multiplied, so a wave alone on its SIMD keeps the matrix pipe busy.  Before the
// last step of a stage the waves meet: by then each has read all of stage t, whose
// buffer stage t + NS is requested into, and waited for its own loads of stage
// t + 1, which all may read after.
//
// A launch of few tiles runs at the pace at which a compute unit takes in a tile's
// operands (105 GB/s here, whatever the waves' shares: 0.16 us for a stage of 64 x 64, of f16
// and of pairs alike); one group of waves reaches 0.25 - 0.28, two 0.17 - 0.21.
//
// Afterwards a wave's blocks of 32 x 32 sums go through LDS, so that a lane has
// four neighbours of a row and memory is read and written in whole lines.
constexpr int MM_PITCH = 36;                        // words of a column of a block in LDS
constexpr int MM_BLOCK = 32 * MM_PITCH * 4;         // bytes of a block in LDS

template <int KIND, int BM, int BN, int WM, int WN, int NS, int G>
struct MmTile {
  static constexpr int NW = (BM / WM) * (BN / WN), THREADS = NW * G * 64;
  static constexpr int TM = WM / 32, TN = WN / 32, BLOCKS = TM * TN;
  static constexpr int STAGE = (BM + BN) * MM_STAGE, LDS = G * NS * STAGE;
  static constexpr int STEPS = KIND == MM_PARTS2 ? 2 : 4;   // of a stage
  static constexpr int P = KIND == MM_PARTS2 ? 2 : 1;       // parts of a value
  static constexpr int ROUNDS = 4 / G;                      // of 8 rows of a block that a wave finishes
  typedef typename MmAcc<KIND>::type Acc;
  typedef StageLoader<BM, NW> LA;
  typedef StageLoader<BN, NW> LB;
  static constexpr int PER = LA::N + LB::N;     // a wave's loads of a stage
  static_assert(NS >= 2 && (NS - 1) * PER < 64, "loads that the counter can hold");
  static_assert(G * NW * MM_BLOCK <= LDS, "a block of each wave in LDS");
  static_assert(G == 1 || G == 2 || G == 4, "whole rounds");

  int lane, wave, group;                        // wave: of the group
  int wm, wn;                                   // the wave's place in the tile
  char* lds;
  Acc acc[TM][TN];

  __device__ __forceinline__ void run(const MmRows& A, const MmRows& B, int bytes, int m0, int n0, char* shared) {
    lane = threadIdx.x & 63;
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    group = G == 1 ? 0 : all / NW;
    wave = G == 1 ? all : all % NW;
    wm = (wave % (BM / WM)) * WM;
    wn = (wave / (BM / WM)) * WN;
    lds = shared;
    LA la;
    LB lb;
    la.init(A, m0, wave, lane);
    lb.init(B, n0, wave, lane);
    const int stages = ((bytes + MM_STAGE - 1) / MM_STAGE + G - 1) / G;      // of each group
    const int kbeg = group * stages * MM_STAGE, kend = min(bytes, kbeg + stages * MM_STAGE);
    char* const mine = lds + group * (NS * STAGE);
    const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)mine;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0;

    // load i of stage t.  Behind the last stage it is of no bytes and loads zeros,
    // so that the number of loads behind a stage's own stays the same.
    auto request = [&](int i, int t, int buf, bool in) {
      const unsigned to = base + buf * STAGE;
      const int k0 = __builtin_amdgcn_readfirstlane(min(kbeg + t * MM_STAGE, bytes));
      if (i < LA::N) la.load(i, to, k0, in, wave);
      else lb.load(i - LA::N, to + BM * MM_STAGE, k0, in, wave);
    };
    const int piece = ((lane & 7) ^ (lane >> 3)) << 4;        // of a lane's loads
    auto inside = [&](int t) { return piece < kend - kbeg - t * MM_STAGE; };
    int at[4];                                  // places of pieces 2 s + lane / 32 in a lane's row
#pragma unroll
    for (int s = 0; s < 4; ++s) at[s] = ((2 * s + (lane >> 5)) ^ (lane & 7)) << 4;
    const int ra = (wm + (lane & 31)) * MM_STAGE, rb = (BM + wn + (lane & 31)) * MM_STAGE;
    mm_i32x4 a[2][TM][P], b[2][TN][P];
    auto fetch = [&](int set, int buf, int s) {
      const char* const p = mine + buf * STAGE;
#pragma unroll
      for (int q = 0; q < P; ++q) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
          a[set][i][q] = *reinterpret_cast<const mm_i32x4*>(p + ra + i * 32 * MM_STAGE + at[s + 2 * q]);
#pragma unroll
        for (int j = 0; j < TN; ++j)
          b[set][j][q] = *reinterpret_cast<const mm_i32x4*>(p + rb + j * 32 * MM_STAGE + at[s + 2 * q]);
      }
    };
    constexpr int NM = (P == 2 ? 3 : 1) * TM * TN;      // products of a step
    // products n0 .. n1 - 1 of a step, f(n) behind product n
    auto multiply = [&](int set, int n0, int n1, auto&& f) {
#pragma unroll
      for (int n = n0; n < n1; ++n) {
        const int x = n / (TM * TN), i = n % (TM * TN) / TN, j = n % TN;
        mm_product(acc[i][j], a[set][i][P == 2 && x == 1], b[set][j][P == 2 && x == 0]);
        f(n);
      }
    };

#pragma unroll
    for (int t = 0; t < NS; ++t) {
      const bool in = inside(t);
#pragma unroll
      for (int i = 0; i < PER; ++i) request(i, t, t, in);
    }
    wait_loads<(NS - 1) * PER>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    fetch(0, 0, 0);
    int buf = 0;
    for (int t = 0; t < stages; ++t) {
      const int next = buf + 1 == NS ? 0 : buf + 1;
#pragma unroll
      for (int s = 0; s < STEPS; ++s) {
        constexpr int HALF = NM / 2;
        if (s + 1 < STEPS) {
          fetch((s + 1) & 1, buf, s + 1);
          __builtin_amdgcn_sched_barrier(0);
          multiply(s & 1, 0, NM, [](int) {});
        } else {
          multiply(s & 1, 0, HALF, [](int) {});
          __builtin_amdgcn_sched_barrier(0);
          wait_loads<(NS - 2) * PER>();
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          fetch(0, next, 0);
          __builtin_amdgcn_sched_barrier(0);
          const bool in = inside(t + NS);
          // the loads between the products, as evenly as they go
          multiply(s & 1, HALF, NM, [&](int n) {
#pragma unroll
            for (int i = (n - HALF) * PER / (NM - HALF); i < (n + 1 - HALF) * PER / (NM - HALF); ++i) {
              __builtin_amdgcn_sched_barrier(0);
              request(i, t + NS, buf, in);
              __builtin_amdgcn_sched_barrier(0);
            }
          });
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      buf = next;
    }
    wait_loads<0>();                            // nothing may write LDS after the tile
    __syncthreads();
  }

  // What a block in LDS needs between writing and reading: the groups meet, a
  // wave alone only keeps its own order.
  __device__ __forceinline__ static void meet() {
    if constexpr (G > 1) {
      __syncthreads();
    } else {
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }
  }
  __device__ __forceinline__ int* block_of(int g) const {
    return reinterpret_cast<int*>(lds + (g * NW + wave) * MM_BLOCK);
  }
  // the row of the block, and the first of its four columns, that a lane has in a round
  __device__ __forceinline__ int row(int round) const { return (group * ROUNDS + round) * 8 + (lane >> 3); }
  __device__ __forceinline__ int col() const { return (lane & 7) * 4; }

  // A block's sums: register v of a lane is row 8 (v / 4) + 4 (lane / 32) + v % 4 of
  // column lane % 32.  In LDS they lie by column.
  __device__ __forceinline__ void spread(int b) {
    int* const p = block_of(group) + (lane & 31) * MM_PITCH + 4 * (lane >> 5);
    const Acc& c = acc[b / TN][b % TN];
    meet();                                     // what was read of the block before
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      mm_i32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const auto x = c[4 * q + e];            // (a cast of the element itself takes the vector's first)
        v[e] = __builtin_bit_cast(int, x);
      }
      *reinterpret_cast<mm_i32x4*>(p + 8 * q) = v;
    }
    meet();
  }
  template <class S>
  __device__ __forceinline__ void sums(int round, S (&x)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = S(0);
#pragma unroll
      for (int g = 0; g < G; ++g)
        x[e] += __builtin_bit_cast(S, block_of(g)[(col() + e) * MM_PITCH + row(round)]);
    }
  }
  // values of the block back into LDS, and four of a column as neighbours: element
  // (col() + e, row(round)) of the block
  __device__ __forceinline__ void put_back(int round, const float (&x)[4]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      block_of(0)[(col() + e) * MM_PITCH + row(round)] = __builtin_bit_cast(int, x[e]);
  }
  __device__ __forceinline__ void crossed(int round, float (&x)[4]) const {
    const mm_i32x4 v = *reinterpret_cast<const mm_i32x4*>(block_of(0) + row(round) * MM_PITCH + col());
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int y = v[e];
      x[e] = __builtin_bit_cast(float, y);
    }
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
