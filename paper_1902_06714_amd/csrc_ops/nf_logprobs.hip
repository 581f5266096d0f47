// Log probabilities of given classes, entropies and the largest alternatives of
// rows of logits, and the gradient of a weighted sum of them.
//
// With z = scale x, m = max z, s = sum exp(z - m):
//   log p_j = (z_j - m) - log s,   H = log s - sum exp(z - m) (z - m) / s,
//   d(g log p_t + h H)/dx_j = scale (g ([j = t] - p_j) - h p_j (log p_j + H)).
//
// What bounds it: the bytes of the logits.  A row of up to 64 KB with a gradient or of at
// most as many rows as compute units, and of up to 8 KB else, is read once into registers,
// and the maximum, the sums, the alternatives and the gradient all come from that
// read; a longer row is read with a running maximum and sum, and again for each of
// the others.  Rows of at most 128 classes take 8 to 64 lanes of a wave.  Measured (us):
// the loss with its gradient of 4096 x 32768 bf16 114 (4.7 TB/s, a copy 4.9 - 5.0); of rows
// past 64 KB, whose second read does not all come from caches, 600 x 50000 bf16 40 where a read and a
// write take 24, 1000 x 131072 bf16 171 for 105; 10000 x 10 f32 4.3 and 1 x 32768 bf16 7.5 (a launch
// alone takes 3.5).  Scores of 2049 x 50021 bf16 with 8 alternatives 72 for 41 of bytes: 15 vector
// instructions a value fill 56% of the issue cycles, and of the 6 waves a SIMD that 72 registers
// leave room for 4.5 are there on average, too few for the loads and the instructions to hide
// one another.
//
// Alternatives: ordered(z) is a whole number in z's order, so (ordered(z),
// ~index) orders by value and then by the lower index, and no two are equal.
// The row's values fall into 64 groups, by the lanes that hold them; the n_top-th largest
// of the groups' maxima (32 ballots of one wave) is at most the row's n_top-th largest
// value, so the values from there on hold all alternatives (not many more, on
// logits of some spread): the lanes whose own maximum is that large put them into LDS,
// and each counts the larger ones.  More than fit there (rows of equal values)
// are found by n_top searches for the next largest instead.
#include <initializer_list>

#include "ops_common.h"

namespace nf {
namespace {

static_assert(NF_TOP_MAX <= 64, "a wave's lanes hold enough maxima for the threshold");
constexpr int TOP_CAP = 1024;    // candidates held in LDS
constexpr int SMALL_MAX = 128;   // classes of the kernel that shares a wave among rows

template <class T>
struct LogpArgs {
  const T* x;
  int64_t rows, ld, ld_dx;
  int classes, n_top;
  float scale;
  const int64_t* target;         // or null: no row has one
  const float* g;                // gradient: weights of the log probabilities ...
  const float* h;                // ... and of the entropies, each or null
  float* logp;                   // outputs, each or null
  float* entropy;
  float* stat;                   // [rows][2]: m, log s
  int* top_ids;                  // [rows][n_top]
  float* top_logp;
  T* dx;
  // rows in slices: their number, classes, and what each leaves
  int slices, slice;
  float4* part;                  // [rows][slices]: m, sum, sum of exp times d
  unsigned long long* keys;      // [rows][slices][n_top]

  LogpArgs of_rows(int64_t first, int64_t n) const {       // (of whole rows)
    LogpArgs a = *this;
    a.rows = n;
    a.x += first * ld;
    if (target) a.target += first;
    if (g) a.g += first;
    if (h) a.h += first;
    if (logp) a.logp += first;
    if (entropy) a.entropy += first;
    if (stat) a.stat += 2 * first;
    if (top_ids) a.top_ids += first * n_top;
    if (top_logp) a.top_logp += first * n_top;
    if (dx) a.dx += first * ld_dx;
    return a;
  }
};

// NaN above all numbers, -0 as 0, and nothing at 0 but places that hold no value
__device__ __forceinline__ unsigned ordered(float z) {
  if (z != z) return 0xffffffffu;
  const unsigned b = __builtin_bit_cast(unsigned, z + 0.0f);
  return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(unsigned k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// z = scale x rounded to fp32, the same wherever it is formed (never half of a
// fused multiply-add: z - m of the largest must be 0)
template <class T>
__device__ __forceinline__ float z_of(T x, float scale) {
#pragma clang fp contract(off)
  return to_float(x) * scale;
}

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LEAST = -1e5f;     // exp of it is 0, and 0 times it is 0

__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * LOG2E); }

// exp(d) and its share of sum exp(d) d; a NaN comes through the exponential
__device__ __forceinline__ void add_exp(float d, float& s, float& q) {
  const float w = exp_of(d);
  s += w;
  q = fmaf(w, fmaxf(d, LEAST), q);
}

// What a row's sums come to.  A row whose classes are all at minus infinity has
// no probabilities: its log probabilities are minus infinity, its entropy and
// its gradient 0.  A NaN or an infinity of the other sign makes everything NaN.
struct RowSums {
  float m, ln, entropy;
  bool empty;
};
__device__ __forceinline__ RowSums row_sums(float m, float s, float t) {
  RowSums r;
  r.empty = s == 0.f;
  r.m = r.empty ? -__builtin_inff() : m;
  r.ln = r.empty ? -__builtin_inff() : logf(s);
  r.entropy = r.empty ? 0.f : r.ln - t / s;
  return r;
}
__device__ __forceinline__ float log_prob(const RowSums& r, float z) {
  return r.empty ? -__builtin_inff() : (z - r.m) - r.ln;
}

// A value's place in the gradient, without the target's own share:
// -scale p (g + h (log p + H)), p = exp(z - m - log s).
struct Slope {
  float m, k, own;               // k = -log2 s; own: the target's share
  float g, h, add;               // -scale g, -scale h, H - log s
  bool entropies;
  // a row that `has` a target of log probability, and its sums
  __device__ __forceinline__ void set(float row_m, float ln, float entropy, float gi, float hi, float scale, bool none) {
    // (of a row without probabilities every p is exp(-infinity), and no weight counts:
    // one made from its log probability may be no number)
    if (none) gi = hi = 0.f;
    m = none ? 0.f : row_m;
    k = none ? -__builtin_inff() : -ln * LOG2E;
    own = scale * gi;
    g = -scale * gi;
    h = -scale * hi;
    add = none ? 0.f : entropy - ln;
    entropies = hi != 0.f;         // NaN too
  }
  // EH: with the entropies' share
  template <bool EH>
  __device__ __forceinline__ float at(float z) const {
    const float d = z - m;
    const float p = __builtin_amdgcn_exp2f(fmaf(d, LOG2E, k));
    if constexpr (!EH) return g * p;
    // (0 times the logarithm of 0 is 0: d is bounded, a NaN comes through p)
    return p * fmaf(h, fmaxf(d, LEAST) + add, g);
  }
};

template <class T>
__device__ __forceinline__ void put_row(const LogpArgs<T>& a, int64_t row, const RowSums& r, int64_t t, float zt) {
  if (a.logp)
    a.logp[row] = t < 0 ? 0.f : t >= a.classes ? __builtin_nanf("") : log_prob(r, zt);
  if (a.entropy) a.entropy[row] = r.entropy;
  if (a.stat) {
    a.stat[2 * row] = r.m;
    a.stat[2 * row + 1] = r.ln;
  }
}

template <class T>
__device__ __forceinline__ Slope slope_of(const LogpArgs<T>& a, int64_t row, const RowSums& r, int64_t t) {
  Slope s;
  // a row without a target has no log probability to change; a target past the
  // classes leaves no gradient that could be taken for one
  const float g = t < 0 || !a.g ? 0.f : t >= a.classes ? __builtin_nanf("") : a.g[row];
  s.set(r.m, r.ln, r.entropy, g, a.h ? a.h[row] : 0.f, a.scale, r.empty && t < a.classes);
  return s;
}

// A row's gradient: f(EH) with whether it has an entropies' share.
template <class F>
__device__ __forceinline__ void with_share(const Slope& sl, F&& f) {
  if (sl.entropies) f(std::true_type());
  else f(std::false_type());
}

// One vector's gradient; x0: its first class.
template <bool EH, class T>
__device__ __forceinline__ void put_slope(const Slope& sl, const Vec16<T>& v, float scale, T* dx, int j, int V, int64_t t) {
  constexpr int E = Vec16<T>::N;
  Vec16<T> o;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float y = sl.at<EH>(z_of(v.v[e], scale));
    o.v[e] = from_float<T>(y);
  }
  if (t >= j && t < j + E) {             // the vector that holds the target
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (j + e == t) o.v[e] = from_float<T>(sl.at<EH>(z_of(v.v[e], scale)) + sl.own);
  }
  if (j + E <= V) {
    store16(dx + j, o);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (j + e < V) dx[j + e] = o.v[e];
  }
}

// ---- rows of at most SMALL_MAX classes: G lanes a row, two values a lane -----
template <class T, int G, bool GRAD>
__global__ void __launch_bounds__(256) logp_small_kernel(const LogpArgs<T> a) {
  const int lane = threadIdx.x & 63, at = lane & (G - 1);
  const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / G;
  const bool live = row < a.rows;
  const int64_t r0 = live ? row : a.rows - 1;
  const T* const x = a.x + r0 * a.ld;
  const int64_t t = a.target ? a.target[r0] : -1;
  float z[2];
  bool in[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int j = at + e * G;
    in[e] = j < a.classes;
    z[e] = in[e] ? z_of(x[j], a.scale) : -__builtin_inff();
  }
  float m = fmaxf(z[0], z[1]);
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  const float mm = m == -__builtin_inff() ? 0.f : m;
  float s = 0.f, q = 0.f;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    add_exp(z[e] - mm, s, q);
  }
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) {
    s += __shfl_xor(s, o, 64);
    q += __shfl_xor(q, o, 64);
  }
  const RowSums r = row_sums(mm, s, q);
  if (live && at == 0) put_row(a, row, r, t, t >= 0 && t < a.classes ? z_of(x[t], a.scale) : 0.f);
  if (a.n_top > 0) {
    unsigned k[2];
    int rank[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 2; ++e) k[e] = in[e] ? ordered(z[e]) : 0u;
    for (int c = 0; c < G; ++c) {
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const unsigned other = __shfl(k[f], c, G);
        const int oj = c + f * G;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          rank[e] += other > k[e] || (other == k[e] && oj < at + e * G);
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (live && in[e] && rank[e] < a.n_top) {
        const int64_t o = row * a.n_top + rank[e];
        if (a.top_ids) a.top_ids[o] = at + e * G;
        if (a.top_logp) a.top_logp[o] = log_prob(r, z[e]);
      }
  }
  if constexpr (GRAD) {
    const Slope sl = slope_of(a, r0, r, t);
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (live && in[e]) {
        const int j = at + e * G;
        const float y = sl.entropies ? sl.at<true>(z[e]) : sl.at<false>(z[e]);
        a.dx[row * a.ld_dx + j] = from_float<T>(y + (j == t ? sl.own : 0.f));
      }
  }
}

// ---- longer rows: one workgroup each ----------------------------------------
template <int W>
struct BlockShare {
  float m[W], s[W], q[W];
  unsigned lane[64 * W];
  unsigned from;
  int count;
  unsigned long long best[W];
  unsigned long long key[TOP_CAP];
};

// NV: 16-byte vectors of the row that a thread holds; 0: none, the row is read
// anew for each pass over it.  PART: a slice of the row, whose sums and
// alternatives logp_join_kernel puts together.
template <class T, int THREADS, int NV, bool GRAD, bool PART = false>
__global__ void __launch_bounds__(THREADS) logp_row_kernel(const LogpArgs<T> a) {
  constexpr int E = Vec16<T>::N, W = THREADS / 64;
  __shared__ BlockShare<W> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = PART ? blockIdx.y : blockIdx.x;
  const int start = PART ? (int)blockIdx.x * a.slice : 0;
  const T* const x = a.x + row * a.ld + start;
  const int V = PART ? min(a.slice, a.classes - start) : a.classes;

  auto load = [&](int j) {           // E values from class j on, minus infinity past the last
    if (j + E <= V) return load16(x + j);
    // (j may lie past the row altogether)
    Vec16<T> r;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      r.v[e] = from_float<T>(-__builtin_inff());
      if (j + e < V) r.v[e] = x[j + e];
    }
    return r;
  };
  Vec16<T> keep[NV > 0 ? NV : 1];
  if constexpr (NV > 0) {
#pragma unroll
    for (int v = 0; v < NV; ++v) keep[v] = load((v * THREADS + tid) * E);
  }
  // The row's values are wanted anew: what was made of them is not kept in registers.
  auto again = [&] {
    if constexpr (NV > 0) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        uint4 u = __builtin_bit_cast(uint4, keep[v]);
        asm volatile("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));
        keep[v] = __builtin_bit_cast(Vec16<T>, u);
      }
    }
  };
  // f(j, vector): each of the thread's vectors that begins inside the row
  auto each = [&](auto&& f) {
    if constexpr (NV > 0) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int j = (v * THREADS + tid) * E;
        if (j < V) f(j, keep[v]);
      }
    } else {
      constexpr int U = 4;
      int j = tid * E;
      for (; j + (U - 1) * THREADS * E < V; j += U * THREADS * E) {
        Vec16<T> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) r[u] = load(j + u * THREADS * E);
#pragma unroll
        for (int u = 0; u < U; ++u) f(j + u * THREADS * E, r[u]);
      }
      for (; j < V; j += THREADS * E) f(j, load(j));
    }
  };
  const int64_t t = !PART && a.target ? a.target[row] : -1;
  float zt = 0.f;
  if (tid == 0 && t >= 0 && t < V) zt = z_of(x[t], a.scale);

  // maximum and sums
  float m = -__builtin_inff(), s = 0.f, q = 0.f, lane_max;
  auto add = [&](const Vec16<T>& r, float mm) {
#pragma unroll
    for (int e = 0; e < E; ++e) add_exp(z_of(r.v[e], a.scale) - mm, s, q);
  };
  if constexpr (NV > 0) {
    // (scale > 0 keeps the order, also as rounded)
    each([&](int, const Vec16<T>& r) {
#pragma unroll
      for (int e = 0; e < E; ++e) m = fmaxf(m, to_float(r.v[e]));
    });
    lane_max = m = z_of(m, a.scale);
    m = wave_max(m);
    if constexpr (W > 1) {
      if (lane == 0) sh.m[wave] = m;
      __syncthreads();
      m = sh.m[0];
#pragma unroll
      for (int w = 1; w < W; ++w) m = fmaxf(m, sh.m[w]);
    }
    m = m == -__builtin_inff() ? 0.f : m;
    again();
    each([&](int, const Vec16<T>& r) { add(r, m); });
  } else {
    // running: the sums are relative to the thread's maximum so far, looked at once
    // for U vectors (whose places past the row hold minus infinity)
    float run = -__builtin_inff();
    m = 0.f;
    constexpr int U = 4;
    for (int j = tid * E; j < V; j += U * THREADS * E) {
      Vec16<T> r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = load(j + u * THREADS * E);
      float c = -__builtin_inff();
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) c = fmaxf(c, to_float(r[u].v[e]));
      c = z_of(c, a.scale);
      if (c > run) {
        const float d = run - c, w = exp_of(d);       // run may be minus infinity: s is 0 then
        q = w == 0.f ? 0.f : w * (q + s * d);
        s *= w;
        run = m = c;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) add(r[u], m);
    }
    const float own = run;
    lane_max = run;
    m = wave_max(run);
    if (lane == 0) sh.m[wave] = m;
    __syncthreads();
    m = sh.m[0];
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, sh.m[w]);
    m = m == -__builtin_inff() ? 0.f : m;
    const float d = own - m, w = exp_of(d);
    // a thread without a finite value may still hold a NaN
    if (own != -__builtin_inff()) {
      q = w == 0.f ? 0.f * q : w * (q + s * d);
      s *= w;
    }
  }
  s = wave_sum(s);
  q = wave_sum(q);
  if constexpr (W > 1) {
    if (lane == 0) {
      sh.s[wave] = s;
      sh.q[wave] = q;
    }
    if (tid == 0) sh.count = 0;
    __syncthreads();
    s = q = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      s += sh.s[w];
      q += sh.q[w];
    }
  } else {
    if (tid == 0) sh.count = 0;
  }
  const RowSums r = row_sums(m, s, q);
  const int64_t piece = PART ? row * a.slices + blockIdx.x : 0;
  if (tid == 0) {
    if constexpr (PART) a.part[piece] = make_float4(m, s, q, 0.f);
    else put_row(a, row, r, t, zt);
  }

  if constexpr (GRAD) {
    const Slope sl = slope_of(a, row, r, t);
    T* const dx = a.dx + row * a.ld_dx;
    again();
    with_share(sl, [&](auto eh) {
      each([&](int j, const Vec16<T>& v) { put_slope<eh.value>(sl, v, a.scale, dx, j, V, t); });
    });
    return;
  }
  if (a.n_top <= 0) return;

  // The n_top-th largest of 64 maxima, each of the lanes of one place in all waves.
  // (A lane that met nothing but NaN has minus infinity: no more than the values there.)
  unsigned from = ordered(lane_max);
  if constexpr (W > 1) {
    sh.lane[tid] = from;
    __syncthreads();
  }
  if (wave == 0) {
    unsigned most = from;
#pragma unroll
    for (int w = 1; w < W; ++w) most = max(most, sh.lane[w * 64 + lane]);
    from = 0;
#pragma unroll
    for (int b = 31; b >= 0; --b) {
      const unsigned c = from | (1u << b);
      if (__popcll(__ballot(most >= c)) >= a.n_top) from = c;
    }
    if constexpr (W > 1)
      if (lane == 0) sh.from = from;
  }
  __syncthreads();
  if constexpr (W > 1) from = sh.from;
  const float least = unordered(from);
  again();
  const bool bad = s != s;                       // a NaN in the row: no maximum tells where
  if (lane_max >= least || bad)
    each([&](int j, const Vec16<T>& v) {
      float top = to_float(v.v[0]);
#pragma unroll
      for (int e = 1; e < E; ++e) top = fmaxf(top, to_float(v.v[e]));
      if (z_of(top, a.scale) < least && !bad) return;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float z = z_of(v.v[e], a.scale);
        if (!(z < least) && j + e < V) {         // a NaN too
          const int at = atomicAdd(&sh.count, 1);
          if (at < TOP_CAP) sh.key[at] = (unsigned long long)ordered(z) << 32 | (unsigned)~(unsigned)(start + j + e);
        }
      }
    });
  __syncthreads();
  const int n = sh.count;
  auto put = [&](int rank, unsigned long long key) {
    if constexpr (PART) {
      a.keys[piece * a.n_top + rank] = key;
      return;
    }
    const int64_t o = row * a.n_top + rank;
    if (a.top_ids) a.top_ids[o] = (int)~(unsigned)key;
    if (a.top_logp) a.top_logp[o] = log_prob(r, unordered((unsigned)(key >> 32)));
  };
  if (n <= TOP_CAP) {
    if constexpr (PART)                          // a slice of fewer classes than alternatives
      for (int k = V + tid; k < a.n_top; k += THREADS) put(k, 0);
    for (int c = tid; c < n; c += THREADS) {
      const unsigned long long key = sh.key[c];
      int rank = 0;
      for (int o = 0; o < n; ++o) rank += sh.key[o] > key;
      if (rank < a.n_top) put(rank, key);
    }
    return;
  }
  unsigned long long last = ~0ull;      // above every key: the lowest index of a NaN has a smaller one
  for (int k = 0; k < a.n_top; ++k) {
    unsigned long long best = 0;
    again();
    each([&](int j, const Vec16<T>& v) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const unsigned o = j + e < V ? ordered(z_of(v.v[e], a.scale)) : 0u;
        const unsigned long long key = (unsigned long long)o << 32 | (unsigned)~(unsigned)(start + j + e);
        if (o && (k == 0 || key < last) && key > best) best = key;
      }
    });
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      const unsigned long long other = __shfl_xor(best, o, 64);
      best = other > best ? other : best;
    }
    if (lane == 0) sh.best[wave] = best;
    __syncthreads();
    best = sh.best[0];
    for (int w = 1; w < W; ++w) best = sh.best[w] > best ? sh.best[w] : best;
    __syncthreads();
    last = best;
    if (tid == 0) put(k, best);
  }
}

// ---- few long rows: the slices of a row put together -----------------------------
constexpr int MAX_SLICES = 64;
constexpr int JOIN_KEYS = 512;       // at most; slices times alternatives

template <class T>
__global__ void __launch_bounds__(256) logp_join_kernel(const LogpArgs<T> a) {
  __shared__ unsigned long long key[JOIN_KEYS];
  __shared__ float sums[3];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, n = a.slices * a.n_top;
  for (int k = tid; k < n; k += 256) key[k] = a.keys[row * n + k];
  if (tid < 64) {
    const float4 p = tid < a.slices ? a.part[row * a.slices + tid] : make_float4(0.f, 0.f, 0.f, 0.f);
    const bool some = p.y != 0.f;    // a NaN too
    float m = wave_max(some ? p.x : -__builtin_inff());
    m = m == -__builtin_inff() ? 0.f : m;
    const float d = p.x - m, w = exp_of(d);
    const float s = wave_sum(some ? p.y * w : 0.f);
    const float q = wave_sum(!some ? 0.f : w == 0.f ? 0.f * p.z : w * (p.z + p.y * d));
    if (tid == 0) {
      sums[0] = m;
      sums[1] = s;
      sums[2] = q;
    }
  }
  __syncthreads();
  const RowSums r = row_sums(sums[0], sums[1], sums[2]);
  if (tid == 0) {
    const int64_t t = a.target ? a.target[row] : -1;
    put_row(a, row, r, t, t >= 0 && t < a.classes ? z_of(a.x[row * a.ld + t], a.scale) : 0.f);
  }
  for (int c = tid; c < n; c += 256) {
    const unsigned long long own = key[c];
    if (own == 0) continue;
    int rank = 0;
    for (int o = 0; o < n; ++o) rank += key[o] > own;
    if (rank >= a.n_top) continue;
    const int64_t o = row * a.n_top + rank;
    if (a.top_ids) a.top_ids[o] = (int)~(unsigned)own;
    if (a.top_logp) a.top_logp[o] = log_prob(r, unordered((unsigned)(own >> 32)));
  }
}

// ---- the gradient from statistics kept earlier ------------------------------
template <class T>
struct GradArgs {
  const T* x;
  T* dx;
  int64_t ld, ld_dx;
  int64_t rows;
  int classes, per_row;            // workgroups a row
  float scale;
  const int64_t* target;
  const float* stat;
  const float* entropy;
  const float* g;
  const float* h;

  GradArgs of_rows(int64_t first, int64_t n) const {
    GradArgs a = *this;
    a.rows = n;
    a.x += first * ld;
    a.dx += first * ld_dx;
    if (target) a.target += first;
    a.stat += 2 * first;
    if (entropy) a.entropy += first;
    if (g) a.g += first;
    if (h) a.h += first;
    return a;
  }
};

constexpr int GRAD_VECS = 2;

// L threads a row and GRAD_VECS vectors each, or of longer rows 256 and several
// workgroups a row.  Bound by the bytes (16000 x 2000 bf16 32 us, 4.0 TB/s); us by 256 threads
// and by the fewest that hold a row: 16000 x 10 f32 12.2, 3.3; x 100 f32 13.6, 5.1; x 500 bf16
// 16.9, 13.1.  Vectors a thread, 4, 2, 1: 16000 x 2000 bf16 38.7, 32.1, 33.0; 1001 x 5003 f32
// 12.0, 9.5, 9.2.
template <class T, int L>
__global__ void __launch_bounds__(256) logp_grad_kernel(const GradArgs<T> a) {
  constexpr int E = Vec16<T>::N;
  const int64_t row = L == 256 ? blockIdx.x / a.per_row : (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
  if (row >= a.rows) return;
  const int first = L == 256 ? (int)(blockIdx.x - row * a.per_row) * 256 * E * GRAD_VECS : 0;
  const int lane = threadIdx.x % L;
  const int V = a.classes;
  const T* const x = a.x + row * a.ld;
  T* const dx = a.dx + row * a.ld_dx;
  Vec16<T> v[GRAD_VECS];
#pragma unroll
  for (int u = 0; u < GRAD_VECS; ++u) {
    const int j = first + (u * L + lane) * E;
    if (j + E <= V) {
      v[u] = load16(x + j);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[u].v[e] = from_float<T>(0.f);
        if (j + e < V) v[u].v[e] = x[j + e];
      }
    }
  }
  const int64_t t = a.target ? a.target[row] : -1;
  Slope sl;
  const float ln = a.stat[2 * row + 1];
  sl.set(a.stat[2 * row], ln, a.h ? a.entropy[row] : 0.f, t < 0 || !a.g ? 0.f : t >= V ? __builtin_nanf("") : a.g[row],
         a.h ? a.h[row] : 0.f, a.scale, ln == -__builtin_inff() && t < V);
  with_share(sl, [&](auto eh) {
#pragma unroll
    for (int u = 0; u < GRAD_VECS; ++u) {
      const int j = first + (u * L + lane) * E;
      if (j < V) put_slope<eh.value>(sl, v[u], a.scale, dx, j, V, t);
    }
  });
}

// ---- launches ----------------------------------------------------------------
// How a call's rows are cut, and where its workspace holds what.
struct LogpPlan {
  int slices = 0, slice = 0;     // 0: rows stay whole
  int64_t keys = 0, stat = 0, entropy = 0, bytes = 0;
};
// Few long rows would leave most of the card idle: they are cut so that about 256
// workgroups have 16 KB or more each.  Another launch or two costs about 4 us each, so rows
// stay whole below 96 KB, with a gradient below 256 KB (us, cut and whole: 1 x 131072 f32
// 10.3, 20, with its gradient 9.8, 29; 20 x 50000 f32 11.1, 15), and 65 or more always (100 x 131072
// f16 with 20 alternatives 23.7, 24.1; 100 x 50000 f32 16.8, 12.7; 128 x 131072 f32 17.2, 15.8).
LogpPlan logp_plan(int64_t size, int64_t rows, int64_t classes, int n_top, bool grad) {
  LogpPlan p;
  const int64_t bytes = classes * size;
  if (rows < 1 || rows > 64 || bytes < (grad ? 256 : 96) * 1024) return p;
  int64_t s = 256 / rows;
  if (s > MAX_SLICES) s = MAX_SLICES;
  if (s > bytes / 16384) s = bytes / 16384;
  if (n_top > 0 && s > JOIN_KEYS / n_top) s = JOIN_KEYS / n_top;
  if (s < 2) return p;
  p.slice = (int)(((classes + s - 1) / s + 63) / 64 * 64);
  p.slices = (int)((classes + p.slice - 1) / p.slice);
  p.keys = rows * p.slices * 16;
  p.stat = p.keys + rows * p.slices * n_top * 8;
  p.entropy = p.stat + rows * 8;
  p.bytes = p.entropy + rows * 4;
  return p;
}

template <class T>
hipError_t launch_parts(LogpArgs<T> a, const LogpPlan& p, char* work, hipStream_t s) {
  a.slices = p.slices;
  a.slice = p.slice;
  a.part = reinterpret_cast<float4*>(work);
  a.keys = reinterpret_cast<unsigned long long*>(work + p.keys);
  const dim3 grid((unsigned)p.slices, (unsigned)a.rows);
  const int64_t vecs = p.slice / Vec16<T>::N;
  hipError_t e;
  if (vecs <= 1024) e = op_launch(logp_row_kernel<T, 256, 4, false, true>, grid, dim3(256), s, a);
  else if (vecs <= 4096) e = op_launch(logp_row_kernel<T, 1024, 4, false, true>, grid, dim3(1024), s, a);
  else e = op_launch(logp_row_kernel<T, 1024, 0, false, true>, grid, dim3(1024), s, a);
  if (e != hipSuccess) return e;
  return op_launch(logp_join_kernel<T>, dim3((unsigned)a.rows), dim3(256), s, a);
}

template <class T>
hipError_t launch_grad(GradArgs<T> a, hipStream_t s) {
  constexpr int64_t per = Vec16<T>::N * GRAD_VECS;        // of a thread
  a.per_row = (int)((a.classes + 256 * per - 1) / (256 * per));
  auto go = [&](auto l) {
    constexpr int L = decltype(l)::value;
    const int64_t per_row = L == 256 ? a.per_row : 1;
    return op_each_launch(a.rows, 256, 256 / L, per_row, [&](int64_t first, int64_t n) {
      return op_launch(logp_grad_kernel<T, L>, dim3((unsigned)((n * per_row + 256 / L - 1) / (256 / L))), dim3(256), s,
                       a.of_rows(first, n));
    });
  };
  if (a.classes <= 4 * per) return go(std::integral_constant<int, 4>());
  if (a.classes <= 16 * per) return go(std::integral_constant<int, 16>());
  if (a.classes <= 64 * per) return go(std::integral_constant<int, 64>());
  return go(std::integral_constant<int, 256>());
}

template <class T, bool GRAD>
hipError_t launch_logp(const LogpArgs<T>& a, int units, hipStream_t s) {
  if (a.classes <= SMALL_MAX) {
    const int half = (a.classes + 1) / 2;
    auto go = [&](auto g) {
      constexpr int G = decltype(g)::value;
      return op_each_launch(a.rows, 256, 256 / G, 1, [&](int64_t first, int64_t n) {
        return op_launch(logp_small_kernel<T, G, GRAD>, dim3((unsigned)((n + 256 / G - 1) / (256 / G))), dim3(256), s,
                         a.of_rows(first, n));
      });
    };
    if (half <= 8) return go(std::integral_constant<int, 8>());
    if (half <= 16) return go(std::integral_constant<int, 16>());
    if (half <= 32) return go(std::integral_constant<int, 32>());
    return go(std::integral_constant<int, 64>());
  }
  const int64_t vecs = (a.classes + Vec16<T>::N - 1) / Vec16<T>::N;
  // Threads of a workgroup and vectors in a thread's registers, as measured (us, MI355X):
  //   no gradient, 256 threads and 2 vectors, against none in registers: 8192 x 2500 bf16 with 8
  //   alternatives 27, 33.  Longer rows are read in passes, the second (for alternatives) by few
  //   lanes: 8192 x 16000 bf16 by 256 threads 101, 512 137, 512 and 4 vectors 126;
  //   2049 x 50021 bf16 by 256 80, by 512 75; 1000 x 131072 f32 by 256 119, 512 107, 1024 102.
  //   Gradient: 8192 x 5000 bf16, 256 and 4 46, 256 and none 58; 4096 x 32768 bf16, 512 and 8 120,
  //   1024 and 4 124, 512 and none 147; 4096 x 16384 f32 113, 108, 123; 600 x 50000 bf16, 512 and none 41,
  //   1024 54, 1024 and 8 51; 1000 x 131072 bf16 by 512 177, by 1024 170.
  //   Few rows wait for one another's steps, so more threads: 1 x 32768 bf16, 1024 and 4 7.5, 512 and 8
  //   8.2; 20 x 50000 f32 by 1024 15, by 512 17.
#define NF_ROW(TH, NV)                                                                               \
  return op_each_launch(a.rows, TH, 1, 1, [&](int64_t first, int64_t n) {                            \
    return op_launch(logp_row_kernel<T, TH, NV, GRAD>, dim3((unsigned)n), dim3(TH), s, a.of_rows(first, n)); \
  })
  const bool few = a.rows <= units;
  if (vecs <= 64) NF_ROW(64, 1);
  if (vecs <= 256) NF_ROW(64, 4);
  if (vecs <= 512) NF_ROW(256, 2);
  if constexpr (GRAD) {
    if (vecs <= 1024) NF_ROW(256, 4);
    if (vecs <= 2048) NF_ROW(512, 4);
    if (vecs <= 4096) {
      if (sizeof(T) == 4 || few) NF_ROW(1024, 4);
      NF_ROW(512, 8);
    }
  } else {
    if (few && vecs <= 4096) NF_ROW(1024, 4);
    if (!few && vecs <= 4096) NF_ROW(256, 0);
  }
  if (!few && vecs <= 16384) NF_ROW(512, 0);
  NF_ROW(1024, 0);
#undef NF_ROW
}

nf_status check_logits(const void* x, int dtype, int64_t rows, int64_t classes, int64_t ld, float scale) {
  if (!op_float_type(dtype)) return op_fail(NF_EINVAL, "logits must be fp32, bf16 or fp16 (dtype %d)", dtype);
  if (rows < 0 || classes < 1) return op_fail(NF_EINVAL, "rows must be at least 0, classes at least 1");
  if (rows > 0x7fffffff || classes > (1 << 30))
    return op_fail(NF_ESHAPE, "at most 2^31 - 1 rows of 2^30 classes");
  if (ld < classes) return op_fail(NF_ESHAPE, "the row pitch is smaller than the classes");
  if (rows > 0 && ld > INT64_MAX / 4 / rows) return op_fail(NF_ESHAPE, "rows times pitch does not fit");
  if (!(scale > 0.f && scale < __builtin_inff())) return op_fail(NF_EINVAL, "scale must be positive and finite");
  if (rows > 0 && !x) return op_fail(NF_EINVAL, "NULL logits");
  if (!op_aligned(x, (uintptr_t)op_size(dtype))) return op_fail(NF_EINVAL, "logits are not aligned to their elements");
  return NF_OK;
}

// The gradient may be written over the logits themselves, and over nothing else
// that the call reads.
nf_status check_gradient(const void* x, int64_t ld, const void* dx, int64_t ld_dx, int dtype, int64_t rows,
                         int64_t classes) {
  if (!dx) return op_fail(NF_EINVAL, "NULL gradient");
  if (ld_dx < classes) return op_fail(NF_ESHAPE, "the gradient's row pitch is smaller than the classes");
  if (ld_dx > INT64_MAX / 4 / rows) return op_fail(NF_ESHAPE, "rows times pitch does not fit");
  if (!op_aligned(dx, (uintptr_t)op_size(dtype))) return op_fail(NF_EINVAL, "the gradient is not aligned to its elements");
  const int64_t e = op_size(dtype);
  const OpArray in{x, 1, 0, rows, ld * e, classes * e}, out{dx, 1, 0, rows, ld_dx * e, classes * e};
  if (op_share(in, out) && !op_same(in, out))
    return op_fail(NF_EINVAL, "the gradient overlaps the logits without being them");
  return NF_OK;
}

// A row's results are written while others' inputs are read: no output shares bytes with the
// targets, weights or statistics.  (The gradient and the logits: check_gradient.)
nf_status check_apart(std::initializer_list<OpArray> out, std::initializer_list<OpArray> in) {
  for (const OpArray& a : out)
    for (const OpArray& b : in)
      if (op_overlap(a.p, a.span(), b.p, b.span()) && op_share(a, b))
        return op_fail(NF_EINVAL, "an output overlaps the logits, targets, weights or statistics");
  return NF_OK;
}
OpArray column(const void* p, int64_t rows, int64_t bytes) { return {p, 1, 0, 1, 0, rows * bytes}; }

// The workspace may be left out: rows then stay whole.
nf_status check_logp_work(const void* work, int64_t have, const LogpPlan& p) {
  if (!work || !p.slices) return NF_OK;
  if (!op_aligned(work, 16)) return op_fail(NF_EINVAL, "the workspace is not aligned to 16 bytes");
  if (have < p.bytes)
    return op_fail(NF_ESHAPE, "the workspace has %lld bytes, %lld are needed", (long long)have, (long long)p.bytes);
  return NF_OK;
}

}  // namespace

int op_compute_units() {
  thread_local int at = -1, units = 0;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return 0;
  }
  if (dev != at) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) {
      (void)hipGetLastError();
      return 0;
    }
    at = dev;
    units = n;
  }
  return units;
}

}  // namespace nf

using namespace nf;

extern "C" {

int64_t nf_logprobs_work(int32_t dtype, int64_t rows, int64_t classes, int32_t n_top, int32_t gradient) {
  op_begin();
  if (!op_float_type(dtype) || rows < 0 || rows > 0x7fffffff || classes < 1 || classes > (1 << 30) || n_top < 0 ||
      n_top > NF_TOP_MAX || (!gradient && n_top > classes)) {
    op_fail(NF_EINVAL, "sizes or type that the call would refuse");
    return -1;
  }
  return logp_plan(op_size(dtype), rows, classes, gradient ? 0 : n_top, gradient != 0).bytes;
}

nf_status nf_logprobs(const void* d_logits, int32_t dtype, int64_t rows, int64_t classes, int64_t ld, float scale,
                      const int64_t* d_targets, int32_t n_top, float* d_logp, float* d_entropy, float* d_stat,
                      int32_t* d_top_ids, float* d_top_logp, void* d_work, int64_t work_bytes, void* stream) {
  op_begin();
  const nf_status st = check_logits(d_logits, dtype, rows, classes, ld, scale);
  if (st != NF_OK) return st;
  if (n_top < 0 || n_top > NF_TOP_MAX) return op_fail(NF_EINVAL, "n_top must be in 0 .. %d", NF_TOP_MAX);
  if (n_top > classes) return op_fail(NF_ESHAPE, "more alternatives than classes");
  if (n_top > 0 && !d_top_ids && !d_top_logp) return op_fail(NF_EINVAL, "alternatives without a place for them");
  if (rows == 0) return NF_OK;
  const LogpPlan plan = logp_plan(op_size(dtype), rows, classes, n_top, false);
  nf_status more = check_logp_work(d_work, work_bytes, plan);
  if (more != NF_OK) return more;
  const int64_t size = op_size(dtype);
  more = check_apart({column(d_logp, rows, 4), column(d_entropy, rows, 4), column(d_stat, rows, 8),
                      column(d_top_ids, rows, 4 * n_top), column(d_top_logp, rows, 4 * n_top)},
                     {{d_logits, 1, 0, rows, ld * size, classes * size}, column(d_targets, rows, 8)});
  if (more != NF_OK) return more;
  const int units = op_compute_units();
  if (units <= 0) return op_fail(NF_EDEVICE, "no usable HIP device");
  return with_type(dtype, [&](auto e) {
    typedef decltype(e) T;
    LogpArgs<T> a{};
    a.x = static_cast<const T*>(d_logits);
    a.rows = rows;
    a.ld = ld;
    a.classes = (int)classes;
    a.n_top = n_top;
    a.scale = scale;
    a.target = d_targets;
    a.logp = d_logp;
    a.entropy = d_entropy;
    a.stat = d_stat;
    a.top_ids = d_top_ids;
    a.top_logp = d_top_logp;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return op_result(plan.slices && d_work ? launch_parts<T>(a, plan, static_cast<char*>(d_work), s)
                                           : launch_logp<T, false>(a, units, s),
                     "log probabilities");
  });
}

nf_status nf_logprobs_train(const void* d_logits, int32_t dtype, int64_t rows, int64_t classes, int64_t ld,
                            float scale, const int64_t* d_targets, const float* d_g_logp, const float* d_g_entropy,
                            float* d_logp, float* d_entropy, float* d_stat, void* d_dlogits, int64_t ld_d,
                            void* d_work, int64_t work_bytes, void* stream) {
  op_begin();
  nf_status st = check_logits(d_logits, dtype, rows, classes, ld, scale);
  if (st != NF_OK) return st;
  if (rows == 0) return NF_OK;
  if (d_g_logp && !d_targets) return op_fail(NF_EINVAL, "weights of log probabilities without targets");
  st = check_gradient(d_logits, ld, d_dlogits, ld_d, dtype, rows, classes);
  if (st != NF_OK) return st;
  const LogpPlan plan = logp_plan(op_size(dtype), rows, classes, 0, true);
  st = check_logp_work(d_work, work_bytes, plan);
  if (st != NF_OK) return st;
  const int64_t size = op_size(dtype);
  const OpArray targets = column(d_targets, rows, 8), g = column(d_g_logp, rows, 4), h = column(d_g_entropy, rows, 4);
  const OpArray sums[] = {column(d_logp, rows, 4), column(d_entropy, rows, 4), column(d_stat, rows, 8)};
  st = check_apart({sums[0], sums[1], sums[2]}, {{d_logits, 1, 0, rows, ld * size, classes * size}, targets, g, h});
  if (st == NF_OK)
    st = check_apart({{d_dlogits, 1, 0, rows, ld_d * size, classes * size}}, {targets, g, h, sums[0], sums[1], sums[2]});
  if (st != NF_OK) return st;
  const int units = op_compute_units();
  if (units <= 0) return op_fail(NF_EDEVICE, "no usable HIP device");
  return with_type(dtype, [&](auto e) {
    typedef decltype(e) T;
    LogpArgs<T> a{};
    a.x = static_cast<const T*>(d_logits);
    a.rows = rows;
    a.ld = ld;
    a.ld_dx = ld_d;
    a.classes = (int)classes;
    a.scale = scale;
    a.target = d_targets;
    a.g = d_g_logp;
    a.h = d_g_entropy;
    a.logp = d_logp;
    a.entropy = d_entropy;
    a.stat = d_stat;
    a.dx = static_cast<T*>(d_dlogits);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!plan.slices || !d_work) return op_result(launch_logp<T, true>(a, units, s), "log probabilities and gradient");
    // the slices' sums, and the gradient from what they come to
    char* const work = static_cast<char*>(d_work);
    if (!a.stat) a.stat = reinterpret_cast<float*>(work + plan.stat);
    if (!a.entropy) a.entropy = reinterpret_cast<float*>(work + plan.entropy);
    hipError_t he = launch_parts<T>(a, plan, work, s);
    if (he != hipSuccess) return op_result(he, "log probabilities");
    GradArgs<T> g{};
    g.x = a.x;
    g.dx = a.dx;
    g.ld = ld;
    g.ld_dx = ld_d;
    g.rows = rows;
    g.classes = (int)classes;
    g.scale = scale;
    g.target = d_targets;
    g.stat = a.stat;
    g.entropy = a.entropy;
    g.g = d_g_logp;
    g.h = d_g_entropy;
    return op_result(launch_grad<T>(g, s), "gradient of log probabilities");
  });
}

nf_status nf_logprobs_grad(const void* d_logits, int32_t dtype, int64_t rows, int64_t classes, int64_t ld,
                           float scale, const int64_t* d_targets, const float* d_stat, const float* d_entropy,
                           const float* d_g_logp, const float* d_g_entropy, void* d_dlogits, int64_t ld_d,
                           void* stream) {
  op_begin();
  nf_status st = check_logits(d_logits, dtype, rows, classes, ld, scale);
  if (st != NF_OK) return st;
  if (rows == 0) return NF_OK;
  if (!d_stat) return op_fail(NF_EINVAL, "NULL statistics");
  if (d_g_logp && !d_targets) return op_fail(NF_EINVAL, "weights of log probabilities without targets");
  if (d_g_entropy && !d_entropy) return op_fail(NF_EINVAL, "weights of entropies without the entropies");
  st = check_gradient(d_logits, ld, d_dlogits, ld_d, dtype, rows, classes);
  if (st != NF_OK) return st;
  const int64_t size = op_size(dtype);
  st = check_apart({{d_dlogits, 1, 0, rows, ld_d * size, classes * size}},
                   {column(d_targets, rows, 8), column(d_stat, rows, 8), column(d_entropy, rows, 4),
                    column(d_g_logp, rows, 4), column(d_g_entropy, rows, 4)});
  if (st != NF_OK) return st;
  const int units = op_compute_units();
  if (units <= 0) return op_fail(NF_EDEVICE, "no usable HIP device");
  return with_type(dtype, [&](auto e) {
    typedef decltype(e) T;
    GradArgs<T> a{};
    a.x = static_cast<const T*>(d_logits);
    a.dx = static_cast<T*>(d_dlogits);
    a.ld = ld;
    a.ld_dx = ld_d;
    a.rows = rows;
    a.classes = (int)classes;
    a.scale = scale;
    a.target = d_targets;
    a.stat = d_stat;
    a.entropy = d_entropy;
    a.g = d_g_logp;
    a.h = d_g_entropy;
    return op_result(launch_grad<T>(a, static_cast<hipStream_t>(stream)), "gradient of log probabilities");
  });
}

}  // extern "C"
