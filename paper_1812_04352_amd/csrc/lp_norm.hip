// Layer norm over the features of every row, y = gamma (x - mean) / sqrt(var + eps) + beta, and its gradients.
//   forward:   one read of x, one write of y: a group of TPR threads holds a row in registers (C pieces of
//              16 bytes a thread), so the mean and then the mean square of x - mean, which does not cancel
//              as the mean square of x minus that of the mean would, cost no second read
//   backward:  with g = gamma dy, xh = (x - mean) r, r = 1 / sqrt(var + eps), over a row's q features
//                dx = r (g - mean g - xh mean(g xh)) (+ dr),  dgamma = sum_rows dy xh,  dbeta = sum_rows dy
//              one read of x, dy (and dr), one write of dx: the statistics are formed again from the row at
//              hand, in two rounds of exchanges (the sums of x and g, then of x - mean, its square and its product
//              with g).
//              A thread keeps the same features of all its rows, so it sums their dgamma and dbeta in
//              registers; a workgroup adds its groups' in order and writes one row of partial sums, which a
//              second kernel adds in fp64 (a single workgroup writes the gradients themselves).
//   The first mean is rounded, and so is the sum that it comes from: a row's x - mean does not sum to 0, but to what that
//   mean is off by. Its mean is taken off x - mean, and the square of it off the mean square, so that a row whose mean
//   exceeds its spread by far loses nothing, and equal values leave 0 (without that a row of 223 values 3300 in fp32
//   was off by hundredths). bf16 rows that a group holds do not need it: where the mean exceeds the spread, the values
//   are multiples of one step, 2^9 at most, and 2^15 of them sum exactly; the mean is then off by half an fp32 step,
//   2^-17 of the values' own, and the spread is at least that by the root of q: off by 2^-9.5 of it at most. (It takes
//   1 to 8 % of the time back, 8192 x 4096 f32 97 -> 98 us, 20000 x 700 f32 49 -> 52, 5003 x 1111 f16 19.1 -> 20.5.)
// Bound by memory: 8192 x 4096 bf16 24 us forward (5.6 TB/s), 64 us back with dr (4.2; the sum of 256 rows of partial sums,
// one of each workgroup, of which there is one a CU, 4.7 of them; without the next rows requested ahead and with sums by
// LDS exchanges 97). Rows that no group can hold are read again for every pass.
#include <algorithm>
#include <type_traits>

#include "lp_internal.h"
#include "lp_mm.h"

namespace lp {
namespace norm {

using mm::GVec;

// Threads of a workgroup whose groups have TPR each: whole groups, about 256 forward and about 1024 back, where every
// workgroup leaves a row of partial sums.
constexpr int threads_forward(int tpr) { return tpr > 256 ? tpr : 256 / tpr * tpr; }
constexpr int threads_back(int tpr) { return 1024 / tpr * tpr; }

// A thread's pieces of a row: features (c TPR + t) V .. of the group's thread t
template <typename T, int TPR, int C>
struct Piece {
  static constexpr int V = 16 / (int)sizeof(T);
  typedef typename GVec<T, V>::type Vec;
  Vec v[C];
  static __device__ __forceinline__ int first(int t, int c) { return (c * TPR + t) * V; }
  // Whole pieces: one that the row's end cuts is read from V values before that end, and those behind it from there too
  // (so that no lane branches and nothing waits for the load); cut() makes them what they stand for.
  __device__ __forceinline__ void load(const T* row, int t, int q) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (q >= V) {
        v[c] = *reinterpret_cast<const Vec*>(row + min(first(t, c), q - V));
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) v[c][k] = first(t, c) + k < q ? row[first(t, c) + k] : (T)0.f;
      }
    }
  }
  // What follows converts the values again: kept as floats from pass to pass they would not fit the registers.
  __device__ __forceinline__ void forget() {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
    for (int c = 0; c < C; ++c) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      u32x4 x = __builtin_bit_cast(u32x4, v[c]);
      asm volatile("" : "+v"(x));
      v[c] = __builtin_bit_cast(Vec, x);
    }
#endif
  }
  // zeros behind the row's end
  __device__ __forceinline__ void cut(int t, int q) {
    if (q < V) return;
    const int bits = (V - q % V) % V * 8 * (int)sizeof(T);  // of the values before the cut piece
#pragma unroll
    for (int c = 0; c < C; ++c) {
      typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
      const int n = first(t, c);
      const u64x2 x = __builtin_bit_cast(u64x2, v[c]);
      u64x2 y = {0, 0};
      if (bits >= 64) y[0] = x[1] >> (bits - 64);
      else if (bits > 0) y[0] = x[0] >> bits | x[1] << (64 - bits), y[1] = x[1] >> bits;
      const bool whole = n + V <= q, none = n >= q;
      y[0] = whole ? x[0] : none ? 0 : y[0];
      y[1] = whole ? x[1] : none ? 0 : y[1];
      v[c] = __builtin_bit_cast(Vec, y);
    }
  }
  static __device__ __forceinline__ void store(T* row, int t, int q, int c, const float (&f)[V]) {
    const int n = first(t, c);
    if (n + V <= q) {
      Vec x;
#pragma unroll
      for (int k = 0; k < V; ++k) x[k] = (T)f[k];
      *reinterpret_cast<Vec*>(row + n) = x;
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (n + k < q) row[n + k] = (T)f[k];
    }
  }
};

// A value's sum over rows of 16 lanes, the same in all of them, by data-parallel moves, whose latency is a vector
// instruction's
__device__ __forceinline__ float row_sum(float v) {
#ifdef __HIP_DEVICE_COMPILE__
#define LP_ADD_MOVED(ctrl) v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, 0xf, 0xf, true))
  LP_ADD_MOVED(0xb1);   // quad_perm 1, 0, 3, 2
  LP_ADD_MOVED(0x4e);   // quad_perm 2, 3, 0, 1
  LP_ADD_MOVED(0x141);  // the other quad of eight lanes: row_half_mirror
  LP_ADD_MOVED(0x140);  // the other half of sixteen: row_mirror
#undef LP_ADD_MOVED
#endif
  return v;
}

// The wave's sum of a value in every lane: its four rows' sums in order
__device__ __forceinline__ float wave_sum(float v) {
  v = row_sum(v);
#ifdef __HIP_DEVICE_COMPILE__
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 16 * i));
  v = (r[0] + r[1]) + (r[2] + r[3]);
#endif
  return v;
}

// Sums of up to M values (two or four) over a group of TPR threads, the same in all of them. Groups wider than a wave
// exchange through the LDS, where every lane adds its group's waves in order; of many waves (M W > 16: 8192 x 4096 f32
// back 98 us, 116 in order) every row of 16 lanes reads one a lane. `at` alternates between two halves, so that one
// barrier a sum is enough (a wave that writes a half again has passed the barrier behind which all have read it).
template <int TPR, int NT, int M>
struct GroupSum {
  static constexpr int W = TPR / 64;  // waves of a group
  typedef float Values __attribute__((ext_vector_type(M)));
  typedef Values Lds[2][NT / 64];
  Lds& lds;
  int at = 0;
  template <int N>
  __device__ __forceinline__ void operator()(float (&s)[N]) {
    if constexpr (TPR < 64) {
#pragma unroll
      for (int o = TPR / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += __shfl_xor(s[i], o, 64);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
    }
    if constexpr (TPR > 64) {
      static_assert(W <= 16, "a row of lanes");
      const int wave = threadIdx.x >> 6, w = threadIdx.x & 15;
      Values v = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = s[i];
      if ((threadIdx.x & 63) == 0) lds[at][wave] = v;
      __syncthreads();
      const Values* g = lds[at] + wave / W * W;
      if constexpr (M * W > 16) {
        v = g[min(w, W - 1)];
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = row_sum(w < W ? v[i] : 0.f);
      } else {
#pragma unroll
        for (int k = 0; k < W; ++k) {
          v = g[k];
#pragma unroll
          for (int i = 0; i < N; ++i) s[i] = k ? s[i] + v[i] : v[i];
        }
      }
      at ^= 1;
    }
  }
};

// Values of this type are taken about the mean of x - mean
template <typename T> constexpr bool CENTRE = !std::is_same<T, __bf16>::value;

// The mean square of x - mean less the square of its mean, `off` (never below 0; a NaN stays one)
__device__ __forceinline__ float variance(float square, float off) {
  const float v = square - off * off;
  return v < 0.f ? 0.f : v;
}

template <typename T, int TPR, int C, int NT>
__global__ __launch_bounds__(NT) void k_forward(const T* x, const T* gamma, const T* beta, T* y, int B, int q, float eps) {
  typedef Piece<T, TPR, C> P;
  constexpr int V = P::V, G = NT / TPR;
  typedef GroupSum<TPR, NT, 2> Sum;
  __shared__ typename Sum::Lds lds;
  Sum sum{lds};
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  P ga, be;
  if (gamma) ga.load(gamma, t, q), ga.cut(t, q);
  if (beta) be.load(beta, t, q), be.cut(t, q);
  const float n = (float)q;
  for (long r0 = (long)blockIdx.x * G; r0 < B; r0 += (long)gridDim.x * G) {  // (the same rounds for every thread)
    const long r = r0 + g;
    P p;
    p.load(x + min(r, (long)B - 1) * q, t, q);
    p.cut(t, q);
    float s1[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < V; ++k) s1[0] += (float)p.v[c][k];
    sum(s1);
    const float mean = s1[0] / n;
    float s2[CENTRE<T> ? 2 : 1] = {};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = P::first(t, c) + k < q ? (float)p.v[c][k] - mean : 0.f;
        s2[0] = fmaf(d, d, s2[0]);
        if constexpr (CENTRE<T>) s2[1] += d;
      }
    sum(s2);
    float off = 0.f;
    if constexpr (CENTRE<T>) off = s2[1] / n;
    const float rstd = 1.f / sqrtf(variance(s2[0] / n, off) + eps);
    if (r >= B) continue;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float f[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        f[k] = ((float)p.v[c][k] - mean - off) * rstd;
        if (gamma) f[k] *= (float)ga.v[c][k];
        if (beta) f[k] += (float)be.v[c][k];
      }
      P::store(y + r * q, t, q, c, f);
    }
  }
}

struct BackArgs {
  const void *x, *gamma, *dy, *dr;  // gamma, dr nullable
  void *dx, *dgamma, *dbeta;        // nullable
  float* part;                      // [workgroups][2][q] partial sums of dgamma and dbeta
  int B, q;
  int rows;                         // of a workgroup
  float eps;
};

// A workgroup's sums of one array, of its groups in order: to the array itself or to a row of partial sums
template <typename T, int TPR, int C>
__device__ __forceinline__ void add_groups(const float (&acc)[C][16 / sizeof(T)], float* lds, int q, T* out, float* part) {
  typedef Piece<T, TPR, C> P;
  constexpr int V = P::V, NT = threads_back(TPR), G = NT / TPR, ROW = TPR * C * V;
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  if constexpr (G == 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int n = P::first(t, c) + k;
        if (n < q) {
          if (part) part[n] = acc[c][k];
          else out[n] = (T)acc[c][k];
        }
      }
    }
  } else {
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < V; k += 4)
        *reinterpret_cast<float4*>(lds + g * ROW + P::first(t, c) + k) = make_float4(acc[c][k], acc[c][k + 1], acc[c][k + 2], acc[c][k + 3]);
    __syncthreads();
    for (int n = threadIdx.x; n < q; n += NT) {
      float s = lds[n];
#pragma unroll
      for (int i = 1; i < G; ++i) s += lds[i * ROW + n];
      if (part) part[n] = s;
      else out[n] = (T)s;
    }
  }
}

// FULL: q = TPR C V, no piece behind the row's end. The next round's rows are requested before this one's sums (one
// piece a thread: registers), so that a workgroup a CU keeps memory busy.
template <typename T, int TPR, int C, bool FULL>
__global__ __launch_bounds__(threads_back(TPR)) void k_backward(BackArgs a) {
  typedef Piece<T, TPR, C> P;
  constexpr int V = P::V, NT = threads_back(TPR), G = NT / TPR;
  constexpr bool AHEAD = C == 1;
  typedef GroupSum<TPR, NT, CENTRE<T> ? 4 : 2> Sum;
  __shared__ typename Sum::Lds lds;
  __shared__ __attribute__((aligned(16))) float sums[G == 1 ? 4 : NT * C * V];
  Sum sum{lds};
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR, q = FULL ? TPR * C * V : a.q;
  const T *x = static_cast<const T*>(a.x), *dy = static_cast<const T*>(a.dy), *dr = a.dx ? static_cast<const T*>(a.dr) : nullptr;
  T* dx = static_cast<T*>(a.dx);
  P ga;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int k = 0; k < V; ++k) ga.v[c][k] = (T)1.f;
  if (a.gamma) ga.load(static_cast<const T*>(a.gamma), t, q), ga.cut(t, q);
  const float n = (float)q;
  float dg[C][V] = {}, db[C][V] = {};
  const long r1 = min((long)a.B, (long)(blockIdx.x + 1) * a.rows);
  struct {
    P x, d, r;
  } now, next;
  const auto load = [&](auto& to, long r) {
    const long at = min(r, r1 - 1) * q;
    to.x.load(x + at, t, q);
    to.d.load(dy + at, t, q);
    if (dr) to.r.load(dr + at, t, q);
  };
  long r0 = (long)blockIdx.x * a.rows;
  if (AHEAD && r0 < r1) load(now, r0 + g);
  for (; r0 < r1; r0 += G) {  // (the same rounds for every thread)
    const long r = r0 + g;
    if constexpr (AHEAD) {
      if (r0 + G < r1) load(next, r + G);
    } else {
      load(now, r);
    }
    if constexpr (!FULL) now.x.cut(t, q), now.d.cut(t, q);  // (dr's values behind the end are not used, those of a cut piece are)
    if constexpr (!FULL) {
      if (dr) now.r.cut(t, q);
    }
    float s1[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        s1[0] += (float)now.x.v[c][k];
        s1[1] = fmaf((float)now.d.v[c][k], (float)ga.v[c][k], s1[1]);
      }
    sum(s1);
    const float mean = s1[0] / n, m1 = s1[1] / n;
    float s2[CENTRE<T> ? 3 : 2] = {};
    if constexpr (!AHEAD) now.x.forget(), now.d.forget(), ga.forget();
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = FULL || P::first(t, c) + k < q ? (float)now.x.v[c][k] - mean : 0.f;
        s2[0] = fmaf(d, d, s2[0]);
        s2[1] = fmaf((float)now.d.v[c][k] * (float)ga.v[c][k], d, s2[1]);
        if constexpr (CENTRE<T>) s2[2] += d;
      }
    sum(s2);
    float off = 0.f;
    if constexpr (CENTRE<T>) off = s2[2] / n;
    const float rstd = 1.f / sqrtf(variance(s2[0] / n, off) + a.eps), m2 = (s2[1] / n - off * m1) * rstd;
    if constexpr (!AHEAD) now.x.forget(), now.d.forget(), ga.forget();
    if (r < r1) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float f[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float dk = (float)now.d.v[c][k], xh = ((float)now.x.v[c][k] - mean - off) * rstd;
          f[k] = rstd * (dk * (float)ga.v[c][k] - m1 - xh * m2);
          if (dr) f[k] += (float)now.r.v[c][k];
          dg[c][k] = fmaf(dk, xh, dg[c][k]);
          db[c][k] += dk;
        }
        if (dx) P::store(dx + r * q, t, q, c, f);
      }
    }
    if constexpr (AHEAD) now = next;
  }
  float* part = a.part ? a.part + (size_t)blockIdx.x * 2 * q : nullptr;
  if (a.dgamma) add_groups<T, TPR, C>(dg, sums, q, static_cast<T*>(a.dgamma), part);
  if (a.dbeta) add_groups<T, TPR, C>(db, sums, q, static_cast<T*>(a.dbeta), part ? part + q : nullptr);
}

// dgamma and dbeta from the partial sums, in fp64 and in order: 64 features by 16 runs of rows a workgroup
template <typename T>
__global__ __launch_bounds__(1024) void k_sum(const float* part, int rows, int q, T* dgamma, T* dbeta) {
  __shared__ double sh[16][64];
  const int half = (q + 63) / 64, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const bool second = (int)blockIdx.x >= half;
  const int n = ((int)blockIdx.x - (second ? half : 0)) * 64 + lane;
  T* out = second ? dbeta : dgamma;
  const int per = (rows + 15) / 16, i1 = min(rows, (w + 1) * per);
  double s = 0.0;
  if (n < q && out) {
    const float* p = part + (second ? q : 0) + n;
    int i = w * per;
    for (; i + 8 <= i1; i += 8) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = p[(size_t)(i + k) * 2 * q];
#pragma unroll
      for (int k = 0; k < 8; ++k) s += (double)v[k];
    }
    for (; i < i1; ++i) s += (double)p[(size_t)i * 2 * q];
  }
  sh[w][lane] = s;
  __syncthreads();
  if (w || n >= q || !out) return;
  for (int k = 1; k < 16; ++k) s += sh[k][lane];
  out[n] = (T)(float)s;
}

// ---- rows that no group holds: every pass reads them again

typedef GroupSum<1024, 1024, 4> LongSum;

// A row's statistics: its first mean, what that is off by, 1 / sqrt(var + eps), and with dy the means of g and g xh
struct LongStats {
  float mean, off, rstd, m1, m2;
  __device__ __forceinline__ float xh(float x) const { return (x - mean - off) * rstd; }
};

// over a workgroup of 1024
template <typename T>
__device__ __forceinline__ LongStats long_stats(const T* x, const T* dy, const T* gamma, int q, float eps, LongSum& sum) {
  const float n = (float)q;
  LongStats r;
  float s1[2] = {0.f, 0.f};
  for (int i = threadIdx.x; i < q; i += 1024) {
    s1[0] += (float)x[i];
    if (dy) s1[1] += (gamma ? (float)gamma[i] : 1.f) * (float)dy[i];
  }
  sum(s1);
  r.mean = s1[0] / n, r.m1 = s1[1] / n;
  float s2[3] = {0.f, 0.f, 0.f};
  for (int i = threadIdx.x; i < q; i += 1024) {
    const float d = (float)x[i] - r.mean;
    s2[0] = fmaf(d, d, s2[0]);
    s2[1] += d;
    if (dy) s2[2] = fmaf((gamma ? (float)gamma[i] : 1.f) * (float)dy[i], d, s2[2]);
  }
  sum(s2);
  r.off = s2[1] / n;
  r.rstd = 1.f / sqrtf(variance(s2[0] / n, r.off) + eps);
  r.m2 = (s2[2] / n - r.off * r.m1) * r.rstd;
  return r;
}

template <typename T>
__global__ __launch_bounds__(1024) void k_forward_long(const T* x, const T* gamma, const T* beta, T* y, int B, int q, float eps) {
  __shared__ LongSum::Lds lds;
  LongSum sum{lds};
  for (long r = blockIdx.x; r < B; r += gridDim.x) {
    const LongStats s = long_stats<T>(x + r * q, nullptr, nullptr, q, eps, sum);
    for (int i = threadIdx.x; i < q; i += 1024) {
      float f = s.xh((float)x[r * q + i]);
      if (gamma) f *= (float)gamma[i];
      if (beta) f += (float)beta[i];
      y[r * q + i] = (T)f;
    }
  }
}

// dx, and the statistics of every row (mean, off, rstd) for the weights' gradients
template <typename T>
__global__ __launch_bounds__(1024) void k_backward_long(BackArgs a, float4* stats) {
  __shared__ LongSum::Lds lds;
  LongSum sum{lds};
  const T *x = static_cast<const T*>(a.x), *dy = static_cast<const T*>(a.dy), *dr = static_cast<const T*>(a.dr);
  const T* gamma = static_cast<const T*>(a.gamma);
  T* dx = static_cast<T*>(a.dx);
  const int q = a.q;
  for (long r = blockIdx.x; r < a.B; r += gridDim.x) {
    const LongStats s = long_stats<T>(x + r * q, dy + r * q, gamma, q, a.eps, sum);
    if (threadIdx.x == 0) stats[r] = make_float4(s.mean, s.off, s.rstd, 0.f);
    if (!dx) continue;
    for (int i = threadIdx.x; i < q; i += 1024) {
      float f = s.rstd * ((gamma ? (float)gamma[i] : 1.f) * (float)dy[r * q + i] - s.m1 - s.xh((float)x[r * q + i]) * s.m2);
      if (dr) f += (float)dr[r * q + i];
      dx[r * q + i] = (T)f;
    }
  }
}

// partial sums of dgamma and dbeta: a thread's feature over a run of rows (grid y)
template <typename T>
__global__ __launch_bounds__(256) void k_weights_long(BackArgs a, const float4* stats) {
  const int i = blockIdx.x * 256 + threadIdx.x, q = a.q;
  if (i >= q) return;
  const T *x = static_cast<const T*>(a.x), *dy = static_cast<const T*>(a.dy);
  float dg = 0.f, db = 0.f;
  const long r1 = min((long)a.B, (long)(blockIdx.y + 1) * a.rows);
  for (long r = (long)blockIdx.y * a.rows; r < r1; ++r) {
    const float4 s = stats[r];
    const float d = (float)dy[r * q + i];
    dg = fmaf(d, ((float)x[r * q + i] - s.x - s.y) * s.z, dg);
    db += d;
  }
  float* part = a.part + (size_t)blockIdx.y * 2 * q;
  part[i] = dg;
  part[q + i] = db;
}

// ---------------------------------------------------------------- launches

// The group that holds a row of q values: threads and pieces a thread (tpr = 0: none does).
struct Group {
  int tpr, c;
};

#define LP_FORWARD_GROUPS(CASE)                                                                                        \
  CASE(4, 1) CASE(8, 1) CASE(16, 1) CASE(32, 1) CASE(64, 1) CASE(64, 2) CASE(64, 3) CASE(64, 4) CASE(128, 3) CASE(256, 2) \
  CASE(256, 3) CASE(256, 4) CASE(512, 3) CASE(1024, 2) CASE(1024, 3) CASE(1024, 4)
#define LP_BACKWARD_GROUPS(CASE)                                                                                   \
  CASE(4, 1) CASE(8, 1) CASE(16, 1) CASE(32, 1) CASE(64, 1) CASE(128, 1) CASE(192, 1) CASE(256, 1) CASE(320, 1) \
  CASE(384, 1) CASE(512, 1) CASE(768, 1) CASE(1024, 1) CASE(1024, 2)

// The first group of the list (by its pieces) that holds the row
inline Group forward_group(size_t esz, int q) {
  const int pieces = mm::ceil_div(q * (long)esz, 16);
#define LP_CASE(TPR, C) \
  if (pieces <= TPR * C) return {TPR, C};
  LP_FORWARD_GROUPS(LP_CASE)
#undef LP_CASE
  return {0, 0};
}

inline Group backward_group(size_t esz, int q) {
  const int pieces = mm::ceil_div(q * (long)esz, 16);
#define LP_CASE(TPR, C) \
  if (pieces <= TPR * C) return {TPR, C};
  LP_BACKWARD_GROUPS(LP_CASE)
#undef LP_CASE
  return {0, 0};
}

// Rows of a backward workgroup: a round of its groups, more where 256 workgroups (one a CU, each with all the waves it can
// hold) would not take all rows so. A round is a chain of load, two sums and store, longer than what the second kernel
// takes for another row of partial sums; with at least one round (two, four), microseconds in a graph: 1000 x 220 f32 7.5
// (8.8, 12.4), 64 x 4096 bf16 7.8 (9.2, 13.0), 512 x 4096 11.9 (11.5, 15.0), 8192 x 64 7.9 (8.6, 10.9), 2000 x 1111 f16 14.2
// (14.2, 19.4); dx alone 4.0 (5.9, 9.8), 3.9 (5.8, 9.8), 4.5 (6.3, 10.3), 3.2 (4.5, 6.9), 8.6 (8.7, 14.3).
inline int backward_rows(int groups, int B) {
  const int most = 256;
  const int rows = std::max(mm::ceil_div(B, most), groups);
  return mm::ceil_div(std::min(rows, 2048 * groups), groups) * groups;  // (at most 2048 rows in a sum of fp32)
}

template <typename T, int TPR, int C>
hipError_t forward_g(const NormArgs& a, hipStream_t st) {
  constexpr int NT = threads_forward(TPR), G = NT / TPR;
  const unsigned grid = (unsigned)std::min<long>(mm::ceil_div(a.B, G), 4096);
  k_forward<T, TPR, C, NT><<<grid, NT, 0, st>>>((const T*)a.x, (const T*)a.gamma, (const T*)a.beta, (T*)a.y, a.B, a.q, (float)a.eps);
  return hipGetLastError();
}

template <typename T>
hipError_t forward_t(const NormArgs& a, hipStream_t st) {
  const Group g = forward_group(sizeof(T), a.q);
#define LP_CASE(TPR, C) \
  if (g.tpr == TPR && g.c == C) return forward_g<T, TPR, C>(a, st);
  LP_FORWARD_GROUPS(LP_CASE)
#undef LP_CASE
  k_forward_long<T><<<(unsigned)std::min(a.B, 2048), 1024, 0, st>>>((const T*)a.x, (const T*)a.gamma, (const T*)a.beta, (T*)a.y, a.B,
                                                                  a.q, (float)a.eps);
  return hipGetLastError();
}

template <typename T>
hipError_t backward_t(const NormArgs& a, hipStream_t st) {
  const NormLayout l = norm_layout(a.dtype, a.B, a.q);
  char* w = static_cast<char*>(a.ws);
  const bool weights = a.dgamma || a.dbeta;
  BackArgs b{a.x, a.gamma, a.dy, a.dr, a.dx, a.dgamma, a.dbeta, l.groups > 1 ? reinterpret_cast<float*>(w + l.part) : nullptr,
             a.B, a.q, l.rows, (float)a.eps};
  const Group g = backward_group(sizeof(T), a.q);
  if (g.tpr) {
    const bool full = a.q == g.tpr * g.c * (16 / (int)sizeof(T));
#define LP_CASE(TPR, C)                                                                                \
  if (g.tpr == TPR && g.c == C) {                                                                      \
    if (full) k_backward<T, TPR, C, true><<<(unsigned)l.groups, threads_back(TPR), 0, st>>>(b);        \
    else k_backward<T, TPR, C, false><<<(unsigned)l.groups, threads_back(TPR), 0, st>>>(b);            \
  }
    LP_BACKWARD_GROUPS(LP_CASE)
#undef LP_CASE
  } else {
    float4* stats = reinterpret_cast<float4*>(w + l.stats);
    b.part = reinterpret_cast<float*>(w + l.part);
    if (a.B) k_backward_long<T><<<(unsigned)std::min(a.B, 2048), 1024, 0, st>>>(b, stats);
    if (weights) k_weights_long<T><<<dim3((unsigned)mm::ceil_div(a.q, 256), (unsigned)l.groups), 256, 0, st>>>(b, stats);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && weights && b.part) {
    k_sum<T><<<2 * (unsigned)mm::ceil_div(a.q, 64), 1024, 0, st>>>(b.part, l.groups, a.q, (T*)a.dgamma, (T*)a.dbeta);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace norm

NormLayout norm_layout(int dtype, int B, int q) {
  const norm::Group g = norm::backward_group(dtype == 0 ? 4 : 2, q);
  NormLayout l{};
  if (g.tpr) {
    l.rows = norm::backward_rows(norm::threads_back(g.tpr) / g.tpr, B);
  } else {
    l.rows = std::min(2048, std::max(16, mm::ceil_div(B, 1024)));
    l.stats = ((size_t)B * 16 + 255) / 256 * 256;
  }
  l.groups = std::max(1, mm::ceil_div(B, l.rows));
  l.part = l.stats;  // (the rows' statistics come first)
  l.stats = 0;
  l.total = std::max<size_t>(l.part + (l.groups > 1 || !g.tpr ? (size_t)l.groups * 2 * q * 4 : 0), 256);
  return l;
}

hipError_t norm_forward_f32(const NormArgs& a, hipStream_t st) { return norm::forward_t<float>(a, st); }
hipError_t norm_forward_bf16(const NormArgs& a, hipStream_t st) { return norm::forward_t<__bf16>(a, st); }
hipError_t norm_forward_f16(const NormArgs& a, hipStream_t st) { return norm::forward_t<_Float16>(a, st); }
hipError_t norm_backward_f32(const NormArgs& a, hipStream_t st) { return norm::backward_t<float>(a, st); }
hipError_t norm_backward_bf16(const NormArgs& a, hipStream_t st) { return norm::backward_t<__bf16>(a, st); }
hipError_t norm_backward_f16(const NormArgs& a, hipStream_t st) { return norm::backward_t<_Float16>(a, st); }

}  // namespace lp
