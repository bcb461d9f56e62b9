// Orthogonalised updates W = alpha O + beta r of a batch of matrices [no][ni] (included by one translation
// unit per type of the products, T). O comes from the momentum v by an iteration whose products are all
// there is to it: X = v / (|v| + eps), |v| the root of the sum of squares, so that no singular value exceeds
// one, then `steps` times, with A the short side's A = X X^T (X^T X of a tall matrix),
//   X <- a X + (b A + c A^2) X   (tall: a X + X (b A + c A^2)),
// which maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.
// fp32 gradients: X, A and P are kept as sums of two f16 values (mm::Duo), a product of which is three of f16: half of
// what splitting floats into three bf16 parts costs, and no split in the products' loop. O is off by as much as with fp32
// products (of its norm, five steps with 3.4445, -4.775, 2.0315: noise of 220 x 220 1.2e-6, those 1.7e-6; of 4096 x 4096 3.2e-6,
// 4.8e-6; four directions a hundredfold 1.7e-5, 2.3e-5), but for matrices that one value carries (1e-6, 1e-7).
//   A and P = b A + c A^2 are symmetric: only tiles on and below the diagonal are formed, and stored on both sides of
//   it. a X is added in fp32 in the last product's epilogue, that of the last step updates W.
// 16-bit gradients: the products' operands X, A and P are in f16 whatever the gradient's type is. No singular value
// exceeds 1.3 or so, so that A and P are in range: f16 then rounds eight times finer than bf16 does. What rounding costs
// is kept down in two ways.
//   A rounding error of X grows like the small singular values do, by a factor a a step, where it is added to them, in
//   a X: the X of a X has 8 bits more, in an array of their own (2^-19 relative; an f16 more is no better), but for
//   the last two steps, behind which little grows. It takes 4096 x 4096 bf16 3 % more time, 2048 of 220 x 220 10 % (2846
//   -> 3124 us; by an f16 more in every step 3461).
//   In those, where X is nearly orthogonal, P is nearly (b + c) I and a X + P X a small difference: they form
//   (a + b + c) X + (P - (b + c) I) X, whose product is small and its rounding with it. (While singular values still
//   differ much it would mix strong directions into small ones.)
// O is off by 5e-4 to 1.5e-3 of its norm for noise, strong rows or columns, a few strong directions or singular values
// down to a thousandth (by X in f16 alone and P as it is 1e-3 to 1.5e-2), by 1.6e-3 where four directions exceed the noise
// a hundredfold (4e-2), by 2.2e-3 where a single value does (3.6e-3).
// Bound by the products: steps (3 n^2 k + n^3) operations, n the short and k the long side: 4096 x 4096 bf16 1585 us (0.87
// PFLOP/s of those; a symmetric product 83 us, the other one 139), 2048 of 220 x 220 f32 4593 us (95 TFLOP/s:
// memory, 3.6 to 5.4 TB/s, since X, A and P pass through it for every product).
#pragma once

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "lp_internal.h"
#include "lp_mm.h"

namespace lp {
namespace orth {

using mm::f32x16;
using mm::f32x4;
using mm::GVec;
using mm::Place;

// A and P are kept times A_UP, X times X_UP: as large as f16 holds where singular values stay below 3 (X 49152, P about
// 53000), so that what is small beside a matrix's largest values keeps its bits. (X times the root of n k, which
// brings the values of noise to 1, O of 220 x 220 f32 is off by 7e-6 to 1.1e-5 of its norm where a row, a column or a value
// carries that; so by 3e-7 to 1.4e-6.)
constexpr float A_UP = 256.f, X_UP = 16384.f;

// ---------------------------------------------------------------- v, its norm, and X

// m' = mu m + g (g without an m) to mo, and v = m' or g + mu m' (g without an mo)
template <typename TI, int V>
struct Momentum {
  const TI* g;
  const float* m;
  float* mo;
  float mu;
  int nesterov;
  typedef typename GVec<TI, V>::type VecI;
  typedef typename GVec<float, V>::type VecF;
  // v from g and m', of V values or the first n of them
  __device__ __forceinline__ void value(const float (&gf)[V], const float (&mf)[V], float (&v)[V]) const {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = !mo ? gf[k] : nesterov ? fmaf(mu, mf[k], gf[k]) : mf[k];
  }
  template <typename T>
  static __device__ __forceinline__ void get(const T* a, int n, float (&f)[V]) {
    if (n == V) {
      const auto x = *reinterpret_cast<const typename GVec<T, V>::type*>(a);
#pragma unroll
      for (int k = 0; k < V; ++k) f[k] = (float)x[k];
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) f[k] = k < n ? (float)a[k] : 0.f;
    }
  }
  // writes m' of the values from index i on
  __device__ __forceinline__ void update(size_t i, int n, float (&v)[V]) const {
    float gf[V], mf[V];
    get(g + i, n, gf);
    if (mo) {
      if (m) get(m + i, n, mf);
#pragma unroll
      for (int k = 0; k < V; ++k) mf[k] = m ? fmaf(mu, mf[k], gf[k]) : gf[k];
      if (n == V) {
        VecF x;
#pragma unroll
        for (int k = 0; k < V; ++k) x[k] = mf[k];
        *reinterpret_cast<VecF*>(mo + i) = x;
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (k < n) mo[i + k] = mf[k];
      }
    }
    value(gf, mf, v);
  }
  // v again, from m'
  __device__ __forceinline__ void again(size_t i, int n, float (&v)[V]) const {
    float gf[V] = {}, mf[V] = {};
    if (!mo || nesterov) get(g + i, n, gf);
    if (mo) get(static_cast<const float*>(mo) + i, n, mf);
    value(gf, mf, v);
  }
};

constexpr int VV = 4;           // values a thread takes at a time

// m', and partial sums of v's squares in fp64 (grid y: the matrix)
template <typename TI>
__global__ __launch_bounds__(256) void k_momentum(Momentum<TI, VV> u, size_t size, double* part) {
  __shared__ double sh[4];
  const size_t base = (size_t)blockIdx.y * size;
  double s = 0.0;
  for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * VV; i < size; i += (size_t)gridDim.x * 256 * VV) {
    float v[VV];
    u.update(base + i, (int)(size - i < VV ? size - i : VV), v);
#pragma unroll
    for (int k = 0; k < VV; ++k) s += (double)v[k] * (double)v[k];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = ((sh[0] + sh[1]) + sh[2]) + sh[3];
}

// Eight bits more than f16's: what it rounds off v, in 256ths of its value's last place, and the value with that (2^e: the
// place of a value h is 2^(e - 25), below 2^-14 that of 2^-14)
__device__ __forceinline__ int place(float h) { return max((int)(__builtin_bit_cast(uint32_t, h) >> 23 & 255) - 112, 1); }
__device__ __forceinline__ float rest(float v) {
  const float h = (float)(mm::f16)v;
  const float r = (v - h) * __builtin_bit_cast(float, (uint32_t)(127 + 33 - place(h)) << 23);
  return fminf(fmaxf(rintf(r), -127.f), 127.f);  // (a NaN gives -127, with its h a NaN again)
}
__device__ __forceinline__ float with_rest(float h, float r) {
  return fmaf(r, __builtin_bit_cast(float, (uint32_t)(127 - 33 + place(h)) << 23), h);
}

template <typename T>
__device__ __forceinline__ void put_values(T* row, int c, const float (&v)[8]) {
  if constexpr (std::is_same<T, mm::Duo>::value) {
    mm::BlockIO<mm::Duo>::put(reinterpret_cast<unsigned char*>(row + c), f32x4{v[0], v[1], v[2], v[3]});
    mm::BlockIO<mm::Duo>::put(reinterpret_cast<unsigned char*>(row + c) + 8, f32x4{v[4], v[5], v[6], v[7]});
  } else {
    typename GVec<T, 8>::type x;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (T)v[k];
    *reinterpret_cast<typename GVec<T, 8>::type*>(row + c) = x;
  }
}

// X = v up / (|v| + eps) in rows of ld values, zeros behind the ni that count (grid y: the matrix); lo (f16, nullable):
// its rest
template <typename TI, typename T>
__global__ __launch_bounds__(256) void k_scale(Momentum<TI, 8> u, int no, int ni, int ld, const double* part, int parts, double eps,
                                               double up, T* X, int8_t* lo, int ldlo) {
  __shared__ double sh;
  if (threadIdx.x < 64) {
    const double* p = part + (size_t)blockIdx.y * parts;
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 64) s += p[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (threadIdx.x == 0) sh = up / (sqrt(s) + eps);
  }
  __syncthreads();
  const double scale = sh;
  const size_t base = (size_t)blockIdx.y * no * ni;
  const uint32_t per = (uint32_t)(ld / 8);
  const size_t all = (size_t)no * per;
  X += (size_t)blockIdx.y * no * ld;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (size_t)gridDim.x * 256) {
    const size_t r = i / per;
    const int c = (int)(i - r * per) * 8, n = min(8, ni - c);
    float v[8] = {};
    if (n > 0) {
      u.again(base + r * ni + c, n, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k < n ? (float)((double)v[k] * scale) : 0.f;
    }
    put_values(X + r * ld, c, v);
    if constexpr (std::is_same<T, mm::f16>::value) {
      if (lo) {
        typename GVec<int8_t, 8>::type y;
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = (int8_t)rest(v[k]);
        *reinterpret_cast<typename GVec<int8_t, 8>::type*>(lo + ((size_t)blockIdx.y * no + r) * ldlo + c) = y;
      }
    }
  }
}

// ---------------------------------------------------------------- small matrices

// A matrix whose short side is at most SMALL_N and its long one at most SMALL_K takes one workgroup and one launch: X stays
// in registers in fp32 (as the accumulators of its product, the short side on rows: a tall matrix is
// turned as it is read and written), and the LDS holds what the products read, X and then A and P in its place,
// as the sum of two f16 values each (2^-22 relative): three instructions a product of two such values.
//   wave (wi, wj): rows 32 wi .., of A and P columns 32 wj .., of X the blocks wj, wj + 2, .. of 32 columns.
// 2048 of 64 x 64 f32 74 us (2.3 TB/s of g, m, r in and m, W out; 384 us by a launch for every product).
constexpr int SMALL_N = 64, SMALL_K = 256;

struct Half2 {
  mm::h16x8 h, l;
};

// KB: columns of X in blocks of 64
template <int KB>
struct SmallLds {
  static constexpr int XP = (64 * KB + 8) * 2, AP = (64 + 8) * 2;  // bytes a row
  __attribute__((aligned(16))) unsigned char x[2][64 * XP];
  __attribute__((aligned(16))) unsigned char a[2][64 * AP];
  double sum[4];
};

// a 32 x 32 block of values to both parts: rows m0 + lane % 32, columns n0 ..
template <int PITCH, int SIZE>
__device__ __forceinline__ void put_parts(unsigned char (&at)[2][SIZE], int m0, int n0, int lane, const f32x16& v, float up) {
  typedef _Float16 h16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    h16x4 h, l;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float f = v[4 * q + k] * up;
      h[k] = (_Float16)f;
      l[k] = (_Float16)(f - (float)h[k]);
    }
    const int o = (m0 + (lane & 31)) * PITCH + (n0 + 8 * q + 4 * (lane >> 5)) * 2;
    *reinterpret_cast<h16x4*>(at[0] + o) = h;
    *reinterpret_cast<h16x4*>(at[1] + o) = l;
  }
}

// eight contraction values from 16 kk + 8 (lane / 32) on of row r0 + lane % 32
template <int PITCH, int SIZE>
__device__ __forceinline__ Half2 get_rows(const unsigned char (&at)[2][SIZE], int r0, int kk, int lane) {
  const int o = (r0 + (lane & 31)) * PITCH + (16 * kk + 8 * (lane >> 5)) * 2;
  return {*reinterpret_cast<const mm::h16x8*>(at[0] + o), *reinterpret_cast<const mm::h16x8*>(at[1] + o)};
}
// and where the contraction runs over the rows: of column c0 + lane % 32 (transposing LDS reads, as in lp_mm.h)
template <int PITCH, int SIZE>
__device__ __forceinline__ Half2 get_columns(const unsigned char (&at)[2][SIZE], int c0, int kk, int lane) {
  Half2 r;
#ifdef __HIP_DEVICE_COMPILE__
  typedef __attribute__((address_space(3))) mm::s16x4 lds4;
  const int o = (16 * kk + 8 * (lane >> 5) + ((lane >> 2) & 3)) * PITCH + (c0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
  mm::s16x4 v[2][2];
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int j = 0; j < 2; ++j) v[p][j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(at[p] + o + 4 * j * PITCH));
  r.h = __builtin_bit_cast(mm::h16x8, __builtin_shufflevector(v[0][0], v[0][1], 0, 1, 2, 3, 4, 5, 6, 7));
  r.l = __builtin_bit_cast(mm::h16x8, __builtin_shufflevector(v[1][0], v[1][1], 0, 1, 2, 3, 4, 5, 6, 7));
#endif
  return r;
}
__device__ __forceinline__ f32x16 mma2(const Half2& n, const Half2& m, f32x16 c) {
  c = mm::mma(n.l, m.h, c);
  c = mm::mma(n.h, m.l, c);
  return mm::mma(n.h, m.h, c);
}

struct SmallArgs {
  int no, ni, steps;
  float a, b, c, alpha, beta;
  double eps, up;  // X is kept times up
};

// f(0) .. f(N - 1), the index a constant: registers have no other
template <int N, typename F>
__device__ __forceinline__ void blocks(F f) {
  if constexpr (N > 0) {
    blocks<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

template <typename TI, int KB, bool TALL>
__global__ __launch_bounds__(256) void k_small(Momentum<TI, 4> u, const TI* r, TI* W, SmallArgs a) {
  typedef SmallLds<KB> Lds;
  __shared__ Lds lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave >> 1, wj = wave & 1;
  const int n = TALL ? a.ni : a.no, k = TALL ? a.no : a.ni, m = 32 * wi + (lane & 31);
  const size_t base = (size_t)blockIdx.x * a.no * a.ni;
  // Block t of an array [no][ni], zeros behind the matrix (loads without a branch: those are of its first value), and back.
  // Pieces of four values of a wide matrix whose rows are such pieces.
  const bool pieces = !TALL && k % 4 == 0;
  const auto fetch = [&](auto* p, int t) {
    p += base;
    int ni = a.ni;
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("" : "+s"(ni));  // the indices are formed anew each time: kept, they would not fit the registers
#endif
    f32x16 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = 32 * (wj + 2 * t) + 8 * q + 4 * (lane >> 5);
      if (pieces) {
        const bool in = m < n && c < k;
        const auto y = *reinterpret_cast<const typename GVec<std::remove_cv_t<std::remove_pointer_t<decltype(p)>>, 4>::type*>(p + (in ? m * ni + c : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] = in ? (float)y[e] : 0.f;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = m < n && c + e < k;
          const float y = (float)p[in ? (TALL ? (c + e) * ni + m : m * ni + c + e) : 0];
          v[4 * q + e] = in ? y : 0.f;
        }
      }
    }
    return v;
  };
  const auto store = [&](auto* p, int t, const f32x16& v) {
    typedef std::remove_pointer_t<decltype(p)> TO;
    p += base;
    int ni = a.ni;
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("" : "+s"(ni));
#endif
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = 32 * (wj + 2 * t) + 8 * q + 4 * (lane >> 5);
      if (pieces) {
        typename GVec<TO, 4>::type y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (TO)v[4 * q + e];
        if (m < n && c < k) *reinterpret_cast<typename GVec<TO, 4>::type*>(p + m * ni + c) = y;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (m < n && c + e < k) p[TALL ? (c + e) * ni + m : m * ni + c + e] = (TO)v[4 * q + e];
      }
    }
  };
  f32x16 x[KB];
  double s = 0.0;
  blocks<KB>([&](auto t) {
    x[t] = fetch(u.g, t);
    if (u.mo) {
      f32x16 mo = x[t];
      if (u.m) {
        const f32x16 old = fetch(u.m, t);
#pragma unroll
        for (int e = 0; e < 16; ++e) mo[e] = fmaf(u.mu, old[e], mo[e]);
      }
      store(u.mo, t, mo);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][e] = u.nesterov ? fmaf(u.mu, mo[e], x[t][e]) : mo[e];
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) s += (double)x[t][e] * (double)x[t][e];
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) lds.sum[wave] = s;
  __syncthreads();
  const double scale = a.up / (sqrt(((lds.sum[0] + lds.sum[1]) + lds.sum[2]) + lds.sum[3]) + a.eps);
#pragma unroll
  for (int t = 0; t < KB; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) x[t][e] = (float)((double)x[t][e] * scale);
  const float down = (float)(1.0 / (a.up * a.up));
  for (int step = 0; step < a.steps; ++step) {
#pragma unroll
    for (int t = 0; t < KB; ++t) put_parts<Lds::XP>(lds.x, 32 * wi, 32 * (wj + 2 * t), lane, x[t], 1.f);
    __syncthreads();
    f32x16 A = 0.f, P = 0.f;
#pragma unroll 4
    for (int kk = 0; kk < 4 * KB; ++kk)
      A = mma2(get_rows<Lds::XP>(lds.x, 32 * wj, kk, lane), get_rows<Lds::XP>(lds.x, 32 * wi, kk, lane), A);
#pragma unroll
    for (int e = 0; e < 16; ++e) A[e] *= down;
    put_parts<Lds::AP>(lds.a, 32 * wi, 32 * wj, lane, A, A_UP);
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      P = mma2(get_rows<Lds::AP>(lds.a, 32 * wj, kk, lane), get_rows<Lds::AP>(lds.a, 32 * wi, kk, lane), P);
#pragma unroll
    for (int e = 0; e < 16; ++e) P[e] = a.b * A[e] + (a.c / (A_UP * A_UP)) * P[e];
    __syncthreads();  // every wave has read A
    put_parts<Lds::AP>(lds.a, 32 * wi, 32 * wj, lane, P, A_UP);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < KB; ++t) {
      f32x16 D = 0.f;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        D = mma2(get_columns<Lds::XP>(lds.x, 32 * (wj + 2 * t), kk, lane), get_rows<Lds::AP>(lds.a, 32 * wi, kk, lane), D);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][e] = a.a * x[t][e] + D[e] * (1.f / A_UP);
    }
    __syncthreads();  // and X and P
  }
  const float alpha = (float)(a.alpha / a.up);
  blocks<KB>([&](auto t) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[t][e] *= alpha;
    if (r) {
      const f32x16 old = fetch(r, t);
#pragma unroll
      for (int e = 0; e < 16; ++e) x[t][e] = fmaf(a.beta, old[e], x[t][e]);
    }
    store(W, t, x[t]);
  });
}

template <typename TI, int KB>
hipError_t small_t(const OrthArgs& a, hipStream_t st) {
  const double up = ldexp(1.0, (int)lround(0.5 * log2((double)a.no * a.ni)));
  const SmallArgs s{a.no, a.ni, a.steps, (float)a.a, (float)a.b, (float)a.c, (float)a.alpha, (float)a.beta, a.eps, up};
  constexpr int MOST = 1 << 22;  // workgroups a launch (2^32 threads are too many)
  for (int z0 = 0; z0 < a.N; z0 += MOST) {
    const size_t from = (size_t)z0 * a.no * a.ni;
    const unsigned grid = (unsigned)std::min(MOST, a.N - z0);
    const Momentum<TI, 4> u{(const TI*)a.g + from, a.m ? a.m + from : nullptr, a.mo ? a.mo + from : nullptr, (float)a.mu, a.nesterov};
    const TI* r = a.r ? (const TI*)a.r + from : nullptr;
    if (a.no > a.ni) k_small<TI, KB, true><<<grid, 256, 0, st>>>(u, r, (TI*)a.W + from, s);
    else k_small<TI, KB, false><<<grid, 256, 0, st>>>(u, r, (TI*)a.W + from, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ---------------------------------------------------------------- products

// A 32 x 32 block of a symmetric D (rows of ld values, whole 16-byte pieces) to its place on the other side of the diagonal:
// turned by way of the wave's LDS. Columns behind the last row of D get v's zeros.
template <typename T>
__device__ __forceinline__ void put_mirror(T* a, long ld, const Place& c, int i, int j, unsigned char* buf, const f32x4 (&v)[4]) {
  typedef mm::BlockIO<T> IO;
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      *reinterpret_cast<T*>(buf + (8 * q + 4 * (c.lane >> 5) + k) * IO::PITCH + (c.lane & 31) * sizeof(T)) = (T)v[q][k];
  mm::wave_in_order();
#pragma unroll
  for (int t = 0; t < IO::ITER; ++t) {
    const int id = c.lane + 64 * t, n = c.nw + 32 * j + id / IO::CPR, m = c.mw + 32 * i + id % IO::CPR * IO::V;
    const typename IO::Piece x = *reinterpret_cast<const typename IO::LPiece*>(buf + id / IO::CPR * IO::PITCH + id % IO::CPR * 16);
    if (n < c.N && m < ld) *reinterpret_cast<typename IO::Piece*>(a + (size_t)n * ld + m) = x;
  }
  mm::wave_in_order();
}

__device__ __forceinline__ void put_mirror(mm::Duo* a, long ld, const Place& c, int i, int j, unsigned char* buf, const f32x4 (&v)[4]) {
  typedef mm::BlockIO<mm::Duo> IO;
  const int m = c.lane & 31;
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      unsigned char* at = buf + (8 * q + 4 * (c.lane >> 5) + k) * IO::PITCH + m / 8 * 32 + m % 8 * 2;
      const _Float16 h = (_Float16)v[q][k];
      *reinterpret_cast<_Float16*>(at) = h;
      *reinterpret_cast<_Float16*>(at + 16) = (_Float16)(v[q][k] - (float)h);
    }
  IO::flush(a, ld, c.nw + 32 * j, c.N, c.mw + 32 * i, c.lane, buf);
}

// f D + b A + d I of a symmetric D, rows of ld values (A nullable)
template <typename T>
struct EpSym {
  struct Args {
    const T* A;
    T* out;
    int ld;
    size_t stride;  // of a matrix
    float f, b, d;
  };
  static __device__ __forceinline__ Args at(Args a, int z) {
    if (a.A) a.A += z * a.stride;
    a.out += z * a.stride;
    return a;
  }
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    mm::Rows<WHOLE, T, FM, FN> old(a.A, a.ld, c);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4];
        old.get(c, i, j, buf, v);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v[q][k] = c.row(i) < c.M && (WHOLE || c.feature(j, q) + k < c.lim) ? a.f * acc[i][j][4 * q + k] + a.b * v[q][k] : 0.f;
        if constexpr (std::is_same<T, mm::f16>::value) {
          if (a.d != 0.f && c.mt == c.nt) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int k = 0; k < 4; ++k) v[q][k] += c.row(i) == c.feature(j, q) + k && c.row(i) < c.M ? a.d : 0.f;
          }
        }
        mm::put_rows<WHOLE>(a.out, a.ld, c.upto(a.ld), c, i, j, buf, v);
        if (c.mt != c.nt) put_mirror(a.out, a.ld, c, i, j, buf, v);
      }
  }
};

// The array of rests, rows of ld values in whole 16-byte pieces, as a lane's quads block by block (compare mm::Rows), and back
template <int FM, int FN>
struct RestRows {
  typedef mm::BlockIO<int8_t> IO;
  int8_t* a;
  long ld;
  typename IO::Block next;
  __device__ __forceinline__ typename IO::Block fetch(const Place& c, int i, int j) const {
    static_assert(IO::ITER == 1 && IO::CPR == 2 && IO::V == 16, "a lane's piece");
    const int m = min(c.mw + 32 * i + c.lane / 2, c.M - 1), n = c.nw + 32 * j + c.lane % 2 * 16;
    return {{*reinterpret_cast<const typename IO::LPiece*>(a + (size_t)m * ld + min((long)n, ld - 16))}};
  }
  __device__ __forceinline__ RestRows(int8_t* a_, long ld_, const Place& c) : a(a_), ld(ld_) {
    if (a) next = fetch(c, 0, 0);
  }
  __device__ __forceinline__ void get(const Place& c, int i, int j, unsigned char* buf, f32x4 (&v)[4]) {
    const typename IO::Block b = next;
    if (i + 1 < FM) next = fetch(c, i + 1, j);
    else if (j + 1 < FN) next = fetch(c, 0, j + 1);
    IO::quads(b, buf, c, v);
  }
  __device__ __forceinline__ void put(const Place& c, int i, int j, unsigned char* buf, const f32x4 (&v)[4]) const {
    unsigned char* w = buf + (c.lane & 31) * IO::PITCH + (c.lane >> 5) * 4;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      typename IO::Quad x;
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = (int8_t)v[q][k];
      *reinterpret_cast<typename IO::Quad*>(w + 8 * q) = x;
    }
    mm::wave_in_order();
    const int m = c.mw + 32 * i + c.lane / 2, n = c.nw + 32 * j + c.lane % 2 * 16;
    const auto x = *reinterpret_cast<const typename IO::LPiece*>(buf + c.lane / 2 * IO::PITCH + c.lane % 2 * 16);
    if (m < c.M && n < ld) *reinterpret_cast<typename IO::LPiece*>(a + (size_t)m * ld + n) = x;
    mm::wave_in_order();
  }
};

// a X + d D. f16: lo (nullable) is the rest of X, and becomes that of the result (more: it will be asked for).
template <typename T>
struct EpNext {
  static constexpr bool LO = std::is_same<T, mm::f16>::value;
  struct Args {
    const T* X;
    T* out;
    int ld;
    size_t stride;
    float a, d;
    int8_t* lo;
    int ldlo;
    size_t slo;
    bool more;
  };
  static __device__ __forceinline__ Args at(Args a, int z) {
    a.X += z * a.stride;
    a.out += z * a.stride;
    if (LO && a.lo) a.lo += z * a.slo;
    return a;
  }
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    mm::Rows<WHOLE, T, FM, FN> X(a.X, a.ld, c);
    RestRows<FM, FN> lo(LO ? a.lo : nullptr, a.ldlo, c);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4];
        X.get(c, i, j, buf, v);
        if (LO && a.lo) {
          f32x4 w[4];
          lo.get(c, i, j, buf, w);
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[q][k] = with_rest(v[q][k], w[q][k]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v[q][k] = WHOLE || c.feature(j, q) + k < c.lim ? a.a * v[q][k] + a.d * acc[i][j][4 * q + k] : 0.f;
        mm::put_rows<WHOLE>(a.out, a.ld, c.upto(a.ld), c, i, j, buf, v);
        if (LO && a.more) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int k = 0; k < 4; ++k) v[q][k] = rest(v[q][k]);
          lo.put(c, i, j, buf, v);
        }
      }
  }
};

// W = alpha (a X + d D) + beta r, rows of N values (r nullable)
template <typename T, typename TO>
struct EpUpdate {
  struct Args {
    const T* X;
    int ld;
    size_t stride;   // of a matrix of X
    const TO* r;
    TO* W;
    size_t wstride;  // of r and W
    float a, d, alpha, beta;
  };
  static __device__ __forceinline__ Args at(Args a, int z) {
    a.X += z * a.stride;
    if (a.r) a.r += z * a.wstride;
    a.W += z * a.wstride;
    return a;
  }
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    mm::Rows<WHOLE, T, FM, FN> X(a.X, a.ld, c);
    mm::Rows<WHOLE, TO, FM, FN, false> r(a.r, c.N, c);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4], w[4];
        X.get(c, i, j, buf, v);
        r.get(c, i, j, buf, w);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (v[q] * a.a + mm::quad(acc[i][j], q) * a.d) * a.alpha + w[q] * a.beta;
        mm::put_rows<WHOLE>(a.W, c.N, c.lim, c, i, j, buf, v);
      }
  }
};

// The partial sums of a split contraction, a workgroup's own place
struct EpPart {
  struct Args {
    f32x4* part;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float*) {
    constexpr int NT = 64 * WGM * WGN;
    f32x4* out = a.part + threadIdx.x;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (c.row(i) >= c.M) continue;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) out[((i * FN + j) * 4 + q) * NT] = mm::quad(acc[i][j], q);
    }
  }
};

// A workgroup's matrix, tile and split. Workgroups go to the eight XCDs in turn, each with its own L2: of many matrices
// each keeps its tiles on one of them, where they share its operands (grid: 8 times the splits, tiles, matrices by
// eight); of few the tiles are spread over all (grid: tiles, splits, matrices; tile_of). Times of the first against the second:
// 64 to 1024 matrices of 100 x 100 to 2000 x 800 0.76 to 1.0 (64 of 512 x 512 f32 833 us, 971; bf16 498, 597); 8 to 60 of
// them 0.81 to 1.31, by how evenly they go into eight (9 of 2000 x 800 f32 1182 us, 899). (No division: the compiler makes
// those in vector registers and leaves what follows from them there, where no descriptor can be formed.)
constexpr int MANY = 64;
struct Where {
  int z, tile, tiles, split, splits;
};
__device__ __forceinline__ Where where(int batch) {
  if (batch >= MANY)
    return {(int)(blockIdx.x & 7) + 8 * (int)blockIdx.z, (int)blockIdx.y, (int)gridDim.y, (int)(blockIdx.x >> 3), (int)(gridDim.x >> 3)};
  return {(int)blockIdx.z, (int)blockIdx.x, (int)gridDim.x, (int)blockIdx.y, (int)gridDim.y};
}
inline dim3 grid_of(int batch, int tiles, int splits) {
  if (batch >= MANY) return dim3(8u * splits, tiles, mm::ceil_div(batch, 8));
  return dim3(tiles, splits, batch);
}

template <class S> struct Symmetric : S { static constexpr bool SYM = true; };
template <class S, bool SYM> using ShapeOf = std::conditional_t<SYM, Symmetric<S>, S>;

// The products of a batch: operands' distances in bytes
template <typename T, class S, bool AT, bool BT, class E>
__global__ __launch_bounds__(S::NT, S::WAVES) void k_bmm(mm::Prob p, int batch, size_t sa, size_t sb, typename E::Args ea) {
  __shared__ mm::Stages<S> stages;
  const Where w = where(batch);
  if (w.z >= batch) return;
  p.A = static_cast<const unsigned char*>(p.A) + w.z * sa;
  p.B = static_cast<const unsigned char*>(p.B) + w.z * sb;
  if constexpr (std::is_same<E, EpPart>::value) {
    ea.part += (((size_t)w.z * w.splits + w.split) * w.tiles + w.tile) * (S::BM * S::BN / 4);
    mm::mm_tile<T, S, AT, BT, E>(p, ea, w.tile, stages, w.split);
  } else {
    mm::mm_tile<T, S, AT, BT, E>(p, E::at(ea, w.z), w.tile, stages, w.split);
  }
}

template <class S, class E>
__global__ __launch_bounds__(S::NT) void k_bfinish(mm::Prob p, int batch, const f32x4* part, int splits, typename E::Args ea) {
  const Where w = where(batch);
  if (w.z >= batch) return;
  mm::finish_tile<S, E>(p, w.tile, part, (size_t)w.z * splits * w.tiles + w.tile, w.tiles, splits, E::at(ea, w.z));
}

// A product of the batch and how it runs
struct Product {
  mm::Prob p;
  size_t sa, sb;
  mm::Plan pl;
  int batch;
  mm::f32x4* part;
  hipStream_t st;
};

template <typename T, class S0, bool AT, bool BT, bool SYM, class E>
hipError_t launch_shape(Product w, const typename E::Args& ea) {
  typedef ShapeOf<S0, SYM> S;
  constexpr int BK = S::KB / (int)sizeof(T);
  mm::Prob& p = w.p;
  p.tm = w.pl.tm, p.tn = w.pl.tn;
  p.kper = std::max(1, mm::ceil_div(mm::ceil_div(p.K, BK), w.pl.splits)) * BK;
  const int tiles = (int)tiles_of(w.pl, SYM);
  if (S::BM > 128 || w.pl.splits == 1) {
    k_bmm<T, S, AT, BT, E><<<grid_of(w.batch, tiles, 1), S::NT, 0, w.st>>>(p, w.batch, w.sa, w.sb, ea);
  } else if constexpr (S::BM <= 128) {
    typedef ShapeOf<mm::Shape<S::BM, S::BN, S::WGM, S::WGN, 128, 2, 2>, SYM> SF;
    k_bmm<T, S, AT, BT, EpPart><<<grid_of(w.batch, tiles, w.pl.splits), S::NT, 0, w.st>>>(p, w.batch, w.sa, w.sb, {w.part});
    k_bfinish<SF, E><<<grid_of(w.batch, tiles, 1), S::NT, 0, w.st>>>(p, w.batch, w.part, w.pl.splits, ea);
  }
  return hipGetLastError();
}

template <typename T, bool AT, bool BT, bool SYM, class E>
hipError_t launch_product(const Product& w, const typename E::Args& ea) {
  if constexpr (SYM && !AT && !BT) {
    if (w.pl.tile == 192) return launch_shape<T, std::conditional_t<sizeof(T) == 2, mm::Tile192, mm::Tile192d>, AT, BT, SYM, E>(w, ea);
  }
  if constexpr (sizeof(T) == 2) {
    if (w.pl.tile == 256) return launch_shape<T, mm::Tile256, AT, BT, SYM, E>(w, ea);
    if (w.pl.tile == 128) return launch_shape<T, mm::Tile128, AT, BT, SYM, E>(w, ea);
    return launch_shape<T, mm::Tile64, AT, BT, SYM, E>(w, ea);
  } else {
    if (w.pl.tile == 256) return launch_shape<T, mm::Tile256f, AT, BT, SYM, E>(w, ea);
    if (w.pl.tile == 128) return launch_shape<T, mm::Tile128f, AT, BT, SYM, E>(w, ea);
    return launch_shape<T, mm::Tile64f, AT, BT, SYM, E>(w, ea);
  }
}

inline mm::Prob prob(const void* A, long lda, const void* B, long ldb, int M, int N, int K) {
  return mm::Prob{A, B, lda, ldb, M, N, K, nullptr, 0, 0, 0, 0, 0};
}

// TI: gradient and weights, T: the products
template <typename TI, typename T>
hipError_t update_t(const OrthArgs& a, hipStream_t st) {
  if (orth_small(a.no, a.ni)) {
    const int k = std::max(a.no, a.ni);
    return k <= 64 ? small_t<TI, 1>(a, st) : k <= 128 ? small_t<TI, 2>(a, st) : small_t<TI, 4>(a, st);
  }
  const OrthLayout l = orth_layout(a.dtype, a.N, a.no, a.ni);
  char* w = static_cast<char*>(a.ws);
  double* norms = reinterpret_cast<double*>(w + l.norms);
  T* X[2] = {reinterpret_cast<T*>(w + l.X[0]), reinterpret_cast<T*>(w + l.X[1])};
  T *A = reinterpret_cast<T*>(w + l.A), *P = reinterpret_cast<T*>(w + l.P);
  constexpr bool LO = std::is_same<T, mm::f16>::value;
  int8_t* lo = LO && a.steps > 2 ? reinterpret_cast<int8_t*>(w + l.lo) : nullptr;
  const bool tall = a.no > a.ni;
  const int n = std::min(a.no, a.ni), k = std::max(a.no, a.ni), ld = l.ld, lda = l.lda;
  const size_t size = (size_t)a.no * a.ni, sx = (size_t)a.no * ld, sA = (size_t)n * lda;
  constexpr float down = 1.f / X_UP;
  for (int z0 = 0; z0 < a.N; z0 += l.chunk) {
    const int batch = std::min(l.chunk, a.N - z0);
    const size_t from = z0 * size;
    const TI* g = (const TI*)a.g + from;
    float* mo = a.mo ? a.mo + from : nullptr;
    const unsigned gx = (unsigned)std::min<size_t>((sx + 4095) / 4096, 2048);
    k_momentum<TI><<<dim3((unsigned)l.parts, (unsigned)batch), 256, 0, st>>>({g, a.m ? a.m + from : nullptr, mo, (float)a.mu, a.nesterov}, size, norms);
    k_scale<TI, T><<<dim3(gx, (unsigned)batch), 256, 0, st>>>({g, nullptr, mo, (float)a.mu, a.nesterov}, a.no, a.ni, ld, norms, l.parts, a.eps, X_UP, X[0], lo, l.ldlo);
    hipError_t e = hipGetLastError();
    for (int s = 0; s < a.steps && e == hipSuccess; ++s) {
      const T* x = X[s & 1];
      const auto product = [&](const mm::Prob& p, size_t sa, size_t sb, const mm::Plan& pl) {
        return Product{p, sa * sizeof(T), sb * sizeof(T), pl, batch, reinterpret_cast<mm::f32x4*>(w + l.part), st};
      };
      // what goes from P to a (its multiple of I has to be in f16's range too: far from it)
      const double move = LO && s + 2 >= a.steps && fabs(a.b + a.c) <= 8 ? a.b + a.c : 0.0;
      // A, the scale of X taken out; P = b A + c A^2
      const typename EpSym<T>::Args ea{nullptr, A, lda, sA, down * down * A_UP, 0.f, 0.f},
          ep{A, P, lda, sA, (float)a.c / A_UP, (float)a.b, (float)-move * A_UP};
      const Product gram = product(prob(x, ld, x, ld, n, n, k), sx, sx, l.gram);
      e = tall ? launch_product<T, true, true, true, EpSym<T>>(gram, ea) : launch_product<T, false, false, true, EpSym<T>>(gram, ea);
      if (e != hipSuccess) break;
      e = launch_product<T, false, false, true, EpSym<T>>(product(prob(A, lda, A, lda, n, n, n), sA, sA, l.poly), ep);
      if (e != hipSuccess) break;
      const Product next = tall ? product(prob(x, ld, P, lda, a.no, a.ni, n), sx, sA, l.next)
                                : product(prob(P, lda, x, ld, a.no, a.ni, n), sA, sx, l.next);
      if (s + 1 < a.steps) {
        const typename EpNext<T>::Args en{x, X[~s & 1], ld, sx, (float)(a.a + move), 1.f / A_UP, s + 2 < a.steps ? lo : nullptr, l.ldlo, (size_t)a.no * l.ldlo, LO && s + 3 < a.steps};
        e = tall ? launch_product<T, false, false, false, EpNext<T>>(next, en) : launch_product<T, false, true, false, EpNext<T>>(next, en);
      } else {
        const typename EpUpdate<T, TI>::Args eu{x, ld, sx, a.r ? (const TI*)a.r + from : nullptr, (TI*)a.W + from, size,
                                                (float)(a.a + move), 1.f / A_UP, (float)(a.alpha * down), (float)a.beta};
        e = tall ? launch_product<T, false, false, false, EpUpdate<T, TI>>(next, eu)
                 : launch_product<T, false, true, false, EpUpdate<T, TI>>(next, eu);
      }
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace orth
}  // namespace lp
