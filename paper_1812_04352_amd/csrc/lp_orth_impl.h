// Orthogonalised updates W = alpha O + beta r of a batch of matrices [no][ni] (included by one translation
// unit per type of the products, T). O comes from the momentum v by an iteration whose products are all
// there is to it: X = v / (|v| + eps), |v| the root of the sum of squares, so that no singular value exceeds
// one, then `steps` times, with A the short side's A = X X^T (X^T X of a tall matrix),
//   X <- a X + (b A + c A^2) X   (tall: a X + X (b A + c A^2)),
// which maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.
//   A and P = b A + c A^2 are symmetric: only tiles on and below the diagonal are formed, and stored on both sides of
//   it. a X is added in fp32 in the last product's epilogue, that of the last step updates W.
// 16-bit gradients: X, A and P are kept in f16 whatever the gradient's type is. No singular value exceeds 1.3 or
// so, so that A and P are in range, and X is kept times 2^shift, about the root of the long side, which brings
// its values to the size of 1: f16 then rounds eight times finer than bf16 does. Rounding errors grow like the
// small singular values do, by a factor a a step: O is off by 1.2e-3 to 3e-3 of its norm for noise and noise with
// a few strong directions, by 4e-2 (bf16: 0.3) where four directions exceed the noise a hundredfold.
// Bound by the products: steps (3 n^2 k + n^3) operations, n the short and k the long side.
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
constexpr int MOST_PARTS = 128;  // partial sums of a matrix's squares

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

// X = v 2^shift / (|v| + eps) in rows of ld values, zeros behind the ni that count (grid y: the matrix)
template <typename TI, typename T>
__global__ __launch_bounds__(256) void k_scale(Momentum<TI, VV> u, int no, int ni, int ld, const double* part, int parts, double eps,
                                               double up, T* X) {
  __shared__ double sh;
  if (threadIdx.x < 64) {
    const double* p = part + (size_t)blockIdx.y * parts;
    double s = (int)threadIdx.x < parts ? p[threadIdx.x] : 0.0;
    if ((int)threadIdx.x + 64 < parts) s += p[threadIdx.x + 64];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (threadIdx.x == 0) sh = up / (sqrt(s) + eps);
  }
  __syncthreads();
  const double scale = sh;
  const size_t base = (size_t)blockIdx.y * no * ni;
  const uint32_t per = (uint32_t)(ld / VV);
  const size_t all = (size_t)no * per;
  X += (size_t)blockIdx.y * no * ld;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (size_t)gridDim.x * 256) {
    const size_t r = i / per;
    const int c = (int)(i - r * per) * VV, n = min(VV, ni - c);
    typename GVec<T, VV>::type x;
    if (n <= 0) {
#pragma unroll
      for (int k = 0; k < VV; ++k) x[k] = (T)0.f;
    } else {
      float v[VV];
      u.again(base + r * ni + c, n, v);
#pragma unroll
      for (int k = 0; k < VV; ++k) x[k] = k < n ? (T)(float)((double)v[k] * scale) : (T)0.f;
    }
    *reinterpret_cast<typename GVec<T, VV>::type*>(X + r * ld + c) = x;
  }
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

// f D + b A of a symmetric D, rows of ld values (A nullable)
template <typename T>
struct EpSym {
  struct Args {
    const T* A;
    T* out;
    int ld;
    size_t stride;  // of a matrix
    float f, b;
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
        mm::put_rows<WHOLE>(a.out, a.ld, c.upto(a.ld), c, i, j, buf, v);
        if (c.mt != c.nt) put_mirror(a.out, a.ld, c, i, j, buf, v);
      }
  }
};

// a X + D
template <typename T>
struct EpNext {
  struct Args {
    const T* X;
    T* out;
    int ld;
    size_t stride;
    float a;
  };
  static __device__ __forceinline__ Args at(Args a, int z) {
    a.X += z * a.stride;
    a.out += z * a.stride;
    return a;
  }
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    mm::Rows<WHOLE, T, FM, FN> X(a.X, a.ld, c);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4];
        X.get(c, i, j, buf, v);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v[q][k] = WHOLE || c.feature(j, q) + k < c.lim ? a.a * v[q][k] + acc[i][j][4 * q + k] : 0.f;
        mm::put_rows<WHOLE>(a.out, a.ld, c.upto(a.ld), c, i, j, buf, v);
      }
  }
};

// W = alpha (a X + D) + beta r, rows of N values (r nullable)
template <typename T, typename TO>
struct EpUpdate {
  struct Args {
    const T* X;
    int ld;
    size_t stride;   // of a matrix of X
    const TO* r;
    TO* W;
    size_t wstride;  // of r and W
    float a, alpha, beta;
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
        for (int q = 0; q < 4; ++q) v[q] = (v[q] * a.a + mm::quad(acc[i][j], q)) * a.alpha + w[q] * a.beta;
        mm::put_rows<WHOLE>(a.W, c.N, c.lim, c, i, j, buf, v);
      }
  }
};

// the partial sums of a split contraction
struct EpPart : mm::EpRaw {
  typedef mm::EpRaw::Args Args;
};
template <class S>
__device__ __forceinline__ mm::f32x4* part_of(mm::f32x4* part, int splits, int z) {
  return part + (size_t)z * splits * gridDim.x * (S::BM * S::BN / 4);
}

template <class S> struct Symmetric : S { static constexpr bool SYM = true; };
template <class S, bool SYM> using ShapeOf = std::conditional_t<SYM, Symmetric<S>, S>;

// The products of a batch (grid z): operands' distances in bytes
template <typename T, class S, bool AT, bool BT, class E>
__global__ __launch_bounds__(S::NT, S::WAVES) void k_bmm(mm::Prob p, size_t sa, size_t sb, typename E::Args ea) {
  __shared__ mm::Stages<S> stages;
  const int z = blockIdx.z;
  p.A = static_cast<const unsigned char*>(p.A) + z * sa;
  p.B = static_cast<const unsigned char*>(p.B) + z * sb;
  if constexpr (std::is_same<E, EpPart>::value) {
    ea.part = part_of<S>(ea.part, gridDim.y, z);
    mm::mm_tile<T, S, AT, BT, E>(p, ea, blockIdx.x, stages);
  } else {
    mm::mm_tile<T, S, AT, BT, E>(p, E::at(ea, z), blockIdx.x, stages);
  }
}

template <class S, class E>
__global__ __launch_bounds__(S::NT) void k_bfinish(mm::Prob p, mm::f32x4* part, int splits, typename E::Args ea) {
  mm::finish_tile<S, E>(p, part_of<S>(part, splits, blockIdx.z), splits, E::at(ea, blockIdx.z));
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
  const unsigned tiles = (unsigned)tiles_of(w.pl, SYM);
  if (S::BM == 256 || w.pl.splits == 1) {
    k_bmm<T, S, AT, BT, E><<<dim3(tiles, 1, (unsigned)w.batch), S::NT, 0, w.st>>>(p, w.sa, w.sb, ea);
  } else if constexpr (S::BM < 256) {
    typedef ShapeOf<mm::Shape<S::BM, S::BN, S::WGM, S::WGN, 128, 2, 2>, SYM> SF;
    k_bmm<T, S, AT, BT, EpPart><<<dim3(tiles, (unsigned)w.pl.splits, (unsigned)w.batch), S::NT, 0, w.st>>>(p, w.sa, w.sb, {w.part});
    k_bfinish<SF, E><<<dim3(tiles, 1, (unsigned)w.batch), S::NT, 0, w.st>>>(p, w.part, w.pl.splits, ea);
  }
  return hipGetLastError();
}

template <typename T, bool AT, bool BT, bool SYM, class E>
hipError_t launch_product(const Product& w, const typename E::Args& ea) {
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
  const OrthLayout l = orth_layout(a.dtype, a.N, a.no, a.ni);
  char* w = static_cast<char*>(a.ws);
  double* norms = reinterpret_cast<double*>(w + l.norms);
  T* X[2] = {reinterpret_cast<T*>(w + l.X[0]), reinterpret_cast<T*>(w + l.X[1])};
  T *A = reinterpret_cast<T*>(w + l.A), *P = reinterpret_cast<T*>(w + l.P);
  const bool tall = a.no > a.ni;
  const int n = std::min(a.no, a.ni), k = std::max(a.no, a.ni), ld = l.ld, lda = l.lda;
  const size_t size = (size_t)a.no * a.ni, sx = (size_t)a.no * ld, sA = (size_t)n * lda;
  const int shift = sizeof(T) == 2 ? (int)lround(0.5 * log2((double)k)) : 0;
  const float down = ldexpf(1.f, -shift);
  for (int z0 = 0; z0 < a.N; z0 += l.chunk) {
    const int batch = std::min(l.chunk, a.N - z0);
    const size_t from = z0 * size;
    const Momentum<TI, VV> u{(const TI*)a.g + from, a.m ? a.m + from : nullptr, a.mo ? a.mo + from : nullptr, (float)a.mu, a.nesterov};
    const unsigned gx = (unsigned)std::min<size_t>((size * VV + 4095) / 4096, 256);
    k_momentum<TI><<<dim3((unsigned)l.parts, (unsigned)batch), 256, 0, st>>>(u, size, norms);
    k_scale<TI, T><<<dim3(gx, (unsigned)batch), 256, 0, st>>>(u, a.no, a.ni, ld, norms, l.parts, a.eps, ldexp(1.0, shift), X[0]);
    hipError_t e = hipGetLastError();
    for (int s = 0; s < a.steps && e == hipSuccess; ++s) {
      const T* x = X[s & 1];
      const auto product = [&](const mm::Prob& p, size_t sa, size_t sb, const mm::Plan& pl) {
        return Product{p, sa * sizeof(T), sb * sizeof(T), pl, batch, reinterpret_cast<mm::f32x4*>(w + l.part), st};
      };
      // A, the scale of X taken out; P = b A + c A^2
      const typename EpSym<T>::Args ea{nullptr, A, lda, sA, down * down, 0.f}, ep{A, P, lda, sA, (float)a.c, (float)a.b};
      const Product gram = product(prob(x, ld, x, ld, n, n, k), sx, sx, l.gram);
      e = tall ? launch_product<T, true, true, true, EpSym<T>>(gram, ea) : launch_product<T, false, false, true, EpSym<T>>(gram, ea);
      if (e != hipSuccess) break;
      e = launch_product<T, false, false, true, EpSym<T>>(product(prob(A, lda, A, lda, n, n, n), sA, sA, l.poly), ep);
      if (e != hipSuccess) break;
      const Product next = tall ? product(prob(x, ld, P, lda, a.no, a.ni, n), sx, sA, l.next)
                                : product(prob(P, lda, x, ld, a.no, a.ni, n), sA, sx, l.next);
      if (s + 1 < a.steps) {
        const typename EpNext<T>::Args en{x, X[~s & 1], ld, sx, (float)a.a};
        e = tall ? launch_product<T, false, false, false, EpNext<T>>(next, en) : launch_product<T, false, true, false, EpNext<T>>(next, en);
      } else {
        const typename EpUpdate<T, TI>::Args eu{x, ld, sx, a.r ? (const TI*)a.r + from : nullptr, (TI*)a.W + from, size,
                                                (float)a.a, (float)(a.alpha * down), (float)a.beta};
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
