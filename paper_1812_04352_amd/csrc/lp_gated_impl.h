// Gated layers y = s(x Wg^T) (x Wu^T) of any width and their gradients, for one element type
// (included by one translation unit per type).
//   forward:   both products in one kernel: a tile holds the same features of Wg and of Wu, a wave both
//              products of its rows and features, so the activation and the product of the two are its
//              epilogue and neither product is ever stored
//   backward:  dzu = dy s(zg), dzg = dy zu s'(zg)   (both products formed again, as above; kept in the
//                                                    element type, operands of the next two products)
//              dx = dzg Wg + dzu Wu,   dWg = dzg^T x,   dWu = dzu^T x
//              dzg and dzu lie side by side in blocks of PAIR_BLOCK features, dz [B][2 no32]: dx is then
//              one contraction over both (the weights' rows taken from either array in turn), and
//              dz^T x one product whose rows belong to dWg and dWu in turn.
// Bound by the products: 4 B ni no operations forward, 12 B ni no back: 8192 x 4096 -> 10240 bf16 1134 us forward (1.21
// PFLOP/s) and 3486 back (1.18). One token reads both weights at 5.7 TB/s (29 us there); 24 x 2048 -> 5120 f16 take 12.9 us.
// dz is rounded to the element type, which is what the next two products' matrix instructions take: the gradients'
// error in bf16 grows by it from 0.0017 to 0.0023 of their norm.
#pragma once

#include <type_traits>

#include "lp_internal.h"
#include "lp_mm.h"
#include "lp_step_impl.h"

namespace lp {
namespace gated {

using mm::f32x16;
using mm::f32x4;
using mm::Place;

// The logistic function, by e = exp(-|z|), which does not overflow; on the hardware's exp2 and reciprocal for
// the 16-bit types (relative error (|z| + 4) 2^-23 at most: that of the exponent, and a step each; e is 0 where it
// lies below 2^-126, beyond |z| = 87.3).
template <typename T>
__device__ __forceinline__ float logistic(float z) {
  if constexpr (sizeof(T) == 2) {
    const float e = __builtin_amdgcn_exp2f(-1.442695040888963f * fabsf(z));
    return (z < 0.f ? e : 1.f) * __builtin_amdgcn_rcpf(1.f + e);
  } else {
    const float e = expf(-fabsf(z));
    return (z < 0.f ? e : 1.f) / (1.f + e);
  }
}

// The standard normal distribution function of z and its density's exponential e = exp(-z^2 / 2). erfc, not erf, so that
// the tail keeps its relative accuracy; of the 16-bit types by a polynomial in t = 1 / (1 + 0.425 |x|), x = z / sqrt 2,
// fitted to exp(x^2) erfc(x) in relative error over all x >= 0 (1.2e-7; 5.3e-7 evaluated in fp32; the function itself 6e-7
// down to z = -3 and, with the exponential's rounding, which grows with z^2, 1.5e-6 to -5.5 and 8e-6 to -13). With the device
// library's erfc 24 x 2048 -> 5120 f16 takes 14.0 us instead of 12.9.
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  if constexpr (sizeof(T) == 2) {
    e = __builtin_amdgcn_exp2f(-0.7213475204444817f * z * z);
    const float t = __builtin_amdgcn_rcpf(1.f + 0.425f * 0.7071067811865476f * fabsf(z));
    float p = 0.07218405604362488f;
    p = fmaf(p, t, -0.3160977065563202f);
    p = fmaf(p, t, 0.4126853942871094f);
    p = fmaf(p, t, -0.10791664570569992f);
    p = fmaf(p, t, 0.2575562298297882f);
    p = fmaf(p, t, 0.199957013130188f);
    p = fmaf(p, t, 0.2419607788324356f);
    p = fmaf(p, t, 0.2396707832813263f);
    const float tail = 0.5f * p * t * e;
    return z > 0.f ? 1.f - tail : tail;
  } else {
    e = expf(-0.5f * z * z);
    return 0.5f * erfcf(-0.7071067811865476f * z);
  }
}

// s(z) and s'(z). gelu is z times the normal distribution function. A NaN stays one.
template <typename T, int ACT>
__device__ __forceinline__ void gate(float z, float& s, float& ds) {
  if constexpr (ACT == ACT_SILU) {
    const float t = logistic<T>(z);
    s = z * t;
    ds = t * (1.f + z * (1.f - t));
  } else if constexpr (ACT == ACT_GELU) {
    float e;
    const float cdf = normal_cdf<T>(z, e);
    s = z * cdf;
    ds = cdf + z * (0.3989422804014327f * e);
  } else {
    s = wide::sigma<T, ACT>(z);
    ds = wide::dsigma<T, ACT>(z);
  }
}

// Calls f with the activation as a compile-time constant (uniform over the launch).
template <typename F>
__device__ __forceinline__ void with_gate(int act, F f) {
  switch (act) {
    case ACT_SILU: return f(std::integral_constant<int, ACT_SILU>{});
    case ACT_GELU: return f(std::integral_constant<int, ACT_GELU>{});
    default: return wide::with_act(act, f);
  }
}

// y = s(D1) D2
template <typename T>
struct EpGated {
  static constexpr bool ONE = true;
  struct Args {
    T* y;
    int act;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    static_assert(FN == 2, "one block column of each product");
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    if (!WHOLE && c.nw >= c.lim) return;
    with_gate(a.act, [&](auto act) {
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float s, ds;
            gate<T, decltype(act)::value>(acc[i][0][4 * q + k], s, ds);
            v[q][k] = s * acc[i][1][4 * q + k];
          }
        mm::put_rows<WHOLE>(a.y, c.N, c.lim, c, i, 0, buf, v);
      }
    });
  }
};

// dzg = dy D2 s'(D1), dzu = dy s(D1): blocks of dz (whole ones: zeros behind the features that count)
template <typename T>
struct EpGatedGrad {
  static constexpr bool ONE = false;
  struct Args {
    const T* dy;
    T* dz;
    long ld;  // 2 no32
    int act;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    static_assert(FN == 2, "one block column of each product");
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    if (!WHOLE && c.nw >= c.lim) return;
    T* dz = a.dz + c.nw;  // the block of features n.. is at column 2 n
    // (the largest tiles have no registers for dy ahead)
    mm::Rows<WHOLE, T, FM, 1, sizeof(T) == 2 && (FM < 4)> dy(a.dy, c.N, c);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      with_gate(a.act, [&](auto act) {  // in place: s(D1) and D2 s'(D1)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float s, ds;
          gate<T, decltype(act)::value>(acc[i][0][r], s, ds);
          acc[i][0][r] = s;
          acc[i][1][r] *= ds;
        }
      });
      f32x4 d[4], v[4];
      dy.get(c, i, 0, buf, d);
#pragma unroll
      for (int j = 1; j >= 0; --j) {  // dzg, then dzu
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int k = 0; k < 4; ++k) v[q][k] = WHOLE || c.feature(0, q) + k < c.lim ? d[q][k] * acc[i][j][4 * q + k] : 0.f;
        mm::BlockIO<T>::store(dz + (1 - j) * mm::PAIR_BLOCK, a.ld, c, i, 0, buf, v, [](int m) { return m; });
      }
    }
  }
};

// dx = D
template <typename T>
struct EpOut {
  static constexpr bool ONE = false;
  struct Args {
    T* out;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = mm::quad(acc[i][j], q);
        mm::put_rows<WHOLE>(a.out, c.N, c.lim, c, i, j, buf, v);
      }
  }
};

// Rows of D in blocks of PAIR_BLOCK: of dWg and of dWu in turn, no rows each
template <typename T>
struct EpPairRows {
  static constexpr bool ONE = false;
  struct Args {
    T* out[2];  // nullable
    int no;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    static_assert(mm::PAIR_BLOCK == 32, "a block of rows is a wave's");
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int blk = (c.mw + 32 * i) / mm::PAIR_BLOCK;
      T* out = a.out[blk & 1];
      Place at = c;
      at.mw = blk / 2 * mm::PAIR_BLOCK - 32 * i;
      at.M = a.no;
      if (!out || at.mw + 32 * i >= a.no) continue;
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        f32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = mm::quad(acc[i][j], q);
        mm::put_rows<WHOLE>(out, c.N, c.lim, at, i, j, buf, v);
      }
    }
  }
};

// dx and dz^T x, neither of which needs the other, as one launch, the longer contraction's tiles first
template <typename T, class S1, class S2, class E1, class E2>
__global__ __launch_bounds__(S1::NT, S1::WAVES) void k_both(mm::Prob p1, typename E1::Args e1, mm::Prob p2, typename E2::Args e2) {
  static_assert(S1::NT == S2::NT && sizeof(mm::Stages<S1>) == sizeof(mm::Stages<S2>), "the same workgroups");
  __shared__ mm::Stages<S1> stages;
  const int n1 = p1.tm * p1.tn, n2 = p2.tm * p2.tn, id = blockIdx.x;
  const bool swap = p2.K > p1.K;
  const int b1 = swap ? n2 : 0, b2 = swap ? 0 : n1;  // where each product's workgroups begin
  if (id >= b1 && id < b1 + n1) mm::mm_tile<T, S1, false, true, E1>(p1, e1, id - b1, stages);
  else mm::mm_tile<T, S2, true, true, E2>(p2, e2, id - b2, reinterpret_cast<mm::Stages<S2>&>(stages));
}

inline mm::Prob prob(const void* A, long lda, const void* B, const void* B2, long ldb, int M, int N, int K, int kw) {
  mm::Prob p{A, B, lda, ldb, M, N, K, nullptr, 0, 0, 0, 0, 0};
  p.B2 = B2;
  p.kw = kw;
  return p;
}

// Operands of rows of ni values: x and both weights as the products need them
template <typename T>
struct Operands {
  const T *x, *Wg, *Wu;
  long ldx, ldw;
  hipError_t e;
  Operands(const GatedArgs& a, const GatedLayout& l, bool as_is, hipStream_t st) {
    char* w = static_cast<char*>(a.ws);
    // both weights are copied where either has to be: their tiles share a leading dimension
    const bool wa = as_is || (a.ni % (16 / (int)sizeof(T)) == 0 && (uintptr_t)a.Wg % 16 == 0 && (uintptr_t)a.Wu % 16 == 0);
    Wg = static_cast<const T*>(a.Wg), Wu = static_cast<const T*>(a.Wu), ldw = a.ni;
    e = hipSuccess;
    if (!wa) {
      const int lp = mm::padded(sizeof(T), a.ni);
      e = mm::launch_repack<T>(Wg, reinterpret_cast<T*>(w + l.Wg), a.no, Wu, reinterpret_cast<T*>(w + l.Wu), a.no, a.ni, lp, st);
      Wg = reinterpret_cast<const T*>(w + l.Wg), Wu = reinterpret_cast<const T*>(w + l.Wu), ldw = lp;
    }
    if (e != hipSuccess) return;
    const mm::Operands<T> o(a.B ? a.x : nullptr, a.B, w + l.x, nullptr, 0, nullptr, a.ni, as_is, st);
    x = o.p[0], ldx = o.ld[0], e = o.e;
  }
};

template <typename T>
hipError_t forward_t(const GatedArgs& a, hipStream_t st) {
  const GatedLayout l = gated_layout(a.dtype, a.B, a.ni, a.no, false);
  const Operands<T> o(a, l, l.z.tile == 1, st);
  if (o.e != hipSuccess) return o.e;
  const typename EpGated<T>::Args e{(T*)a.y, a.act};
  return mm::launch_mm<T, false, false, EpGated<T>, mm::PAIR_ROWS>(
      prob(o.x, o.ldx, o.Wg, o.Wu, o.ldw, a.B, a.no, a.ni, 0), e, l.z, static_cast<char*>(a.ws) + l.part, st);
}

template <typename T>
hipError_t backward_t(const GatedArgs& a, hipStream_t st) {
  const GatedLayout l = gated_layout(a.dtype, a.B, a.ni, a.no, true);
  char* w = static_cast<char*>(a.ws);
  void* part = w + l.part;
  const Operands<T> o(a, l, false, st);
  hipError_t e = o.e;
  if (e != hipSuccess) return e;
  T* dz = reinterpret_cast<T*>(w + l.dz);
  const int two = 2 * mm::ceil_div(a.no, mm::PAIR_BLOCK) * mm::PAIR_BLOCK;
  if (a.B) {  // (an empty batch leaves zero sums: products over no rows)
    const typename EpGatedGrad<T>::Args eg{(const T*)a.dy, dz, two, a.act};
    e = mm::launch_mm<T, false, false, EpGatedGrad<T>, mm::PAIR_ROWS>(
        prob(o.x, o.ldx, o.Wg, o.Wu, o.ldw, a.B, a.no, a.ni, 0), eg, l.z, part, st);
  }
  const mm::Prob px = prob(dz, two, o.Wg, o.Wu, o.ldw, a.B, a.ni, two, a.no), pw = prob(dz, two, o.x, nullptr, o.ldx, two, a.ni, a.B, 0);
  const typename EpOut<T>::Args ex{(T*)a.dx};
  const typename EpPairRows<T>::Args ew{{(T*)a.dWg, (T*)a.dWu}, a.no};
  const bool weights = a.dWg || a.dWu;
  if (e == hipSuccess && l.both && a.B && a.dx && weights) {
    typedef std::conditional_t<sizeof(T) == 2, mm::Tile64, mm::Tile64f> S;
    const auto whole = [](mm::Prob p) {
      p.tm = mm::ceil_div(p.M, S::BM), p.tn = mm::ceil_div(p.N, S::BN);
      p.kper = mm::ceil_div(p.K * (long)sizeof(T), mm::STAGE_BYTES) * (mm::STAGE_BYTES / (int)sizeof(T));
      return p;
    };
    const mm::Prob x = whole(px), w2 = whole(pw);
    k_both<T, mm::Paired<S, mm::PAIR_COLS>, S, EpOut<T>, EpPairRows<T>>
        <<<(unsigned)(x.tm * x.tn + w2.tm * w2.tn), S::NT, 0, st>>>(x, ex, w2, ew);
    return hipGetLastError();
  }
  if (e == hipSuccess && a.B && a.dx)
    e = mm::launch_mm<T, false, true, EpOut<T>, mm::PAIR_COLS>(px, ex, l.zx, part, st);
  if (e == hipSuccess && weights) e = mm::launch_mm<T, true, true, EpPairRows<T>>(pw, ew, l.zw, part, st);
  return e;
}

}  // namespace gated
}  // namespace lp
