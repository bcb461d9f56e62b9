// One layer step y = r + h sigma(x W^T + b) of any width, its gradients, and 8-bit
// checkpoints, for one element type (included by one translation unit per type).
//   forward:   one product with the bias, activation, residual and checkpoint of y in its epilogue
//   backward:  g = sigma'(x W^T + b) dy   (the pre-activation is formed again; kept in the element
//                                          type, which is what the next products take: h stays out
//                                          of g, so that a small step does not push it out of the
//                                          range of f16)
//              dx = h g W (+ dy),  dW = h g^T x,  db = h sum g (from g before its rounding)
#pragma once

#include "lp_checkpoint.h"
#include "lp_internal.h"
#include "lp_mm.h"

namespace lp {
namespace {

using mm::f32x16;
using mm::f32x4;
using mm::Place;

// tanh for the 16-bit types: (1 - t) / (1 + t) with t = exp(-2|x|) on the hardware's exp2 and
// reciprocal (error below 2^-22 absolute); below 1/4, where the difference would cancel, the odd
// polynomial up to x^7 (its next term is below 4e-7 of the value there).
__device__ __forceinline__ float tanh16(float x) {
  const float a = fabsf(x), t = __builtin_amdgcn_exp2f(-2.885390081777927f * a);  // 2 log2(e) |x|
  const float big = (1.f - t) * __builtin_amdgcn_rcpf(1.f + t), s = a * a;
  const float small = a * (1.f + s * (-0.33333334f + s * (0.13333334f - s * 0.053968254f)));
  return copysignf(a < 0.25f ? small : big, x);
}

// 1 - tanh(x)^2 = 4 t / (1 + t)^2: no cancellation for large |x|
template <typename T>
__device__ __forceinline__ float dtanh(float x) {
  if constexpr (sizeof(T) == 2) {
    const float t = __builtin_amdgcn_exp2f(-2.885390081777927f * fabsf(x)), r = __builtin_amdgcn_rcpf(1.f + t);
    return 4.f * t * r * r;
  } else {
    const float t = expf(-2.f * fabsf(x)), d = 1.f + t;
    return 4.f * t / (d * d);
  }
}

// sigma and sigma' of a run-time activation (uniform over the launch). A NaN stays one.
template <typename T>
__device__ __forceinline__ float sigma(float z, int act) {
  switch (act) {
    case ACT_TANH: return sizeof(T) == 2 ? tanh16(z) : tanhf(z);
    case ACT_RELU: return z != z ? z : act_f<float, ACT_RELU>(z);
    case ACT_SMOOTHRELU: return z != z ? z : act_f<float, ACT_SMOOTHRELU>(z);
    default: return z;
  }
}

template <typename T>
__device__ __forceinline__ float dsigma(float z, int act) {
  switch (act) {
    case ACT_TANH: return dtanh<T>(z);
    case ACT_RELU: return z != z ? z : dact_f<float, ACT_RELU>(z);
    case ACT_SMOOTHRELU: return z != z ? z : dact_f<float, ACT_SMOOTHRELU>(z);
    default: return 1.f;
  }
}

// y = r + h sigma(D + b), optionally with its checkpoint. The 32 features of a block row are a
// checkpoint block, held by lanes l and l ^ 32; the checkpoint is that of y as stored.
template <typename T>
struct EpStep {
  struct Args {
    const T* b;
    const T* r;  // nullable
    T* y;
    int8_t* y8;  // nullable
    uint8_t* ye;
    float h;
    int act;
  };
  template <int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float*) {
    const int half = 4 * (c.lane >> 5);
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int n0 = c.nw + 32 * j;
      if (n0 >= c.N) continue;
      f32x4 bias[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) bias[q] = a.b ? mm::load4(a.b, n0 + 8 * q + half, c.N) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int m = c.mw + 32 * i + (c.lane & 31);
        const bool on = m < c.M;
        const size_t row = (size_t)(on ? m : 0) * c.N;
        f32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = n0 + 8 * q + half;
          const f32x4 z = mm::quad(acc[i][j], q) + bias[q];
          f32x4 r = {0.f, 0.f, 0.f, 0.f};
          if (a.r && on && n < c.N) r = mm::load4(a.r + row, n, c.N);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[q][k] = (float)(T)(r[k] + a.h * sigma<T>(z[k], a.act));
          if (on && n < c.N) mm::store4(a.y + row, n, c.N, v[q]);
        }
        if (a.y8) {  // uniform over the launch
          uint32_t top = 0;
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (n0 + 8 * q + half + k < c.N) top = max(top, abs_bits(v[q][k]));
          top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
          const uint32_t byte = ck_byte<T>(top);
          const float inv = ck_inv(byte);
          if (!on) continue;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int n = n0 + 8 * q + half;
            typename mm::GVec<int8_t, 4>::type w;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = (int8_t)ck_round(v[q][k], inv);
            if (n + 4 <= c.N) {
              *reinterpret_cast<typename mm::GVec<int8_t, 4>::type*>(a.y8 + row + n) = w;
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k)
                if (n + k < c.N) a.y8[row + n + k] = w[k];
            }
          }
          if (half == 0) a.ye[(size_t)m * ((c.N + CK_BLOCK - 1) / CK_BLOCK) + n0 / CK_BLOCK] = (uint8_t)byte;
        }
      }
    }
  }
};

// g = sigma'(D + b) dy, and the sums of its columns over the tile's rows (fp32, before rounding)
template <typename T>
struct EpGrad {
  struct Args {
    const T* b;
    const T* dy;
    T* g;
    float* part;  // [tile rows][N]
    int act;
  };
  template <int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    const int half = 4 * (c.lane >> 5);
    f32x16 sums[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int n0 = c.nw + 32 * j;
      sums[j] = 0.f;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int m = c.mw + 32 * i + (c.lane & 31);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = n0 + 8 * q + half;
          if (m >= c.M || n >= c.N) continue;
          f32x4 z = mm::quad(acc[i][j], q);
          if (a.b) z += mm::load4(a.b, n, c.N);
          f32x4 g = mm::load4(a.dy + (size_t)m * c.N, n, c.N);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            g[k] *= dsigma<T>(z[k], a.act);
            sums[j][4 * q + k] += g[k];
          }
          mm::store4(a.g + (size_t)m * c.N, n, c.N, g);
        }
      }
    }
    mm::column_sums<FN, WGM, WGN>(sums, c, lds, a.part + (size_t)c.mt * c.N);
  }
};

// dx = h D (+ dy)
template <typename T>
struct EpDx {
  struct Args {
    const T* dy;  // nullable
    T* dx;
    float h;
  };
  template <int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float*) {
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = c.mw + 32 * i + (c.lane & 31);
      if (m >= c.M) continue;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = c.nw + 32 * j + 8 * q + 4 * (c.lane >> 5);
          if (n >= c.N) continue;
          f32x4 v = mm::quad(acc[i][j], q) * a.h;
          if (a.dy) v += mm::load4(a.dy + (size_t)m * c.N, n, c.N);
          mm::store4(a.dx + (size_t)m * c.N, n, c.N, v);
        }
    }
  }
};

// Eight lanes per block of 32 features, four features each; the grid walks the blocks.
constexpr unsigned CK_GRID = 1u << 20;

template <typename T>
__global__ __launch_bounds__(256) void k_ck_store(const T* x, int8_t* x8, uint8_t* xe, size_t nblk, int q, int nb) {
  const int part = threadIdx.x & 7;
  for (size_t blk = (size_t)blockIdx.x * 32 + (threadIdx.x >> 3); blk < nblk; blk += (size_t)gridDim.x * 32) {
    const size_t row = blk / nb;
    const int n = (int)(blk - row * nb) * CK_BLOCK + 4 * part;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (n < q) v = mm::load4(x + row * q, n, q);
    uint32_t top = max(max(abs_bits(v[0]), abs_bits(v[1])), max(abs_bits(v[2]), abs_bits(v[3])));
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    const uint32_t byte = ck_byte<T>(top);
    const float inv = ck_inv(byte);
    typename mm::GVec<int8_t, 4>::type w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = (int8_t)ck_round(v[k], inv);
    int8_t* out = x8 + row * q + n;
    if (n + 4 <= q) {
      *reinterpret_cast<typename mm::GVec<int8_t, 4>::type*>(out) = w;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (n + k < q) out[k] = w[k];
    }
    if (part == 0) xe[blk] = (uint8_t)byte;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_ck_load(const int8_t* x8, const uint8_t* xe, T* x, size_t nblk, int q, int nb) {
  for (size_t blk = (size_t)blockIdx.x * 32 + (threadIdx.x >> 3); blk < nblk; blk += (size_t)gridDim.x * 32) {
    const size_t row = blk / nb;
    const int n = (int)(blk - row * nb) * CK_BLOCK + 4 * (threadIdx.x & 7);
    if (n < q) mm::store4(x + row * q, n, q, mm::load4(x8 + row * q, n, q) * ck_scale(xe[blk]));
  }
}

inline unsigned ck_grid(size_t nblk) { return (unsigned)std::min<size_t>((nblk + 31) / 32, CK_GRID); }

template <typename T>
hipError_t ck_store_t(const void* x, int8_t* x8, uint8_t* xe, long B, int q, hipStream_t st) {
  const int nb = mm::ceil_div(q, CK_BLOCK);
  const size_t nblk = (size_t)B * nb;
  k_ck_store<T><<<ck_grid(nblk), 256, 0, st>>>((const T*)x, x8, xe, nblk, q, nb);
  return hipGetLastError();
}

template <typename T>
hipError_t ck_load_t(const int8_t* x8, const uint8_t* xe, void* x, long B, int q, hipStream_t st) {
  const int nb = mm::ceil_div(q, CK_BLOCK);
  const size_t nblk = (size_t)B * nb;
  k_ck_load<T><<<ck_grid(nblk), 256, 0, st>>>(x8, xe, (T*)x, nblk, q, nb);
  return hipGetLastError();
}

inline mm::Prob prob(const void* A, long lda, const void* B, long ldb, int M, int N, int K) {
  return mm::Prob{A, B, lda, ldb, M, N, K, nullptr, 0, 0, 0, 0, 0};
}

template <typename T>
hipError_t step_forward_t(const StepArgs& a, hipStream_t st) {
  typename EpStep<T>::Args e{(const T*)a.b, (const T*)a.r, (T*)a.y, a.y8, a.ye, (float)a.h, a.act};
  return mm::launch_mm<T, false, false, EpStep<T>>(prob(a.x, a.ni, a.W, a.ni, a.B, a.no, a.ni), e, 1, st);
}

template <typename T>
hipError_t step_backward_t(const StepArgs& a, hipStream_t st) {
  const StepLayout l = step_layout(a.dtype, a.B, a.ni, a.no);
  char* w = static_cast<char*>(a.ws);
  T* g = reinterpret_cast<T*>(w + l.g);
  float* colpart = reinterpret_cast<float*>(w + l.col);
  float* part = reinterpret_cast<float*>(w + l.part);
  const void* x = a.x;
  hipError_t e = hipSuccess;
  if (!x) {
    x = w + l.x;
    if (a.B && (e = ck_load_t<T>(a.x8, a.xe, w + l.x, a.B, a.ni, st)) != hipSuccess) return e;
  }
  if (a.B) {  // (an empty batch leaves zero sums: products over no rows)
    typename EpGrad<T>::Args eg{(const T*)a.b, (const T*)a.dy, g, colpart, a.act};
    e = mm::launch_mm<T, false, false, EpGrad<T>>(prob(x, a.ni, a.W, a.ni, a.B, a.no, a.ni), eg, 1, st);
    if (e != hipSuccess) return e;
  }
  const float h = (float)a.h;
  if (a.dx && a.B) {
    typename EpDx<T>::Args ed{a.residual ? (const T*)a.dy : nullptr, (T*)a.dx, h};
    e = mm::launch_mm<T, false, true, EpDx<T>>(prob(g, a.no, a.W, a.ni, a.B, a.ni, a.no), ed, 1, st);
    if (e != hipSuccess) return e;
  }
  if (a.dW) {
    const mm::Prob p = prob(g, a.no, x, a.ni, a.no, a.ni, a.B);
    if (l.splits > 1) {
      e = mm::launch_mm<T, true, true, mm::EpPart>(p, mm::EpPart::Args{part}, l.splits, st);
      if (e != hipSuccess) return e;
      const size_t n = (size_t)a.no * a.ni;
      mm::k_join<T><<<(unsigned)std::min<size_t>((n + 1023) / 1024, 4096), 256, 0, st>>>(part, l.splits, n, (T*)a.dW, h,
                                                                                          nullptr);
      e = hipGetLastError();
    } else {
      e = mm::launch_mm<T, true, true, mm::EpScale<T>>(p, typename mm::EpScale<T>::Args{(T*)a.dW, h, nullptr}, 1, st);
    }
    if (e != hipSuccess) return e;
  }
  if (a.db) {
    mm::k_colsum<T><<<(unsigned)mm::ceil_div(a.no, 256), 256, 0, st>>>(colpart, mm::ceil_div(a.B, mm::TILE), mm::TILE, nullptr,
                                                                     a.no, (T*)a.db, h, nullptr);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace
}  // namespace lp
