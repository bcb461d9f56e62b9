// One layer step y = r + h sigma(x W^T + b) of any width, its gradients, and 8-bit
// checkpoints, for one element type (included by one translation unit per type).
//   forward:   one product with the bias, activation, residual and checkpoint of y in its epilogue
//   backward:  g = sigma'(x W^T + b) dy   (the pre-activation is formed again; kept in the element
//                                          type, which is what the next products take: h stays out
//                                          of g, so that a small step does not push it out of the
//                                          range of f16)
//              dx = h g W (+ dy),  dW = h g^T x,  db = h sum g (from g before its rounding)
// Bound by the products (2 B ni no operations each): 8192 x 4096 -> 4096 bf16 forward with its
// checkpoint 257 us (1.07 PFLOP/s), back 263 + 241 + 214 us, of which the epilogue of g takes some 40:
// the largest tiles fill a CU, so nothing runs beside an epilogue. Small batches are bound by reading W
// (one row of 4096 x 4096: 6.8 us, 4.9 TB/s) and by launches.
#pragma once

#include <type_traits>

#include "lp_checkpoint.h"
#include "lp_internal.h"
#include "lp_mm.h"

namespace lp {
namespace wide {

using mm::f32x16;
using mm::f32x4;
using mm::Place;

// Four values of a checkpoint row of N features.
template <bool WHOLE = false>
__device__ __forceinline__ void store_ck(int8_t* row, int n, int N, f32x4 v, float inv) {
  typename mm::GVec<int8_t, 4>::type w;
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = (int8_t)ck_round(v[k], inv);
  if (WHOLE || n + 4 <= N) {
    *reinterpret_cast<typename mm::GVec<int8_t, 4>::type*>(row + n) = w;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (n + k < N) row[n + k] = w[k];
  }
}

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

// sigma and sigma'. A NaN stays one.
template <typename T, int ACT>
__device__ __forceinline__ float sigma(float z) {
  if constexpr (ACT == ACT_TANH) return sizeof(T) == 2 ? tanh16(z) : tanhf(z);
  else return z != z ? z : act_f<float, ACT>(z);
}

template <typename T, int ACT>
__device__ __forceinline__ float dsigma(float z) {
  if constexpr (ACT == ACT_TANH) return dtanh<T>(z);
  else if constexpr (ACT == ACT_IDENTITY) return 1.f;
  else return z != z ? z : dact_f<float, ACT>(z);
}

// Calls f with the activation as a compile-time constant (uniform over the launch).
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  switch (act) {
    case ACT_TANH: return f(std::integral_constant<int, ACT_TANH>{});
    case ACT_RELU: return f(std::integral_constant<int, ACT_RELU>{});
    case ACT_SMOOTHRELU: return f(std::integral_constant<int, ACT_SMOOTHRELU>{});
    default: return f(std::integral_constant<int, ACT_IDENTITY>{});
  }
}

// y = r + h sigma(D + b), optionally with its checkpoint. The 32 features of a block row are a
// checkpoint block, held by lanes l and l ^ 32; the checkpoint is that of y as stored.
template <typename T>
struct EpStep {
  static constexpr bool ONE = true;
  struct Args {
    const T* b;
    const T* r;  // nullable
    T* y;
    int8_t* y8;  // nullable
    uint8_t* ye;
    float h;
    int act;
    bool blocks_of_32() const { return y8 != nullptr; }  // a workgroup's features are whole checkpoint blocks
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    const int nb = (c.N + CK_BLOCK - 1) / CK_BLOCK;
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    mm::Rows<WHOLE, T, FM, FN> res(a.r, c.N, c);
    with_act(a.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        if (!WHOLE && c.nw + 32 * j >= c.lim) continue;
        f32x4 bias[4];
        mm::get_bias<WHOLE>(a.b, c, j, bias);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          f32x4 v[4];
          res.get(c, i, j, buf, v);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 z = mm::quad(acc[i][j], q) + bias[q];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[q][k] += a.h * sigma<T, decltype(act)::value>(z[k]);
          }
          mm::put_rows<WHOLE>(a.y, c.N, c.lim, c, i, j, buf, v);
          if (a.y8) {
            uint32_t top = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                v[q][k] = (float)(T)v[q][k];
                if (WHOLE || c.feature(j, q) + k < c.lim) top = max(top, abs_bits(v[q][k]));
              }
            top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
            const uint32_t byte = ck_byte<T>(top);
            const float inv = ck_inv(byte);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int k = 0; k < 4; ++k) v[q][k] = (float)ck_round(v[q][k], inv);
            mm::put_rows<WHOLE>(a.y8, c.N, c.lim, c, i, j, buf, v);
            const int m = c.row(i);
            if (m < c.M && c.lane < 32) a.ye[(size_t)m * nb + (c.nw + 32 * j) / CK_BLOCK] = (uint8_t)byte;
          }
        }
      }
    });
  }
};

// g = sigma'(D + b) dy (rows of ld values, zeros behind the N that count), and the sums of its
// columns over the tile's rows (fp32, before rounding)
template <typename T>
struct EpGrad {
  static constexpr bool ONE = true;
  struct Args {
    const T* b;
    const T* dy;
    T* g;
    int ld;
    float* part;  // [tile rows][N]
    T* db;        // with a single tile row: h times the sums themselves
    float h;
    int act;
    bool blocks_of_32() const { return false; }
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    float col[FN];
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    // (the largest tiles have no registers left for dy ahead: with it 90 spilled, 774 us against 751 for
    // the whole way back of 8192 x 4096 -> 4096 bf16. Floats, never read ahead, spill 74 there all the same, 144
    // bytes a lane once a tile: order of the loads and the width of the column sums do not change that)
    mm::Rows<WHOLE, T, FM, FN, sizeof(T) == 2 && (FM * FN < 8)> dy(a.dy, c.N, c);
    with_act(a.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        col[j] = 0.f;
        if (!WHOLE && c.nw + 32 * j >= a.ld) continue;
        f32x16 sums = 0.f;
        f32x4 bias[4];
        mm::get_bias<WHOLE>(a.b, c, j, bias);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
          const bool on = c.row(i) < c.M;
          f32x4 g[4];
          dy.get(c, i, j, buf, g);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4 z = mm::quad(acc[i][j], q) + bias[q];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const bool in = on && (WHOLE || c.feature(j, q) + k < c.lim);
              g[q][k] = in ? g[q][k] * dsigma<T, decltype(act)::value>(z[k]) : 0.f;
              sums[4 * q + k] += g[q][k];
            }
          }
          mm::put_rows<WHOLE>(a.g, a.ld, c.upto(a.ld), c, i, j, buf, g);
        }
        col[j] = mm::fold_columns(sums, c.lane);
      }
    });
    mm::column_sums<FN, WGM, WGN>(col, c, lds, [&](int n, float t) {
      if (a.db) a.db[n] = (T)(a.h * t);
      else a.part[(size_t)c.mt * c.N + n] = t;
    });
  }
};

// dx = h D (+ dy)
template <typename T>
struct EpDx {
  static constexpr bool ONE = false;
  struct Args {
    const T* dy;  // nullable
    T* dx;
    float h;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    mm::Rows<WHOLE, T, FM, FN> dy(a.dy, c.N, c);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4];
        dy.get(c, i, j, buf, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += mm::quad(acc[i][j], q) * a.h;
        mm::put_rows<WHOLE>(a.dx, c.N, c.lim, c, i, j, buf, v);
      }
  }
};

// Checkpoint kernels: four lanes per block of 32 features, eight features each, four blocks a
// thread in flight; bound by memory. FLAT: rows of whole blocks, which follow one another without
// a division. (With four features a thread, one block in flight and 64-bit divisions 16384 x 8192
// bf16 took 127 us to store and 133 us to load.)
constexpr int CK_U = 4;

template <typename T>
__device__ __forceinline__ void load8(const T* row, int n, int q, f32x4 (&v)[2]) {
  v[0] = mm::load4(row, n, q);
  v[1] = mm::load4(row, n + 4, q);
}

template <typename T, bool FLAT>
__global__ __launch_bounds__(256) void k_ck_store(const T* x, int8_t* x8, uint8_t* xe, uint32_t nblk, int q, uint32_t nb) {
  const int part = threadIdx.x & 3;
  const uint32_t stride = gridDim.x * 64u;
  for (uint32_t b0 = blockIdx.x * 64u + (threadIdx.x >> 2); b0 < nblk; b0 += CK_U * stride) {
    f32x4 v[CK_U][2];
    size_t at[CK_U];
    int n[CK_U];
#pragma unroll
    for (int u = 0; u < CK_U; ++u) {
      const uint32_t blk = min(b0 + u * stride, nblk - 1), row = FLAT ? 0 : blk / nb;
      n[u] = FLAT ? 8 * part : (int)(blk - row * nb) * CK_BLOCK + 8 * part;
      at[u] = FLAT ? (size_t)blk * CK_BLOCK : (size_t)row * q;
      if constexpr (FLAT) {
        const auto t = *reinterpret_cast<const typename mm::GVec<T, 8>::type*>(x + at[u] + n[u]);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[u][k >> 2][k & 3] = (float)t[k];
      } else {
        load8(x + at[u], n[u], q, v[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < CK_U; ++u) {
      const uint32_t blk = b0 + u * stride;
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) top = max(top, abs_bits(v[u][k >> 2][k & 3]));
      top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
      top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
      const uint32_t byte = ck_byte<T>(top);
      const float inv = ck_inv(byte);
      if (blk >= nblk) continue;
      if constexpr (FLAT) {
        typename mm::GVec<int8_t, 8>::type w;
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = (int8_t)ck_round(v[u][k >> 2][k & 3], inv);
        *reinterpret_cast<typename mm::GVec<int8_t, 8>::type*>(x8 + at[u] + n[u]) = w;
      } else {
        store_ck(x8 + at[u], n[u], q, v[u][0], inv);
        store_ck(x8 + at[u], n[u] + 4, q, v[u][1], inv);
      }
      if (part == 0) xe[blk] = (uint8_t)byte;
    }
  }
}

// To rows of ld >= q values, zeros behind the q that count (to the end of their last block).
template <typename T, bool FLAT>
__global__ __launch_bounds__(256) void k_ck_load(const int8_t* x8, const uint8_t* xe, T* x, uint32_t nblk, int q, uint32_t nb,
                                                 int ld) {
  const int part = threadIdx.x & 3;
  const uint32_t stride = gridDim.x * 64u;
  for (uint32_t b0 = blockIdx.x * 64u + (threadIdx.x >> 2); b0 < nblk; b0 += CK_U * stride) {
    f32x4 v[CK_U][2];
    float scale[CK_U];
    size_t row[CK_U];
    int n[CK_U];
#pragma unroll
    for (int u = 0; u < CK_U; ++u) {
      const uint32_t blk = min(b0 + u * stride, nblk - 1);
      row[u] = FLAT ? 0 : blk / nb;
      n[u] = FLAT ? 8 * part : (int)(blk - (uint32_t)row[u] * nb) * CK_BLOCK + 8 * part;
      scale[u] = ck_scale(xe[blk]);
      if constexpr (FLAT) {
        row[u] = blk;
        const auto t = *reinterpret_cast<const typename mm::GVec<int8_t, 8>::type*>(x8 + (size_t)blk * CK_BLOCK + n[u]);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[u][k >> 2][k & 3] = (float)t[k];
      } else {
        load8(x8 + row[u] * q, n[u], q, v[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < CK_U; ++u) {
      if (b0 + u * stride >= nblk) continue;
      if constexpr (FLAT) {
        typename mm::GVec<T, 8>::type w;
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = (T)(v[u][k >> 2][k & 3] * scale[u]);
        *reinterpret_cast<typename mm::GVec<T, 8>::type*>(x + row[u] * CK_BLOCK + n[u]) = w;
      } else {
        // (a block that is not finite is NaN in the row's features only: the rest of ld is zero)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[u][k >> 2][k & 3] = n[u] + k < q ? v[u][k >> 2][k & 3] * scale[u] : 0.f;
        mm::store4(x + row[u] * ld, n[u], ld, v[u][0]);
        mm::store4(x + row[u] * ld, n[u] + 4, ld, v[u][1]);
      }
    }
  }
}

// At most 16384 workgroups: CK_U blocks a thread where there are that many, and then again.
inline unsigned ck_grid(size_t nblk) {
  const size_t all = (nblk + 63) / 64;
  return (unsigned)(all <= 1024 ? all : std::min<size_t>((all + CK_U - 1) / CK_U, 16384));
}

template <typename T>
hipError_t ck_store_t(const void* x, int8_t* x8, uint8_t* xe, long B, int q, hipStream_t st) {
  const int nb = mm::ceil_div(q, CK_BLOCK);
  const uint32_t nblk = (uint32_t)(B * nb);
  if (q % CK_BLOCK == 0) k_ck_store<T, true><<<ck_grid(nblk), 256, 0, st>>>((const T*)x, x8, xe, nblk, q, nb);
  else k_ck_store<T, false><<<ck_grid(nblk), 256, 0, st>>>((const T*)x, x8, xe, nblk, q, nb);
  return hipGetLastError();
}

template <typename T>
hipError_t ck_load_t(const int8_t* x8, const uint8_t* xe, void* x, long B, int q, int ld, hipStream_t st) {
  const int nb = mm::ceil_div(q, CK_BLOCK);
  const uint32_t nblk = (uint32_t)(B * nb);
  if (q % CK_BLOCK == 0 && ld == q) k_ck_load<T, true><<<ck_grid(nblk), 256, 0, st>>>(x8, xe, (T*)x, nblk, q, nb, ld);
  else k_ck_load<T, false><<<ck_grid(nblk), 256, 0, st>>>(x8, xe, (T*)x, nblk, q, nb, ld);
  return hipGetLastError();
}

inline mm::Prob prob(const void* A, long lda, const void* B, long ldb, int M, int N, int K) {
  return mm::Prob{A, B, lda, ldb, M, N, K, nullptr, 0, 0, 0, 0, 0};
}

template <typename T>
hipError_t step_forward_t(const StepArgs& a, hipStream_t st) {
  const StepLayout l = step_layout(a.dtype, a.B, a.ni, a.no);
  char* w = static_cast<char*>(a.ws);
  const mm::Operands<T> o(a.x, a.B, w + l.x, a.W, a.no, w + l.W, a.ni, l.z.tile == 1, st);
  if (o.e != hipSuccess) return o.e;
  typename EpStep<T>::Args e{(const T*)a.b, (const T*)a.r, (T*)a.y, a.y8, a.ye, (float)a.h, a.act};
  return mm::launch_mm<T, false, false, EpStep<T>>(prob(o.p[0], o.ld[0], o.p[1], o.ld[1], a.B, a.no, a.ni), e, l.z,
                                                  w + l.part, st);
}

template <typename T>
hipError_t step_backward_t(const StepArgs& a, hipStream_t st) {
  const StepLayout l = step_layout(a.dtype, a.B, a.ni, a.no);
  char* w = static_cast<char*>(a.ws);
  T* g = reinterpret_cast<T*>(w + l.g);
  const int ldg = mm::padded(sizeof(T), a.no), ldck = mm::padded(sizeof(T), a.ni);
  float* colpart = reinterpret_cast<float*>(w + l.col);
  hipError_t e = hipSuccess;
  if (!a.x && a.B && (e = ck_load_t<T>(a.x8, a.xe, w + l.x, a.B, a.ni, ldck, st)) != hipSuccess) return e;
  const mm::Operands<T> o(a.B ? a.x : nullptr, a.B, w + l.x, a.W, a.no, w + l.W, a.ni, false, st);
  if (o.e != hipSuccess) return o.e;
  const T* x = a.x ? o.p[0] : reinterpret_cast<const T*>(w + l.x);
  const long ldx = a.x ? o.ld[0] : ldck;
  const float h = (float)a.h;
  const bool own_db = a.B && a.db && l.z.tm == 1;  // a single tile row leaves db itself
  if (a.B) {  // (an empty batch leaves zero sums: products over no rows)
    typename EpGrad<T>::Args eg{(const T*)a.b, (const T*)a.dy, g, ldg, colpart, own_db ? (T*)a.db : nullptr, h, a.act};
    e = mm::launch_mm<T, false, false, EpGrad<T>>(prob(x, ldx, o.p[1], o.ld[1], a.B, a.no, a.ni), eg, l.z, w + l.part, st);
    if (e != hipSuccess) return e;
  }
  typedef mm::EpScale<T> EpDW;
  const typename EpDx<T>::Args ed{a.residual ? (const T*)a.dy : nullptr, (T*)a.dx, h};
  const typename EpDW::Args ew{(T*)a.dW, h, nullptr};
  const mm::Prob px = prob(g, ldg, o.p[1], o.ld[1], a.B, a.ni, a.no), pw = prob(g, ldg, x, ldx, a.no, a.ni, a.B);
  const bool dx = a.dx && a.B;
  const mm::ColSum<T> cs{colpart, a.B ? l.z.tm : 0, l.z.tile, nullptr, a.no, own_db ? nullptr : (T*)a.db, h, nullptr};
  if (dx && a.dW) return mm::launch_both<T, EpDx<T>, EpDW>(px, ed, l.zx, pw, ew, l.zw, cs, w + l.part, st);
  if (dx) e = mm::launch_mm<T, false, true, EpDx<T>>(px, ed, l.zx, w + l.part, st);
  if (a.dW && e == hipSuccess) e = mm::launch_mm<T, true, true, EpDW>(pw, ew, l.zw, w + l.part, st);
  if (cs.out && e == hipSuccess) e = mm::launch_colsum(cs, st);
  return e;
}

}  // namespace wide
}  // namespace lp
