// Softmax cross-entropy of integer labels over a large vocabulary, for one element type
// (included by one translation unit per type). With z_k = W u_k + mu and the rows k that have
// a label c_k in 0..nc-1 (n of them):
//   lse_k = log sum_j exp z_kj,  loss_k = lse_k - z_k[c_k],  J = (1/n) sum loss_k,
//   P = softmax(z) - onehot,  du = (s/n) P W,  dW = (s/n) P^T u,  dmu = (s/n) sum_k P_k.
// A product over all classes leaves, per tile of classes, each row's maximum and sum of exponentials
// (8 bytes where the tile had 128 logits); they are joined in order into lse. For the gradients a
// piece of the vocabulary is taken after the other: its logits, kept by the first product or, of
// batches too large for that (label_layout), formed a second time, become a piece of P in the
// workspace in the element type (the type of the next products' operands), as P times PSCALE: 2^14
// for f16, whose range would otherwise lose the small probabilities of a large vocabulary (the least
// normal value then stands for 3.7e-9), a power of two that the epilogues take back exactly.
// Bound by the products: 8192 rows of 2048 features, 65536 classes bf16 6.5 ms, of which the three
// products 533, 449 and 433 us a piece of 16384 classes (1.01, 1.20 and 1.24 PFLOP/s for the 98 % of the
// rows that have a label; the first also writes the logits) and P 162 us (reading and writing, 4.9 TB/s).
// Losses alone of 16 rows of 4096 features, 131072 classes: 179 us, reading the weights at 6 TB/s.
// Rows without a label take no part in the gradients, whatever they hold: the labelled rows are
// first copied together, so a product runs over n rows.
#pragma once

#include <type_traits>

#include "lp_internal.h"
#include "lp_mm.h"

namespace lp {
namespace wide {

using mm::f32x16;
using mm::f32x4;
using mm::Place;

template <typename T>
constexpr float PSCALE = std::is_same<T, _Float16>::value ? 16384.f : 1.f;

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(1.4426950408889634f * x); }

struct MaxSum {
  float m, s;  // maximum and sum of exp(z - m); m = -inf, s = 0 where no class is left
};

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return MaxSum{m, a.s + b.s};  // (a NaN's sum stays one)
  return MaxSum{m, a.s * exp_of(a.m - m) + b.s * exp_of(b.m - m)};
}

// Per row: maximum and sum of exponentials over the tile's classes, and the label's logit.
template <typename T>
struct EpLse {
  static constexpr bool ONE = true;
  struct Args {
    const T* mu;            // nullable, of the product's first class
    const int64_t* labels;  // of D's rows
    MaxSum* part;           // [class tiles][rows]
    float* zl;              // [rows]: logit of the label
    long rows;              // row stride of part
    int j0;                 // first class of the product
    float* z;               // logits to keep, rows of ldz values (nullable)
    int ldz;
    bool blocks_of_32() const { return false; }
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    MaxSum* red = reinterpret_cast<MaxSum*>(lds + WGM * WGN * mm::WAVE_LDS / 4);  // [WGN][rows of the tile]
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    constexpr int BM = WGM * FM * 32;
    f32x4 mu[FN][4];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        mu[j][q] = a.mu ? mm::load4<WHOLE>(a.mu, c.feature(j, q), c.lim) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = c.row(i);
      // the label's place among the wave's classes
      const int64_t l = (m < c.M ? a.labels[m] : -1) - a.j0;
      const int at = l >= 0 && l < c.lim ? (int)l - c.nw : -1;
      float top = -INFINITY, zl = 0.f;
      bool mine = false;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int n = c.feature(j, r >> 2) - c.nw + (r & 3);
          const float z = acc[i][j][r] + mu[j][r >> 2][r & 3];
          if (at == n) zl = z, mine = true;
          if (WHOLE || c.nw + n < c.lim) top = fmaxf(top, z);
        }
      if (mine) a.zl[m] = zl;
      if (a.z) {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          f32x4 v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = mm::quad(acc[i][j], q) + mu[j][q];
          mm::put_rows<WHOLE>(a.z, a.ldz, c.lim, c, i, j, buf, v);
        }
      }
      // a NaN is no maximum; it comes back through the sum (exp of NaN)
      const float ref = top == -INFINITY ? 0.f : top;
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (WHOLE || c.feature(j, r >> 2) + (r & 3) < c.lim) s += exp_of((acc[i][j][r] + mu[j][r >> 2][r & 3]) - ref);
      MaxSum v{top, s};
      v = join(v, MaxSum{__shfl_xor(v.m, 32, 64), __shfl_xor(v.s, 32, 64)});
      if (c.lane < 32) red[c.wn * BM + c.wm * FM * 32 + 32 * i + c.lane] = v;
    }
    c.meet<WGM * WGN>();
    for (int r = threadIdx.x; r < BM; r += 64 * WGM * WGN) {
      MaxSum v = red[r];
#pragma unroll
      for (int w = 1; w < WGN; ++w) v = join(v, red[w * BM + r]);
      if (c.m0 + r < c.M) a.part[(size_t)c.nt * a.rows + c.m0 + r] = v;
    }
  }
};

// A piece of P (times PSCALE; rows of ld values, zeros behind the N that count), and its column
// sums over the tile's rows (fp32, before rounding).
template <typename T>
struct EpProb {
  static constexpr bool ONE = false;
  struct Args {
    const T* mu;            // nullable, of the piece
    const int64_t* labels;  // of D's rows
    const float* lse;
    T* P;
    int ld;
    float* part;            // [tile rows][part_ld], from the piece's first class on (nullable)
    long part_ld;
    T* dmu;                 // with a single tile row: scale[0] times the sums themselves (nullable)
    const float* scale;
    int j0;                 // first class of the piece
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    float col[FN];
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    int at[FM];  // the label's place among the wave's classes
    float lse[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = min(c.row(i), c.M - 1);
      const int64_t l = a.labels[m] - a.j0;
      at[i] = l >= 0 && l < c.lim ? (int)l - c.nw : -1;
      lse[i] = a.lse[m];
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      col[j] = 0.f;
      if (!WHOLE && c.nw + 32 * j >= a.ld) continue;
      f32x16 sums = 0.f;
      f32x4 mu[4];
      mm::get_bias<WHOLE>(a.mu, c, j, mu);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const bool on = c.row(i) < c.M;
        f32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 z = mm::quad(acc[i][j], q) + mu[q];
          const int n = c.feature(j, q) - c.nw;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float p = exp_of(z[k] - lse[i]) - (at[i] == n + k ? 1.f : 0.f);
            if (!on || (!WHOLE && c.nw + n + k >= c.lim)) p = 0.f;
            sums[4 * q + k] += p;
            v[q][k] = p * PSCALE<T>;
          }
        }
        mm::put_rows<WHOLE>(a.P, a.ld, c.upto(a.ld), c, i, j, buf, v);
      }
      if (a.part) col[j] = mm::fold_columns(sums, c.lane);
    }
    if (a.part)
      mm::column_sums<FN, WGM, WGN>(col, c, lds, [&](int n, float t) {
        if (a.dmu) a.dmu[n] = (T)(t * a.scale[0]);
        else a.part[(size_t)c.mt * a.part_ld + n] = t;
      });
  }
};

// du of a piece: added to the earlier pieces' sum in fp32, or, with the last piece, scaled,
// rounded and written to the row that the labelled row came from.
template <typename T>
struct EpDu {
  static constexpr bool ONE = false;
  struct Args {
    float* acc32;      // [rows][N]: sum over the pieces
    T* du;
    const int* from;   // row of u that a labelled row came from
    const float* scale;
    float f;
    int first, last;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    const float f = a.f * a.scale[0];
    unsigned char* buf = mm::wave_lds(lds, c, WGN);
    mm::Rows<WHOLE, float, FM, FN> sum(a.first ? nullptr : a.acc32, c.N, c);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4];
        sum.get(c, i, j, buf, v);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v[q] += mm::quad(acc[i][j], q);
          if (a.last) v[q] *= f;
        }
        if (a.last) mm::put_rows<WHOLE>(a.du, c.N, c.lim, c, i, j, buf, v, [&](int m) { return a.from[m]; });
        else mm::put_rows<WHOLE>(a.acc32, c.N, c.lim, c, i, j, buf, v);
      }
  }
};

// Lists the rows that have a label (in order): from[r] = row, to[row] = r or -1, lab[r], their
// number, and gs / max(1, number). One workgroup.
static __global__ __launch_bounds__(1024) void k_rows(const int64_t* labels, int B, int nc, double gs, int* from, int* to,
                                               int64_t* lab, int* count, float* scale) {
  __shared__ int wave_n[16];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  int base = 0;
  for (int b0 = 0; b0 < B; b0 += 1024) {
    const int b = b0 + t;
    const int64_t l = b < B ? labels[b] : -1;
    const bool on = l >= 0 && l < nc;
    const uint64_t mask = __ballot(on);
    if (lane == 0) wave_n[w] = __popcll(mask);
    __syncthreads();
    int at = base, all = 0;
    for (int k = 0; k < 16; ++k) {
      if (k < w) at += wave_n[k];
      all += wave_n[k];
    }
    at += __popcll(mask & ((1ull << lane) - 1));
    if (on) {
      from[at] = b;
      lab[at] = l;
    }
    if (b < B) to[b] = on ? at : -1;
    base += all;
    __syncthreads();
  }
  if (t == 0) {
    count[0] = base;
    scale[0] = (float)(gs / (double)(base > 0 ? base : 1));
  }
}

// Copies the labelled rows together (rows of ld values, zeros behind the q that count); the other
// rows' loss and gradient are zero. A wave per row. Batches of at most ROWS_EACH rows have no k_rows:
// every workgroup then counts the labelled rows before its own (up to 32 KB of labels from cache).
constexpr int ROWS_EACH = 4096;
template <typename T>
__global__ __launch_bounds__(256) void k_gather(const T* u, const int64_t* labels, int B, int q, int nc, double gs, int* from,
                                                int* to, int64_t* lab, int* count, float* scale, T* uc, int ld, T* du,
                                                T* dmu, float* row) {
  __shared__ int sh[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, b0 = blockIdx.x * 4, b = b0 + wave;
  int r = -1;
  if (B <= ROWS_EACH) {  // (the same for all)
    int n = 0;
    for (int i = threadIdx.x; i < b0; i += 256) n += labels[i] >= 0 && labels[i] < nc;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    if (lane == 0) sh[wave] = n;
    __syncthreads();
    int at = sh[0] + sh[1] + sh[2] + sh[3];
    for (int i = 0; i < 4; ++i) {
      const int64_t l = b0 + i < B ? labels[b0 + i] : -1;
      const bool on = l >= 0 && l < nc;
      if (i == wave && on) {
        r = at;
        if (lane == 0) from[at] = b, lab[at] = l;
      }
      at += on;
    }
    if (b0 + 4 >= B) {
      if (threadIdx.x == 0) {
        count[0] = at;
        scale[0] = (float)(gs / (double)(at > 0 ? at : 1));
      }
      if (at == 0 && dmu)  // (with a single column partial the products write dmu, if there are any)
        for (int i = threadIdx.x; i < nc; i += 256) dmu[i] = (T)0.f;
    }
  } else if (b < B) {
    r = to[b];
  }
  if (b >= B) return;
  if (r < 0) {
    if (lane == 0) row[b] = 0.f;
    if (du)
      for (int i = 4 * lane; i < q; i += 256) mm::store4(du + (size_t)b * q, i, q, f32x4{0.f, 0.f, 0.f, 0.f});
    return;
  }
  for (int i = 4 * lane; i < ld; i += 256) mm::store4(uc + (size_t)r * ld, i, ld, mm::load4(u + (size_t)b * q, i, q));
}

// A piece of P (times PSCALE; rows of ldp values, zeros from class n to `to`, a multiple of four) from
// its kept logits z (rows of ldz values; of floats P may be z itself), and its column sums over
// PROB_ROWS rows a workgroup. Four classes a thread.
constexpr int PROB_ROWS = 32;
template <typename T>
__global__ __launch_bounds__(256) void k_prob(const float* z, int ldz, const float* lse, const int64_t* lab, const int* count,
                                              int j0, int n, int to, T* P, int ldp, float* part, T* dmu, const float* scale) {
  const int c = (blockIdx.y * 256 + threadIdx.x) * 4, m0 = blockIdx.x * PROB_ROWS, m1 = min(m0 + PROB_ROWS, *count);
  if (c >= to || m0 >= m1) return;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int m = m0; m < m1; ++m) {
    f32x4 v = mm::load4<true>(z + (size_t)m * ldz, c, to);
    const float l = lse[m];
    const int64_t at = lab[m] - j0 - c;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = c + k < n ? exp_of(v[k] - l) - (at == k ? 1.f : 0.f) : 0.f;
    sum += v;
    mm::store4<true>(P + (size_t)m * ldp, c, to, v * PSCALE<T>);
  }
  if (dmu) mm::store4(dmu, c, n, sum * scale[0]);
  else if (part) mm::store4(part + (size_t)blockIdx.x * n, c, n, sum);
}

// Joins the class tiles of a row: lse and the loss. `per` rows (a power of two) by 256 / per threads
// a workgroup: many threads a row where there are few rows (16 rows of 1024 tiles: 33 us with 16
// threads a row, 5 with 128).
// labels as in EpLse; a row without one has loss 0. from (nullable): where row r's loss goes. J (a single
// workgroup for all rows): the mean of the labelled rows' losses, summed in fp64 in order.
static __global__ __launch_bounds__(256) void k_lse(const MaxSum* part, int tiles, long rows, const int64_t* labels, int nc,
                                                    const float* zl, const int* count, int M, const int* from, float* lse,
                                                    float* loss, int per, float* J) {
  __shared__ MaxSum red[256];
  __shared__ float rows_loss[256];
  if (count) M = min(M, *count);
  const int r = threadIdx.x & (per - 1), g = threadIdx.x / per, groups = 256 / per, m = blockIdx.x * per + r;
  MaxSum v{-INFINITY, 0.f};
  if (m < M) {
    int t = g;
    for (; t + 3 * groups < tiles; t += 4 * groups) {
      MaxSum w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = part[(size_t)(t + k * groups) * rows + m];
#pragma unroll
      for (int k = 0; k < 4; ++k) v = join(v, w[k]);
    }
    for (; t < tiles; t += groups) v = join(v, part[(size_t)t * rows + m]);
  }
  red[threadIdx.x] = v;
  for (int half = groups / 2; half > 0; half /= 2) {
    __syncthreads();
    if (g < half) red[threadIdx.x] = v = join(v, red[threadIdx.x + half * per]);
  }
  if (g == 0 && m < M) {
    const float l = v.m + logf(v.s);
    if (lse) lse[m] = l;
    const int64_t lab = labels[m];
    const bool on = lab >= 0 && lab < nc;
    const float d = on ? l - zl[m] : 0.f;
    loss[from ? from[m] : m] = d;
    rows_loss[r] = d;
  }
  if (!J) return;
  __syncthreads();
  if (threadIdx.x) return;
  double sum = 0.0;
  int n = 0;
  for (int k = 0; k < per && k < M; ++k) {
    const int64_t lab = labels[k];
    if (lab >= 0 && lab < nc) sum += (double)rows_loss[k], ++n;
  }
  J[0] = (float)(sum / (n > 0 ? n : 1));
}

// J = sum of the rows' losses / number of labelled rows, in fp64 and in a fixed order.
static __global__ __launch_bounds__(1024) void k_mean_loss(const float* loss, const int64_t* labels, int B, int nc, float* J) {
  __shared__ double sh[1024];
  double s = 0.0, n = 0.0;
  for (int b = threadIdx.x; b < B; b += 1024) {
    s += (double)loss[b];
    n += labels[b] >= 0 && labels[b] < nc ? 1.0 : 0.0;
  }
  s = block_sum<1024>(s, sh);
  n = block_sum<1024>(n, sh);
  if (threadIdx.x == 0) J[0] = (float)(s / (n > 0.0 ? n : 1.0));
}

template <typename T>
hipError_t loss_labels_t(const LabelArgs& a, hipStream_t st) {
  const bool grad = a.du || a.dW || a.dmu;
  const LabelLayout l = label_layout(a.dtype, a.B, a.q, a.nc, grad);
  char* w = static_cast<char*>(a.ws);
  MaxSum* part = reinterpret_cast<MaxSum*>(w + l.part);
  float* zl = reinterpret_cast<float*>(w + l.zl);
  float* row = a.row ? a.row : reinterpret_cast<float*>(w + l.row);
  const int ldu = mm::padded(sizeof(T), a.q);
  const T* W = static_cast<const T*>(a.W);
  const T* mu = static_cast<const T*>(a.mu);
  int* from = reinterpret_cast<int*>(w + l.from);
  int* to = reinterpret_cast<int*>(w + l.to);
  int64_t* lab = reinterpret_cast<int64_t*>(w + l.lab);
  int* count = reinterpret_cast<int*>(w + l.count);
  float* scale = reinterpret_cast<float*>(w + l.scale);
  float* lse = reinterpret_cast<float*>(w + l.lse);
  T* uc = reinterpret_cast<T*>(w + l.u);
  T* P = reinterpret_cast<T*>(w + l.P);
  float* acc32 = reinterpret_cast<float*>(w + l.du);
  float* col = reinterpret_cast<float*>(w + l.col);
  void* split = w + l.split;
  hipError_t e = hipSuccess;
  const bool as_is = a.q % (16 / (int)sizeof(T)) == 0 && (uintptr_t)W % 16 == 0;  // the weights
  const int piece = as_is ? l.piece : l.copied;
  float* z = l.keep ? reinterpret_cast<float*>(w + l.z) : nullptr;
  const int ldz = mm::padded(sizeof(T), a.nc);
  // rows of the products: u's own, or with gradients the labelled ones
  const T* rows = nullptr;
  long ldr = 0;
  if (grad) {
    if (a.B > ROWS_EACH) k_rows<<<1, 1024, 0, st>>>(a.labels, a.B, a.nc, a.gscale, from, to, lab, count, scale);
    if (a.B)
      k_gather<T><<<(unsigned)mm::ceil_div(a.B, 4), 256, 0, st>>>((const T*)a.u, a.labels, a.B, a.q, a.nc, a.gscale, from, to, lab,
                                                                  count, scale, uc, ldu, (T*)a.du, (T*)a.dmu, row);
    else k_rows<<<1, 1024, 0, st>>>(a.labels, 0, a.nc, a.gscale, from, to, lab, count, scale);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const int* cnt = grad ? count : nullptr;
  const int64_t* labels = grad ? lab : a.labels;
  int tiles = 0;  // class tiles so far
  for (int j0 = 0; j0 < a.nc && a.B; j0 += piece) {
    const int n = std::min(piece, a.nc - j0);
    const mm::Plan pl = mm::plan_rows(sizeof(T), a.B, n, a.q);
    // (u is copied, if it has to be, with the first piece)
    const mm::Operands<T> o(grad || j0 ? nullptr : a.u, a.B, uc, W + (size_t)j0 * a.q, n, w + l.W, a.q, pl.tile == 1, st);
    if (o.e != hipSuccess) return o.e;
    if (j0 == 0) {
      rows = grad ? uc : o.p[0];
      ldr = grad ? ldu : o.ld[0];
    }
    typename EpLse<T>::Args ea{mu ? mu + j0 : nullptr, labels, part + (size_t)tiles * a.B, zl, a.B, j0, z ? z + j0 : nullptr, ldz};
    const mm::Prob p{rows, o.p[1], ldr, o.ld[1], a.B, n, a.q, cnt, 1, 0, 0, 0, 0};
    if ((e = mm::launch_mm<T, false, false, EpLse<T>>(p, ea, pl, split, st)) != hipSuccess) return e;
    tiles += pl.tn;
  }
  // few rows and tiles: one workgroup joins them all and takes the mean
  const bool small = a.B <= 64 && (long)a.B * tiles <= 4096;
  if (a.B) {
    int per = a.B >= 2048 ? 16 : 2;
    if (small)
      while (per < a.B) per *= 2;
    k_lse<<<(unsigned)mm::ceil_div(a.B, per), 256, 0, st>>>(part, tiles, a.B, labels, a.nc, zl, cnt, a.B, grad ? from : nullptr,
                                                            grad ? lse : nullptr, row, per, small ? a.J : nullptr);
  }
  if (!a.B || !small) k_mean_loss<<<1, 1024, 0, st>>>(row, a.labels, a.B, a.nc, a.J);
  if ((e = hipGetLastError()) != hipSuccess || !grad) return e;
  for (int j0 = 0; j0 < a.nc; j0 += piece) {
    const int n = std::min(piece, a.nc - j0);
    // (the weights' copy of a single piece is still there; of one row's product there was none)
    const bool again = a.B && (piece < a.nc || a.B == 1);
    const mm::Operands<T> o(nullptr, 0, nullptr, W + (size_t)j0 * a.q, again ? n : 0, w + l.W, a.q, false, st);
    if (o.e != hipSuccess) return o.e;
    T* dmu = a.dmu ? (T*)a.dmu + j0 : nullptr;
    int col_rows = 0, col_step = 1;  // column partials, and the rows of one
    const bool place = z && sizeof(T) == 4;  // P takes its logits' place: the last piece ends with their rows
    const int wide = place && j0 + n == a.nc ? ldz - j0 : mm::padded(sizeof(T), n), ldp = place ? ldz : wide;
    if (place) P = reinterpret_cast<T*>(z + j0);
    if (a.B && z) {
      col_rows = mm::ceil_div(a.B, PROB_ROWS), col_step = PROB_ROWS;
      const bool own = col_rows == 1;
      k_prob<T><<<dim3((unsigned)col_rows, (unsigned)mm::ceil_div(wide, 1024)), 256, 0, st>>>(
          z + j0, ldz, lse, lab, count, j0, n, wide, P, ldp, dmu ? col : nullptr, own ? dmu : nullptr, scale);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    } else if (a.B) {
      const mm::Plan pl = mm::plan_of(sizeof(T), a.B, n, a.q);  // (one row's logits are always kept)
      col_rows = pl.tm, col_step = pl.tile;
      typename EpProb<T>::Args ep{mu ? mu + j0 : nullptr, lab, lse, P, ldp, dmu ? col : nullptr, n,
                                  col_rows == 1 ? dmu : nullptr, scale, j0};
      const mm::Prob pp{uc, o.p[1], ldu, o.ld[1], a.B, n, a.q, count, 1, 0, 0, 0, 0};
      if ((e = mm::launch_mm<T, false, false, EpProb<T>>(pp, ep, pl, split, st)) != hipSuccess) return e;
    }
    // (a single column partial's kernel has left dmu itself)
    const mm::ColSum<T> cs{col, col_rows, col_step, a.B ? count : nullptr, n, col_rows != 1 ? dmu : nullptr, 1.f, scale};
    typedef mm::EpScale<T> EpDW;
    const typename EpDu<T>::Args ed{acc32, (T*)a.du, from, scale, 1.f / PSCALE<T>, j0 == 0, j0 + n == a.nc};
    const typename EpDW::Args ew{a.dW ? (T*)a.dW + (size_t)j0 * a.q : nullptr, 1.f / PSCALE<T>, scale};
    const mm::Prob pd{P, o.p[1], ldp, o.ld[1], a.B, a.q, n, count, 1, 0, 0, 0, 0}, pw{P, uc, ldp, ldu, n, a.q, a.B, count, 0, 1, 0, 0, 0};
    const mm::Plan zd = mm::plan_of(sizeof(T), a.B, a.q, n), zw = mm::plan_of(sizeof(T), n, a.q, a.B);
    const bool du = a.du && a.B;
    if (du && a.dW) {
      e = mm::launch_both<T, EpDu<T>, EpDW>(pd, ed, zd, pw, ew, zw, cs, split, st);
    } else {
      if (du) e = mm::launch_mm<T, false, true, EpDu<T>>(pd, ed, zd, split, st);
      if (a.dW && e == hipSuccess) e = mm::launch_mm<T, true, true, EpDW>(pw, ew, zw, split, st);
      if (cs.out && e == hipSuccess) e = mm::launch_colsum(cs, st);
    }
    if (e != hipSuccess) return e;
  }
  return hipGetLastError();
}

}  // namespace wide
}  // namespace lp
