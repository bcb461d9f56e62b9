// Matrix products with fused epilogues for layers of any width and heads over large
// vocabularies: D[m][n] = sum_k A[m][k] B[n][k], one tile of D per workgroup, handed to
// an epilogue (bias, activation, residual, softmax statistics, ...) while it is still in
// registers. Element types bf16, f16 and float, accumulation in fp32.
//
// Each operand is stored either with the contraction index running fastest ("rows":
// A[m][k], leading dimension lda) or with it running slowest ("columns": A[k][m]), so the
// three products of a layer (z = x W^T, dx = g W, dW = g^T x) read the caller's arrays as
// they are.
//
// Matrix instructions: 32 x 32 x 16 (bf16, f16) and 32 x 32 x 2 (float), with n on the
// instruction's rows and m on its columns. Lane l then holds, of each 32 x 32 block, the 16
// values n = 8 (r / 4) + 4 (l / 32) + r % 4, r = 0..15, of the single row m = l % 32: four
// consecutive features at a time (vector loads and stores of rows), and sums over a row
// need one exchange with lane l ^ 32.
//
// LDS holds KB = 128 bytes of the contraction (64 values of 16 bits, 32 floats) of every
// row of the tile, twice (one stage is filled while the other is read; one barrier a
// stage), in 16-byte chunks.
//   rows:    chunk c of row r lies at r * 8 + (c ^ (r & 7)): the eight chunks of a bank
//            cycle that a fragment read takes (eight rows, one chunk index) hit different
//            banks, and so do the writes.
//   columns: row k of the stage holds its R columns; fragments of 16-bit types are read
//            with the transposing LDS load, which hands lane i of 16 the values (k0..k0+3,
//            column i) from four rows' 32-byte pieces. Chunks are exchanged by 64 bytes
//            times k % 4, so that those four rows lie in different banks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "lp_device.h"

namespace lp {
namespace mm {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int KB = 128;  // bytes of the contraction per row and stage

// N consecutive values in global memory, with their element's alignment
template <typename T, int N> struct GVec { typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };

template <typename T> struct Frag;  // the 16 bytes a lane feeds to the matrix instructions
template <> struct Frag<bf16> { typedef b16x8 type; };
template <> struct Frag<f16> { typedef h16x8 type; };
template <> struct Frag<float> { typedef f32x4 type; };

__device__ __forceinline__ f32x16 mma(b16x8 a, b16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(h16x8 a, h16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f32x4 a, f32x4 b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// Four values of a row of N features from feature n on, as floats (0 past the row's end;
// WHOLE: they are all there).
template <bool WHOLE = false, typename T>
__device__ __forceinline__ f32x4 load4(const T* row, int n, int N) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (WHOLE || n + 4 <= N) {
    const auto x = *reinterpret_cast<const typename GVec<T, 4>::type*>(row + n);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = (float)x[k];
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (n + k < N) v[k] = (float)row[n + k];
  }
  return v;
}

template <bool WHOLE = false, typename T>
__device__ __forceinline__ void store4(T* row, int n, int N, f32x4 v) {
  if (WHOLE || n + 4 <= N) {
    typename GVec<T, 4>::type x;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = (T)v[k];
    *reinterpret_cast<typename GVec<T, 4>::type*>(row + n) = x;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (n + k < N) row[n + k] = (T)v[k];
  }
}

// One operand's tile of R rows of D, straight from global memory to LDS. Arrays start on 16
// bytes and so do their rows.
template <typename T, int R, int NT, bool COLS>
struct Stage {
  static constexpr int V = 16 / sizeof(T);           // values per chunk
  static constexpr int BK = KB / (int)sizeof(T);     // contraction values per stage
  static constexpr int PER = R * 8 / NT;             // chunks per thread
  static constexpr int CH = R / V;                   // columns: chunks per row of the stage
  static constexpr int SWZ = (sizeof(T) == 2 ? 12 : 8) & (CH - 1);
  static_assert(R * 8 % NT == 0, "whole chunks per thread");
  static_assert(NT % 64 == 0 && (COLS ? NT / CH % 4 == 0 : true), "the exchange is the same for all of a thread's chunks");

  static __device__ __forceinline__ int swz(int k) {  // columns: chunk exchange of row k
    return (sizeof(T) == 2 ? k << 2 : k << 1) & SWZ;
  }

  const unsigned char* base;  // of the next stage (uniform)
  long left;                  // bytes from base to the end of the last row that counts
  long step;                  // bytes per stage
  uint32_t off[PER];
  int kc;                     // rows: first contraction index of this thread's chunks
  int k, k1;

  // rows r0.. of `rows`, contraction k0.. up to k1
  __device__ __forceinline__ void start(const void* p, long ld, int r0, int rows, int k0, int k1_) {
    const int t = threadIdx.x;
    k = k0;
    k1 = k1_;
    if constexpr (!COLS) {
      const int c = (t & 7) ^ ((t >> 3) & 7);
      kc = c * V;
      base = static_cast<const unsigned char*>(p) + ((long)r0 * ld + k0) * (long)sizeof(T);
      left = ((long)(rows - r0) * ld - k0) * (long)sizeof(T);
      step = KB;
#pragma unroll
      for (int i = 0; i < PER; ++i) off[i] = (uint32_t)((t + i * NT) >> 3) * (uint32_t)(ld * sizeof(T)) + c * 16;
    } else {
      const int c = (t % CH) ^ swz(t / CH);
      kc = 0;
      base = static_cast<const unsigned char*>(p) + ((long)k0 * ld + r0) * (long)sizeof(T);
      left = ((long)(k1 - k0) * ld - r0) * (long)sizeof(T);
      step = BK * ld * (long)sizeof(T);
#pragma unroll
      for (int i = 0; i < PER; ++i) off[i] = (uint32_t)((t + i * NT) / CH) * (uint32_t)(ld * sizeof(T)) + c * 16;
    }
  }

  // Requests the next stage. Loads past `left` give zeros: rows past the last (rows), contraction
  // indices past the last (columns); so does an offset of 2^31 (rows: past the contraction's end).
  __device__ __forceinline__ void load(unsigned char* lds) {
#ifdef __HIP_DEVICE_COMPILE__  // (buffer resources are no type of the host compilation)
    typedef __attribute__((address_space(3))) void lds_void;
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, left < 0x7fffffff ? (int)left : 0x7fffffff, 0x00020000);
    const bool past = !COLS && k + kc >= k1;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(lds + (i * NT + (threadIdx.x & ~63)) * 16), 16,
                                               past ? 0x80000000u : off[i], 0, 0, 0);
    base += step;
    left -= step;
    k += BK;
#endif
  }

  // the fragment of rows r0..r0+31 and contraction step kk (two chunks) of a stage
  static __device__ __forceinline__ typename Frag<T>::type frag(const unsigned char* lds, int r0, int kk, int lane) {
    typedef typename Frag<T>::type F;
    if constexpr (!COLS) {
      const int r = r0 + (lane & 31), c = 2 * kk + (lane >> 5);
      return *reinterpret_cast<const F*>(lds + (r * 8 + (c ^ (r & 7))) * 16);
    } else if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) s16x4 lds4;
      const int col = r0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      s16x4 h[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int k = 16 * kk + 8 * (lane >> 5) + 4 * j + ((lane >> 2) & 3);
        const unsigned char* a = lds + (k * CH + ((col / V) ^ swz(k))) * 16 + (col % V) * 2;
        h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)a);
      }
      return __builtin_bit_cast(F, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      F v;
      const int col = r0 + (lane & 31);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = 8 * kk + 4 * (lane >> 5) + j;
        v[j] = *reinterpret_cast<const float*>(lds + (k * CH + ((col / V) ^ swz(k))) * 16 + (col % V) * 4);
      }
      return v;
    }
  }
};

struct Prob {
  const void* A;
  const void* B;
  long lda, ldb;
  int M, N, K;
  const int* count;  // device count of rows that replaces M or K where it is smaller (nullable)
  int count_m, count_k;
  int tm, tn;        // tiles of D
  int kper;          // contraction per split (grid y), a multiple of a stage's
};

// What an epilogue knows of its place: row m of D is mw + 32 i + lane % 32 of block row i,
// feature n = nw + 32 j + 8 q + 4 (lane / 32) of quad q of block column j.
struct Place {
  int M, N;
  int m0, n0;      // the workgroup's tile
  int mw, nw;      // the wave's part of it
  int wm, wn;      // the wave's place in the workgroup
  int mt, nt;      // tile indices
  int split;
  int lane;
  __device__ __forceinline__ int row(int i) const { return mw + 32 * i + (lane & 31); }
  __device__ __forceinline__ int feature(int j, int q) const { return nw + 32 * j + 8 * q + 4 * (lane >> 5); }
};

// Workgroups go to the eight XCDs in turn, each with its own L2: an XCD takes a run of
// tiles, ordered in groups of GROUP tile rows by all tile columns, so that neighbours in
// time share their operands.
constexpr int GROUP = 8;
__device__ __forceinline__ void tile_of(int id, int tm, int tn, int& mt, int& nt) {
  const int total = tm * tn, q = total / 8, r = total % 8, x = id % 8;
  const int at = x * q + min(x, r) + id / 8;
  const int g = at / (GROUP * tn), in = at - g * GROUP * tn, rows = min(tm - g * GROUP, GROUP);
  mt = g * GROUP + in % rows;
  nt = in / rows;
}

template <typename T, int BM, int BN, int WGM, int WGN, bool AT, bool BT, class E>
__global__ __launch_bounds__(64 * WGM * WGN) void k_mm(Prob p, typename E::Args ea) {
  constexpr int NT = 64 * WGM * WGN, FM = BM / WGM / 32, FN = BN / WGN / 32;
  typedef Stage<T, BM, NT, AT> SA;
  typedef Stage<T, BN, NT, BT> SB;
  __shared__ __attribute__((aligned(16))) unsigned char lds[2][(BM + BN) * KB];
  Place c;
  int K = p.K;
  c.M = p.M;
  c.N = p.N;
  if (p.count) {
    const int n = *p.count;
    if (p.count_m) c.M = min(c.M, n);
    if (p.count_k) K = min(K, n);
  }
  tile_of(blockIdx.x, p.tm, p.tn, c.mt, c.nt);
  c.m0 = c.mt * BM;
  c.n0 = c.nt * BN;
  if (c.m0 >= c.M) return;
  c.lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  c.wm = wave / WGN;
  c.wn = wave % WGN;
  c.mw = c.m0 + c.wm * (BM / WGM);
  c.nw = c.n0 + c.wn * (BN / WGN);
  c.split = blockIdx.y;
  const int k0 = blockIdx.y * p.kper, k1 = min(K, k0 + p.kper);
  const int steps = k1 > k0 ? (k1 - k0 + SA::BK - 1) / SA::BK : 0;
  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = 0.f;
  SA sa;
  SB sb;
  sa.start(p.A, p.lda, c.m0, c.M, k0, k1);
  sb.start(p.B, p.ldb, c.n0, c.N, k0, k1);
  if (steps) {
    sa.load(lds[0]);
    sb.load(lds[0] + BM * KB);
  }
  for (int s = 0; s < steps; ++s) {
    unsigned char* la = lds[s & 1];
    unsigned char* lb = la + BM * KB;
    __syncthreads();
    if (s + 1 < steps) {
      sa.load(lds[(s + 1) & 1]);
      sb.load(lds[(s + 1) & 1] + BM * KB);
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      typename Frag<T>::type fa[FM], fb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = SA::frag(la, c.wm * (BM / WGM) + 32 * i, kk, c.lane);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = SB::frag(lb, c.wn * (BN / WGN) + 32 * j, kk, c.lane);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mma(fb[j], fa[i], acc[i][j]);
    }
  }
  __syncthreads();  // the epilogue may use the stages' LDS
  float* el = reinterpret_cast<float*>(&lds[0][0]);
  // whole quads of features everywhere: straight-line code, no test per quad
  if (c.n0 + BN <= c.N) E::template run<true, FM, FN, WGM, WGN>(ea, c, acc, el);
  else E::template run<false, FM, FN, WGM, WGN>(ea, c, acc, el);
}

// The four values of quad q of a block
__device__ __forceinline__ f32x4 quad(const f32x16& a, int q) {
  f32x4 v;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = a[4 * q + k];
  return v;
}

// Sums over the rows of a tile of one value per feature: v[j][r] holds a lane's sum over its
// own block rows. Halving exchanges over the 32 lanes that share features leave one feature
// block's value per lane, then the waves' sums are added in order. Result: out[n], n = n0.. .
template <int FN, int WGM, int WGN>
__device__ __forceinline__ void column_sums(f32x16 (&v)[FN], const Place& c, float* lds, float* out) {
  const int BNW = 32 * FN;
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    // after the exchange over bit b the lane keeps the values r whose bit matches its own
    float w[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) w[r] = v[j][r];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int half = 8 >> b, bit = 16 >> b;
      const bool up = c.lane & bit;
#pragma unroll
      for (int r = 0; r < half; ++r) {
        const float mine = up ? w[r + half] : w[r], other = up ? w[r] : w[r + half];
        w[r] = mine + __shfl_xor(other, bit, 64);
      }
    }
    // lane bits 4..1 now name r (most significant first); bit 0 still to add
    const float s = w[0] + __shfl_xor(w[0], 1, 64);
    const int r = (c.lane >> 1) & 15;
    if (!(c.lane & 1)) lds[c.wm * (WGN * BNW) + c.wn * BNW + 32 * j + 8 * (r >> 2) + 4 * (c.lane >> 5) + (r & 3)] = s;
  }
  __syncthreads();
  for (int n = threadIdx.x; n < WGN * BNW; n += 64 * WGM * WGN) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WGM; ++w) s += lds[w * (WGN * BNW) + n];
    if (c.n0 + n < c.N) out[c.n0 + n] = s;
  }
}

// Partial sums of a split contraction, joined by k_join in the order of the splits.
struct EpPart {
  struct Args {
    float* part;  // [splits][M][N]
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float*) {
    float* out = a.part + (size_t)c.split * c.M * c.N;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = c.row(i);
      if (m >= c.M) continue;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) store4<WHOLE>(out + (size_t)m * c.N, c.feature(j, q), c.N, quad(acc[i][j], q));
    }
  }
};

// out = f * scale[0] * D (scale: device value, nullable)
template <typename T>
struct EpScale {
  struct Args {
    T* out;  // [M][N]
    float f;
    const float* scale;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float*) {
    const float f = a.scale ? a.f * a.scale[0] : a.f;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = c.row(i);
      if (m >= c.M) continue;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) store4<WHOLE>(a.out + (size_t)m * c.N, c.feature(j, q), c.N, quad(acc[i][j], q) * f);
    }
  }
};

// out[i] = f * scale[0] * sum over splits of part[split][i]
template <typename T>
__global__ __launch_bounds__(256) void k_join(const float* part, int splits, size_t n, T* out, float f,
                                              const float* scale) {
  const float g = scale ? f * scale[0] : f;
  for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (size_t)gridDim.x * 1024) {
    const int left = (int)(n - i < 4 ? n - i : 4);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < splits; ++k) s += load4(part + (size_t)k * n + i, 0, left);
    store4(out + i, 0, left, s * g);
  }
}

// out[n] = f * scale[0] * sum over tile rows of part[t][n], in fp64 and in order. With
// `count` given, only the tile rows that hold rows below it were written.
template <typename T>
__global__ __launch_bounds__(256) void k_colsum(const float* part, int tiles, int bm, const int* count, int n, T* out,
                                                float f, const float* scale) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  if (count) tiles = min(tiles, (*count + bm - 1) / bm);
  double s = 0.0;
  for (int t = 0; t < tiles; ++t) s += (double)part[(size_t)t * n + i];
  out[i] = (T)((float)s * (scale ? f * scale[0] : f));
}

// Rows of `cols` values to rows of ld values, zeros behind them (ld a multiple of a chunk): a
// copy whose rows start on 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void k_repack(const T* in, T* out, size_t rows, int cols, int ld) {
  constexpr int V = 16 / sizeof(T);
  const int per = ld / V;
  for (size_t id = (size_t)blockIdx.x * 256 + threadIdx.x; id < rows * per; id += (size_t)gridDim.x * 256) {
    const size_t r = id / per;
    const int c = (int)(id - r * per) * V;
    const T* p = in + r * cols + c;
    typename GVec<T, V>::type v;
    if (c + V <= cols) {
      v = *reinterpret_cast<const typename GVec<T, V>::type*>(p);
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = c + k < cols ? p[k] : (T)0.f;
    }
    *reinterpret_cast<typename GVec<T, V>::type*>(out + r * ld + c) = v;
  }
}

// ---------------------------------------------------------------- launches

// Tile sizes: 4 waves of 64 x 64.
constexpr int TILE = 128;

inline int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

// The leading dimension of a row of n values that starts on 16 bytes.
inline int padded(size_t esz, int n) { return ceil_div(n, 16 / (int)esz) * (16 / (int)esz); }

// An operand as the products need it: the caller's array where its rows start on 16 bytes,
// else a copy in the workspace.
template <typename T>
struct Operand {
  const T* p;
  long ld;
  hipError_t e;
  Operand(const void* in, size_t rows, int cols, void* copy, hipStream_t st)
      : p(static_cast<const T*>(in)), ld(cols), e(hipSuccess) {
    if (cols * sizeof(T) % 16 == 0 && (uintptr_t)in % 16 == 0) return;
    ld = padded(sizeof(T), cols);
    p = static_cast<const T*>(copy);
    const size_t n = rows * (ld * sizeof(T) / 16);
    if (n == 0) return;
    k_repack<T><<<(unsigned)std::min<size_t>((n + 255) / 256, 1u << 20), 256, 0, st>>>(
        static_cast<const T*>(in), static_cast<T*>(copy), rows, cols, (int)ld);
    e = hipGetLastError();
  }
};

template <typename T, bool AT, bool BT, class E>
hipError_t launch_mm(Prob p, const typename E::Args& ea, int splits, hipStream_t st) {
  constexpr int BK = KB / (int)sizeof(T);
  p.tm = ceil_div(p.M, TILE);
  p.tn = ceil_div(p.N, TILE);
  p.kper = ceil_div(ceil_div(p.K, BK), splits) * BK;
  if (p.kper == 0) p.kper = BK;
  k_mm<T, TILE, TILE, 2, 2, AT, BT, E><<<dim3((unsigned)(p.tm * p.tn), (unsigned)splits), 256, 0, st>>>(p, ea);
  return hipGetLastError();
}

// Splits of a contraction of K values for an M x N result: enough for two workgroups a
// CU, each with at least four stages.
inline int splits_of(size_t esz, int M, int N, long K) {
  const long tiles = (long)ceil_div(M, TILE) * ceil_div(N, TILE), steps = ceil_div(K * (long)esz, KB);
  long s = 512 / (tiles > 0 ? tiles : 1);
  if (s > steps / 4) s = steps / 4;
  return (int)(s < 1 ? 1 : s > 32 ? 32 : s);
}

}  // namespace mm
}  // namespace lp
