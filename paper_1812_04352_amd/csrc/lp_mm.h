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
// Matrix instructions: 32 x 32 x 16 in bf16 or f16 (floats as split bf16 products), with n on the
// instruction's rows and m on its columns. Lane l then holds, of each 32 x 32 block, the 16
// values n = 8 (r / 4) + 4 (l / 32) + r % 4, r = 0..15, of the single row m = l % 32: four
// consecutive features at a time (vector loads and stores of rows), and sums over a row
// need one exchange with lane l ^ 32.
//
// LDS holds several stages of KB bytes of the contraction of every row of the tile (some are
// filled while one is read; one barrier a stage), in 16-byte chunks.
//   rows:    the chunks of a row are exchanged by a part of the row's index, so that the eight
//            chunks of a bank cycle that a fragment read takes (eight rows, one chunk index)
//            lie in different banks.
//   columns: row k of the stage holds its R columns; fragments of 16-bit types are read
//            with the transposing LDS load, which hands lane i of 16 the values (k0..k0+3,
//            column i) from four rows' 32-byte pieces. Chunks are exchanged by 64 bytes
//            times k % 4, so that those four rows lie in different banks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "lp_device.h"
#include "lp_internal.h"
#include "lp_split.h"

namespace lp {
namespace mm {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
using lp::f32x8;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// N consecutive values in global memory, with their element's alignment
template <typename T, int N> struct GVec { typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };

// A value as the sum of two f16 ones, hi + lo (2^-22 relative, 2^-25 absolute): rows of such values hold eight hi and the
// same eight lo in turn, 4 bytes a value; rows have a multiple of eight of them. Workspace arrays only.
struct Duo {
  uint32_t bits;
};
struct DuoFrag {
  h16x8 hi, lo;
};

// What a lane reads of one operand for a step of 16 contraction values (eight of them), and what
// the matrix instructions take: floats are split into three bf16 parts (lp_split.h), six products
// of which make one of floats: 2.4 times the float instructions' rate, with a smaller error.
template <typename T> struct Frag;
template <> struct Frag<bf16> { typedef b16x8 type; typedef b16x8 ready; };
template <> struct Frag<f16> { typedef h16x8 type; typedef h16x8 ready; };
template <> struct Frag<float> { typedef f32x8 type; typedef Split8 ready; };
template <> struct Frag<Duo> { typedef DuoFrag type; typedef DuoFrag ready; };

__device__ __forceinline__ b16x8 prepare(b16x8 x) { return x; }
__device__ __forceinline__ h16x8 prepare(h16x8 x) { return x; }
__device__ __forceinline__ Split8 prepare(f32x8 x) { return split8(x); }
__device__ __forceinline__ DuoFrag prepare(const DuoFrag& x) { return x; }
// of sign * x (sign = 1 or -1, the same for the wave; 16-bit types have none)
template <typename F>
__device__ __forceinline__ auto prepare(F x, float sign) {
  if constexpr (std::is_same<F, f32x8>::value) return split8(x, sign);
  else return x;
}

__device__ __forceinline__ f32x16 mma(b16x8 a, b16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(h16x8 a, h16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const DuoFrag& a, const DuoFrag& b, f32x16 c) {  // (lo lo is below 2^-22)
  c = mma(a.lo, b.hi, c);
  c = mma(a.hi, b.lo, c);
  return mma(a.hi, b.hi, c);
}
__device__ __forceinline__ f32x16 mma(const Split8& a, const Split8& b, f32x16 c) {
  constexpr int ia[6] = {0, 2, 1, 0, 1, 0}, ib[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
  for (int k = 0; k < 6; ++k) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.p[ia[k]], b.p[ib[k]], c, 0, 0, 0);
  return c;
}
// the float instructions, for tiles whose split products are not finite
template <typename F>
__device__ __forceinline__ f32x16 mma_float(F a, F b, f32x16 c) {
  if constexpr (std::is_same<F, f32x8>::value) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  }
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

// One operand's tile of R rows of D, KB bytes of the contraction a row, straight from global
// memory to LDS. Arrays start on 16 bytes and so do their rows.
template <typename T, int R, int KB, int NT, bool COLS>
struct Stage {
  static constexpr int V = 16 / sizeof(T);           // values per chunk
  static constexpr int BK = KB / (int)sizeof(T);     // contraction values per stage
  static constexpr int RC = KB / 16;                 // rows: chunks per row
  static constexpr int PER = R * RC / NT;            // chunks per thread
  static constexpr int CH = R / V;                   // columns: chunks per row of the stage
  static constexpr bool TURNS = !std::is_same<T, float>::value;  // columns: read by transposing loads
  static constexpr int SWZ = (TURNS ? 12 : 8) & (CH - 1);
  static constexpr int UNIT = std::is_same<T, Duo>::value ? 8 : V;  // values that lie together
  static_assert(R * RC % NT == 0, "whole chunks per thread");
  static_assert(KB == 64 || KB == 128, "the rows' exchange");

  static __device__ __forceinline__ int swz(int k) {  // columns: chunk exchange of row k
    return (TURNS ? k << 2 : k) & SWZ;
  }
  static __device__ __forceinline__ int rswz(int r) {  // rows: chunk exchange of row r
    return KB == 128 ? r & 7 : (r >> 1) & 3;
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
      const int c = (t % RC) ^ rswz(t / RC);
      kc = c * V / UNIT * UNIT;
      base = static_cast<const unsigned char*>(p) + ((long)r0 * ld + k0) * (long)sizeof(T);
      left = ((long)(rows - r0) * ld - k0) * (long)sizeof(T);
      step = KB;
#pragma unroll
      for (int i = 0; i < PER; ++i) off[i] = (uint32_t)((t + i * NT) / RC) * (uint32_t)(ld * sizeof(T)) + c * 16;
    } else {
      kc = 0;
      base = static_cast<const unsigned char*>(p) + ((long)k0 * ld + r0) * (long)sizeof(T);
      // (to the last chunk of row k1 - 1 that counts: behind it may lie what no kernel has written, which
      // must not decide whether a float tile is formed again)
      left = ((long)(k1 - k0 - 1) * ld + (rows + UNIT - 1) / UNIT * UNIT - r0) * (long)sizeof(T);
      step = BK * ld * (long)sizeof(T);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int r = (t + i * NT) / CH;
        off[i] = (uint32_t)r * (uint32_t)(ld * sizeof(T)) + ((t % CH) ^ swz(r)) * 16;
      }
    }
  }

  // Requests the next stage; wave: the wave's index in a scalar register. Loads past `left` give
  // zeros: rows past the last (rows), contraction indices past the last (columns); so does an
  // offset of 2^31 (rows: past the contraction's end, which only the last stage can hold).
  // (The instruction is written out: of the builtin's loads the compiler believes that a transposing
  // LDS read may depend on every one in flight, and waits for all of them before it. The program's LDS
  // accesses stay on their side of it. The compiler does not see its hazards: s_nop 0 is the wait state
  // between m0 and a load, and the five between a vector instruction that writes a scalar of the
  // descriptor, such as a spilled one's return, and a load are there since the descriptor is formed by
  // scalar instructions: tests/test_wide_code.py reads the generated code for it. Waiting for them here
  // costs the large products 1 %.)
  __device__ __forceinline__ void load(unsigned char* lds, int wave) {
    last_stage();
    request<0, PER>(base, left, lds, wave);
    advance();
  }
  __device__ __forceinline__ void last_stage() {  // (it ends with the contraction)
    if (!COLS && k + BK > k1) {
#pragma unroll
      for (int i = 0; i < PER; ++i) off[i] = k + kc >= k1 ? 0x80000000u : off[i];
    }
  }
  __device__ __forceinline__ void advance() {
    base += step;
    left -= step;
    k += BK;
  }
  // the thread's chunks I0 .. I1 - 1
  template <int I0, int I1>
  __device__ __forceinline__ void request(const unsigned char* base, long left, unsigned char* lds, int wave) {
#ifdef __HIP_DEVICE_COMPILE__
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const i32x4 r = {(int)(uint32_t)at, (int)(uint32_t)(at >> 32) & 0xffff, (left >> 31) != 0 ? 0x7fffffff : (int)left, 0x00020000};
    const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)lds + wave * 1024;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is reserved: a note that it may be needed around the statement, where nothing holds it)
#pragma unroll
    for (int i = I0; i < I1; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to + i * NT * 16), "v"(off[i]),
                   "s"(r)
                   : "m0", "memory");
#pragma clang diagnostic pop
#endif
  }
};

// The weights' tile of a pair of arrays of rows of the same shape: RR rows of the first, then the same
// rows of the second.
template <typename T, int R, int KB, int NT>
struct PairRows : Stage<T, R / 2, KB, NT, false> {
  typedef Stage<T, R / 2, KB, NT, false> S;
  static constexpr int PER = 2 * S::PER;
  long hop;  // from the first array to the second
  __device__ __forceinline__ void start(const void* p, const void* p2, long ld, int r0, int rows, int k0, int k1) {
    S::start(p, ld, r0, rows, k0, k1);
    hop = static_cast<const unsigned char*>(p2) - static_cast<const unsigned char*>(p);
  }
  __device__ __forceinline__ void load(unsigned char* lds, int wave) {
    this->last_stage();
    this->template request<0, S::PER>(this->base, this->left, lds, wave);
    this->template request<0, S::PER>(this->base + hop, this->left, lds + R / 2 * KB, wave);
    this->advance();
  }
};

// The tile of a pair of arrays of `rows` columns whose contraction indices alternate: PAIR_BLOCK rows of the
// first, the same rows of the second, and so on, zeros behind the kw rows that each has. A stage of
// 16-bit values holds a block of each, one of floats a block of either in turn. (k0: a multiple of a stage.)
constexpr int PAIR_BLOCK = 32;
template <typename T, int R, int KB, int NT>
struct PairCols : Stage<T, R, KB, NT, true> {
  typedef Stage<T, R, KB, NT, true> S;
  static constexpr bool BOTH = S::BK == 2 * PAIR_BLOCK;
  static_assert(BOTH || S::BK == PAIR_BLOCK, "whole blocks");
  static_assert(!BOTH || (S::PER % 2 == 0 && S::PER / 2 * NT / S::CH == PAIR_BLOCK), "a load's chunks lie in one block");
  long hop, lhop;  // BOTH: from the first array to the second; else what the next stage adds to base and takes off left
  __device__ __forceinline__ void start(const void* p, const void* p2, long ld, int r0, int rows, int kw, int k0) {
    const int k = k0 / (2 * PAIR_BLOCK) * PAIR_BLOCK;  // the row of both arrays that k0 lies in
    S::start(p, ld, r0, rows, k, kw);
    hop = static_cast<const unsigned char*>(p2) - static_cast<const unsigned char*>(p);
    this->step = PAIR_BLOCK * ld * (long)sizeof(T);
    if constexpr (BOTH) {
      const uint32_t back = (uint32_t)(PAIR_BLOCK * ld * (long)sizeof(T));
#pragma unroll
      for (int i = S::PER / 2; i < S::PER; ++i) this->off[i] -= back;
    } else {
      lhop = 0;
      if (k0 / PAIR_BLOCK % 2) turn();
    }
  }
  __device__ __forceinline__ void turn() {  // the other array's rows are next
    this->base += hop, this->left -= lhop;
    hop = this->step - hop, lhop = this->step - lhop;
  }
  __device__ __forceinline__ void load(unsigned char* lds, int wave) {
    if constexpr (BOTH) {
      this->template request<0, S::PER / 2>(this->base, this->left, lds, wave);
      this->template request<S::PER / 2, S::PER>(this->base + hop, this->left, lds, wave);
      this->base += this->step, this->left -= this->step;
    } else {
      this->template request<0, S::PER>(this->base, this->left, lds, wave);
      turn();
    }
  }
};

// Reads a wave's fragments of one operand: NF blocks of 32 rows of D from row r0 of the tile on.
// A lane's offsets into a stage are kept in registers as far as the exchange of chunks makes them
// differ (rows: per contraction step; columns: per block), the rest is the load's own offset.
template <typename T, class S, int KB, int NF, bool COLS>
struct Reader {
  typedef typename Frag<T>::type F;
  static constexpr int N = COLS ? NF : KB / (sizeof(T) == 2 ? 32 : 16);
  uint32_t at[N];

  __device__ __forceinline__ Reader(int r0, int lane) {
#pragma unroll
    for (int x = 0; x < N; ++x) {
      if constexpr (!COLS) {  // 16 bits: step x; float: chunk x % 2 of step x / 2
        const int r = r0 + (lane & 31), c = sizeof(T) == 2 ? 2 * x + (lane >> 5) : 4 * (x / 2) + 2 * (lane >> 5) + x % 2;
        at[x] = (r * S::RC + (c ^ S::rswz(r))) * 16;
      } else if constexpr (std::is_same<T, Duo>::value) {
        const int col = r0 + 32 * x + 16 * ((lane >> 4) & 1) + 4 * (lane & 3), k = 8 * (lane >> 5) + ((lane >> 2) & 3);
        at[x] = (k * S::CH + ((col / 8 * 2) ^ S::swz(k))) * 16 + (col % 8) * 2;
      } else if constexpr (sizeof(T) == 2) {
        const int col = r0 + 32 * x + 16 * ((lane >> 4) & 1) + 4 * (lane & 3), k = 8 * (lane >> 5) + ((lane >> 2) & 3);
        at[x] = (k * S::CH + ((col / S::V) ^ S::swz(k))) * 16 + (col % S::V) * 2;
      } else {
        const int col = r0 + 32 * x + (lane & 31), k = 8 * (lane >> 5);
        at[x] = (k * S::CH + ((col / S::V) ^ S::swz(k))) * 16 + (col % S::V) * 4;
      }
    }
  }

  // block i, step kk (16 contraction values, eight of them this lane's) of the stage at lds
  __device__ __forceinline__ F operator()(const unsigned char* lds, int i, int kk) const {
    if constexpr (!COLS) {
      if constexpr (sizeof(T) == 2) {
        return *reinterpret_cast<const F*>(lds + at[kk] + i * 32 * KB);
      } else if constexpr (std::is_same<T, Duo>::value) {
        return F{*reinterpret_cast<const h16x8*>(lds + at[2 * kk] + i * 32 * KB),
                 *reinterpret_cast<const h16x8*>(lds + at[2 * kk + 1] + i * 32 * KB)};
      } else {
        const f32x4 lo = *reinterpret_cast<const f32x4*>(lds + at[2 * kk] + i * 32 * KB);
        const f32x4 hi = *reinterpret_cast<const f32x4*>(lds + at[2 * kk + 1] + i * 32 * KB);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    } else if constexpr (std::is_same<T, Duo>::value) {
      typedef __attribute__((address_space(3))) s16x4 lds4;
      s16x4 h[2][2];
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          h[p][j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + at[i] + 16 * p + (16 * kk + 4 * j) * S::CH * 16));
      return F{__builtin_bit_cast(h16x8, __builtin_shufflevector(h[0][0], h[0][1], 0, 1, 2, 3, 4, 5, 6, 7)),
               __builtin_bit_cast(h16x8, __builtin_shufflevector(h[1][0], h[1][1], 0, 1, 2, 3, 4, 5, 6, 7))};
    } else if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) s16x4 lds4;
      s16x4 h[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        h[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + at[i] + (16 * kk + 4 * j) * S::CH * 16));
      return __builtin_bit_cast(F, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      F v;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const float*>(lds + at[i] + (16 * kk + j) * S::CH * 16);
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
  const void* B2 = nullptr;  // pairs of arrays: the second one
  int kw = 0;                // PAIR_COLS: rows of each
};

// A wave's LDS writes before its other lanes' reads and the other way round: the wave's accesses are
// made in order, so the compiler alone has to be kept from exchanging them.
__device__ __forceinline__ void wave_in_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What an epilogue knows of its place: row m of D is mw + 32 i + lane % 32 of block row i,
// feature n = nw + 32 j + 8 q + 4 (lane / 32) of quad q of block column j.
struct Place {
  int M, N;
  int lim;         // end of the workgroup's features
  int m0, n0;      // the workgroup's tile
  int mw, nw;      // the wave's part of it
  int wm, wn;      // the wave's place in the workgroup
  int mt, nt;      // tile indices
  int split;
  int lane;
  // the end of what is written of rows of ld >= N values (the last tile also writes what is behind N)
  __device__ __forceinline__ int upto(int ld) const { return lim == N ? ld : lim; }
  // the workgroup's waves meet (a single wave's LDS accesses are in order by themselves)
  template <int WAVES>
  __device__ __forceinline__ void meet() const {
    if constexpr (WAVES == 1) wave_in_order();
    else __syncthreads();
  }
  __device__ __forceinline__ int row(int i) const { return mw + 32 * i + (lane & 31); }
  __device__ __forceinline__ int feature(int j, int q) const { return nw + 32 * j + 8 * q + 4 * (lane >> 5); }
};

// The LDS of an epilogue: a part per wave for a 32 x 32 block of floats in padded rows, and behind
// them 8 bytes per row of the tile and wave column.
constexpr int WAVE_LDS = 32 * (32 * 4 + 16);
constexpr int epilogue_lds(int waves, int bm, int wgn) { return waves * WAVE_LDS + bm * wgn * 8; }

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

// Tiles of a symmetric D on and below its diagonal, tm (tm + 1) / 2 of them: a run of tile rows an XCD.
__device__ __forceinline__ void tile_below(int id, int tm, int& mt, int& nt) {
  const int total = tm * (tm + 1) / 2, q = total / 8, r = total % 8, x = id % 8;
  const int at = x * q + min(x, r) + id / 8;
  mt = (int)((sqrtf(8.f * (float)at + 1.f) - 1.f) * 0.5f);  // (off by one at most: settled below)
  while ((mt + 1) * (mt + 2) / 2 <= at) ++mt;
  while (mt * (mt + 1) / 2 > at) --mt;
  nt = at - mt * (mt + 1) / 2;
}

// What B is: one array; a pair of arrays in rows, D1 and D2 formed side by side, half a tile's features
// of each (an epilogue finds those of D1 in block column 0, those of D2 in block column 1); a pair of arrays in
// columns whose contraction indices alternate by PAIR_BLOCK.
enum { PAIR_NONE = 0, PAIR_ROWS = 1, PAIR_COLS = 2 };

// Tile shapes: BM x BN values of D by WGM x WGN waves; NS stages of KB bytes in LDS; fragments
// are read GK steps at a time, a group ahead of their products.
template <int BM_, int BN_, int WGM_, int WGN_, int KB_, int NS_, int GK_>
struct Shape {
  static constexpr int PAIR = PAIR_NONE, BNO = BN_;  // BNO: features of D a tile
  static constexpr bool SYM = false;
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, KB = KB_, NS = NS_, GK = GK_, NT = 64 * WGM_ * WGN_;
  // waves a SIMD has to hold: two workgroups of four waves where their LDS fits twice
  static constexpr int WAVES = NT == 512 || 2 * NS_ * (BM_ + BN_) * KB_ <= 160 * 1024 ? 2 : 1;
  static_assert((NS & (NS - 1)) == 0, "a stage's place is its index modulo NS");
};

// The same tiles for a pair of arrays
template <class S, int PAIR_>
struct PairShape : S {
  static constexpr int PAIR = PAIR_, BNO = PAIR_ == PAIR_ROWS ? S::BN / 2 : S::BN;
  static_assert(PAIR_ != PAIR_ROWS || S::BN / S::WGN == 64, "one block column of each");
};
template <class S, int PAIR> using Paired = std::conditional_t<PAIR == PAIR_NONE, S, PairShape<S, PAIR>>;

// All but N of the wave's loads to LDS have landed, and every wave is here. (The compiler does not
// count those loads: nothing else waits for them.)
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// id: the workgroup's index among the product's. SCALAR: the tile's place is put into scalar registers by force: it comes
// from divisions, which are made in vector registers, and beside a large epilogue the compiler may leave the
// operands' addresses there too, of which no descriptor can be formed. (The compiler does not see the written-out
// instruction's hazards: a wait state between a vector instruction's result and its reading, and five until a scalar that
// it writes may be read by any other instruction.)
template <class S, bool SCALAR = false>
__device__ __forceinline__ Place place(const Prob& p, int id, int split, int wave, int& K) {
  Place c;
  K = p.K;
  c.M = p.M;
  c.N = p.N;
  if (p.count) {
    const int n = *p.count;
    if (p.count_m) c.M = min(c.M, n);
    if (p.count_k) K = min(K, n);
  }
  if constexpr (S::SYM) tile_below(id, p.tm, c.mt, c.nt);
  else tile_of(id, p.tm, p.tn, c.mt, c.nt);
#ifdef __HIP_DEVICE_COMPILE__
  if constexpr (SCALAR) {
    asm volatile("s_nop 1\n\tv_readfirstlane_b32 %0, %2\n\tv_readfirstlane_b32 %1, %3\n\ts_nop 4"
                 : "=&s"(c.mt), "=&s"(c.nt)
                 : "v"(c.mt), "v"(c.nt));
  }
#endif
  c.m0 = c.mt * S::BM;
  c.n0 = c.nt * S::BNO;
  c.lim = min(c.N, c.n0 + S::BNO);
  c.lane = threadIdx.x & 63;
  c.wm = wave / S::WGN;
  c.wn = wave % S::WGN;
  c.mw = c.m0 + c.wm * (S::BM / S::WGM);
  c.nw = c.n0 + c.wn * (S::BNO / S::WGN);
  c.split = split;
  return c;
}

// LDS of a workgroup: the stages
template <class S>
struct Stages {
  __attribute__((aligned(16))) unsigned char at[S::NS][(S::BM + S::BN) * S::KB];
};

template <typename T, class S, bool AT, bool BT, class E>
__device__ __forceinline__ void mm_tile(const Prob& p, const typename E::Args& ea, int id, Stages<S>& stages, int split = blockIdx.y) {
  constexpr int BM = S::BM, BN = S::BN, WGM = S::WGM, WGN = S::WGN, KB = S::KB, NS = S::NS, NT = S::NT;
  constexpr int FM = BM / WGM / 32, FN = BN / WGN / 32, GK = S::GK;
  constexpr int NG = KB / (16 * (int)sizeof(T)) / GK;
  static_assert(NG % 2 == 0, "the fragment sets alternate within a stage");
  typedef Stage<T, BM, KB, NT, AT> SA;
  constexpr int PAIR = S::PAIR;
  static_assert(PAIR == PAIR_NONE || BT == (PAIR == PAIR_COLS), "how the pair lies");
  typedef std::conditional_t<PAIR == PAIR_ROWS, PairRows<T, BN, KB, NT>,
                             std::conditional_t<PAIR == PAIR_COLS, PairCols<T, BN, KB, NT>, Stage<T, BN, KB, NT, BT>>>
      SB;
  constexpr int LOADS = SA::PER + SB::PER;
  auto& lds = stages.at;
  static_assert(epilogue_lds(WGM * WGN, BM, WGN) <= NS * (BM + BN) * KB, "the epilogue's LDS");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int K;
  const Place c = place<S, std::is_same<T, Duo>::value || S::SYM || S::PAIR != PAIR_NONE>(p, id, split, wave, K);
  if (c.m0 >= c.M) return;
  const int k0 = split * p.kper, k1 = min(K, k0 + p.kper);
  const int steps = k1 > k0 ? (k1 - k0 + SA::BK - 1) / SA::BK : 0;
  const Reader<T, SA, KB, FM, AT> ra(c.wm * (BM / WGM), c.lane);
  // (of a pair in rows: the blocks of both halves, which lie BN / 2 rows apart)
  const Reader<T, Stage<T, BN, KB, NT, BT>, KB, PAIR == PAIR_ROWS ? 1 : FN, BT> rb(c.wn * (S::BNO / WGN), c.lane);
  f32x16 acc[FM][FN];
  // The contraction. A group's fragments are read during the products of the group before; the
  // last group of a stage reads the next stage's first fragments, behind the stage's one barrier:
  // every wave has then read all of this stage, and the next one has landed, so the stage NS
  // further on is requested into this one's place.
  const auto contract = [&](auto as_float) {
    SA sa;
    SB sb;
    sa.start(p.A, p.lda, c.m0, c.M, k0, k1);
    if constexpr (PAIR == PAIR_ROWS) sb.start(p.B, p.B2, p.ldb, c.n0, c.N, k0, k1);
    else if constexpr (PAIR == PAIR_COLS) sb.start(p.B, p.B2, p.ldb, c.n0, c.N, p.kw, k0);
    else sb.start(p.B, p.ldb, c.n0, c.N, k0, k1);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = 0.f;
    typename Frag<T>::type fa[2][GK][FM], fb[2][GK][FN];
    const auto frags = [&](int s, int g, int to) {
      const unsigned char* la = lds[s & (NS - 1)];
#pragma unroll
      for (int k = 0; k < GK; ++k) {
#pragma unroll
        for (int i = 0; i < FM; ++i) fa[to][k][i] = ra(la, i, g * GK + k);
#pragma unroll
        for (int j = 0; j < FN; ++j)
          fb[to][k][j] = PAIR == PAIR_ROWS ? rb(la + (BM + j * (BN / 2)) * KB, 0, g * GK + k) : rb(la + BM * KB, j, g * GK + k);
      }
    };
    const auto request = [&](int s) {
      sa.load(lds[s & (NS - 1)], wave);
      sb.load(lds[s & (NS - 1)] + BM * KB, wave);
    };
    float sign = 1.f;
    const auto products = [&](int at, int k) {
      if constexpr (decltype(as_float)::value) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = mma_float(fb[at][k][j], fa[at][k][i], acc[i][j]);
      } else {
        typename Frag<T>::ready ga[FM], gb[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) gb[j] = prepare(fb[at][k][j], sign);
#pragma unroll
        for (int i = 0; i < FM; ++i) ga[i] = prepare(fa[at][k][i]);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = mma(gb[j], ga[i], acc[i][j]);
      }
    };
    // more: the stage NS further on exists; next: the next one does
    const auto stage = [&](int s, auto more, auto next) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const int at = g & 1;
        if (g < NG - 1) {
          frags(s, g + 1, at ^ 1);
        } else if (decltype(next)::value) {
          wait_and_meet<decltype(more)::value ? (NS - 2) * LOADS : 0>();
          __builtin_amdgcn_sched_barrier(0);
          if (decltype(more)::value) request(s + NS);
          frags(s + 1, 0, at ^ 1);
        }
#pragma unroll
        for (int k = 0; k < GK; ++k) products(at, k);
      }
    };
    // The instruction's sums round towards minus infinity by a small part of their last place
    // (lp_split.h). Of floats the middle half of the stages is therefore summed with the other sign, minus
    // the sum so far and minus the products: the error of the first and last quarter then cancels that of
    // the middle, in sums that grow with the contraction as in those that stay small. Mean error of sums of
    // 220, 1024 and 8192 positive products: -1.3e-8, -6.1e-9 and -2.1e-8 without, -2.5e-9, -0.7e-9 and -0.1e-9
    // with it (a sum of 220 is off by 1.8e-7 either way; one of a single stage, 32 products, keeps its
    // -2.3e-9). It takes 1 to 2 % of the time of large products, 5 % of 1000 x 220 -> 220. (Of 16-bit types
    // the results' own rounding is 2^-9 and more.)
    constexpr bool SIGNS = std::is_same<T, float>::value && !decltype(as_float)::value;
    const int minus = steps / 4, plus = minus + (steps + 1) / 2;  // (a single stage keeps its sign)
    const auto turn = [&](int s) {
      if (SIGNS && steps > 1 && (s == minus || s == plus)) {
        sign = -sign;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = -acc[i][j];
      }
    };
    if (steps) {
#pragma unroll
      for (int s = 0; s < NS; ++s)
        if (s < steps) request(s);
      if (steps >= NS) wait_and_meet<(NS - 1) * LOADS>();
      else wait_and_meet<0>();
      frags(0, 0, 0);
      int s = 0;
      for (; s + NS < steps; ++s) {
        turn(s);
        stage(s, std::true_type{}, std::true_type{});
      }
      for (; s + 1 < steps; ++s) {
        turn(s);
        stage(s, std::false_type{}, std::true_type{});
      }
      turn(s);
      stage(s, std::false_type{}, std::false_type{});
    }
  };
  contract(std::false_type{});
  if constexpr (std::is_same<T, float>::value) {
    // An operand that is infinite or beyond the largest bf16 value makes split products NaN: a tile
    // with a result that is not finite is formed again by the float instructions, which give
    // infinities and overflow as fp32 has them.
    bool finite = true;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) finite = finite && fabsf(acc[i][j][r]) < INFINITY;
    if (__syncthreads_or(!finite)) contract(std::true_type{});
  }
  __syncthreads();  // the epilogue may use the stages' LDS
  float* el = reinterpret_cast<float*>(&lds[0][0]);
  // whole quads of features everywhere: straight-line code, no test per quad
  if (c.n0 + S::BNO <= c.N) E::template run<true, FM, FN, WGM, WGN>(ea, c, acc, el);
  else E::template run<false, FM, FN, WGM, WGN>(ea, c, acc, el);
}

template <typename T, class S, bool AT, bool BT, class E>
__global__ __launch_bounds__(S::NT, S::WAVES) void k_mm(Prob p, typename E::Args ea) {
  __shared__ Stages<S> stages;
  mm_tile<T, S, AT, BT, E>(p, ea, blockIdx.x, stages);
}

// The four values of quad q of a block
__device__ __forceinline__ f32x4 quad(const f32x16& a, int q) {
  f32x4 v;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = a[4 * q + k];
  return v;
}

// A wave's 32 x 32 blocks of D between global memory, in rows of 16-byte pieces, and the quads that
// the lanes hold, by way of the wave's own part of the LDS. Quads alone would be 8 bytes a lane from
// 32 rows at a time.
template <typename T>
struct BlockIO {
  static constexpr int W = 32 * (int)sizeof(T), PITCH = W + 16, CPR = W / 16, V = 16 / (int)sizeof(T);
  static constexpr int ITER = (32 * CPR + 63) / 64, BYTES = 32 * PITCH;
  typedef typename GVec<T, V>::type Piece;
  typedef T LPiece __attribute__((ext_vector_type(V)));
  typedef T Quad __attribute__((ext_vector_type(4)));
  struct Block {
    Piece p[ITER];
  };

  // pieces of block (i, j) of an array of rows of ld values (rows past the last are the last: not used)
  static __device__ __forceinline__ Block fetch(const T* a, long ld, const Place& c, int i, int j) {
    Block b;
#pragma unroll
    for (int t = 0; t < ITER; ++t) {
      const int id = c.lane + 64 * t, m = min(c.mw + 32 * i + id / CPR, c.M - 1);
      b.p[t] = *reinterpret_cast<const Piece*>(a + (size_t)m * ld + c.nw + 32 * j + id % CPR * V);
    }
    return b;
  }

  static __device__ __forceinline__ void quads(const Block& b, unsigned char* buf, const Place& c, f32x4 (&v)[4]) {
#pragma unroll
    for (int t = 0; t < ITER; ++t) {
      const int id = c.lane + 64 * t;
      *reinterpret_cast<LPiece*>(buf + id / CPR * PITCH + id % CPR * 16) = b.p[t];
    }
    wave_in_order();
    const unsigned char* r = buf + (c.lane & 31) * PITCH + (c.lane >> 5) * 4 * sizeof(T);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const Quad x = *reinterpret_cast<const Quad*>(r + 8 * q * sizeof(T));
#pragma unroll
      for (int k = 0; k < 4; ++k) v[q][k] = (float)x[k];
    }
    wave_in_order();
  }

  // row(m): the index of row m in the array
  template <typename F>
  static __device__ __forceinline__ void store(T* a, long ld, const Place& c, int i, int j, unsigned char* buf,
                                               const f32x4 (&v)[4], F row) {
    unsigned char* w = buf + (c.lane & 31) * PITCH + (c.lane >> 5) * 4 * sizeof(T);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      Quad x;
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = (T)v[q][k];
      *reinterpret_cast<Quad*>(w + 8 * q * sizeof(T)) = x;
    }
    wave_in_order();
#pragma unroll
    for (int t = 0; t < ITER; ++t) {
      const int id = c.lane + 64 * t, m = c.mw + 32 * i + id / CPR;
      const Piece x = *reinterpret_cast<const LPiece*>(buf + id / CPR * PITCH + id % CPR * 16);
      if (m < c.M) *reinterpret_cast<Piece*>(a + (size_t)row(m) * ld + c.nw + 32 * j + id % CPR * V) = x;
    }
    wave_in_order();
  }
};

// Of values in two parts: an array's rows are whole pieces, ld of them; what lies behind them is not touched.
template <>
struct BlockIO<Duo> {
  static constexpr int W = 128, PITCH = W + 16, CPR = W / 16, V = 4;
  static constexpr int ITER = 32 * CPR / 64, BYTES = 32 * PITCH;
  typedef f32x4 Piece;
  typedef _Float16 Quad __attribute__((ext_vector_type(4)));

  static __device__ __forceinline__ void put(unsigned char* at, f32x4 v) {
    Quad h, l;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      h[k] = (_Float16)v[k];
      l[k] = (_Float16)(v[k] - (float)h[k]);
    }
    *reinterpret_cast<Quad*>(at) = h;
    *reinterpret_cast<Quad*>(at + 16) = l;
  }
  struct Block {
    Piece p[ITER];
  };
  static __device__ __forceinline__ Block fetch(const Duo* a, long ld, const Place& c, int i, int j) {
    Block b;
#pragma unroll
    for (int t = 0; t < ITER; ++t) {
      const int id = c.lane + 64 * t, m = min(c.mw + 32 * i + id / CPR, c.M - 1), n = c.nw + 32 * j + id % CPR * V;
      b.p[t] = *reinterpret_cast<const Piece*>(a + (size_t)m * ld + min((long)n, ld - V));  // (pieces behind a row: not used)
    }
    return b;
  }
  static __device__ __forceinline__ void quads(const Block& b, const Place& c, unsigned char* buf, f32x4 (&v)[4]) {
#pragma unroll
    for (int t = 0; t < ITER; ++t) {
      const int id = c.lane + 64 * t;
      *reinterpret_cast<Piece*>(buf + id / CPR * PITCH + id % CPR * 16) = b.p[t];
    }
    wave_in_order();
    const unsigned char* r = buf + (c.lane & 31) * PITCH + (c.lane >> 5) * 8;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const Quad h = *reinterpret_cast<const Quad*>(r + 32 * q), l = *reinterpret_cast<const Quad*>(r + 32 * q + 16);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[q][k] = (float)h[k] + (float)l[k];
    }
    wave_in_order();
  }
  // rows m0 .. m0 + 31 below M, columns n0 .. from the wave's LDS
  static __device__ __forceinline__ void flush(Duo* a, long ld, int m0, int M, int n0, int lane, const unsigned char* buf) {
    wave_in_order();
#pragma unroll
    for (int t = 0; t < ITER; ++t) {
      const int id = lane + 64 * t, m = m0 + id / CPR, n = n0 + id % CPR * V;
      const Piece x = *reinterpret_cast<const Piece*>(buf + id / CPR * PITCH + id % CPR * 16);
      if (m < M && n < ld) *reinterpret_cast<Piece*>(a + (size_t)m * ld + n) = x;
    }
    wave_in_order();
  }
  static __device__ __forceinline__ void store(Duo* a, long ld, const Place& c, int i, int j, unsigned char* buf, const f32x4 (&v)[4]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) put(buf + (c.lane & 31) * PITCH + 32 * q + (c.lane >> 5) * 8, v[q]);
    flush(a, ld, c.mw + 32 * i, c.M, c.nw + 32 * j, c.lane, buf);
  }
};

static_assert(WAVE_LDS == BlockIO<float>::BYTES && WAVE_LDS == BlockIO<Duo>::BYTES, "a wave's part of the LDS");
__device__ __forceinline__ unsigned char* wave_lds(float* lds, const Place& c, int wgn) {
  return reinterpret_cast<unsigned char*>(lds) + (c.wm * wgn + c.wn) * WAVE_LDS;
}

// An array of rows of ld values, those below c.lim of which count (WHOLE: all of the tile's), as a lane's quads,
// block by block in the order i = 0.. within j = 0..
template <bool WHOLE, typename T, int FM, int FN, bool AHEAD = sizeof(T) == 2>
struct Rows {
  typedef BlockIO<T> IO;
  const T* a;
  long ld;
  typename IO::Block next;
  __device__ __forceinline__ Rows(const T* a_, long ld_, const Place& c) : a(a_), ld(ld_) {
    if constexpr (WHOLE && AHEAD) {
      if (a) next = IO::fetch(a, ld, c, 0, 0);
    }
  }
  // the quads of block (i, j) (zeros without an array); requests the next block's (AHEAD: of floats
  // there are too many registers in use for that)
  __device__ __forceinline__ void get(const Place& c, int i, int j, unsigned char* buf, f32x4 (&v)[4]) {
    if (!a) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = 0.f;
    } else if constexpr (WHOLE) {
      const typename IO::Block b = AHEAD ? next : IO::fetch(a, ld, c, i, j);
      if (AHEAD && i + 1 < FM) next = IO::fetch(a, ld, c, i + 1, j);
      else if (AHEAD && j + 1 < FN) next = IO::fetch(a, ld, c, 0, j + 1);
      IO::quads(b, buf, c, v);
    } else {
      const T* row = a + (size_t)min(c.row(i), c.M - 1) * ld;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = load4(row, c.feature(j, q), c.lim);
    }
  }
};

template <bool WHOLE, int FM, int FN, bool AHEAD>
struct Rows<WHOLE, Duo, FM, FN, AHEAD> {
  typedef BlockIO<Duo> IO;
  static constexpr bool NEXT = FM * FN <= 4;  // (larger tiles have no registers for it)
  const Duo* a;
  long ld;
  IO::Block next;
  __device__ __forceinline__ Rows(const Duo* a_, long ld_, const Place& c) : a(a_), ld(ld_) {
    if (NEXT && a) next = IO::fetch(a, ld, c, 0, 0);
  }
  __device__ __forceinline__ void get(const Place& c, int i, int j, unsigned char* buf, f32x4 (&v)[4]) {
    if (a) {
      const IO::Block b = NEXT ? next : IO::fetch(a, ld, c, i, j);
      if (NEXT && i + 1 < FM) next = IO::fetch(a, ld, c, i + 1, j);
      else if (NEXT && j + 1 < FN) next = IO::fetch(a, ld, c, 0, j + 1);
      IO::quads(b, c, buf, v);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = 0.f;
    }
  }
};

// The quads of block (i, j) to an array of rows of ld values, n of which are written.
template <bool WHOLE, typename T, typename F>
__device__ __forceinline__ void put_rows(T* a, long ld, int n, const Place& c, int i, int j, unsigned char* buf,
                                         const f32x4 (&v)[4], F row) {
  if constexpr (WHOLE) {
    BlockIO<T>::store(a, ld, c, i, j, buf, v, row);
  } else if (c.row(i) < c.M) {
    T* r = a + (size_t)row(c.row(i)) * ld;
#pragma unroll
    for (int q = 0; q < 4; ++q) store4(r, c.feature(j, q), n, v[q]);
  }
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void put_rows(T* a, long ld, int n, const Place& c, int i, int j, unsigned char* buf,
                                         const f32x4 (&v)[4]) {
  put_rows<WHOLE>(a, ld, n, c, i, j, buf, v, [](int m) { return m; });
}

// (values in two parts: whole rows)
template <bool WHOLE>
__device__ __forceinline__ void put_rows(Duo* a, long ld, int, const Place& c, int i, int j, unsigned char* buf, const f32x4 (&v)[4]) {
  BlockIO<Duo>::store(a, ld, c, i, j, buf, v);
}

// Four features of a row vector (a bias) for each quad of block column j; zeros without one.
template <bool WHOLE, typename T>
__device__ __forceinline__ void get_bias(const T* b, const Place& c, int j, f32x4 (&v)[4]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = b ? load4<WHOLE>(b, c.feature(j, q), c.lim) : f32x4{0.f, 0.f, 0.f, 0.f};
}

// Sums over a wave's rows of the features of a block column: v holds a lane's sums over its own
// rows. Halving exchanges over the 32 lanes that share features leave one feature's sum per pair of
// lanes: that of feature 8 (r / 4) + 4 (lane / 32) + r % 4, r = lane / 2 % 16.
__device__ __forceinline__ float fold_columns(const f32x16& v, int lane) {
  // after the exchange over a lane bit the lane keeps the values r whose bit matches its own
  float w[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) w[r] = v[r];
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int half = 8 >> b, bit = 16 >> b;
    const bool up = lane & bit;
#pragma unroll
    for (int r = 0; r < half; ++r) {
      const float mine = up ? w[r + half] : w[r], other = up ? w[r] : w[r + half];
      w[r] = mine + __shfl_xor(other, bit, 64);
    }
  }
  return w[0] + __shfl_xor(w[0], 1, 64);
}

// The waves' folded sums of each block column, added in order: out(n, sum), n = n0 ..
template <int FN, int WGM, int WGN, typename F>
__device__ __forceinline__ void column_sums(const float (&s)[FN], const Place& c, float* lds, F out) {
  constexpr int BNW = 32 * FN;
  const int r = (c.lane >> 1) & 15;
  c.meet<WGM * WGN>();  // the waves' parts of the LDS are free
  if (!(c.lane & 1)) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
      lds[c.wm * (WGN * BNW) + c.wn * BNW + 32 * j + 8 * (r >> 2) + 4 * (c.lane >> 5) + (r & 3)] = s[j];
  }
  c.meet<WGM * WGN>();
  for (int n = threadIdx.x; n < WGN * BNW; n += 64 * WGM * WGN) {
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < WGM; ++w) t += lds[w * (WGN * BNW) + n];
    if (c.n0 + n < c.lim) out(c.n0 + n, t);
  }
}

// The partial sums of a split contraction as the lanes hold them; k_finish adds them in the order
// of the splits and runs the product's epilogue.
struct EpRaw {
  static constexpr bool ONE = false;
  struct Args {
    f32x4* part;  // [splits][tiles][quads of a lane][threads]
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float*) {
    constexpr int NT = 64 * WGM * WGN, Q = 4 * FM * FN;
    f32x4* out = a.part + ((size_t)c.split * gridDim.x + blockIdx.x) * (Q * NT) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (c.row(i) >= c.M) continue;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) out[((i * FN + j) * 4 + q) * NT] = quad(acc[i][j], q);
    }
  }
};

// out = f * scale[0] * D (scale: device value, nullable)
template <typename T>
struct EpScale {
  static constexpr bool ONE = false;
  struct Args {
    T* out;  // [M][N]
    float f;
    const float* scale;
  };
  template <bool WHOLE, int FM, int FN, int WGM, int WGN>
  static __device__ __forceinline__ void run(const Args& a, const Place& c, f32x16 (&acc)[FM][FN], float* lds) {
    const float f = a.scale ? a.f * a.scale[0] : a.f;
    unsigned char* buf = wave_lds(lds, c, WGN);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        f32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = quad(acc[i][j], q) * f;
        put_rows<WHOLE>(a.out, c.N, c.lim, c, i, j, buf, v);
      }
  }
};

// Adds the partial sums of a split contraction, a tile's from `first` on `step` tiles apart, in order and runs the epilogue.
template <class S, class E>
__device__ __forceinline__ void finish_tile(const Prob& p, int id, const f32x4* part, size_t first, size_t step, int splits,
                                            const typename E::Args& ea) {
  constexpr int WGM = S::WGM, WGN = S::WGN, FM = S::BM / WGM / 32, FN = S::BN / WGN / 32, Q = 4 * FM * FN;
  __shared__ __attribute__((aligned(16))) float lds[epilogue_lds(WGM * WGN, S::BM, WGN) / 4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int K;
  const Place c = place<S>(p, id, 0, wave, K);
  if (c.m0 >= c.M) return;
  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = 0.f;
#pragma unroll 2
  for (int k = 0; k < splits; ++k) {
    const f32x4* in = part + (first + k * step) * (Q * S::NT) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (c.row(i) >= c.M) continue;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const f32x4 v = in[((i * FN + j) * 4 + q) * S::NT];
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][4 * q + r] += v[r];
        }
    }
  }
  if (c.n0 + S::BNO <= c.N) E::template run<true, FM, FN, WGM, WGN>(ea, c, acc, lds);
  else E::template run<false, FM, FN, WGM, WGN>(ea, c, acc, lds);
}

template <class S, class E>
__global__ __launch_bounds__(S::NT) void k_finish(Prob p, const f32x4* part, int splits, typename E::Args ea) {
  finish_tile<S, E>(p, blockIdx.x, part, blockIdx.x, gridDim.x, splits, ea);
}

// A product of one row of A (both operands in rows): bound by reading B once. A workgroup takes NF
// features, a wave R of them: it reads whole runs of their rows (64 lanes, 16 bytes each, one after the
// other, U of them in flight), multiplies in fp32 on the vector ALU, and adds over its lanes in a fixed
// order; the sums go through the LDS into the layout that an epilogue expects of one wave. Any alignment.
// NF (one_features): a CU reads about 23 GB/s from memory, so few features a workgroup where there are
// few in all: 1024 x 8192 bf16 7.5 us with 8, 9.5 with 16, 14.2 with 32; 4096 x 4096 8.9 with 16, 11.4 with
// 32; 65536 x 4096 90 with 8, 87.5 with 16 (6.1 TB/s), 98 with 32. A checkpoint's blocks need 32.
// (Matrix instructions fed from 16 rows' 64-byte pieces took 13 to 15 us there, split tiles 12 in two launches;
// two to four rows on the vector ALU 21, where split tiles still take 12.)
inline int one_features(long N) { return N <= 16384 ? 8 : 16; }

// PAIR: of a pair of weight arrays in rows, NF rows of the two together a workgroup, a wave those of one feature.
template <typename T, int NF, class E, bool PAIR = false>
__global__ __launch_bounds__(32 * NF) void k_one(Prob p, typename E::Args ea) {
  constexpr int V = 16 / (int)sizeof(T), RUN = 64 * V, R = 2, U = 4, FN = PAIR ? 2 : 1, NFO = NF / FN;
  typedef typename GVec<T, V>::type GChunk;
  __shared__ __attribute__((aligned(16))) float lds[epilogue_lds(1, 32, 1) / 4];
  __shared__ float sums[32 * FN];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (p.count && *p.count == 0) return;
  const int n0 = blockIdx.x * NFO;
  const T* a = static_cast<const T*>(p.A);
  const T* b[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    if constexpr (PAIR) b[j] = static_cast<const T*>(j ? p.B2 : p.B) + (long)min(n0 + wave, p.N - 1) * p.ldb;
    else b[j] = static_cast<const T*>(p.B) + (long)min(n0 + wave * R + j, p.N - 1) * p.ldb;
  }
  float acc[R] = {};
  const auto add = [&](const GChunk (&w)[R], const GChunk& x) {
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
      for (int j = 0; j < R; ++j) acc[j] = fmaf((float)w[j][k], (float)x[k], acc[j]);
  };
  int k = lane * V;
  for (; k - lane * V + U * RUN <= p.K; k += U * RUN) {  // U whole runs
    GChunk w[U][R], x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int j = 0; j < R; ++j) w[u][j] = *reinterpret_cast<const GChunk*>(b[j] + k + u * RUN);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const GChunk*>(a + k + u * RUN);
#pragma unroll
    for (int u = 0; u < U; ++u) add(w[u], x[u]);
  }
  for (; k < p.K; k += RUN) {  // this lane's chunks of the rest
    GChunk w[R], x;
    if (k + V <= p.K) {
#pragma unroll
      for (int j = 0; j < R; ++j) w[j] = *reinterpret_cast<const GChunk*>(b[j] + k);
      x = *reinterpret_cast<const GChunk*>(a + k);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int j = 0; j < R; ++j) w[j][e] = k + e < p.K ? b[j][k + e] : (T)0.f;
        x[e] = k + e < p.K ? a[k + e] : (T)0.f;
      }
    }
    add(w, x);
  }
  if (threadIdx.x < 32 * FN) sums[threadIdx.x] = 0.f;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < R; ++j) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) acc[j] += __shfl_xor(acc[j], o, 64);
    if (lane == 0) sums[PAIR ? 32 * j + wave : wave * R + j] = acc[j];
  }
  __syncthreads();
  if (wave) return;
  // lane l's quad q: row m = l % 32 (of which there is one), features 8 q + 4 (l / 32) ..
  f32x16 d[1][FN];
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int r = 0; r < 16; ++r) d[0][j][r] = sums[32 * j + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)];
  Place c;
  c.M = 1, c.N = p.N, c.lim = min(p.N, n0 + NFO), c.m0 = 0, c.n0 = n0, c.mw = 0, c.nw = n0, c.wm = 0, c.wn = 0;
  c.mt = 0, c.nt = blockIdx.x, c.split = 0, c.lane = lane;
  if (n0 + 32 <= c.lim) E::template run<true, 1, FN, 1, 1>(ea, c, d, lds);
  else E::template run<false, 1, FN, 1, 1>(ea, c, d, lds);
}

// out[n] = f * scale[0] * sum over tile rows of part[t][n], in fp64 and in order (64 columns by 4
// runs of tile rows a workgroup). With `count` given, only the tile rows that hold rows below it
// were written.
template <typename T>
struct ColSum {
  const float* part;
  int tiles, bm;
  const int* count;  // nullable
  int n;
  T* out;
  float f;
  const float* scale;  // nullable
  unsigned blocks() const { return (unsigned)((n + 63) / 64); }
};

template <typename T>
__device__ __forceinline__ void col_sum(const ColSum<T>& a, int id, double (*sh)[64]) {
  const int i = id * 64 + (threadIdx.x & 63), g = threadIdx.x >> 6, n = a.n;
  const float* part = a.part;
  const int tiles = a.count ? min(a.tiles, (*a.count + a.bm - 1) / a.bm) : a.tiles;
  const int per = (tiles + 3) / 4, t1 = min(tiles, (g + 1) * per);
  double s = 0.0;
  if (i < n) {
    int t = g * per;
    for (; t + 8 <= t1; t += 8) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = part[(size_t)(t + k) * n + i];
#pragma unroll
      for (int k = 0; k < 8; ++k) s += (double)v[k];
    }
    for (; t < t1; ++t) s += (double)part[(size_t)t * n + i];
  }
  sh[g][threadIdx.x & 63] = s;
  __syncthreads();
  if (g || i >= n) return;
  s = ((sh[0][threadIdx.x] + sh[1][threadIdx.x]) + sh[2][threadIdx.x]) + sh[3][threadIdx.x];
  a.out[i] = (T)((float)s * (a.scale ? a.f * a.scale[0] : a.f));
}

template <typename T>
__global__ __launch_bounds__(256) void k_colsum(ColSum<T> a) {
  __shared__ double sh[4][64];
  col_sum(a, blockIdx.x, sh);
}

// The products that follow a gradient's first one, and its column sums, none of which needs another's
// result, as one launch: A B in (rows, columns), A^T B in (columns, columns), the longer contraction's
// tiles first, so that they are not what the launch ends with (931 x 4269 -> 186 f32 79 us against 88), then
// the sums.
template <typename T, class S, class E1, class E2>
__global__ __launch_bounds__(S::NT, S::WAVES) void k_both(Prob p1, typename E1::Args e1, Prob p2, typename E2::Args e2, ColSum<T> cs) {
  __shared__ Stages<S> stages;
  const int n1 = p1.tm * p1.tn, n2 = p2.tm * p2.tn, id = blockIdx.x;
  const bool swap = p2.K > p1.K;
  const int b1 = swap ? n2 : 0, b2 = swap ? 0 : n1;  // where each product's workgroups begin
  if (id >= b1 && id < b1 + n1) mm_tile<T, S, false, true, E1>(p1, e1, id - b1, stages);
  else if (id < n1 + n2) mm_tile<T, S, true, true, E2>(p2, e2, id - b2, stages);
  else col_sum(cs, id - n1 - n2, reinterpret_cast<double(*)[64]>(&stages));
}

// Rows of `cols` values to rows of ld values, zeros behind them (ld a multiple of a chunk): copies of
// two arrays whose rows then start on 16 bytes. 1 << shift threads a row.
template <typename T>
__global__ __launch_bounds__(256) void k_repack(const T* in0, T* out0, long rows0, const T* in1, T* out1, long rows1, int cols,
                                                int ld, int shift) {
  constexpr int V = 16 / sizeof(T);
  const int per = ld / V, tpr = 1 << shift, t = threadIdx.x & (tpr - 1);
  const long step = (long)gridDim.x * (256 >> shift);
  for (long r = (long)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift); r < rows0 + rows1; r += step) {
    const T* in = r < rows0 ? in0 + r * cols : in1 + (r - rows0) * cols;
    T* out = r < rows0 ? out0 + r * ld : out1 + (r - rows0) * ld;
    for (int i = t; i < per; i += tpr) {
      const int c = i * V;
      typename GVec<T, V>::type v;
      if (c + V <= cols) {
        v = *reinterpret_cast<const typename GVec<T, V>::type*>(in + c);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = c + k < cols ? in[c + k] : (T)0.f;
      }
      *reinterpret_cast<typename GVec<T, V>::type*>(out + c) = v;
    }
  }
}

// ---------------------------------------------------------------- launches

inline int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

// The leading dimension of the workspace's rows of n values: they start on 16 bytes, long ones on 128, a
// cache line and a stage's row (9990 x 3136 x 6849 bf16: 405 us with rows of 6912 values, 533 with 6856).
inline int padded(size_t esz, int n) {
  const int unit = (n * (long)esz > 1024 ? 128 : 16) / (int)esz;
  return ceil_div(n, unit) * unit;
}

template <typename T>
hipError_t launch_repack(const T* in0, T* out0, size_t rows0, const T* in1, T* out1, size_t rows1, int cols, int ld, hipStream_t st) {
  int shift = 0;
  while (shift < 8 && (1 << shift) < ld * (int)sizeof(T) / 16) ++shift;
  const size_t blocks = (rows0 + rows1 + (256 >> shift) - 1) / (256 >> shift);
  k_repack<T><<<(unsigned)std::min<size_t>(blocks, 1u << 20), 256, 0, st>>>(in0, out0, (long)rows0, in1, out1, (long)rows1, cols, ld,
                                                                          shift);
  return hipGetLastError();
}

// Two operands of rows of `cols` values as the products need them: the caller's arrays where their
// rows start on 16 bytes, else copies in the workspace (one launch for both).
template <typename T>
struct Operands {
  const T* p[2];
  long ld[2];
  hipError_t e = hipSuccess;
  // as_is: any alignment will do
  Operands(const void* in0, size_t rows0, void* copy0, const void* in1, size_t rows1, void* copy1, int cols, bool as_is,
           hipStream_t st) {
    const void* in[2] = {in0, in1};
    void* copy[2] = {copy0, copy1};
    size_t rows[2] = {rows0, rows1};
    const int lp = padded(sizeof(T), cols);
    for (int i = 0; i < 2; ++i) {
      p[i] = static_cast<const T*>(in[i]);
      ld[i] = cols;
      if (as_is || !in[i] || (cols % (16 / (int)sizeof(T)) == 0 && (uintptr_t)in[i] % 16 == 0)) {
        rows[i] = 0;
      } else {
        p[i] = static_cast<const T*>(copy[i]);
        ld[i] = lp;
      }
    }
    if (rows[0] + rows[1])
      e = launch_repack<T>(static_cast<const T*>(in0), static_cast<T*>(copy0), rows[0], static_cast<const T*>(in1),
                           static_cast<T*>(copy1), rows[1], cols, lp, st);
  }
};

// Tile shapes. Large: a wave's 128 x 64 values reuse every LDS read most. Middle: two workgroups a
// CU, one's epilogue beside the other's products. Small: four stages in flight for short grids.
typedef Shape<256, 256, 2, 4, 128, 2, 2> Tile256;
typedef Shape<128, 128, 2, 2, 128, 2, 2> Tile128;
typedef Shape<128, 128, 2, 2, 128, 4, 2> Tile128d;  // four stages, where a CU holds one workgroup at most
typedef Shape<64, 64, 2, 2, 128, 4, 2> Tile64;  // (eight stages are no faster: 12.7 to 13.9 us on 24 x 8192 x 2048)
typedef Shape<256, 256, 2, 4, 128, 2, 1> Tile256f;  // float: two steps a stage; bound by the split's vector instructions
typedef Shape<128, 128, 2, 2, 128, 2, 1> Tile128f;
typedef Shape<64, 64, 2, 2, 128, 4, 1> Tile64f;
// between: symmetric results whose tiles of 256 leave much of the card idle (both operands in rows)
typedef Shape<192, 192, 2, 3, 128, 2, 2> Tile192;
typedef Shape<192, 192, 2, 3, 128, 2, 1> Tile192d;
// of a pair of arrays in rows: 32 features of each, a wave holds both products of its rows
typedef Shape<64, 64, 2, 1, 128, 4, 2> Tile64p;
typedef Shape<64, 64, 2, 1, 128, 4, 1> Tile64pf;
constexpr int STAGE_BYTES = 128;

// The plan with the least estimated time, from measured times of a stage (us) with one workgroup on
// a CU and with two (of 256: two in turn; one on every CU takes 1.8). A split writes and reads its
// partial sums (3 TB/s both ways) and takes a second launch (3 us). The epilogue is not in it: short
// contractions and heavy epilogues (gradients, losses) take up to twice the estimate. Measured against the other choices,
// bf16: 1024 x 1024 x 4096 21 us by tiles of 64 (128: 34, 256: 89); 2048 x 2048 x 4096 39 by 128 with four
// stages (two: 45, 64: 55, 256: 88); 4096 x 2048 x 4096 63 us by 128 with two stages (four: 75); 8192 x 4096 x
// 4096 230 us by 256 (128: 256, 64: over 370). float: 4096 x 1024 x 1024 60 us by 128 (64: 74, 256: 134);
// 1024 x 1024 x 4096 (columns) 70 by 128 in eight splits, which the estimate takes, 68 in four (64 in two: 77,
// 256: 501); 4096 x 4096 x 4096 545 by 256 (128: 600 to 694, 64: 1008).
// batch: products of this size in one launch; sym: only the tiles on and below the diagonal; duo: values in two
// parts (half again the products of 16-bit values a stage).
inline Plan plan_of(size_t esz, long M, long N, long K, long batch = 1, bool sym = false, bool duo = false) {
  const int steps = ceil_div(K * (long)esz, STAGE_BYTES);
  const double stage[3][3][2] = {
      {{1.4, 3.6}, {0.60, 1.0}, {0.30, 0.45}}, {{4.1, 8.7}, {1.8, 2.7}, {0.75, 1.15}}, {{2.1, 5.4}, {0.9, 1.5}, {0.40, 0.65}}};
  const auto& us = stage[duo ? 2 : esz == 4];
  Plan best{};
  double least = 1e30;
  for (int s = 0; s < 3; ++s) {
    const int tile = 256 >> s;
    const long tm = ceil_div(M, tile), tn = ceil_div(N, tile), tiles = batch * (sym ? tm * (tm + 1) / 2 : tm * tn);
    // (one tile row reads its weights once, from memory: 0.42 a stage with one workgroup on a CU)
    const double two = us[s][1],
                 one = tile == 256 && tiles > 128 ? two / 2 : tile == 64 && tm == 1 && esz == 2 ? 0.42 : us[s][0];
    for (int splits : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      if (splits > 1 && (steps < 4 * splits || tile == 256)) break;  // (a split large tile would be two middle ones)
      const long n = ceil_div(tiles * splits, 256);
      double t = ceil_div(steps, splits) * ((n / 2) * two + (n % 2) * one);
      if (splits > 1) t += 3.0 + 2.0 * splits * M * tn * tile * 4 * (sym ? 0.5 : 1.0) * batch / 3e6;
      if (t < least) {
        least = t;
        best = Plan{tile, splits, (int)tm, (int)tn, t};
      }
    }
  }
  return best;
}

// The plan of a product whose operands are both in rows: k_one for one row.
inline Plan plan_rows(size_t esz, long M, long N, long K) {
  if (M == 1) return Plan{1, 1, 1, ceil_div(N, one_features(N))};
  return plan_of(esz, M, N, K);
}

template <typename T>
hipError_t launch_colsum(const ColSum<T>& cs, hipStream_t st) {
  k_colsum<T><<<cs.blocks(), 256, 0, st>>>(cs);
  return hipGetLastError();
}

template <typename T, class S, bool AT, bool BT, class E>
hipError_t launch_shape(Prob p, const typename E::Args& ea, const Plan& pl, void* part, hipStream_t st) {
  constexpr int BK = S::KB / (int)sizeof(T);
  p.tm = pl.tm;
  p.tn = pl.tn;
  p.kper = std::max(1, ceil_div(ceil_div(p.K, BK), pl.splits)) * BK;
  const unsigned tiles = (unsigned)(p.tm * p.tn);
  if (S::BM == 256 || pl.splits == 1) {
    k_mm<T, S, AT, BT, E><<<dim3(tiles), S::NT, 0, st>>>(p, ea);
  } else if constexpr (S::BM < 256) {
    k_mm<T, S, AT, BT, EpRaw><<<dim3(tiles, (unsigned)pl.splits), S::NT, 0, st>>>(p, EpRaw::Args{static_cast<f32x4*>(part)});
    k_finish<Paired<Shape<S::BM, S::BN, S::WGM, S::WGN, 128, 2, 2>, S::PAIR>, E><<<dim3(tiles), S::NT, 0, st>>>(p, static_cast<const f32x4*>(part), pl.splits, ea);
  }
  return hipGetLastError();
}

// part: pl.part_bytes() of workspace. Epilogues of products that one row may have (ONE) come in one-row kernels too.
template <typename T, bool AT, bool BT, class E, int PAIR = PAIR_NONE>
hipError_t launch_mm(const Prob& p, const typename E::Args& ea, const Plan& pl, void* part, hipStream_t st) {
  if constexpr (!AT && !BT && E::ONE) {
    if (pl.tile == 1) {
      if constexpr (PAIR == PAIR_ROWS) {
        if (one_features(2L * p.N) == 8) k_one<T, 8, E, true><<<(unsigned)pl.tn, 256, 0, st>>>(p, ea);
        else k_one<T, 16, E, true><<<(unsigned)pl.tn, 512, 0, st>>>(p, ea);
      } else {
        if (ea.blocks_of_32()) k_one<T, 32, E><<<(unsigned)ceil_div(p.N, 32), 1024, 0, st>>>(p, ea);
        else if (one_features(p.N) == 8) k_one<T, 8, E><<<(unsigned)pl.tn, 256, 0, st>>>(p, ea);
        else k_one<T, 16, E><<<(unsigned)pl.tn, 512, 0, st>>>(p, ea);
      }
      return hipGetLastError();
    }
  }
  if constexpr (sizeof(T) == 2) {
    if (pl.tile == 256) return launch_shape<T, Paired<Tile256, PAIR>, AT, BT, E>(p, ea, pl, part, st);
    if (pl.tile == 128) {
      if ((long)pl.tm * pl.tn * pl.splits <= 256) return launch_shape<T, Paired<Tile128d, PAIR>, AT, BT, E>(p, ea, pl, part, st);
      return launch_shape<T, Paired<Tile128, PAIR>, AT, BT, E>(p, ea, pl, part, st);
    }
    return launch_shape<T, Paired<std::conditional_t<PAIR == PAIR_ROWS, Tile64p, Tile64>, PAIR>, AT, BT, E>(p, ea, pl, part, st);
  } else {
    if (pl.tile == 256) return launch_shape<T, Paired<Tile256f, PAIR>, AT, BT, E>(p, ea, pl, part, st);
    if (pl.tile == 128) return launch_shape<T, Paired<Tile128f, PAIR>, AT, BT, E>(p, ea, pl, part, st);
    return launch_shape<T, Paired<std::conditional_t<PAIR == PAIR_ROWS, Tile64pf, Tile64f>, PAIR>, AT, BT, E>(p, ea, pl, part, st);
  }
}

// Two products and a gradient's column sums (cs.out nullable): one launch where both take the small
// tiles unsplit and contract over at most BOTH_STAGES stages, else one each. 98 shapes of 2 to 2000
// workgroups, one launch against three, times of the whole way back: 11.7 us against 18.2 (93 x 32 -> 62 bf16) to
// 0.95 times (564 x 6751 -> 567 f32); 9 % less with 61 and 48 stages (3010 x 499 -> 3868 bf16), 3 % with 51 and
// 50 of floats (1598 x 2483 -> 1614). Beyond, launches do not count: with 109 stages each 1 % less, with 102 and
// 179 (11419 x 266 -> 6519 bf16) 2 % more, since the launch ends unevenly.
constexpr int BOTH_STAGES = 64;
template <typename T, class E1, class E2>
hipError_t launch_both(Prob p1, const typename E1::Args& e1, const Plan& pl1, Prob p2, const typename E2::Args& e2,
                       const Plan& pl2, const ColSum<T>& cs, void* part, hipStream_t st) {
  const auto one = [](Prob& p, const Plan& pl) {
    const int stages = std::max(1, ceil_div(p.K * (long)sizeof(T), STAGE_BYTES));
    if (pl.tile != 64 || pl.splits != 1 || stages > BOTH_STAGES) return false;
    p.tm = pl.tm, p.tn = pl.tn;
    p.kper = stages * (STAGE_BYTES / (int)sizeof(T));
    return true;
  };
  if (one(p1, pl1) && one(p2, pl2)) {
    typedef std::conditional_t<sizeof(T) == 2, Tile64, Tile64f> S;
    const unsigned grid = (unsigned)(p1.tm * p1.tn + p2.tm * p2.tn) + (cs.out ? cs.blocks() : 0);
    k_both<T, S, E1, E2><<<grid, S::NT, 0, st>>>(p1, e1, p2, e2, cs);
    return hipGetLastError();
  }
  hipError_t e = launch_mm<T, false, true, E1>(p1, e1, pl1, part, st);
  if (e == hipSuccess) e = launch_mm<T, true, true, E2>(p2, e2, pl2, part, st);
  if (e == hipSuccess && cs.out) e = launch_colsum(cs, st);
  return e;
}

}  // namespace mm
}  // namespace lp
