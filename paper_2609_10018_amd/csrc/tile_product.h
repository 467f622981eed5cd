// Tile products of the linear layer's cross-entropy: D = A B^T over K for one
// workgroup's BM x BN tile, with either operand lying straight (rows of K
// contiguous values) or turned (K rows of contiguous columns), in bf16 or fp32.
//
// A step is 128 bytes of K of a straight operand (64 bf16, 32 fp32 values), 64 or
// 32 rows of a turned one.  Tiles go to LDS by direct 16-byte loads, two stages.
//  * Straight: 128-byte LDS rows, 16-byte chunk c of row r at c ^ ((r ^ r>>3) & 7).
//    bf16: a lane's chunk is its operand.  fp32: four values of K a lane and read,
//    each the operand of one 32x32x2 product (which two values of K meet in a
//    product is free as long as both operands agree).
//  * Turned: a row of LDS for each k.  bf16: the operand, eight k of one column, comes
//    through the transposing read (in a group of 16 lanes, lane i receives column i of
//    the four rows whose 8-byte pieces the group addresses).  The chunks are exchanged
//    so that the four rows x 64 bytes that 32 lanes read lie in different banks.
//    fp32: single values, the two half-waves' rows four apart, in different banks.
// The products are taken transposed (D^T = B A^T): a lane holds one row of A and,
// in groups of four consecutive, columns 8 (e / 4) + 4 (lane / 32) + e % 4.
//
// What lies outside an operand gets an offset past every buffer and arrives as zeros.
#pragma once

#include "common.h"
#include "lds_load.h"

namespace elasto {

// A matrix as it lies in memory.
struct Matrix {
  const char* p = nullptr;
  int64_t ld = 0;  // bytes between its rows
};

template <typename T>
struct Step {
  static constexpr int K = 128 / (int)sizeof(T);  // values of K
};

// TURNED: whether K is the operand's row.  B: the tile's size along the other axis.
template <typename T, bool TURNED, int B, int THREADS>
struct Operand {
  static constexpr int kBytes = B * 128;
  static constexpr int kRow = TURNED ? B * (int)sizeof(T) : 128;  // bytes of an LDS row
  static constexpr int kChunks = kRow / 16;
  static constexpr int kLoads = kBytes / (16 * THREADS);
  static_assert(kBytes % (16 * THREADS) == 0, "whole loads");

  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (!TURNED) return (r ^ (r >> 3)) & 7;
    if constexpr (sizeof(T) == 4) return ((r >> 2) & 1) * 8;
    if constexpr (B == 64) return ((r >> 1) & 1) * 4;
    return (r & 3) * 4;
  }

  // Where this thread's loads of a step lie, from the tile's corner.
  uint32_t at[kLoads];
  static __device__ __forceinline__ int row(int i, int tid) { return (i * THREADS + tid) / kChunks; }
  static __device__ __forceinline__ int chunk(int i, int tid) {
    return ((i * THREADS + tid) % kChunks) ^ swizzle(row(i, tid));
  }
  // size: rows or columns of the operand from the tile's corner on.
  __device__ __forceinline__ Operand(int64_t ld, int64_t size, int tid) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = row(i, tid), c = chunk(i, tid);
      const bool in = TURNED ? (int64_t)c * (16 / (int)sizeof(T)) < size : r < size;
      at[i] = in ? (uint32_t)r * (uint32_t)ld + (uint32_t)c * 16 : kOutOfRange;
    }
  }
  // The loads of a step that starts at `from`, of which k values of K are there.  live:
  // one bit for each of the step's K rows (turned operands).
  template <bool LIVE>
  __device__ __forceinline__ void issue(char* stage, const char* from, int k, const uint32_t* live,
                                        int tid) const {
    const __amdgpu_buffer_rsrc_t src =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from), (short)0, 0x7fffffff, kRsrcWord3);
    uint32_t bits[2] = {~0u, ~0u};
    if constexpr (LIVE) {
      bits[0] = live[0];
      if constexpr (Step<T>::K == 64) bits[1] = live[1];
    }
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = row(i, tid);
      bool in = true;
      if constexpr (TURNED)
        in = r < k;
      else
        in = chunk(i, tid) * (16 / (int)sizeof(T)) < k;
      if constexpr (LIVE) in = in && ((bits[r >> 5] >> (r & 31)) & 1);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          src, (lds_void*)(stage + (i * THREADS + wave * 64) * 16), 16, (int)(in ? at[i] : kOutOfRange),
          0, 0, 0);
    }
  }

  // The values of quarter kk of a step in the 32 rows (columns) from `first` on.
  static __device__ __forceinline__ u32x4 read(const char* stage, int first, int kk, int lane) {
    const int lr = lane & 31, lg = lane >> 5;
    if constexpr (!TURNED) {
      const int r = first + lr;
      return *reinterpret_cast<const u32x4*>(stage + r * 128 + (((2 * kk + lg) ^ swizzle(r)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      typedef short i16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
      const int lq = lane & 15, g = lane >> 4;
      const int r = kk * 16 + 8 * lg + (lq >> 2), c = first + 16 * (g & 1) + 4 * (lq & 3);
      const char* p = stage + r * kRow + (((c >> 3) ^ swizzle(r)) << 4) + (c & 7) * 2;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p));
      const u32x2 hi =
          __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * kRow)));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      u32x4 v;
      const int c = first + lr;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 8 * kk + 4 * lg + e;
        v[e] = *reinterpret_cast<const uint32_t*>(stage + r * kRow + (((c >> 2) ^ swizzle(r)) << 4) + (c & 3) * 4);
      }
      return v;
    }
  }
};

// acc[i][j] += the product of A's 32-row block i and B's block j of this wave.
template <typename T, int TM, int TN>
__device__ __forceinline__ void multiply(const u32x4 (&a)[TM], const u32x4 (&b)[TN], f32x16 (&acc)[TM][TN]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8, b[j]), __builtin_bit_cast(bf16x8, a[i]), acc[i][j], 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(b[j][e]), __uint_as_float(a[i][e]),
                                                           acc[i][j], 0, 0, 0);
  }
}

template <typename T_, int BM_, int BN_, int WM_, int WN_>
struct Shape {
  typedef T_ T;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int kThreads = 64 * WM * WN;
  static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  static constexpr int kStage = (BM + BN) * 128;
};

template <bool LIVE, typename OA, typename OB>
__device__ __forceinline__ void issue_step(const OA& oa, const OB& ob, char* st, const char* pa, const char* pb,
                                           int k, const uint32_t* bits, int tid) {
  oa.template issue<false>(st, pa, k, nullptr, tid);
  ob.template issue<LIVE>(st + OA::kBytes, pb, k, bits, tid);
}

// One step: the next one's loads into `fill`, the products from `st`.
template <typename S, bool LIVE, typename OA, typename OB>
__device__ __forceinline__ void product_step(const OA& oa, const OB& ob, char* __restrict__ fill,
                                             const char* __restrict__ st, bool more, const char* pa,
                                             const char* pb, int k, const uint32_t* bits,
                                             f32x16 (&acc)[S::TM][S::TN]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN;
  if (more) issue_step<LIVE>(oa, ob, fill, pa, pb, k, bits, tid);
#pragma unroll
  for (int kk = 0; kk < 4; ++kk) {
    u32x4 a[S::TM], b[S::TN];
#pragma unroll
    for (int i = 0; i < S::TM; ++i) a[i] = OA::read(st, wm * S::WTM + 32 * i, kk, lane);
#pragma unroll
    for (int j = 0; j < S::TN; ++j) b[j] = OB::read(st + OA::kBytes, wn * S::WTN + 32 * j, kk, lane);
    multiply<typename S::T>(a, b, acc);
  }
}

// The sums of K values [k0, k1) (k0 a whole step) of the tile at (m0, n0), into acc, which
// holds what they start from.  M, N: the operands' sizes.  LIVE: bits of K's rows, of which
// the others are not read in B (in A they hold zeros).
template <typename S, bool TA, bool TB, bool LIVE>
__device__ __forceinline__ void tile_product(char* smem, const Matrix& A, const Matrix& B, int64_t M, int64_t N,
                                             int64_t m0, int64_t n0, int64_t k0, int64_t k1, const uint32_t* live,
                                             f32x16 (&acc)[S::TM][S::TN]) {
  typedef typename S::T T;
  constexpr int K = Step<T>::K, ES = (int)sizeof(T);
  typedef Operand<T, TA, S::BM, S::kThreads> OA;
  typedef Operand<T, TB, S::BN, S::kThreads> OB;
  const int tid = threadIdx.x;
  const OA oa(A.ld, M - m0, tid);
  const OB ob(B.ld, N - n0, tid);
  const char* pa = A.p + (TA ? k0 * A.ld + m0 * ES : m0 * A.ld + k0 * ES);
  const char* pb = B.p + (TB ? k0 * B.ld + n0 * ES : n0 * B.ld + k0 * ES);
  const int64_t sa = TA ? A.ld * K : 128, sb = TB ? B.ld * K : 128;
  const int nk = (int)((k1 - k0 + K - 1) / K);
  const uint32_t* bits = LIVE ? live + k0 / 32 : nullptr;
  auto left = [&](int kt) { return (int)min((int64_t)K, k1 - k0 - (int64_t)kt * K); };
  auto stage = [&](int kt) { return smem + (kt & 1) * S::kStage; };
  auto bits_of = [&](int kt) { return LIVE ? bits + kt * (K / 32) : nullptr; };
  if (nk > 0) issue_step<LIVE>(oa, ob, stage(0), pa, pb, left(0), bits_of(0), tid);
  for (int kt = 0; kt < nk; ++kt) {
    wait_vm_lds<0>();
    __syncthreads();
    const bool more = kt + 1 < nk;
    product_step<S, LIVE>(oa, ob, stage(kt + 1), stage(kt), more, pa + (kt + 1) * sa, pb + (kt + 1) * sb,
                          more ? left(kt + 1) : 0, more ? bits_of(kt + 1) : nullptr, acc);
  }
}

}  // namespace elasto
