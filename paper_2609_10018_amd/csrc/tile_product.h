// Tile products of the linear layer's cross-entropy: D = A B^T over K for one
// workgroup's BM x BN tile, with either operand lying straight (rows of K
// contiguous values) or turned (K rows of contiguous columns), in bf16 or fp32.
//
// A step is KB = 128 bytes of K of a straight operand, and as many rows of a turned one as that
// holds values.  Tiles go to LDS by direct 16-byte loads, in two to four stages.
//  * Straight: LDS rows of KB bytes, 16-byte chunk c of row r at c ^ (r>>1 & 7).
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

#include <type_traits>

#include "common.h"
#include "lds_load.h"

namespace elasto {

// A matrix as it lies in memory.
struct Matrix {
  const char* p = nullptr;
  int64_t ld = 0;  // bytes between its rows
};

constexpr int KB = 128;

// TURNED: whether K is the operand's row.  B: the tile's size along the other axis.
template <typename T, bool TURNED, int B, int THREADS>
struct Operand {
  static constexpr int kBytes = B * KB, kK = KB / (int)sizeof(T), kQuarters = KB / 32;
  static constexpr int kRow = TURNED ? B * (int)sizeof(T) : KB;  // bytes of an LDS row
  static constexpr int kChunks = kRow / 16;
  static constexpr int kReads = !TURNED ? 1 : sizeof(T) == 2 ? 2 : 4;  // LDS reads of a quarter
  static constexpr int kLoads = kBytes / (16 * THREADS);
  static_assert(kBytes % (16 * THREADS) == 0, "whole loads");

  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (!TURNED) return (r >> 1) & 7;
    if constexpr (B == 32) return 0;  // four rows are 256 bytes (fp32: the half-waves' rows share banks)
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
  __device__ __forceinline__ void issue(char* stage, const char* from, int k, uint64_t live, int tid) const {
    const __amdgpu_buffer_rsrc_t src =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from), (short)0, 0x7fffffff, kRsrcWord3);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    auto load = [&](int i, uint32_t off) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void*)(stage + (i * THREADS + wave * 64) * 16), 16,
                                               (int)off, 0, 0, 0);
    };
    if (k == kK && (!LIVE || live == ~0ull)) {  // a whole step
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load(i, at[i]);
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = row(i, tid);
        bool in = TURNED ? r < k : chunk(i, tid) * (16 / (int)sizeof(T)) < k;
        if constexpr (LIVE) in = in && ((live >> r) & 1);
        load(i, in ? at[i] : kOutOfRange);
      }
    }
  }

  // A lane's addresses in a stage, for a wave whose rows (columns) start at `first`, a multiple of 32:
  // straight, one for each quarter, blocks 32 rows apart; turned, one for each block of 32 columns,
  // quarters a fixed number of rows apart.
  template <int BLOCKS>
  struct Reader {
    int at[TURNED ? BLOCKS : kQuarters];
    // from: the quarter that counts as the first.
    __device__ __forceinline__ Reader(int first, int lane, int from) {
      const int lr = lane & 31, lg = lane >> 5;
      if constexpr (!TURNED) {
#pragma unroll
        for (int kk = 0; kk < kQuarters; ++kk) at[kk] = (first + lr) * KB + (((2 * (kk + from) + lg) ^ swizzle(lr)) << 4);
      } else {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
          if constexpr (sizeof(T) == 2) {
            const int lq = lane & 15, g = lane >> 4;
            const int r = 8 * lg + (lq >> 2), c = first + 32 * i + 16 * (g & 1) + 4 * (lq & 3);
            at[i] = (r + 16 * from) * kRow + (((c >> 3) ^ swizzle(r)) << 4) + (c & 7) * 2;
          } else {
            const int r = 4 * lg, c = first + 32 * i + lr;
            at[i] = (r + 8 * from) * kRow + (((c >> 2) ^ swizzle(r)) << 4) + (c & 3) * 4;
          }
        }
      }
    }
    // The values of quarter kk of block i.
    __device__ __forceinline__ u32x4 read(const char* stage, int i, int kk) const {
      if constexpr (!TURNED) {
        return *reinterpret_cast<const u32x4*>(stage + at[kk] + i * 32 * KB);
      } else if constexpr (sizeof(T) == 2) {
        typedef short i16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        const char* p = stage + at[i] + kk * 16 * kRow;
        const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)p));
        const u32x2 hi =
            __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 4 * kRow)));
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
      } else {
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = *reinterpret_cast<const uint32_t*>(stage + at[i] + (8 * kk + e) * kRow);
        return v;
      }
    }
  };
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

// GROUPS: workgroups that a CU holds by their registers and LDS.  KS: 4 where each of four groups of WM x
// WN waves takes one quarter of every step (small launches: a tile's chain of products is a quarter as
// long); their sums are added at the end, in the groups' order, in all of them.
template <typename T_, int BM_, int BN_, int WM_, int WN_, int STAGES_, int GROUPS_, int KS_ = 1>
struct Shape {
  typedef T_ T;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
  static constexpr int kK = KB / (int)sizeof(T_);  // values of K of a step
  static constexpr int KS = KS_, kTeam = WM * WN, kThreads = 64 * kTeam * KS;
  static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 32, TN = WTN / 32;
  static constexpr int kStage = (BM + BN) * KB;
  static constexpr bool kFew = TM * TN <= 2;  // few accumulators
  static constexpr int kGroups = GROUPS_, kWaves = kGroups * kTeam * KS / 4;  // kWaves: on a SIMD
  static_assert(STAGES * kStage * kGroups <= 160 * 1024, "LDS of a CU");
  static_assert(KS == 1 || (KS == 4 && KS * kTeam * TM * TN * 4096 <= STAGES * kStage), "quarters");
};

// The operands' values of one quarter of a step.
template <typename S>
struct Quarter {
  u32x4 a[S::TM], b[S::TN];
};
template <typename S, typename OA, typename OB>
struct Readers {
  typename OA::template Reader<S::TM> a;
  typename OB::template Reader<S::TN> b;
  __device__ __forceinline__ Readers(int wave, int lane)
      : a(wave % S::kTeam / S::WN * S::WTM, lane, wave / S::kTeam),
        b(wave % S::WN * S::WTN, lane, wave / S::kTeam) {}
  __device__ __forceinline__ void read(Quarter<S>& q, const char* st, int kk) const {
#pragma unroll
    for (int i = 0; i < S::TM; ++i) q.a[i] = a.read(st, i, kk);
#pragma unroll
    for (int j = 0; j < S::TN; ++j) q.b[j] = b.read(st + OA::kBytes, j, kk);
  }
};

template <int G, int NM, int NR>
struct Interleave {
  static __device__ __forceinline__ void go() {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    constexpr int n = NR * (G + 1) / NM - NR * G / NM;
    if constexpr (n > 0) __builtin_amdgcn_sched_group_barrier(0x100, n, 0);
    if constexpr (G + 1 < NM) Interleave<G + 1, NM, NR>::go();
  }
};

// Where a step's operands lie, and how much of it there is.
struct StepAt {
  const char *a, *b;
  int k;
  uint64_t live;  // one bit for each of its rows of K
};
template <bool LIVE, typename OA, typename OB>
__device__ __forceinline__ void issue_step(const OA& oa, const OB& ob, char* st, const StepAt& at, int tid) {
  oa.template issue<false>(st, at.a, at.k, ~0ull, tid);
  ob.template issue<LIVE>(st + OA::kBytes, at.b, at.k, at.live, tid);
}

// One step: the loads of a later one into `fill`, the products from `st`.  Each quarter's operands
// are read while the one before is multiplied; q[1] comes with the last quarter of the step before (not of
// the first) and leaves with this one's.  `fill` and `st` are different stages: said so that the
// compiler does not make the reads of one wait for the loads of the other.
template <typename S, bool LIVE, bool FIRST, typename OA, typename OB>
__device__ __forceinline__ void product_step(const OA& oa, const OB& ob, const Readers<S, OA, OB>& rd, char* __restrict__ fill,
                                             const char* __restrict__ st, bool more, const StepAt& at,
                                             Quarter<S> (&q)[2], f32x16 (&acc)[S::TM][S::TN]) {
  typedef typename S::T T;
  const int tid = threadIdx.x;
  constexpr int NR = OA::kReads * S::TM + OB::kReads * S::TN, NM = (sizeof(T) == 2 ? 1 : 4) * S::TM * S::TN;
  if constexpr (S::KS > 1) {  // this group's quarter, multiplied a step later
    rd.read(q[0], st, 0);
    if (more) issue_step<LIVE>(oa, ob, fill, at, tid);
    if constexpr (!FIRST) multiply<T>(q[1].a, q[1].b, acc);
    q[1] = q[0];
    return;
  }
  __builtin_amdgcn_sched_barrier(0);
  rd.read(q[0], st, 0);
  if constexpr (!FIRST) {
    multiply<T>(q[1].a, q[1].b, acc);
    Interleave<0, NM, NR>::go();
    __builtin_amdgcn_sched_barrier(0);
  }
  if (more) issue_step<LIVE>(oa, ob, fill, at, tid);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int kk = 1; kk < OA::kQuarters; ++kk) {
    rd.read(q[kk & 1], st, kk);
    multiply<T>(q[~kk & 1].a, q[~kk & 1].b, acc);
    Interleave<0, NM, NR>::go();
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Whether this wave's group starts from acc (the others from zeros) and hands the results out.
template <typename S>
__device__ __forceinline__ bool leads() {
  return S::KS == 1 || (int)threadIdx.x < 64 * S::kTeam;
}

// The sums of K values [k0, k1) (k0 a whole step) of the tile at (m0, n0), into acc, which
// holds what they start from.  M, N: the operands' sizes.  LIVE: bits of K's rows, of which
// the others are not read in B (in A they hold zeros).  Ends with all loads and reads done in this wave;
// others may still read their last quarter.
template <typename S, bool TA, bool TB, bool LIVE>
__device__ __forceinline__ void tile_product(char* smem, const Matrix& A, const Matrix& B, int64_t M, int64_t N,
                                             int64_t m0, int64_t n0, int64_t k0, int64_t k1, const uint32_t* live,
                                             f32x16 (&acc)[S::TM][S::TN]) {
  typedef typename S::T T;
  constexpr int K = S::kK, ES = (int)sizeof(T);
  typedef Operand<T, TA, S::BM, S::kThreads> OA;
  typedef Operand<T, TB, S::BN, S::kThreads> OB;
  constexpr int kLoads = OA::kLoads + OB::kLoads, kAhead = S::STAGES - 1;
  const int tid = threadIdx.x;
  const OA oa(A.ld, M - m0, tid);
  const OB ob(B.ld, N - n0, tid);
  const Readers<S, OA, OB> rd(__builtin_amdgcn_readfirstlane(tid >> 6), tid & 63);
  const char* pa = A.p + (TA ? k0 * A.ld + m0 * ES : m0 * A.ld + k0 * ES);
  const char* pb = B.p + (TB ? k0 * B.ld + n0 * ES : n0 * B.ld + k0 * ES);
  const int64_t sa = TA ? A.ld * K : KB, sb = TB ? B.ld * K : KB;
  const int nk = (int)((k1 - k0 + K - 1) / K);
  if (nk <= 0) return;
  const uint32_t* words = live + k0 / 32;
  auto bits_of = [&](int kt) -> uint64_t {
    if constexpr (!LIVE) return ~0ull;
    if constexpr (K == 64) return (uint64_t)words[2 * kt] | (uint64_t)words[2 * kt + 1] << 32;
    return (uint64_t)words[kt] | ~0ull << 32;
  };
  // Read a step ahead of their use, so that nothing waits for them.
  uint64_t bits = bits_of(0);
  auto step = [&](int kt) {
    const StepAt at = {pa + kt * sa, pb + kt * sb, (int)min((int64_t)K, k1 - k0 - (int64_t)kt * K), bits};
    bits = bits_of(min(kt + 1, nk - 1));
    return at;
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (i < nk) issue_step<LIVE>(oa, ob, smem + i * S::kStage, step(i), tid);
  Quarter<S> q[2];
  int use = 0, fill = kAhead;  // stages
  auto one = [&](int kt, auto first) {
    // This step's loads are back: all but those of the steps behind it.
    if (kAhead > 1 && kt + kAhead <= nk)
      wait_vm_lds<(kAhead - 1) * kLoads>();
    else
      wait_vm_lds<0>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const bool more = kt + kAhead < nk;
    product_step<S, LIVE, decltype(first)::value>(oa, ob, rd, smem + fill * S::kStage, smem + use * S::kStage, more,
                                                  step(more ? kt + kAhead : nk - 1), q, acc);
    use = use + 1 == S::STAGES ? 0 : use + 1;
    fill = fill + 1 == S::STAGES ? 0 : fill + 1;
  };
  one(0, std::true_type());
  if constexpr (S::kFew && sizeof(T) == 4) {
    // fp32 in small tiles: the sums of eight steps (256 values of K) are added up by themselves, so
    // that an error does not grow with the root of K.
    f32x16 sum[S::TM][S::TN] = {};
    for (int kt = 1; kt < nk;) {
      const int end = min(nk, kt + 8);
#pragma clang loop unroll(disable)
      for (; kt < end; ++kt) one(kt, std::false_type());
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
          sum[i][j] += acc[i][j];
          acc[i][j] = f32x16{};
        }
    }
    multiply<T>(q[1].a, q[1].b, acc);
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j) acc[i][j] += sum[i][j];
  } else {
    for (int kt = 1; kt < nk; ++kt) one(kt, std::false_type());
    multiply<T>(q[1].a, q[1].b, acc);
  }
  if constexpr (S::KS > 1) {
    __syncthreads();
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), team = wave % S::kTeam, lane = tid & 63;
    auto slot = [&](int ks, int i, int j, int g) {
      return reinterpret_cast<f32x4*>(smem) + ((((ks * S::kTeam + team) * S::TM + i) * S::TN + j) * 4 + g) * 64 + lane;
    };
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *slot(wave / S::kTeam, i, j, g) = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 s = *slot(0, i, j, g);
#pragma unroll
          for (int ks = 1; ks < S::KS; ++ks) s += *slot(ks, i, j, g);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] = s[e];
        }
  }
}

}  // namespace elasto
