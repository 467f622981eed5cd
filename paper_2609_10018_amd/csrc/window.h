// Shared by the forward and backward kernels of the windowed attention: the
// mask, packed query rows, LDS tiles and the operands of the matrix
// instructions.
//
// Packed rows: the G = heads / kv_heads query heads of a key head are taken
// together, row r = i * G + g being query i of the group's head g, so that a
// tile of rows reads each key once for the whole group and stays within few
// positions.
//
// Positions: query i of a sequence with ql queries and kl keys stands at
// p = i + kl - ql, key j at j.  p sees j < kl if (|p - j| < window or
// j < sinks) and, causal, j <= p.
//
// Matrix instructions (32x32, 16 k-slots): lane l holds row (A) or column (B)
// l % 32 and k-slots 8 * (l / 32) + 0..7; of the result, column l % 32 and rows
// 8 * (i / 4) + 4 * (l / 32) + i % 4, i < 16.  k-slots are only labels: a
// transposed score block's registers 8t .. 8t + 7 are rows 16t + 4h + 0..3 and
// 16t + 8 + 4h + 0..3 (h = l / 32) of a column, and serve as they stand as the
// B operand of the next product, whose A operand is read from LDS with the same
// assignment (transposed_operand).  fp32 uses 32x32x2 instructions, one per
// pair of k-slots, in the same layout.
#pragma once

#include "common.h"
#include "heads.h"
#include "lds_load.h"

namespace elasto {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Mask {
  int causal, window, sinks;
};

// Keys that position pos sees among kl: [0, hs] and [lo, hi] (hi < lo: none).
struct Keys {
  int hs, lo, hi;
};
__device__ __forceinline__ Keys keys_of(const Mask& m, int pos, int kl) {
  const int last = m.causal ? min(pos, kl - 1) : kl - 1;
  Keys k;
  k.hs = min(m.sinks - 1, last);
  k.lo = max(pos - m.window + 1, 0);
  k.hi = min(last, pos + m.window - 1);
  return k;
}

// What a block of scores starts from where the mask hides some of them: 0, or
// -infinity, so that the branch over it leaves the scores where they are.  x[i]
// is for row `from` + 8 * (i / 4) + i % 4 of a range of len.
__device__ __forceinline__ f32x16 hidden(int from, unsigned len) {
  f32x16 x;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    x[i] = (unsigned)(from + 8 * (i >> 2) + (i & 3)) < len ? 0.0f : -INFINITY;
  return x;
}
// Keys j + 8 * (i / 4) + i % 4.  low, high: some of the block's keys may lie
// before a row's window, behind it (one of them: one comparison a score);
// sinks: some may be sinks.
__device__ __forceinline__ f32x16 hidden(int j, const Keys& k, bool low, bool high, bool sinks) {
  f32x16 x;
  const int first = k.lo - j, last = k.hi - j, sink = k.hs - j;
  if (low && high) {
    x = hidden(-first, (unsigned)max(k.hi - k.lo + 1, 0));
  } else if (high) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 8 * (i >> 2) + (i & 3) <= last ? 0.0f : -INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 8 * (i >> 2) + (i & 3) >= first ? 0.0f : -INFINITY;
  }
  if (sinks)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = sink >= 8 * (i >> 2) + (i & 3) ? 0.0f : x[i];
  return x;
}

__device__ __forceinline__ int clamp_len(const int32_t* lens, int b, int longest) {
  return lens ? min(max(lens[b], 0), longest) : longest;
}

// Consecutive workgroups go to the eight XCDs in turn, each with an L2 of its
// own: give each XCD a contiguous run of the work, so that the tiles that read
// the same keys share an L2.
__device__ __forceinline__ int64_t xcd_order(int64_t id, int64_t n) {
  const int64_t x = id & 7, q = n >> 3, rem = n & 7;
  return x * q + (x < rem ? x : rem) + (id >> 3);
}

// Keeps an accumulator where it is across a branch: without this the compiler
// moves whole accumulators (16 instructions each) at the join.  FEW: the kernel
// needs no more than 256 registers a lane; otherwise its accumulators lie in the
// second file (fp32, heads of 128, backward 2 x 2048 tokens x 8 heads: 411 us
// untied, with spills, 372 tied).
template <bool FEW>
__device__ __forceinline__ void stay(f32x16& x) {
  if constexpr (FEW) asm volatile("" : "+v"(x));
  else asm volatile("" : "+a"(x));
}

// The other half-wave's value.
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ void zero(f32x16& v) {
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = 0.0f;
}

// Keys that some of the rows between two positions see (their keys_of: a0, a1):
// [0, last] without [gap0, gap1).
struct SeenKeys {
  int last, gap0, gap1;
  __device__ __forceinline__ SeenKeys(const Keys& a0, const Keys& a1)
      : last(max(a1.hs, a1.hi)), gap0(max(a1.hs + 1, 0)), gap1(a0.lo) {}
};

// `bytes` bytes at p as a buffer (at most kReach of them; an offset of kReach
// lies outside, as do the row's bytes that follow it).
constexpr uint32_t kReach = 0xfffff000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const char* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), (short)0,
                                           (int)(bytes < (int64_t)kReach ? (uint32_t)bytes : kReach),
                                           kRsrcWord3);
}

// One head of k or v of one sequence: rows st bytes apart.  Keys that none of
// the workgroup's rows sees arrive as zeros: what their memory holds (pages that
// a cache has given up, say) never meets a product.
struct KeyRows {
  const char* p;
  int64_t st;
  SeenKeys seen;
  bool near;                   // all of it within 32-bit offsets: one buffer for every tile
  __amdgpu_buffer_rsrc_t all;
  __device__ __forceinline__ KeyRows(const char* base, int64_t stride, const SeenKeys& keys, int row_bytes)
      : p(base), st(stride), seen(keys) {
    const int64_t bytes = (int64_t)max(seen.last, 0) * st + row_bytes;
    near = bytes < ((int64_t)1 << 31);
    all = buffer_of(p, bytes);
  }
  // The tile that starts at row j0, to LDS.
  template <typename L>
  __device__ __forceinline__ void issue(char* tile, int wave, int lane, int j0, int row_bytes) const {
    if (j0 < seen.gap1 && j0 + L::kTileRows > seen.gap0)
      L::issue(tile, wave, lane, buffer_of(p + j0 * st, (seen.last - j0) * st + row_bytes), [&](int i) {
        const int r = L::row(i, wave, lane), key = j0 + r;
        return key >= seen.gap0 && key < seen.gap1 ? kReach : (uint32_t)r * (uint32_t)st;
      });
    else if (near)
      L::issue(tile, wave, lane, all, (uint32_t)j0 * (uint32_t)st, (uint32_t)st);
    else
      L::issue(tile, wave, lane, buffer_of(p + j0 * st, (seen.last - j0) * st + row_bytes), 0, (uint32_t)st);
  }
};

template <typename T>
struct Frag;
template <>
struct Frag<uint16_t> {
  bf16x8 v;
};
template <>
struct Frag<float> {
  float v[8];
};

__device__ __forceinline__ f32x16 mma(const Frag<uint16_t>& a, const Frag<uint16_t>& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
  return c;
}

// Registers 8t .. 8t + 7 of a result as an operand (bf16: rounded).
__device__ __forceinline__ void as_operand(const f32x16& x, int t, Frag<uint16_t>& f) {
  const u32x4 w = {pack_bf16x2(x[8 * t], x[8 * t + 1]), pack_bf16x2(x[8 * t + 2], x[8 * t + 3]),
                   pack_bf16x2(x[8 * t + 4], x[8 * t + 5]), pack_bf16x2(x[8 * t + 6], x[8 * t + 7])};
  f.v = __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ void as_operand(const f32x16& x, int t, Frag<float>& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = x[8 * t + e];
}

// Features 16kk + 8h + 0..7 of a row in memory.
__device__ __forceinline__ void load_operand(const char* row, int kk, int h, Frag<uint16_t>& f) {
  f.v = *reinterpret_cast<const bf16x8*>(row + kk * 32 + h * 16);
}
__device__ __forceinline__ void load_operand(const char* row, int kk, int h, Frag<float>& f) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(row + kk * 64 + h * 32);
  const f32x4 b = *reinterpret_cast<const f32x4*>(row + kk * 64 + h * 32 + 16);
#pragma unroll
  for (int e = 0; e < 4; ++e) f.v[e] = a[e], f.v[4 + e] = b[e];
}
__device__ __forceinline__ float dot(const Frag<uint16_t>& a, const Frag<uint16_t>& b, float s) {
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf((float)a.v[e], (float)b.v[e], s);
  return s;
}
__device__ __forceinline__ float dot(const Frag<float>& a, const Frag<float>& b, float s) {
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(a.v[e], b.v[e], s);
  return s;
}

// Four consecutive features of a result row.
__device__ __forceinline__ void store4(uint16_t* p, float a, float b, float c, float d) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(a, b), pack_bf16x2(c, d)};
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<f32x4*>(p) = f32x4{a, b, c, d};
}

// A tile of rows of HD features in LDS: blocks of 1 KB, which one load of a wave
// fills (16 bytes a lane, in the lanes' order), 64 bytes apart.  Row r lies in
// block r % 4 of each four, (r / 4) % kBlockRows rows down, its 16-byte pieces
// XORed in their low two bits with (r / 4) % 4.  The LDS is 256 bytes wide:
// the 16 rows whose same piece one step of a row read takes, and the four rows
// x 32 bytes of a group of a transposed read, then lie side by side in it.  All
// of a lane's reads are at constant offsets from four addresses (Reader).
template <typename T, int HD>
struct Tile {
  static constexpr int kRow = HD * (int)sizeof(T);  // bytes of a row
  static constexpr int kPieces = kRow / 16;
  static constexpr int kBlockRows = 64 / kPieces;
  static constexpr int kBlock = 1024 + 64;
  template <int ROWS>
  static constexpr int bytes() {
    return ROWS / kBlockRows * kBlock;
  }
  // Where row r, a multiple of 4, starts.
  static __host__ __device__ constexpr int row_at(int r) {
    return (r >> 2) / kBlockRows * 4 * kBlock + (r >> 2) % kBlockRows * kRow;
  }

  // Loads of ROWS rows straight to LDS, the blocks shared out over WAVES waves.
  template <int ROWS, int WAVES>
  struct Loads {
    static constexpr int kTileRows = ROWS;
    static constexpr int kLoads = ROWS / kBlockRows / WAVES;
    static_assert(ROWS % (kBlockRows * WAVES) == 0 && (WAVES == 1 || WAVES == 4), "whole blocks a wave");
    // Row of the tile that a lane loads from at load i, and its piece there.
    static __device__ __forceinline__ int row(int i, int wave, int lane) {
      const int blk = wave + WAVES * i;
      return (blk & 3) + 4 * (lane / kPieces + kBlockRows * (blk >> 2));
    }
    static __device__ __forceinline__ int piece(int i, int wave, int lane) {
      return (lane % kPieces) ^ ((row(i, wave, lane) >> 2) & 3);
    }
    // offset(i): where the lane's row of load i lies in src; what lies past its
    // end arrives as zeros.
    template <typename F>
    static __device__ __forceinline__ void issue(char* tile, int wave, int lane,
                                                 __amdgpu_buffer_rsrc_t src, F&& offset) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void*)(tile + (wave + WAVES * i) * kBlock), 16,
                                                 (int)(offset(i) + piece(i, wave, lane) * 16), 0, 0, 0);
    }
    // Rows st bytes apart, the first at `at`.
    static __device__ __forceinline__ void issue(char* tile, int wave, int lane,
                                                 __amdgpu_buffer_rsrc_t src, uint32_t at, uint32_t st) {
      const uint32_t first = (uint32_t)row(0, wave, lane) * st;
      issue(tile, wave, lane, src, [&](int i) {
        // The rows of two loads are the same number apart in every lane.
        return first + (at + (uint32_t)(row(i, 0, 0) - row(0, 0, 0)) * st);
      });
    }
  };

  // A lane's addresses in a tile.
  struct Reader {
    int even, odd;  // of row l % 32: pieces 2kk + h of even and odd kk (fp32: pieces 2h and 2h + 1)
    int lo, hi;     // transposed: rows 4h .., 8 + 4h ..
    __device__ __forceinline__ explicit Reader(int lane) {
      const int r = lane & 31, h = lane >> 5, x = (r >> 2) & 3;
      const int at = (r & 3) * kBlock + row_at(r & ~3);
      if constexpr (sizeof(T) == 2) {
        even = at + ((h ^ x) << 4);
        odd = at + (((h + 2) ^ x) << 4);
        const int c = ((lane & 16) >> 3) | ((lane & 2) >> 1), sub = (lane & 1) * 8;
        const int from = ((lane & 15) >> 2) * kBlock + h * kRow + sub;
        lo = from + ((c ^ h) << 4);
        hi = from + row_at(8) + ((c ^ h ^ 2) << 4);
      } else {
        even = at + (((2 * h) ^ x) << 4);
        odd = at + (((2 * h + 1) ^ x) << 4);
        const int c = (r >> 2) & 3, from = h * kRow + (r >> 4) * 64 + (lane & 3) * 4;
        lo = from + ((c ^ h) << 4);
        hi = from + row_at(8) + ((c ^ h ^ 2) << 4);
      }
    }

    // Row r0 + l % 32 (r0 a multiple of 32), features 16kk + 8h + 0..7.
    __device__ __forceinline__ void operand(const char* tile, int r0, int kk, Frag<T>& f) const {
      if constexpr (sizeof(T) == 2) {
        f.v = *reinterpret_cast<const bf16x8*>(tile + ((kk & 1) ? odd : even) + (kk >> 1) * 64 + row_at(r0));
      } else {
        const f32x4 a = *reinterpret_cast<const f32x4*>(tile + even + kk * 64 + row_at(r0));
        const f32x4 b = *reinterpret_cast<const f32x4*>(tile + odd + kk * 64 + row_at(r0));
#pragma unroll
        for (int e = 0; e < 4; ++e) f.v[e] = a[e], f.v[4 + e] = b[e];
      }
    }

    // Feature 32n + l % 32 of rows r0 + 4h + 0..3 and r0 + 8 + 4h + 0..3 (r0 a
    // multiple of 16).  bf16: the transposing LDS read; in each group of 16
    // lanes, lane i addresses columns 4 (i % 4) .. + 3 of row i / 4 and receives
    // column i of the four rows.
    __device__ __forceinline__ void transposed(const char* tile, int r0, int n, Frag<T>& f) const {
      if constexpr (sizeof(T) == 2) {
        typedef short i16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
        const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(tile + lo + row_at(r0) + n * 64)));
        const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(tile + hi + row_at(r0) + n * 64)));
        const u32x4 w = {a[0], a[1], b[0], b[1]};
        f.v = __builtin_bit_cast(bf16x8, w);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f.v[e] = *reinterpret_cast<const float*>(tile + lo + row_at(r0) + n * 128 + e * kBlock);
          f.v[4 + e] = *reinterpret_cast<const float*>(tile + hi + row_at(r0) + n * 128 + e * kBlock);
        }
      }
    }
  };
};

// Waits for all of this wave's loads: ahead of a loop over tiles, so that inside
// it nothing waits for the operands loaded before it, and with them for tiles.
__device__ __forceinline__ void settle() {
  asm volatile("" ::: "memory");
  wait_vm_lds<0>();
  asm volatile("" ::: "memory");
}

// Waits until at most N of this wave's loads are in flight and its LDS reads
// are done, then for the workgroup's waves.
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("" ::: "memory");
  wait_vm_lds<N>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace elasto
