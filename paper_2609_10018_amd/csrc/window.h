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

// A tile of rows of HD features in LDS, in the order of memory but for the
// 16-byte pieces of a row, which are XORed with the row number: the 32 rows (or
// 4 x 4 pieces) that one read takes then lie in different banks.
template <typename T, int HD>
struct Tile {
  static constexpr int kRow = HD * (int)sizeof(T);  // bytes of a row
  static constexpr int kPieces = kRow / 16;
  static constexpr int kXor = (kPieces < 16 ? kPieces : 16) - 1;
  static constexpr int kBlockRows = 64 / kPieces;  // rows of the 1 KB that a wave loads at once

  static __device__ __forceinline__ int at(int r, int piece) {
    return r * kRow + ((piece ^ (r & kXor)) << 4);
  }

  // Loads of ROWS rows straight to LDS, the blocks of 1 KB shared out over
  // WAVES waves: kLoads a wave, each lane 16 bytes at a constant offset from
  // the tile's first row.
  template <int ROWS, int WAVES>
  struct Loads {
    static constexpr int kLoads = ROWS / kBlockRows / WAVES;
    static_assert(ROWS % (kBlockRows * WAVES) == 0, "every wave loads the same number of blocks");
    uint32_t off[kLoads];

    // offset(r): where row r lies after the first.
    template <typename F>
    __device__ __forceinline__ void set(int wave, int lane, F&& offset) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = (wave + WAVES * i) * kBlockRows + lane / kPieces;
        off[i] = offset(r) + (((lane % kPieces) ^ (r & kXor)) << 4);
      }
    }
    // From `bytes` bytes at base; what lies past them arrives as zeros.
    __device__ __forceinline__ void issue(char* tile, int wave, const char* base, int64_t bytes) const {
      const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<char*>(base), (short)0, (int)(uint32_t)(bytes < 0xffffffffll ? bytes : 0xffffffffll),
          kRsrcWord3);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void*)(tile + (wave + WAVES * i) * 1024), 16,
                                                 (int)off[i], 0, 0, 0);
    }
  };

  // Row r, features 16kk + 8h + 0..7.
  static __device__ __forceinline__ void operand(const char* tile, int r, int kk, int h, Frag<T>& f) {
    if constexpr (sizeof(T) == 2) {
      f.v = *reinterpret_cast<const bf16x8*>(tile + at(r, 2 * kk + h));
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(tile + at(r, 4 * kk + 2 * h));
      const f32x4 b = *reinterpret_cast<const f32x4*>(tile + at(r, 4 * kk + 2 * h + 1));
#pragma unroll
      for (int e = 0; e < 4; ++e) f.v[e] = a[e], f.v[4 + e] = b[e];
    }
  }

  // Feature 32n + l % 32 of rows r0 + 4h + 0..3 and r0 + 8 + 4h + 0..3.
  // bf16: the transposing LDS read.  In each group of 16 lanes, lane i addresses
  // columns 4 (i % 4) .. + 3 of row i / 4 and receives column i of the four rows.
  static __device__ __forceinline__ void transposed(const char* tile, int r0, int n, int lane,
                                                    Frag<T>& f) {
    const int h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      typedef short i16x4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
      const int r = r0 + 4 * h + ((lane & 15) >> 2);
      const int col = n * 32 + (lane & 16) + 4 * (lane & 3);
      const int sub = (col & 4) * 2;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(tile + at(r, col >> 3) + sub)));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(tile + at(r + 8, col >> 3) + sub)));
      const u32x4 w = {lo[0], lo[1], hi[0], hi[1]};
      f.v = __builtin_bit_cast(bf16x8, w);
    } else {
      const int col = n * 32 + (lane & 31);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = r0 + 4 * h + (e & 3) + (e & 4) * 2;
        f.v[e] = *reinterpret_cast<const float*>(tile + at(r, col >> 2) + (col & 3) * 4);
      }
    }
  }
};

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
