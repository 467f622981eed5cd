// Rows of logits read by a whole workgroup in aligned runs of eight, whatever
// the row's first address is (an odd number of classes moves it row by row).
#pragma once

#include "common.h"

namespace elasto {

// Rows of one launch, a workgroup each: a launch holds fewer than 2^32 threads.
constexpr int64_t kLaunchRows = 1 << 21;

__device__ __forceinline__ void load8(const uint16_t* p, float* v) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float* v) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
__device__ __forceinline__ float load1(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float load1(const float* p) { return *p; }

// Past the caches: what is written is not read again here, and the row that is
// read twice keeps its place in them.
__device__ __forceinline__ void store8(uint16_t* p, const float* v) {
  const u32x4 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                   pack_bf16x2(v[6], v[7])};
  __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4*>(p));
  __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, reinterpret_cast<f32x4*>(p + 4));
}
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// Row of C values: `head` single ones up to a 16-byte boundary, `runs` of
// eight, then the rest; the single ones are numbered 0 .. singles - 1.
template <typename T>
struct RowSpan {
  int head, runs, singles;
  __device__ __forceinline__ RowSpan(const T* z, int C) {
    const int off = (int)(reinterpret_cast<uintptr_t>(z) & 15) / (int)sizeof(T);
    head = min(C, off ? 16 / (int)sizeof(T) - off : 0);
    runs = (C - head) >> 3;
    singles = C - (runs << 3);
  }
  __device__ __forceinline__ int single(int i) const { return i < head ? i : (runs << 3) + i; }
  __device__ __forceinline__ int run(int c) const { return head + (c << 3); }
};

// each(first index, eight values) over the runs of thread tid of N, four loads
// in flight; then one(index, value) over its single values.
template <int N, typename T, typename R, typename S>
__device__ __forceinline__ void walk_row(const T* z, const RowSpan<T>& s, int tid, R&& each, S&& one) {
  int c = tid;
  for (; c + 3 * N < s.runs; c += 4 * N) {
    float v[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u) load8(z + s.run(c + u * N), v[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u) each(s.run(c + u * N), v[u]);
  }
  for (; c < s.runs; c += N) {
    float v[8];
    load8(z + s.run(c), v);
    each(s.run(c), v);
  }
  for (int i = tid; i < s.singles; i += N) one(s.single(i), load1(z + s.single(i)));
}

}  // namespace elasto
