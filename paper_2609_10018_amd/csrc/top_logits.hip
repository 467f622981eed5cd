// The largest logits of each row, largest first, the lower index first among
// equal ones: what a teacher's answer is reduced to for distillation.
//
// Values and indices are ordered together: key = (order of the value, ~index),
// so keys differ and ties need no care.  One workgroup a row:
//  1. every thread finds the largest key of its share.  Each of the W waves
//     sorts its 64 and gives the ceil(top / W)-th: at least `top` keys of the
//     row are no smaller than the least of those;
//  2. the keys from that bound on, hardly more than `top` of them, are
//     collected in LDS.  Where they are too many to hold (the largest ones lie
//     in few threads' shares), the top-th of those held is the next bound: each
//     round drops all but `top` of what it held, so the rounds end;
//  3. the collected keys are sorted, up to 512 of them by one wave in registers,
//     and the first `top` written.
// The order of collecting does not matter to the result.
//
// A thread keeps the largest value of each of its runs of eight, so the second
// walk reads only runs that hold a key from the bound on again: one pass over the
// logits.  1024 x 100003 bf16, top 64: 55-59 us by the card, 3.5-3.7 TB/s.  Kernels that
// only read reach 5.1 on as many bytes; here two rows on a CU read, sort, collect and
// sort one after the other, and their waves wait 70% of the time.  64 x 1000 fp32, top
// 16: 6 us, a launch and the chain of one wave; 4096 x 1000 12 us (1.4 TB/s): 16 KB of
// LDS a row leave a SIMD two or three waves.
#include <algorithm>
#include <type_traits>

#include "layout.h"
#include "logits.h"

namespace elasto {
namespace {

constexpr int kHold = 2048;  // keys held in LDS

// Order of floats as unsigned integers, -0 as 0, NaN above all.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  const uint32_t o = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
  return x == x ? o : 0xffffffffu;
}
__device__ __forceinline__ uint64_t key_of(uint32_t order, int i) {
  return (uint64_t)order << 32 | (uint32_t)~i;
}

// v of lane ^ STEP, by lane moves rather than through LDS: half the time of a sort
// is the wait for them.
template <int STEP>
__device__ __forceinline__ uint32_t moved(uint32_t v, int lane) {
  auto dpp = [](uint32_t x, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true);
  };
  if constexpr (STEP == 1) return dpp(v, std::integral_constant<int, 0xB1>());
  else if constexpr (STEP == 2) return dpp(v, std::integral_constant<int, 0x4E>());
  else if constexpr (STEP == 4)  // ^ 3, then ^ 7
    return dpp(dpp(v, std::integral_constant<int, 0x1B>()), std::integral_constant<int, 0x141>());
  else if constexpr (STEP == 8) return dpp(v, std::integral_constant<int, 0x128>());
  else if constexpr (STEP == 16) {
    const auto x = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return lane & 16 ? x[0] : x[1];
  } else {
    const auto x = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return lane & 32 ? x[0] : x[1];
  }
}

// One step of a bitonic sort of the wave's keys: key 64 r + lane in k[r].
template <int K, int SIZE, int STEP>
__device__ __forceinline__ void sort_step(uint64_t (&k)[K], int lane) {
  if constexpr (STEP >= 64) {
#pragma unroll
    for (int r = 0; r < K; ++r) {
      constexpr int D = STEP / 64;
      if (r & D) continue;
      const bool down = (64 * r & SIZE) == 0;
      const uint64_t a = k[r], b = k[r | D];
      if ((a < b) == down) k[r] = b, k[r | D] = a;
    }
  } else {
#pragma unroll
    for (int r = 0; r < K; ++r) {
      const uint64_t o = (uint64_t)moved<STEP>((uint32_t)(k[r] >> 32), lane) << 32 |
                         moved<STEP>((uint32_t)k[r], lane);
      const bool down = ((64 * r + lane) & SIZE) == 0, low = (lane & STEP) == 0;
      k[r] = (low == down) == (k[r] > o) ? k[r] : o;
    }
  }
  if constexpr (STEP > 1) sort_step<K, SIZE, STEP / 2>(k, lane);
}
// The wave's 64 K keys, largest first.
template <int K, int SIZE = 2>
__device__ __forceinline__ void wave_sort(uint64_t (&k)[K], int lane) {
  sort_step<K, SIZE, SIZE / 2>(k, lane);
  if constexpr (SIZE < 64 * K) wave_sort<K, SIZE * 2>(k, lane);
}

// The largest `top` of n <= 64 K keys in LDS, by one wave.
template <int K, typename F>
__device__ __forceinline__ void write_sorted(const uint64_t* keys, int n, int top, int lane, F&& write) {
  uint64_t k[K];
#pragma unroll
  for (int r = 0; r < K; ++r) k[r] = 64 * r + lane < n ? keys[64 * r + lane] : 0;
  wave_sort(k, lane);
#pragma unroll
  for (int r = 0; r < K; ++r)
    if (64 * r + lane < top) write(64 * r + lane, k[r]);
}

// keys[0, n) largest first; n a power of two.
template <int N>
__device__ __forceinline__ void block_sort(uint64_t* keys, int n, int tid) {
  for (int size = 2; size <= n; size *= 2)
    for (int step = size / 2; step >= 1; step /= 2) {
      for (int t = tid; t < n / 2; t += N) {
        const int i = 2 * t - (t & (step - 1)), j = i + step;
        const uint64_t a = keys[i], b = keys[j];
        if ((a < b) == ((i & size) == 0)) {
          keys[i] = b;
          keys[j] = a;
        }
      }
      __syncthreads();
    }
}

// The largest of eight values, NaN if there is one.
__device__ __forceinline__ float top8(const float* v) {
  float m = v[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) m = __builtin_elementwise_maximum(m, v[e]);
  return m;
}

// RUNS: runs of eight a thread, whose largest values it keeps for the second
// walk; 0: more, which are all read again.
template <typename T, int N, int RUNS>
__global__ __launch_bounds__(N, (N == 1024 ? 8 : 2)) void top_logits_kernel(
    const T* logits, int64_t ld, int C, int top, float* values, int32_t* indices) {
  __shared__ uint64_t held[kHold];
  __shared__ uint64_t bounds[N / 64];
  __shared__ int count;
  const int tid = threadIdx.x, lane = tid & 63;
  const T* z = logits + (int64_t)blockIdx.x * ld;
  RowSpan<T> span(z, C);
  // Few classes: one by one, so that all threads have some and the bound is close
  // (422 bf16, top 54: with runs for 52 lanes alone every key is collected, 25 us).
  if (C <= 8 * N) span.head = span.singles = C, span.runs = 0;
  // f(index, value) over the thread's single values, eight loads in flight.
  auto each_single = [&](auto&& f) __attribute__((always_inline)) {
    for (int i0 = tid; i0 < span.singles; i0 += 8 * N) {
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        v[u] = i0 + u * N < span.singles ? load1(z + span.single(i0 + u * N)) : 0.0f;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u * N < span.singles) f(span.single(i0 + u * N), v[u]);
    }
  };

  // The thread's largest key, or rather one that is no larger: of a run, its
  // largest value at its last index.
  uint64_t best = 0;  // less than any key
  uint32_t most[RUNS > 0 ? RUNS : 1];  // order of each run's largest value
  uint32_t bo = 0;
  int bi = 0;
  auto take = [&](uint32_t o, int last) {
    bi = o > bo ? last : bi;
    bo = o > bo ? o : bo;
  };
  if constexpr (RUNS > 0) {
    constexpr int kBatch = RUNS < 4 ? RUNS : 4;
#pragma unroll
    for (int r0 = 0; r0 < RUNS; r0 += kBatch) {
      float v[kBatch][8];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int c = tid + (r0 + u) * N;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[u][e] = 0.0f;
        if (c < span.runs) load8(z + span.run(c), v[u]);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int c = tid + (r0 + u) * N;
        most[r0 + u] = c < span.runs ? order_of(top8(v[u])) : 0;
        take(most[r0 + u], span.run(c) + 7);
      }
      asm volatile("" ::: "memory");  // four loads in flight are enough, and their registers
    }
    each_single([&](int i, float v) {
      const uint64_t k = key_of(order_of(v), i);
      best = k > best ? k : best;
    });
  } else {
    walk_row<N>(z, span, tid, [&](int i, const float* v) { take(order_of(top8(v)), i + 7); },
                [&](int i, float v) {
                  const uint64_t k = key_of(order_of(v), i);
                  best = k > best ? k : best;
                });
  }
  if (bo) {
    const uint64_t k = key_of(bo, bi);
    best = k > best ? k : best;
  }
  constexpr int W = N / 64;
  uint64_t sorted[1] = {best};
  wave_sort(sorted, lane);
  if (lane == (top + W - 1) / W - 1) bounds[tid >> 6] = sorted[0];
  __syncthreads();
  uint64_t bound = bounds[0];
#pragma unroll
  for (int w = 1; w < W; ++w) bound = bounds[w] < bound ? bounds[w] : bound;

  auto write = [&](int t, uint64_t k) {
    const int i = (int)~(uint32_t)k;
    values[(int64_t)blockIdx.x * top + t] = load1(z + i);
    indices[(int64_t)blockIdx.x * top + t] = i;
  };
  while (true) {
    if (tid == 0) count = 0;
    __syncthreads();
    auto keep = [&](uint64_t k) {
      const int at = atomicAdd(&count, 1);
      if (at < kHold) held[at] = k;
    };
    const uint32_t bh = (uint32_t)(bound >> 32);
    auto keep8 = [&](int i, const float* v) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint64_t k = key_of(order_of(v[e]), i + e);
        if (k >= bound) keep(k);
      }
    };
    auto keep1 = [&](int i, float v) {
      const uint64_t k = key_of(order_of(v), i);
      if (k >= bound) keep(k);
    };
    if constexpr (RUNS > 0) {
      unsigned hits = 0;
#pragma unroll
      for (int r = 0; r < RUNS; ++r) hits |= most[r] >= bh && most[r] ? 1u << r : 0u;
      for (; hits; hits &= hits - 1) {
        const int i = span.run(tid + (__ffs((int)hits) - 1) * N);
        float v[8];
        load8(z + i, v);
        keep8(i, v);
      }
      each_single(keep1);
    } else {
      walk_row<N>(z, span, tid,
                  [&](int i, const float* v) {
                    if (order_of(top8(v)) >= bh) keep8(i, v);
                  },
                  keep1);
    }
    __syncthreads();
    const int n = count;
    // The rule: few more than top.  (512 keys take 16 registers more than 1024
    // threads, two rows to a CU, have.)
    constexpr int kInWave = N < 1024 ? 512 : 256;
    if (n <= kInWave) {
      if (tid >= 64) return;
      if (n <= 64) write_sorted<1>(held, n, top, lane, write);
      else if (n <= 128) write_sorted<2>(held, n, top, lane, write);
      else if (N == 1024 || n <= 256) write_sorted<4>(held, n, top, lane, write);
      else write_sorted<8>(held, n, top, lane, write);
      return;
    }
    const int got = n < kHold ? n : kHold;
    int p2 = 1;
    while (p2 < got) p2 *= 2;
    for (int t = got + tid; t < p2; t += N) held[t] = 0;
    __syncthreads();
    block_sort<N>(held, p2, tid);
    if (n <= kHold) break;
    bound = held[top - 1];
    __syncthreads();
  }
  for (int t = tid; t < top; t += N) write(t, held[t]);
}

template <typename T, int N, int RUNS>
void start(const T* z, int64_t ld, int64_t rows, int C, int top, float* values, int32_t* indices,
           hipStream_t s) {
  for (int64_t r = 0; r < rows; r += kLaunchRows)
    hipLaunchKernelGGL((top_logits_kernel<T, N, RUNS>), dim3((unsigned)std::min(rows - r, kLaunchRows)),
                       dim3(N), 0, s, z + r * ld, ld, C, top, values + r * top, indices + r * top);
}

template <typename T>
hipError_t launch(const void* logits, int64_t ld, int64_t rows, int C, int top, float* values,
                  int32_t* indices, hipStream_t s) {
  const T* z = static_cast<const T*>(logits);
  // The bound is each wave's ceil(top / W)-th of 64, and loose where that is one of
  // its last: most keys are then collected and sorted.  One wave a row, four: 4096
  // x 1000, top 16 11 and 18 us, top 56 18 and 20, top 64 75 and 20.  Four waves,
  // eight: top 128 25 and 46, top 250 84 and 56.
  if (C <= 2048 && top <= 56)
    start<T, 64, 4>(z, ld, rows, C, top, values, indices, s);
  else if (C < 8192 && top <= 224)
    start<T, 256, 4>(z, ld, rows, C, top, values, indices, s);
  else if (C < 8192)
    start<T, 512, 2>(z, ld, rows, C, top, values, indices, s);
  else if (C <= 65536)
    start<T, 1024, 8>(z, ld, rows, C, top, values, indices, s);
  else if (C <= 131072)
    start<T, 1024, 16>(z, ld, rows, C, top, values, indices, s);
  else
    start<T, 1024, 0>(z, ld, rows, C, top, values, indices, s);
  return hipGetLastError();
}

}  // namespace
}  // namespace elasto

using namespace elasto;

extern "C" elasto_status_t elasto_op_top_logits(int32_t dtype, const void* logits, int64_t ld,
                                                int64_t rows, int32_t classes, int32_t top,
                                                float* values, int32_t* indices, void* hip_stream) {
  if (dtype != ELASTO_BF16 && dtype != ELASTO_FP32) return fail(ELASTO_ERR_INVALID_ARG, "bad dtype %d", dtype);
  if (rows < 0 || rows > 0x7fffffff || classes < 1 || classes > (1 << 30) || ld < classes)
    return fail(ELASTO_ERR_INVALID_ARG, "top_logits: bad rows, classes or row stride");
  if (top < 1 || top > 256 || top > classes)
    return fail(ELASTO_ERR_INVALID_ARG, "top_logits: top %d outside [1, min(256, classes)]", top);
  if (rows == 0) return ELASTO_OK;
  if (!logits || !values || !indices) return fail(ELASTO_ERR_INVALID_ARG, "NULL pointer");
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == ELASTO_BF16 ? 2 : 4) ||
      reinterpret_cast<uintptr_t>(values) % 4 || reinterpret_cast<uintptr_t>(indices) % 4)
    return fail(ELASTO_ERR_INVALID_ARG, "top_logits: misaligned pointer");
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = dtype == ELASTO_BF16
                           ? launch<uint16_t>(logits, ld, rows, classes, top, values, indices, s)
                           : launch<float>(logits, ld, rows, classes, top, values, indices, s);
  if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "top_logits: %s", hipGetErrorString(e));
  return ELASTO_OK;
}
