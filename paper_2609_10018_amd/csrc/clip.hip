// The global L2 norm of many tensors, and their clipping by it:
//   norm = sqrt(sum over all elements of g^2),  out = g min(1, max_norm / norm).
//
// The tensors' addresses and sizes travel in the kernels' arguments, kTensors a launch,
// so a call keeps nothing and a captured graph repeats it.  A launch cuts its tensors into
// chunks of 16 KB, which its workgroups take in turn; the squares are summed in 64 bits (no
// square overflows or vanishes, and the sum of 10^9 of them keeps 32 bits), one partial sum
// a workgroup.  The scaling launches add the partial sums up once more, each workgroup for
// itself and in the same order, which costs less than a launch between the two.  Their
// chunks run from the last to the first: what the norm read last is still in the cache
// behind L2.
//
// Bound by memory: the gradients read (twice where they do not fit the cache) and written.  290 tensors of 2.5
// GB 1375 us (5.6 TB/s over the three passes); 146 of 75 MB 44 in the kernels (3.4 over two), 63 the call, whose
// host side is longer.
#include <math.h>

#include <algorithm>
#include <vector>

#include "common.h"
#include "heads.h"

namespace elasto {
namespace {

constexpr int kTensors = 180;          // of a launch: its arguments stay below 4 KB
constexpr int kChunk = 16384;          // bytes of a chunk
constexpr int kMaxBlocks = 2048;       // workgroups of a call's norm, one partial sum each
constexpr int kThreads = 256;

// The tensors of a launch: 14 bytes each, and 8 for a result.
struct Table {
  uintptr_t at[kTensors];        // address; bit 0: bf16
  uint32_t first[kTensors + 1];  // first chunk of each tensor
  uint16_t last[kTensors];       // elements of the last chunk
  int n;
};
struct Results {
  char* out[kTensors];
};

// Elements of a chunk by bytes of an element.
template <typename T>
constexpr int kPer = kChunk / (int)sizeof(T);

__device__ __forceinline__ void unpack(const u32x4& w, float* v, uint16_t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const u32x4& w, float* v, float) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ float one(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float one(const float* p) { return *p; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

// The tensor that holds chunk c: first[i] <= c < first[i + 1].
template <typename Tab>
__device__ __forceinline__ int find(const Tab& t, uint32_t c) {
  int lo = 0, hi = t.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    (t.first[mid] <= c ? lo : hi) = mid;
  }
  return lo;
}

struct Chunk {
  const char* p;
  int64_t offset;  // bytes, in its tensor
  int tensor, n;
  bool bf16;
  __device__ __forceinline__ Chunk(const Table& t, uint32_t c) {
    tensor = find(t, c);
    offset = (int64_t)(c - t.first[tensor]) * kChunk;
    bf16 = t.at[tensor] & 1;
    p = reinterpret_cast<const char*>(t.at[tensor] & ~(uintptr_t)1) + offset;
    n = c + 1 == t.first[tensor + 1] ? t.last[tensor] : bf16 ? kPer<uint16_t> : kPer<float>;
  }
};

// The n elements of a chunk at p: `head` single ones up to a 16-byte boundary, whole pieces of 16
// bytes, the rest single again.
template <typename T>
struct Span {
  int head, pieces, n;
  __device__ __forceinline__ Span(const T* p, int n_) : n(n_) {
    constexpr int E = 16 / (int)sizeof(T);
    const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15) / (int)sizeof(T);
    head = min(n, off ? E - off : 0);
    pieces = (n - head) / E;
  }
  // Single elements: before the first piece and behind the last.
  __device__ __forceinline__ int singles() const { return n - pieces * (16 / (int)sizeof(T)); }
  __device__ __forceinline__ int single(int i) const {
    return i < head ? i : i + pieces * (16 / (int)sizeof(T));
  }
};

template <typename T>
__device__ __forceinline__ double squares(const T* p, int n) {
  constexpr int E = 16 / (int)sizeof(T);
  const Span<T> s(p, n);
  const u32x4* q = reinterpret_cast<const u32x4*>(p + s.head);
  double sum = 0.0;
  const int tid = threadIdx.x;
  u32x4 w[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    w[u] = u32x4{0, 0, 0, 0};
    if (tid + u * kThreads < s.pieces) w[u] = q[tid + u * kThreads];
  }
  if (tid < s.singles()) {
    const double v = one(p + s.single(tid));
    sum = v * v;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    float v[E];
    unpack(w[u], v, T());
#pragma unroll
    for (int e = 0; e < E; ++e) sum = fma((double)v[e], (double)v[e], sum);
  }
  return sum;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = red[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) s += red[i];
  return s;
}

__global__ __launch_bounds__(kThreads) void norm_kernel(Table t, double* part) {
  __shared__ double red[kThreads / 64];
  const uint32_t chunks = t.first[t.n];
  double sum = 0.0;
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Chunk k(t, c);
    sum += k.bf16 ? squares(reinterpret_cast<const uint16_t*>(k.p), k.n) : squares(reinterpret_cast<const float*>(k.p), k.n);
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__device__ __forceinline__ double total_of(const double* part, int parts, double* red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
  return block_sum(s, red);
}

// What the norm makes of the gradients: g becomes g a b.  A norm that is no finite number scales nothing:
// the factor that is told is 0, for the caller's step to leave out.  A factor below fp32's normal range
// (gradients of 1e30 clipped to 1e-20, say) is taken in two, since the results lie well inside the range,
// and is told as no less than the smallest number above 0.
struct Scale {
  float norm, factor, a, b;
  __device__ __forceinline__ Scale(double sum, float max_norm) : factor(1.0f), a(1.0f), b(1.0f) {
    const double root = sqrt(sum);
    norm = (float)root;
    if (!(norm < INFINITY)) {
      factor = 0.0f;
    } else if (norm > max_norm) {
      const double f = (double)max_norm / root;
      const bool far = f < 0x1p-126;
      a = (float)(far ? f * 0x1p125 : f);
      b = far ? 0x1p-125f : 1.0f;
      factor = fmaxf((float)f, 0x1p-149f);
    }
  }
  __device__ __forceinline__ bool nothing() const { return a == 1.0f && b == 1.0f; }
};

__global__ __launch_bounds__(kThreads) void norm_out_kernel(const double* part, int parts, float* norm) {
  __shared__ double red[kThreads / 64];
  const double s = total_of(part, parts, red);
  if (threadIdx.x == 0) norm[0] = (float)sqrt(s);
}

// PAST: past the caches, where the gradients do not fit them.
template <bool PAST, typename T>
__device__ __forceinline__ void scale(const T* p, T* out, int n, float a, float b) {
  constexpr int E = 16 / (int)sizeof(T);
  const int tid = threadIdx.x;
  const Span<T> s(p, n);
  const bool wide = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  const u32x4* q = reinterpret_cast<const u32x4*>(p + s.head);
  u32x4 w[4];
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (tid + u * kThreads < s.pieces) w[u] = PAST ? __builtin_nontemporal_load(q + tid + u * kThreads) : q[tid + u * kThreads];
  float head = 0.0f;
  if (tid < s.singles()) head = one(p + s.single(tid));
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int i = tid + u * kThreads;
    if (i >= s.pieces) break;
    float v[E];
    unpack(w[u], v, T());
    T* o = out + s.head + i * E;
    if (wide) {
      u32x4 r;
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = pack_bf16x2(v[2 * e] * a * b, v[2 * e + 1] * a * b);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = __float_as_uint(v[e] * a * b);
      }
      if constexpr (PAST)
        __builtin_nontemporal_store(r, reinterpret_cast<u32x4*>(o));
      else
        *reinterpret_cast<u32x4*>(o) = r;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) put(o + e, v[e] * a * b);
    }
  }
  if (tid < s.singles()) put(out + s.single(tid), head * a * b);
}

// stats: where the call's first launch leaves norm and factor.  in_place: where nothing is scaled everything
// is left as it is.
template <bool PAST>
__global__ __launch_bounds__(kThreads) void clip_kernel(Table t, Results r, const double* part, int parts,
                                                        float max_norm, float* stats, bool in_place) {
  __shared__ double red[kThreads / 64];
  const Scale by(total_of(part, parts, red), max_norm);
  if (stats && blockIdx.x == 0 && threadIdx.x == 0) {
    stats[0] = by.norm;
    stats[1] = by.factor;
  }
  if (in_place && by.nothing()) return;
  const uint32_t chunks = t.first[t.n];
  for (uint32_t b = blockIdx.x; b < chunks; b += gridDim.x) {
    const uint32_t c = chunks - 1 - b;
    const Chunk k(t, c);
    char* out = r.out[k.tensor] + k.offset;
    if (k.bf16)
      scale<PAST>(reinterpret_cast<const uint16_t*>(k.p), reinterpret_cast<uint16_t*>(out), k.n, by.a, by.b);
    else
      scale<PAST>(reinterpret_cast<const float*>(k.p), reinterpret_cast<float*>(out), k.n, by.a, by.b);
  }
}

// ---------------------------------------------------------------- host

constexpr int64_t kMaxCount = (int64_t)1 << 40;
static_assert(sizeof(Table) + sizeof(Results) + 64 <= 4096, "kernel arguments");

int64_t chunks_of(const elasto_grad_t& g) {
  const int64_t bytes = g.count * (g.dtype == ELASTO_BF16 ? 2 : 4);
  return (bytes + kChunk - 1) / kChunk;
}

bool check_list(const char* name, const elasto_grad_t* g, int32_t n) {
  if (n < 0 || n > (1 << 20) || (n > 0 && !g))
    return fail(ELASTO_ERR_INVALID_ARG, "clip: bad list of %s", name), false;
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (g[i].dtype != ELASTO_BF16 && g[i].dtype != ELASTO_FP32)
      return fail(ELASTO_ERR_INVALID_ARG, "clip: %s %d: bad dtype %d", name, i, g[i].dtype), false;
    if (g[i].count < 0 || (total += std::min(g[i].count, kMaxCount)) >= kMaxCount)
      return fail(ELASTO_ERR_INVALID_ARG, "clip: %s %d: bad count", name, i), false;
    if (g[i].count > 0 && (!g[i].data || !aligned(g[i].data, g[i].dtype == ELASTO_BF16 ? 2 : 4)))
      return fail(ELASTO_ERR_INVALID_ARG, "clip: %s %d is NULL or misaligned", name, i), false;
  }
  return true;
}

struct Range {
  const char *a, *b;
  bool operator<(const Range& o) const { return a < o.a; }
};
const char* end_of(const elasto_grad_t& g) {
  return static_cast<const char*>(g.data) + g.count * (g.dtype == ELASTO_BF16 ? 2 : 4);
}

// Results that share memory with one another, or with a gradient that is not their own at the
// same place, would be written twice or read after they are written.
bool check_apart(const elasto_grad_t* in, const elasto_grad_t* out, int n) {
  std::vector<Range> w, r;
  w.reserve(n);
  for (int i = 0; i < n; ++i)
    if (out[i].count > 0) w.push_back({static_cast<const char*>(out[i].data), end_of(out[i])});
  if (!std::is_sorted(w.begin(), w.end())) std::sort(w.begin(), w.end());
  for (size_t i = 1; i < w.size(); ++i)
    if (w[i].a < w[i - 1].b) return fail(ELASTO_ERR_INVALID_ARG, "clip: results overlap"), false;
  for (int i = 0; i < n; ++i) {
    if (in[i].count == 0 || in[i].data == out[i].data) continue;
    const char *a = static_cast<const char*>(in[i].data), *b = end_of(in[i]);
    auto it = std::lower_bound(w.begin(), w.end(), Range{a, a});
    if ((it != w.end() && it->a < b) || (it != w.begin() && (it - 1)->b > a))
      return fail(ELASTO_ERR_INVALID_ARG, "clip: gradient %d overlaps a result that is not its own", i), false;
  }
  return true;
}

// Launches of the list: f(table, first entry, chunks).
template <typename F>
hipError_t each_launch(const elasto_grad_t* g, int n, F&& f) {
  Table t;
  int at[kTensors];
  hipError_t e = hipSuccess;
  for (int i = 0; i < n && e == hipSuccess;) {
    t.n = 0;
    t.first[0] = 0;
    int64_t chunks = 0;
    for (; i < n && t.n < kTensors; ++i) {
      if (g[i].count == 0) continue;
      const int64_t c = chunks_of(g[i]);
      if (chunks + c >= ((int64_t)1 << 31)) {
        if (t.n == 0) return hipErrorInvalidValue;  // no tensor of a list has as many
        break;
      }
      const int per = g[i].dtype == ELASTO_BF16 ? kChunk / 2 : kChunk / 4;
      t.at[t.n] = reinterpret_cast<uintptr_t>(g[i].data) | (g[i].dtype == ELASTO_BF16);
      t.last[t.n] = (uint16_t)(g[i].count - (c - 1) * per);
      at[t.n] = i;
      chunks += c;
      t.first[++t.n] = (uint32_t)chunks;
    }
    if (t.n > 0) e = f(t, at, (uint32_t)chunks);
  }
  return e;
}

// Workgroups of each launch's norm: as many as its chunks' share of kMaxBlocks, at least one.
struct Plan {
  std::vector<int> blocks;
  int parts = 0;
  bool past = false;
};
Plan plan_of(const elasto_grad_t* g, int n) {
  int64_t all = 0;
  for (int i = 0; i < n; ++i) all += g[i].count > 0 ? chunks_of(g[i]) : 0;
  Plan p;
  // Gradients of more than the cache behind L2 go past the caches (5.1 GB read and written, 1454 -> 1373
  // us with the norm; 77 MB 44 -> 46 in the kernels).
  p.past = all * kChunk > ((int64_t)256 << 20);
  (void)each_launch(g, n, [&](const Table&, const int*, uint32_t chunks) {
    const int64_t share = ((int64_t)chunks * kMaxBlocks + all - 1) / all;
    p.blocks.push_back((int)std::max<int64_t>(1, std::min<int64_t>(chunks, share)));
    p.parts += p.blocks.back();
    return hipSuccess;
  });
  return p;
}

bool check_workspace(const void* ws, int64_t have, int64_t need) {
  if (need > 0 && (!ws || !aligned(ws, 16) || have < need))
    return fail(ELASTO_ERR_INVALID_ARG, "clip: the workspace holds %lld of %lld bytes (16-byte aligned)",
                (long long)(ws ? have : 0), (long long)need),
           false;
  return true;
}

hipError_t launch_norm(const elasto_grad_t* g, int n, const Plan& plan, double* part, hipStream_t s) {
  size_t k = 0;
  int at = 0;
  return each_launch(g, n, [&](const Table& t, const int*, uint32_t) {
    hipLaunchKernelGGL(norm_kernel, dim3((unsigned)plan.blocks[k]), dim3(kThreads), 0, s, t, part + at);
    at += plan.blocks[k++];
    return hipGetLastError();
  });
}

}  // namespace
}  // namespace elasto

using namespace elasto;

// Nothing may leave a C entry but its status.
#define ELASTO_GUARD(body)                                              \
  try {                                                                 \
    body                                                                \
  } catch (...) {                                                       \
    return fail(ELASTO_ERR_OUT_OF_MEMORY, "clip: out of host memory");  \
  }

extern "C" {

elasto_status_t elasto_grad_norm_workspace(const elasto_grad_t* grads, int32_t n, int64_t* bytes) {
  if (!bytes) return fail(ELASTO_ERR_INVALID_ARG, "NULL argument");
  if (!check_list("gradients", grads, n)) return ELASTO_ERR_INVALID_ARG;
  ELASTO_GUARD(*bytes = (int64_t)plan_of(grads, n).parts * 8; return ELASTO_OK;)
}

elasto_status_t elasto_op_grad_norm(const elasto_grad_t* grads, int32_t n, float* norm, void* workspace,
                                    int64_t workspace_bytes, void* hip_stream) {
  if (!check_list("gradients", grads, n)) return ELASTO_ERR_INVALID_ARG;
  if (!norm || !aligned(norm, 4)) return fail(ELASTO_ERR_INVALID_ARG, "clip: norm is NULL or misaligned");
  ELASTO_GUARD({
    const Plan plan = plan_of(grads, n);
    if (!check_workspace(workspace, workspace_bytes, (int64_t)plan.parts * 8)) return ELASTO_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    double* part = static_cast<double*>(workspace);
    hipError_t e = launch_norm(grads, n, plan, part, s);
    if (e == hipSuccess) {
      hipLaunchKernelGGL(norm_out_kernel, dim3(1), dim3(kThreads), 0, s, part, plan.parts, norm);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "grad_norm: %s", hipGetErrorString(e));
    return ELASTO_OK;
  })
}

elasto_status_t elasto_op_clip_gradients(const elasto_grad_t* grads, const elasto_grad_t* out, int32_t n,
                                         float max_norm, float* stats, void* workspace, int64_t workspace_bytes,
                                         void* hip_stream) {
  if (!check_list("gradients", grads, n) || !check_list("results", out, n)) return ELASTO_ERR_INVALID_ARG;
  if (!(max_norm > 0.0f)) return fail(ELASTO_ERR_INVALID_ARG, "clip: max_norm must be > 0");
  if (!stats || !aligned(stats, 4)) return fail(ELASTO_ERR_INVALID_ARG, "clip: stats is NULL or misaligned");
  bool in_place = true;
  for (int i = 0; i < n; ++i) {
    if (grads[i].count != out[i].count || grads[i].dtype != out[i].dtype)
      return fail(ELASTO_ERR_INVALID_ARG, "clip: result %d has another size or type than its gradient", i);
    in_place = in_place && (grads[i].data == out[i].data || grads[i].count == 0);
  }
  ELASTO_GUARD({
    if (!check_apart(grads, out, n)) return ELASTO_ERR_INVALID_ARG;
    const Plan plan = plan_of(grads, n);
    if (!check_workspace(workspace, workspace_bytes, (int64_t)plan.parts * 8)) return ELASTO_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    double* part = static_cast<double*>(workspace);
    hipError_t e = launch_norm(grads, n, plan, part, s);
    float* st = stats;
    if (e == hipSuccess)
      e = each_launch(grads, n, [&](const Table& t, const int* at, uint32_t chunks) {
        Results r;
        for (int i = 0; i < t.n; ++i) r.out[i] = static_cast<char*>(out[at[i]].data);
        hipLaunchKernelGGL((plan.past ? clip_kernel<true> : clip_kernel<false>),
                           dim3(std::min<uint32_t>(chunks, kMaxBlocks)), dim3(kThreads), 0, s, t, r, part,
                           plan.parts, max_norm, st, in_place);
        st = nullptr;
        return hipGetLastError();
      });
    if (e == hipSuccess && st) {  // no elements at all
      Table t;
      t.n = 0;
      t.first[0] = 0;
      hipLaunchKernelGGL((clip_kernel<false>), dim3(1), dim3(kThreads), 0, s, t, Results(), part, 0, max_norm, st, true);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "clip_gradients: %s", hipGetErrorString(e));
    return ELASTO_OK;
  })
}

}  // extern "C"
