// Distillation from a teacher's largest logits, mixed with the cross-entropy of
// labels: the row losses and, in the same call, the gradient of the student's
// logits z.  With the teacher's values t_i at classes c_i, i < top, temperature
// tau and p = softmax(t / tau) over the entries given:
//   loss = alpha tau^2 sum_i p_i (log p_i - log softmax(z / tau)[c_i])
//          + (1 - alpha) (lse(z) - z_label),
//   dz_j = w (alpha tau (softmax(z / tau)_j - sum of p_i with c_i = j)
//          + (1 - alpha) (softmax(z)_j - [j = label])),
// w the row's weight.  The full softmax enters the gradient of every class, the
// teacher and the label only top + 1 of them.
//
// One workgroup a row.  A first walk takes the maximum and the sums of both
// temperatures together, a second one writes the gradient; the row comes from
// memory once, the second time from the caches behind L2.  The top + 1 special
// classes are then written again by the threads that hold them, from their
// logits gathered before: each sums what all entries of its class take off (a
// class may come twice), so no order of atomics enters.
//
// Bound by memory: the logits once, the gradient once.  2048 x 131072 bf16 with its
// gradient 241 us, 4.45 TB/s (a copy of that size runs at 5.1); the loss alone,
// 1000 x 50021 fp32, 39 us, 5.1.  Both temperatures together take two exponentials
// an element and walk (vector ALU 67% of the cycles), which the memory's time nearly
// covers: 2048 x 131072 bf16 266 us (with labels and one temperature 255).
#include <math.h>

#include <algorithm>

#include "distill.h"
#include "growth_step.h"
#include "heads.h"
#include "logits.h"

namespace elasto {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename T, typename G>
struct DistillP {
  const T* logits;
  int64_t ld;
  const float* teacher;
  const int32_t* index;
  const int32_t* labels;
  const float* weight;
  float* loss;
  G* grad;  // NULL: the loss alone
  int64_t ldg, row0;
  int C, top;
  float alpha, beta;  // of the teacher's and of the labels' part
  float tau, scale;
};

// A reference m near the maximum of x and sums of 2^(c x - c m) for two factors c: the
// exponents as one multiply-add each, with the product c m rounded first.  That
// rounding is the same wherever the maximum is the same, so it cancels in the
// quotients, and what it leaves in the sums' logarithms is known (left).
//
// Beyond |c m| = 2^30 (rows that a mask of the lowest finite value
// fills, say) that rounding would leave the exponents' range.  Numbers that far
// out are 64 or more apart in c x, so only those equal to the maximum count: a
// smaller factor, which brings c m to 2^30, leaves the others nothing either.
constexpr float kFar = 1073741824.0f;
__device__ __forceinline__ bool far_out(float m, float c) { return fabsf(m * c) > kFar; }
struct Power {
  float c, off;
  __device__ __forceinline__ Power(float m, float factor) {
#pragma clang fp contract(off)  // the product rounded, whatever it is added to
    c = m != -INFINITY && far_out(m, factor) ? kFar / fabsf(m) : factor;
    const float r = -m * c;
    off = m == -INFINITY ? 0.0f : r;
  }
  __device__ __forceinline__ float operator()(float x) const {
    return __builtin_amdgcn_exp2f(fmaf(x, c, off));
  }
  __device__ __forceinline__ float left(float m) const { return m == -INFINITY ? 0.0f : fmaf(m, c, off); }
};
struct Sums {
  float m, a, b;
};
// What a sum about m becomes about t, of at least m.
__device__ __forceinline__ float moved(float m, float t, float c) {
#pragma clang fp contract(off)
  const float r = m * c, q = t * c;
  return m == t || m == -INFINITY ? 1.0f
         : far_out(m, c) || far_out(t, c) ? 0.0f : __builtin_amdgcn_exp2f(r - q);
}
__device__ __forceinline__ void move_to(Sums& s, float t, float ca, float cb) {
  s.a *= moved(s.m, t, ca);
  s.b *= moved(s.m, t, cb);
  s.m = t;
}
__device__ __forceinline__ void merge(Sums& s, Sums o, float ca, float cb) {
  const float t = fmaxf(s.m, o.m);
  move_to(s, t, ca, cb);
  move_to(o, t, ca, cb);
  s.a += o.a;
  s.b += o.b;
}

// TWO: the sums of both temperatures are needed and differ.
template <typename T, typename G, int N, bool TWO>
__global__ __launch_bounds__(N) void distill_kernel(DistillP<T, G> p) {
  constexpr int W = N / 64;
  __shared__ float red[W][4];
  __shared__ float amount[kMaxTop + 1];  // what entry i takes off its class
  __shared__ int where[kMaxTop + 1];     // its class, -1: none
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t r = p.row0 + blockIdx.x;
  const T* z = p.logits + r * p.ld;
  const int C = p.C;
  const float weight = (p.weight ? p.weight[r] : 1.0f);
  G* g = p.grad ? p.grad + r * p.ldg : nullptr;
  if (weight == 0.0f) {  // a row left out: its logits are not read
    if (g) {
      const RowSpan<G> gs(g, C);
      const float none[8] = {};
      for (int c = tid; c < gs.runs; c += N) store8(g + gs.run(c), none);
      for (int i = tid; i < gs.singles; i += N) store1(g + gs.single(i), 0.0f);
    }
    if (tid == 0) p.loss[r] = 0.0f;
    return;
  }
  const float w = weight * p.scale;
  const float ct = kLog2e / p.tau;
  const RowSpan<T> span(z, C);

  // The special classes: teacher entries, then the label.
  int cls = -1;
  bool bad = false;
  float tv = -INFINITY, zs = 0.0f;
  if (tid < p.top) {
    const int c = p.index[r * p.top + tid];
    bad = c < -1 || c >= C;
    if (c >= 0 && c < C) {
      cls = c;
      tv = p.teacher[r * p.top + tid];
      bad = tv != tv;
    }
  } else if (tid == p.top && p.labels) {
    const int c = p.labels[r];
    bad = c < 0 || c >= C;
    if (!bad) cls = c;
  }
  if (cls >= 0) zs = load1(z + cls);

  // One walk: reference and sums.
  Sums s = {-INFINITY, 0.0f, 0.0f};
  Power pa(s.m, ct), pb(s.m, kLog2e);
  // The reference follows the maximum only where that has risen by more than
  // 2^kRise (in the sharper sum): terms of up to 2^kRise are as exact, and of
  // a wave's 64 lanes one would raise its own at most runs otherwise.
  constexpr float kRise = 8.0f;
  const float sharp = TWO ? fmaxf(ct, kLog2e) : ct;
  auto raise = [&](float t) {
    if ((t - s.m) * sharp > kRise) {
      move_to(s, t, ct, kLog2e);
      pa = Power(t, ct);
      if constexpr (TWO) pb = Power(t, kLog2e);
    }
  };
  auto add = [&](float x) {
    s.a += pa(x);
    if constexpr (TWO) s.b += pb(x);
  };
  walk_row<N>(z, span, tid,
              [&](int, const float* v) {
                float t = v[0];
#pragma unroll
                for (int e = 1; e < 8; ++e) t = fmaxf(t, v[e]);
                raise(t);
#pragma unroll
                for (int e = 0; e < 8; ++e) add(v[e]);
              },
              [&](int, float v) {
                raise(v);
                add(v);
              });
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1)
    merge(s, Sums{__shfl_xor(s.m, o, 64), __shfl_xor(s.a, o, 64), __shfl_xor(s.b, o, 64)}, ct, kLog2e);
  // The teacher's maximum goes along.
  const float tw = wave_max(tv);
  if (lane == 0) {
    red[wave][0] = s.m;
    red[wave][1] = s.a;
    red[wave][2] = s.b;
    red[wave][3] = tw;
  }
  const bool any_bad = __syncthreads_or(bad);
  s = Sums{red[0][0], red[0][1], red[0][2]};
  float tm = red[0][3];
#pragma unroll
  for (int i = 1; i < W; ++i) {
    merge(s, Sums{red[i][0], red[i][1], red[i][2]}, ct, kLog2e);
    tm = fmaxf(tm, red[i][3]);
  }
  __syncthreads();
  if constexpr (!TWO) s.b = s.a;  // tau 1, or one of the two not needed

  // Teacher probabilities and the row's loss.
  const float tx = (tv - tm) / p.tau;
  const float te = tid < p.top && tm > -INFINITY ? __builtin_amdgcn_exp2f(tx * kLog2e) : 0.0f;
  const float ts = wave_sum(te);
  if (lane == 0) red[wave][0] = ts;
  __syncthreads();
  float tsum = 0.0f;
#pragma unroll
  for (int i = 0; i < W; ++i) tsum += red[i][0];
  __syncthreads();
  const bool taught = p.alpha > 0.0f && tm > -INFINITY;  // the teacher gives the row something
  const float prob = taught ? te / tsum : 0.0f;
  pa = Power(s.m, ct);
  if constexpr (TWO) pb = Power(s.m, kLog2e);
  const Power& p1 = TWO ? pb : pa;  // of the labels' part
  float part = 0.0f;
  if (tid < p.top) {
    // log p - log q, each from differences to its own maximum.
    if (prob > 0.0f || prob != prob)
      part = p.alpha * p.tau * p.tau * prob *
             (tx - log2f(tsum) * kLn2 + ((s.m - zs) / p.tau + (log2f(s.a) - pa.left(s.m)) * kLn2));
  } else if (tid == p.top && p.beta > 0.0f) {
    part = p.beta * ((s.m - zs) + (log2f(s.b) - p1.left(s.m)) * kLn2);
  }
  const float total = wave_sum(part);
  if (lane == 0) red[wave][0] = total;
  if (tid <= p.top) {
    where[tid] = cls;
    amount[tid] = tid < p.top ? p.alpha * p.tau * prob : p.beta;
  }
  __syncthreads();
  if (tid == 0) {
    float sum = 0.0f;
    for (int i = 0; i < W; ++i) sum += red[i][0];
    p.loss[r] = any_bad ? NAN : sum;
  }
  if (!g) return;

  // The gradient: both softmaxes with their weights in the factors.
  const float fa = (taught ? p.alpha * p.tau / s.a : 0.0f) * w;
  const float fb = (p.labels ? p.beta / s.b : 0.0f) * w;
  const float f1 = fa + fb;
  auto value = [&](float x) {
    if constexpr (TWO)
      return fmaf(fa, pa(x), fb * pb(x));
    else
      return f1 * pa(x);
  };
  // Single stores where the two rows reach 16 bytes at different columns (fp32 logits
  // and a bf16 gradient: half of the rows unless classes are a multiple of 8; 1000 x
  // 50021 89 us, 1000 x 50024 82).
  const bool wide = (reinterpret_cast<uintptr_t>(g + span.head) & 15) == 0;
  walk_row<N>(z, span, tid,
              [&](int i, const float* v) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = value(v[e]);
                if (wide) {
                  store8(g + i, o);
                } else {
#pragma unroll
                  for (int e = 0; e < 8; ++e) store1(g + i + e, o[e]);
                }
              },
              [&](int i, float v) { store1(g + i, value(v)); });
  __syncthreads();  // the special classes' values go over those
  if (tid <= p.top && cls >= 0) {
    float off = 0.0f;
    bool first = true;
    for (int i = 0; i <= p.top; ++i)
      if (where[i] == cls) {
        if (i < tid) first = false;
        off += amount[i];
      }
    if (first) store1(g + cls, fmaf(-off, w, value(zs)));
  }
}

// Whether the sums of both temperatures are needed and differ.  With no labels, or
// none of the teacher, one sum does: at the temperature that is needed.
bool two_sums(const DistillArgs& a) {
  return a.labels && a.alpha > 0.0f && a.alpha < 1.0f && a.temperature != 1.0f;
}

template <typename T, typename G, int N>
hipError_t launch(const DistillArgs& a, hipStream_t s) {
  DistillP<T, G> p;
  p.logits = static_cast<const T*>(a.logits);
  p.ld = a.ld;
  p.teacher = a.values;
  p.index = a.indices;
  p.labels = a.labels;
  p.weight = a.row_weight;
  p.loss = a.loss;
  p.grad = static_cast<G*>(a.dlogits);
  p.ldg = a.ldg;
  p.C = a.classes;
  p.top = a.top;
  p.alpha = a.alpha;
  p.beta = a.labels ? 1.0f - a.alpha : 0.0f;
  p.tau = a.alpha == 0.0f ? 1.0f : a.temperature;
  p.scale = a.scale;
  const bool two = two_sums(a);
  hipError_t e = hipSuccess;
  for (p.row0 = 0; p.row0 < a.rows && e == hipSuccess; p.row0 += kLaunchRows) {
    const unsigned rows = (unsigned)std::min<int64_t>(a.rows - p.row0, kLaunchRows);
    if (two)
      hipLaunchKernelGGL((distill_kernel<T, G, N, true>), dim3(rows), dim3(N), 0, s, p);
    else
      hipLaunchKernelGGL((distill_kernel<T, G, N, false>), dim3(rows), dim3(N), 0, s, p);
    e = hipGetLastError();
  }
  return e;
}

// More threads than teacher entries, one for the label among them; and about one run
// of eight a thread for short rows, of which many run at once (4096 x 1000 fp32:
// 34 us with 512 threads, 19 with 256, 14 with 128).  Long rows take 1024, which
// hold two rows on a CU where 512 hold four: the rows at work, read a second time for
// the gradient, would not stay in the cache behind L2 (2048 x 131072 bf16: 257 us
// with 512 threads, 247 with 1024; 4096 x 32000: 122 and 190).  At two temperatures
// 1024 threads take 87 registers, for the sums of 16 waves, and a CU holds one row of
// them: they pay for longer rows only (2048 x 131072 bf16: 266 us with 512 threads,
// 310 with 1024; 1600 x 160000: 292 and 302; 1300 x 200003: 332 and 302; 1024 x
// 65536 fp32: 138 and 158; 400 x 200003: 208 and 200).  The loss alone takes as
// many, so that its bits are the same.
template <typename T, typename G>
hipError_t launch_threads(const DistillArgs& a, hipStream_t s) {
  if (a.classes <= 1024 && a.top < 128) return launch<T, G, 128>(a, s);
  if (a.classes <= 2048 && a.top < 256) return launch<T, G, 256>(a, s);
  if ((int64_t)a.classes * (int)sizeof(T) > (two_sums(a) ? 350 : 200) * 1024) return launch<T, G, 1024>(a, s);
  return launch<T, G, 512>(a, s);
}

}  // namespace

bool check_distill(const DistillArgs& a) {
  const int es = a.dtype == ELASTO_BF16 ? 2 : 4, gs = a.grad_dtype == ELASTO_BF16 ? 2 : 4;
  if ((a.dtype != ELASTO_BF16 && a.dtype != ELASTO_FP32) ||
      (a.grad_dtype != ELASTO_BF16 && a.grad_dtype != ELASTO_FP32))
    return fail(ELASTO_ERR_INVALID_ARG, "distill: bad dtype %d or %d", a.dtype, a.grad_dtype), false;
  if (a.rows < 0 || a.rows > 0x7fffffff || a.classes < 1 || a.classes > (1 << 30) || a.ld < a.classes ||
      (a.dlogits && a.ldg < a.classes))
    return fail(ELASTO_ERR_INVALID_ARG, "distill: bad rows, classes or row strides"), false;
  if (a.top < 0 || a.top > kMaxTop)
    return fail(ELASTO_ERR_INVALID_ARG, "distill: top %d outside [0, %d]", a.top, kMaxTop), false;
  if (!(a.temperature >= 1e-6f) || !(a.temperature <= 1e6f) || !(a.alpha >= 0.0f) || !(a.alpha <= 1.0f) ||
      !(fabsf(a.scale) < INFINITY))
    return fail(ELASTO_ERR_INVALID_ARG, "distill: needs temperature in [1e-6, 1e6], alpha in [0, 1] and a finite scale"), false;
  if (a.alpha > 0.0f && a.top == 0)
    return fail(ELASTO_ERR_INVALID_ARG, "distill: alpha > 0 needs teacher entries"), false;
  if (a.rows == 0) return true;
  if (!a.logits || !a.loss || (a.top > 0 && (!a.values || !a.indices)))
    return fail(ELASTO_ERR_INVALID_ARG, "distill: NULL pointer"), false;
  if (a.alpha < 1.0f && !a.labels) return fail(ELASTO_ERR_INVALID_ARG, "distill: alpha < 1 needs labels"), false;
  if (!aligned(a.logits, es) || !aligned(a.dlogits, gs) || !aligned(a.loss, 4) || !aligned(a.values, 4) ||
      !aligned(a.indices, 4) || !aligned(a.labels, 4) || !aligned(a.row_weight, 4))
    return fail(ELASTO_ERR_INVALID_ARG, "distill: misaligned pointer"), false;
  if (a.dlogits == a.logits && (a.dtype != a.grad_dtype || a.ld != a.ldg))
    return fail(ELASTO_ERR_INVALID_ARG, "distill: dlogits over logits needs the same type and row stride"), false;
  return true;
}

hipError_t launch_distill(const DistillArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (a.dtype == ELASTO_BF16)
    return a.grad_dtype == ELASTO_BF16 ? launch_threads<uint16_t, uint16_t>(a, s)
                                       : launch_threads<uint16_t, float>(a, s);
  return a.grad_dtype == ELASTO_BF16 ? launch_threads<float, uint16_t>(a, s)
                                     : launch_threads<float, float>(a, s);
}

}  // namespace elasto

using namespace elasto;

extern "C" elasto_status_t elasto_op_distill(int32_t dtype, const void* logits, int64_t ld, int64_t rows,
                                             int32_t classes, const float* teacher_values,
                                             const int32_t* teacher_indices, int32_t top,
                                             const int32_t* labels, const float* row_weight,
                                             float temperature, float alpha, float scale, float* loss,
                                             int32_t grad_dtype, void* dlogits, int64_t ldg,
                                             void* hip_stream) {
  DistillArgs a;
  a.dtype = dtype; a.logits = logits; a.ld = ld; a.rows = rows; a.classes = classes;
  a.values = teacher_values; a.indices = teacher_indices; a.top = top; a.labels = labels;
  a.row_weight = row_weight; a.temperature = temperature; a.alpha = alpha; a.scale = scale;
  a.loss = loss; a.grad_dtype = grad_dtype; a.dlogits = dlogits; a.ldg = ldg;
  if (!check_distill(a)) return ELASTO_ERR_INVALID_ARG;
  const hipError_t e = launch_distill(a, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "distill: %s", hipGetErrorString(e));
  return ELASTO_OK;
}

extern "C" elasto_status_t elasto_growth_step_distill(elasto_growth_t g, int32_t mode, const void* images,
                                                      const int32_t* labels, const float* teacher_values,
                                                      const int32_t* teacher_indices, int32_t top,
                                                      float temperature, float alpha, int32_t batch,
                                                      float lr, float clip_norm, float* stats,
                                                      void* hip_stream) {
  if (!g) return fail(ELASTO_ERR_INVALID_ARG, "context is NULL");
  DistillArgs a;
  a.dtype = ELASTO_FP32; a.grad_dtype = ELASTO_BF16;
  a.values = teacher_values; a.indices = teacher_indices; a.top = top; a.labels = labels;
  a.temperature = temperature; a.alpha = alpha;
  // What the step itself fills in is checked there; here the caller's part.
  a.logits = a.loss = reinterpret_cast<float*>(256);
  a.rows = a.classes = a.ld = 1;
  if (!check_distill(a)) return ELASTO_ERR_INVALID_ARG;
  const GrowthLoss loss = {"distillation loss",
                           [](const void* args, const GrowthLogits& z, hipStream_t s) {
                             DistillArgs d = *static_cast<const DistillArgs*>(args);
                             d.logits = z.logits; d.ld = z.ld; d.rows = z.batch; d.classes = z.classes;
                             d.loss = z.rowloss; d.dlogits = z.dlogits; d.ldg = z.ldg;
                             d.scale = 1.0f / (float)z.batch;
                             return launch_distill(d, s);
                           },
                           &a};
  return growth_step(g, mode, images, batch, lr, clip_norm, stats, hip_stream, loss);
}
