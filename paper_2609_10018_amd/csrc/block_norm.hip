// What lies between two blocks of a transformer, in one pass over the tokens: the norm behind a
// block, its gate, the residual addition and the norm ahead of the next block.
//   n = N_post(y)  (or y),  x' = a x + g (.) n,  u = N_pre(x'),
//   N(v) = (v - mean) r (.) gamma + beta,  r = 1 / sqrt(mean((v - mean)^2) + eps)
// (RMS: mean = 0).  Backward, with v^ = (v - mean) r and N'(d) = r (d gamma - v^ mean(d gamma v^)
// - mean(d gamma)) (RMS: without the last term):
//   dX = dx' + N_pre'(du),  dx = a dX,  dn = g (.) dX,  dy = N_post'(dn)  (or dn),
//   dgamma = sum d v^ and dbeta = sum d over the tokens, dg = sum dX (.) n over a gate's tokens.
//
// A row is held in the registers of 16 lanes to sixteen waves, eight or sixteen values a thread, and read
// once; its statistics are taken there, of a layer norm first the mean and then what is about it, so a large
// mean costs no digits.  Everything between the load and the store is fp32; u is taken from x' before x' is
// rounded.  Backward, a workgroup walks the rows of one gate (or a part of them) and sums the weights'
// gradients of its columns in registers; the parts are summed by a second kernel in a fixed order.  Rows of
// more than 8192 leave no registers for the sums: a kernel of its own takes them, column by column, from the
// rows and six numbers that the first one has written of each (568 rows of 8735: 558 us with the sums spilled,
// 50; 6000 rows of 12288, fp32 beside bf16: 477, for ten passes over the rows instead of six).
//
// Bound by memory: forward four passes over the tokens, backward six.  Measured on a card whose copies reach
// 4.75 TB/s: forward, 50432 rows of 768, bf16, layer norm and gate, 62 us (5.0 TB/s); backward, 18700 rows of
// 2048, fp32 beside bf16, norms on both sides and every weight's gradient, 161 us (4.6 TB/s).  Rows of bf16
// under a layer norm of 2048 to 8192 columns wait for their exchanges: 1.5 to 1.9 times the floor.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "heads.h"

namespace elasto {
namespace {

constexpr int kMaxDim = 16384;
constexpr int kSums = 5;                   // pre gamma, pre beta, post gamma, post beta, gate
constexpr int kStats = 6;                  // mean, r, mean(d gamma v^) r and mean(d gamma) r of x', mean and r of y

struct Rows {  // strides in bytes
  char* p;
  int64_t sb, st;
};

struct BlockP {
  Rows x, y, x_out, u;     // backward: x_out and y are inputs,
  Rows dx_out, du, dx, dy;
  const float *pre_gamma, *pre_beta, *post_gamma, *post_beta, *gate;
  int64_t gate_ld;         // 0: one for all sequences
  const int32_t* lens;
  int batch, tokens, dim;
  bool layer, post, has_y;
  float a, eps, inv_dim;
  // Backward.
  float* part;             // [workgroup][4][dim]
  float* gate_part;        // [unit or workgroup][dim]
  bool gate_unit;          // a gate's sums end with the unit
  int slices;              // units of a sequence: runs of its rows
  int wanted;              // bits: the sums that are asked for
  float* stats;            // [row][kStats] of rows whose sums a kernel of their own takes
};

// A row is held by T threads, CH runs of 8 columns each: run i of thread t begins at column (i T + t) 8.  Rows
// reach into the last of the CH (forward_width, backward_width), so the others are there in every thread.
// Runs are loaded and stored whole, at whatever address they lie.  Where dim is no multiple of 8, the row's
// last run is moved back to end with it, and its first `skip` values, which are the run's before it, count
// as 0 and are not stored (CUT; the other dims have kernels without it: 50432 rows of 768, 69 -> 54 us).
template <int T, int CH, bool CUT>
struct Place {
  static constexpr int E = 8 * CH, kLast = CH - 1;
  static constexpr bool kCut = CUT, kShort = CUT && T == 16;   // kShort: rows of fewer than 8
  int dim, t, skip;
  bool cut;       // this thread's last run is the one that was moved
  bool drop[7];   // its values that are not the thread's
  float m;        // 1 where the last run is there, 0 where it is not
  __device__ __forceinline__ Place(int dim_, int t_) : dim(dim_), t(t_), skip(-dim_ & 7) {
    m = there(kLast) ? 1.0f : 0.0f;
    cut = CUT && there(kLast) && column(kLast) + 8 > dim;
#pragma unroll
    for (int e = 0; e < 7; ++e) drop[e] = cut && e < skip;
  }
  __device__ __forceinline__ int column(int i) const { return (i * T + t) * 8; }
  __device__ __forceinline__ int begin(int i) const { return CUT && i == kLast ? min(column(i), dim - 8) : column(i); }
  __device__ __forceinline__ bool there(int i) const { return i < kLast || column(i) < dim; }
  // Whether value e is one of the row's.
  __device__ __forceinline__ bool holds(int e) const {
    return there(e >> 3) && !(CUT && (e >> 3) == kLast && (e & 7) < 7 && drop[e & 7]);
  }
  __device__ __forceinline__ void clean_run(float (&v)[E], int i) const {
    if (CUT && i == kLast)
#pragma unroll
      for (int e = 0; e < 7; ++e) v[8 * i + e] = drop[e] ? 0.0f : v[8 * i + e];
  }

  // v less `less` in the columns that are there; in the others it stays 0.
  __device__ __forceinline__ void subtract_run(float (&v)[E], float less, int i) const {
    const float k = i == kLast ? less * m : less;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[8 * i + e] -= k;
    clean_run(v, i);
  }
  __device__ __forceinline__ void subtract(float (&v)[E], float less) const {
#pragma unroll
    for (int i = 0; i < CH; ++i) subtract_run(v, less, i);
  }
};

typedef u32x4 __attribute__((aligned(2))) bf16_run;    // eight bf16 at any bf16's address
typedef f32x4 __attribute__((aligned(4))) f32_run;

__device__ __forceinline__ void store_value(uint16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_run(uint16_t* p, const float* v) {
  *reinterpret_cast<bf16_run*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                          pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void store_run(float* p, const float* v) {
  *reinterpret_cast<f32_run*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32_run*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

template <typename L, typename T>
__device__ __forceinline__ void store_run(T* p, const L& l, const float (&v)[L::E], int i) {
  if (!l.there(i)) return;
  T* to = p + l.begin(i);
  if (!L::kCut || i != L::kLast || !l.cut)
    store_run(to, v + 8 * i);
  else
#pragma unroll
    for (int e = 1; e < 8; ++e)
      if (e >= l.skip) store_value(to + e, v[8 * i + e]);
}
template <typename L, typename T>
__device__ __forceinline__ void store_row(T* p, const L& l, const float (&v)[L::E]) {
#pragma unroll
  for (int i = 0; i < L::E / 8; ++i) store_run(p, l, v, i);
}

// A row as it was loaded.  A row shorter than a run has it before its begin: it is loaded by values.
template <typename L, typename T>
struct Raw {
  static constexpr bool kPacked = sizeof(T) == 2;
  u32x4 w[kPacked ? L::E / 8 : L::E / 4];
  __device__ __forceinline__ void load_run(const T* p, bool there, const L& l, int i) {
    u32x4* o = w + (kPacked ? i : 2 * i);
    o[0] = u32x4{0, 0, 0, 0};
    if (!kPacked) o[1] = u32x4{0, 0, 0, 0};
    if (!there || !l.there(i)) return;
    const T* from = p + l.begin(i);
    if (L::kShort && l.dim < 8) {
#pragma unroll
      for (int e = 1; e < 8; ++e)
        if (e >= l.skip) {
          if constexpr (kPacked)
            o[0][e >> 1] |= (uint32_t)from[e] << (16 * (e & 1));
          else
            o[e >> 2][e & 3] = __float_as_uint(from[e]);
        }
    } else if constexpr (kPacked) {
      o[0] = *reinterpret_cast<const bf16_run*>(from);
    } else {
      const f32x4 a = *reinterpret_cast<const f32_run*>(from), b = *reinterpret_cast<const f32_run*>(from + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[0][e] = __float_as_uint(a[e]), o[1][e] = __float_as_uint(b[e]);
    }
  }
  __device__ __forceinline__ void load(const T* p, bool there, const L& l) {
#pragma unroll
    for (int i = 0; i < L::E / 8; ++i) load_run(p, there, l, i);
  }
  __device__ __forceinline__ void get_run(float (&v)[L::E], const L& l, int i) const {
#pragma unroll
    for (int e = 8 * i; e < 8 * i + 8; ++e) {
      if constexpr (kPacked)
        v[e] = __uint_as_float((e & 1) ? (w[e >> 3][(e & 7) >> 1] & 0xffff0000u) : (w[e >> 3][(e & 7) >> 1] << 16));
      else
        v[e] = __uint_as_float(w[e >> 2][e & 3]);
    }
    l.clean_run(v, i);
  }
  __device__ __forceinline__ void get(float (&v)[L::E], const L& l) const {
#pragma unroll
    for (int i = 0; i < L::E / 8; ++i) get_run(v, l, i);
  }
};

template <typename L>
__device__ __forceinline__ void load_weight_run(const float* w, float none, const L& l, int i, float (&v)[L::E]) {
  if (w) {
    Raw<L, float> r;
    r.load_run(w, true, l, i);
    r.get_run(v, l, i);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[8 * i + e] = none;
  }
}
template <typename L>
__device__ __forceinline__ void load_weight(const float* w, float none, const L& l, float (&v)[L::E]) {
#pragma unroll
  for (int i = 0; i < L::E / 8; ++i) load_weight_run(w, none, l, i, v);
}

// The sum over groups of 2 to 64 lanes, in all of them: in rows of 16 by lane moves of the adder itself, then the
// rows' sums in their order.
template <int CTRL>
__device__ __forceinline__ float add_moved(float v) {
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                 0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float sum_of_lanes(float v) {
  v = add_moved<0xB1>(v);                               // lane ^ 1
  if constexpr (LANES > 2) v = add_moved<0x4E>(v);      // lane ^ 2
  if constexpr (LANES > 4) v = add_moved<0x141>(v);     // the other quad of eight
  if constexpr (LANES > 8) v = add_moved<0x140>(v);     // the other eight of a row
  if constexpr (LANES <= 16) return v;
  if constexpr (LANES == 32) return v + __shfl_xor(v, 16);
  auto row = [&](int r) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 16 * r)); };
  return (row(0) + row(1)) + (row(2) + row(3));
}

// Sums over a row's T threads, where they are several waves through LDS: two buffers in turn, so that one
// barrier does for each exchange (who writes a buffer again has passed the barrier behind which all have read
// it).
constexpr int kMost = 3;  // sums of an exchange
template <int T>
struct Exchange {
  static constexpr int W = (T + 63) / 64;
  float* buf;  // [2][W][kMost]
  int turn = 0;
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N], int t) {
    static_assert(N <= kMost, "room");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum_of_lanes<T < 64 ? T : 64>(v[i]);
    if constexpr (W > 1) {
      float* b = buf + turn * W * kMost;
      turn ^= 1;
      if ((t & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) b[(t >> 6) * kMost + i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = sum_of_lanes<W>(b[(t & (W - 1)) * kMost + i]);
    }
  }
};

template <typename T>
__device__ __forceinline__ T* at(const Rows& r, int b, int t) {
  return reinterpret_cast<T*>(r.p + b * r.sb + t * r.st);
}

// Whether the weights and the next row's loads stay in registers: not for rows of 1024 threads, which have
// 128 registers.  Backward these still hold the next row's where they can.
template <int T>
constexpr bool kKeep = T < 1024;
template <bool LAYER, int T, int CH>
constexpr bool kAhead = CH == 1 && (T < 1024 || !LAYER);
constexpr int workgroup(int T) { return T > 256 ? T : 256; }

// T: of y and u.  S: of the stream.  TR threads a row; a workgroup of 256 threads holds 256 / TR rows.  Rows
// are taken in strides of the grid's, the next one's loads in flight, the weights in registers.
template <typename T, typename S, bool LAYER, bool CUT, int TR, int CH>
__global__ __launch_bounds__(workgroup(TR)) void block_norm_kernel(BlockP p) {
  typedef Place<TR, CH, CUT> L;
  constexpr int E = L::E, R = workgroup(TR) / TR;
  constexpr bool KEEP = kKeep<TR>;
  __shared__ float red[R][2 * Exchange<TR>::W * kMost];
  const int mine = TR < 64 ? threadIdx.x / TR : __builtin_amdgcn_readfirstlane(threadIdx.x / TR);
  const L l(p.dim, threadIdx.x % TR);
  const int t = l.t;
  Exchange<TR> exchange = {red[mine]};
  const int rows = p.batch * p.tokens, stride = gridDim.x * R;
  float pg[E], pb[E], qg[E], qb[E], g[E];
  auto pre = [&] {
    load_weight(p.pre_gamma, 1.0f, l, pg);
    if constexpr (LAYER) load_weight(p.pre_beta, 0.0f, l, pb);
  };
  auto post = [&] {
    load_weight(p.post_gamma, 1.0f, l, qg);
    if constexpr (LAYER) load_weight(p.post_beta, 0.0f, l, qb);
  };
  if (KEEP && p.u.p) pre();
  if (KEEP && p.post) post();
  if (KEEP) load_weight(p.gate, 1.0f, l, g);  // of the first sequence, or of all
  int gate_of = 0;
  Raw<L, S> rx;
  Raw<L, T> ry;
  int b = 0, tok = 0;
  bool live = false;
  auto fetch = [&](int row) {
    live = row < rows;
    const int r = live ? row : 0;
    b = (int)((unsigned)r / (unsigned)p.tokens);
    tok = r - b * p.tokens;
    if (live && p.lens) live = tok < p.lens[b];
    rx.load(at<const S>(p.x, b, tok), live, l);
    if (p.has_y) ry.load(at<const T>(p.y, b, tok), live, l);
  };
  // All rows of a workgroup take as many rounds: with W > 1 they meet at its barriers.
  int row = blockIdx.x * R;
  if (KEEP) fetch(row + mine);
  for (; row < rows; row += stride) {
    if (!KEEP) fetch(row + mine);
    float x[E], v[E];
    rx.get(x, l);
    const bool now = live;
    const int nb = b, nt = tok;
    if (p.has_y) {
      ry.get(v, l);
      if (KEEP && row + stride < rows) fetch(row + stride + mine);
      if (p.post) {
        if constexpr (LAYER) {
          float s[1] = {0.0f};
#pragma unroll
          for (int e = 0; e < E; ++e) s[0] += v[e];
          exchange(s, t);
          l.subtract(v, s[0] * p.inv_dim);
        }
        float q[1] = {0.0f};
#pragma unroll
        for (int e = 0; e < E; ++e) q[0] = fmaf(v[e], v[e], q[0]);
        exchange(q, t);
        const float r = 1.0f / sqrtf(fmaf(q[0], p.inv_dim, p.eps));
        if (!KEEP) post();
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = LAYER ? fmaf(v[e] * r, qg[e], qb[e]) : v[e] * r * qg[e];
      }
      if (!KEEP && !p.gate_ld) load_weight(p.gate, 1.0f, l, g);
      if (p.gate_ld && (!KEEP || nb != gate_of)) {
        load_weight(p.gate + nb * p.gate_ld, 1.0f, l, g);
        gate_of = nb;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = fmaf(p.a, x[e], g[e] * v[e]);
    } else {
      if (KEEP && row + stride < rows) fetch(row + stride + mine);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] *= p.a;
    }
    if (now && p.x_out.p) store_row(at<S>(p.x_out, nb, nt), l, x);
    if (!p.u.p) continue;
    if constexpr (LAYER) {
      float s[1] = {0.0f};
#pragma unroll
      for (int e = 0; e < E; ++e) s[0] += x[e];
      exchange(s, t);
      l.subtract(x, s[0] * p.inv_dim);
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < E; ++e) q[0] = fmaf(x[e], x[e], q[0]);
    exchange(q, t);
    const float r = 1.0f / sqrtf(fmaf(q[0], p.inv_dim, p.eps));
    if (!KEEP) pre();
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = LAYER ? fmaf(x[e] * r, pg[e], pb[e]) : x[e] * r * pg[e];
    if (now) store_row(at<T>(p.u, nb, nt), l, x);
  }
}

// Three exchanges a row (RMS: two): sums for the means; about them, with what both norms need that the
// gradient of x' does not wait for; and the norm behind the block's.
template <typename T, typename S, bool LAYER, bool CUT, int TR, int CH>
__global__ __launch_bounds__(workgroup(TR), TR > 256 ? 1 : 3) void block_norm_bwd_kernel(BlockP p) {
  typedef Place<TR, CH, CUT> L;
  constexpr int E = L::E, R = workgroup(TR) / TR;
  constexpr bool KEEP = kKeep<TR>, AHEAD = kAhead<LAYER, TR, CH>, SUMS = CH == 1;
  __shared__ float red[R][2 * Exchange<TR>::W * kMost];
  __shared__ float sums[R > 1 ? (R - 1) * TR : 1];
  const int mine = TR < 64 ? threadIdx.x / TR : __builtin_amdgcn_readfirstlane(threadIdx.x / TR);
  const L l(p.dim, threadIdx.x % TR);
  const int t = l.t;
  Exchange<TR> exchange = {red[mine]};
  float pg[E], pb[E], qg[E], qb[E], gg[E];
#pragma unroll
  for (int e = 0; e < E; ++e) pg[e] = pb[e] = qg[e] = qb[e] = gg[e] = 0.0f;
  // The workgroup's rows sum into the first one's thread, value by value, which hands them out.
  auto flush = [&](const float (&v)[E], float* out) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float s = v[e];
      if constexpr (R > 1) {
        __syncthreads();
        if (mine > 0) sums[(mine - 1) * TR + t] = s;
        __syncthreads();
        if (mine == 0)
#pragma unroll
          for (int k = 0; k < R - 1; ++k) s += sums[k * TR + t];
      }
      if (mine == 0 && l.holds(e)) out[l.begin(e >> 3) + (e & 7)] = s;
    }
  };
  float w_pre[E], w_post[E], b_post[E], w_gate[E];
  if (KEEP) {
    load_weight(p.pre_gamma, 1.0f, l, w_pre);
    if (p.post) load_weight(p.post_gamma, 1.0f, l, w_post);
    if (LAYER && p.post) load_weight(p.post_beta, 0.0f, l, b_post);
    load_weight(p.gate, 1.0f, l, w_gate);
  }
  // Run by run.  Where registers are short, what is loaded behind a mark is not loaded ahead of it.
  auto hold_order = [] {
    if constexpr (!KEEP) __builtin_amdgcn_sched_barrier(0);
  };
  auto by_runs = [&](auto f) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      f(i);
      hold_order();
    }
  };
  const int units = p.batch * p.slices;
  for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int b = unit / p.slices, slice = unit - b * p.slices;
    const int n = p.lens ? max(0, min(p.tokens, p.lens[b])) : p.tokens;
    const int share = (n + p.slices - 1) / p.slices, first = slice * share, last = min(n, first + share);
    if (KEEP && p.gate_ld) load_weight(p.gate + b * p.gate_ld, 1.0f, l, w_gate);
    const float* gate = p.gate ? p.gate + b * p.gate_ld : nullptr;
    Raw<L, S> rx, rd;
    Raw<L, T> ru, ry;
    auto load_run = [&](int tok, bool live, int i) {
      const int k = live ? tok : 0;
      if (p.du.p) {
        ru.load_run(at<const T>(p.du, b, k), live, l, i);
        rx.load_run(at<const S>(p.x_out, b, k), live, l, i);
      }
      if (p.has_y) ry.load_run(at<const T>(p.y, b, k), live, l, i);
      if (AHEAD && p.dx_out.p) rd.load_run(at<const S>(p.dx_out, b, k), live, l, i);
    };
    auto load = [&](int tok) {
#pragma unroll
      for (int i = 0; i < CH; ++i) load_run(tok, tok < last, i);
    };
    if (AHEAD && first < last) load(first + mine);
    // Every row of a workgroup takes as many rounds: they meet at its barriers.
    for (int k = first; k < last; k += R) {
      const int tok = k + mine;
      const bool live = tok < last;
      if (!AHEAD) load(tok);
      float d[E], x[E], v[E], s[3] = {0.0f, 0.0f, 0.0f};
      auto get = [&](int i) {
#pragma unroll
        for (int e = 8 * i; e < 8 * i + 8; ++e) d[e] = x[e] = v[e] = 0.0f;
        if (p.du.p) {
          ru.get_run(d, l, i);
          rx.get_run(x, l, i);
        }
        if (p.has_y) ry.get_run(v, l, i);
      };
      float mean_x = 0.0f, mean_y = 0.0f, c = 0.0f;
      auto center = [&](int i) {
        if constexpr (LAYER) {
          if (p.du.p) l.subtract_run(x, mean_x, i);
          if (p.post) l.subtract_run(v, mean_y, i);
        }
      };
      if constexpr (LAYER) {
        by_runs([&](int i) {
          get(i);
          hold_order();
          if (!KEEP) load_weight_run(p.pre_gamma, 1.0f, l, i, w_pre);
#pragma unroll
          for (int e = 8 * i; e < 8 * i + 8; ++e) {
            s[0] += x[e];
            s[1] += v[e];
            s[2] = fmaf(d[e], w_pre[e], s[2]);
          }
        });
        exchange(s, t);
        mean_x = s[0] * p.inv_dim;
        mean_y = s[1] * p.inv_dim;
        c = s[2] * p.inv_dim;
        s[0] = s[1] = s[2] = 0.0f;
      }
      by_runs([&](int i) {
        if constexpr (!LAYER) get(i);
        if (!KEEP) load_weight_run(p.pre_gamma, 1.0f, l, i, w_pre);
        center(i);
#pragma unroll
        for (int e = 8 * i; e < 8 * i + 8; ++e) {
          s[0] = fmaf(x[e], x[e], s[0]);
          s[1] = fmaf(v[e], v[e], s[1]);
          s[2] = fmaf(d[e] * w_pre[e], x[e], s[2]);
        }
      });
      exchange(s, t);
      const float r = 1.0f / sqrtf(fmaf(s[0], p.inv_dim, p.eps)), a = r * s[2] * p.inv_dim;
      const float r_post = p.post ? 1.0f / sqrtf(fmaf(s[1], p.inv_dim, p.eps)) : 1.0f;
      if constexpr (!SUMS)
        if (p.stats && t == 0) {
          float* o = p.stats + ((int64_t)b * p.tokens + tok) * kStats;
          o[0] = mean_x, o[1] = r, o[2] = a, o[3] = r * c, o[4] = mean_y, o[5] = r_post;
        }
      float q[2] = {0.0f, 0.0f};
      by_runs([&](int i) {
        if (!KEEP) load_weight_run(p.pre_gamma, 1.0f, l, i, w_pre);   // again: not held over the exchange
        if (p.du.p) {
#pragma unroll
          for (int e = 8 * i; e < 8 * i + 8; ++e) {
            const float xn = x[e] * r;
            if constexpr (SUMS && LAYER) pb[e] += d[e];
            if constexpr (SUMS) pg[e] = fmaf(d[e], xn, pg[e]);
            d[e] = r * fmaf(d[e], w_pre[e], -xn * a);
          }
          if constexpr (LAYER) l.subtract_run(d, r * c, i);
        }
        if (p.dx_out.p) {
          if (!AHEAD) rd.load_run(at<const S>(p.dx_out, b, live ? tok : 0), live, l, i);
          rd.get_run(x, l, i);
#pragma unroll
          for (int e = 8 * i; e < 8 * i + 8; ++e) d[e] += x[e];
        }
        if (AHEAD && k + R < last) load(tok + R);
        if (p.dx.p && live) {
#pragma unroll
          for (int e = 8 * i; e < 8 * i + 8; ++e) x[e] = p.a * d[e];
          store_run(at<S>(p.dx, b, tok), l, x, i);
        }
        if (!p.has_y) return;
        hold_order();
        if (!KEEP) load_weight_run(gate, 1.0f, l, i, w_gate);
        if (!p.post) {
#pragma unroll
          for (int e = 8 * i; e < 8 * i + 8; ++e) {
            if constexpr (SUMS) gg[e] = fmaf(d[e], v[e], gg[e]);
            d[e] *= w_gate[e];
          }
          return;
        }
        hold_order();
        if (!KEEP) load_weight_run(p.post_gamma, 1.0f, l, i, w_post);
        if (!KEEP && LAYER && SUMS) load_weight_run(p.post_beta, 0.0f, l, i, b_post);
#pragma unroll
        for (int e = 8 * i; e < 8 * i + 8; ++e) {
          v[e] *= r_post;
          if constexpr (SUMS) gg[e] = fmaf(d[e], LAYER ? fmaf(v[e], w_post[e], b_post[e]) : v[e] * w_post[e], gg[e]);
          d[e] *= w_gate[e];
          if constexpr (SUMS) qg[e] = fmaf(d[e], v[e], qg[e]);
          if constexpr (SUMS && LAYER) qb[e] += d[e];
          d[e] *= w_post[e];
          q[0] = fmaf(d[e], v[e], q[0]);
          if constexpr (LAYER) q[1] += d[e];
        }
      });
      if (!p.has_y) continue;
      float am = 0.0f, m = 0.0f;
      if (p.post) {
        exchange(q, t);
        am = q[0] * p.inv_dim;
        m = LAYER ? q[1] * p.inv_dim : 0.0f;
      }
      by_runs([&](int i) {
        if (p.post) {
#pragma unroll
          for (int e = 8 * i; e < 8 * i + 8; ++e) d[e] = r_post * (d[e] - fmaf(v[e], am, m));
        }
        if (p.dy.p && live) store_run(at<T>(p.dy, b, tok), l, d, i);
      });
    }
    if (SUMS && p.gate_unit) {
      flush(gg, p.gate_part + (int64_t)unit * p.dim);
#pragma unroll
      for (int e = 0; e < E; ++e) gg[e] = 0.0f;
    }
  }
  if (!SUMS || !p.part) return;
  float* part = p.part + (int64_t)blockIdx.x * 4 * p.dim;
  if (p.wanted & 1) flush(pg, part);
  if (p.wanted & 2) flush(pb, part + p.dim);
  if (p.wanted & 4) flush(qg, part + 2 * p.dim);
  if (p.wanted & 8) flush(qb, part + 3 * p.dim);
  if ((p.wanted & 16) && !p.gate_unit) flush(gg, p.gate_part + (int64_t)blockIdx.x * p.dim);
}

// The sums of the weights' gradients of rows too long to have them in registers beside the row, from the rows
// and what the kernel above wrote of each: a thread has eight columns, a wave the rows of its units.
template <typename T, typename S, bool LAYER, bool CUT>
__global__ __launch_bounds__(64) void block_columns_kernel(BlockP p) {
  typedef Place<64, 1, CUT> L;
  const L l(p.dim, blockIdx.y * 64 + threadIdx.x);
  float pg[8], pb[8], qg[8], qb[8], gg[8], w_pre[8], w_post[8], b_post[8], w_gate[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) pg[e] = pb[e] = qg[e] = qb[e] = gg[e] = 0.0f;
  load_weight(p.pre_gamma, 1.0f, l, w_pre);
  load_weight(p.post_gamma, 1.0f, l, w_post);
  load_weight(p.post_beta, 0.0f, l, b_post);
  load_weight(p.gate, 1.0f, l, w_gate);
  auto put = [&](const float (&v)[8], float* out) {
    if (l.there(0)) store_run(out, l, v, 0);
  };
  const bool rest = p.has_y && (p.wanted & 28);   // sums that need y and the gradient of x'
  const int units = p.batch * p.slices;
  for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int b = unit / p.slices, slice = unit - b * p.slices;
    const int n = p.lens ? max(0, min(p.tokens, p.lens[b])) : p.tokens;
    const int share = (n + p.slices - 1) / p.slices, first = slice * share, last = min(n, first + share);
    if (p.gate_ld) load_weight(p.gate + b * p.gate_ld, 1.0f, l, w_gate);
#pragma unroll 2
    for (int tok = first; tok < last; ++tok) {
      const float* o = p.stats + ((int64_t)b * p.tokens + tok) * kStats;
      float d[8] = {}, x[8];
      if (p.du.p) {
        Raw<L, T> ru;
        Raw<L, S> rx;
        ru.load(at<const T>(p.du, b, tok), true, l);
        rx.load(at<const S>(p.x_out, b, tok), true, l);
        ru.get(d, l);
        rx.get(x, l);
        if constexpr (LAYER) l.subtract(x, o[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float xn = x[e] * o[1];
          if constexpr (LAYER) pb[e] += d[e];
          pg[e] = fmaf(d[e], xn, pg[e]);
          d[e] = o[1] * fmaf(d[e], w_pre[e], -xn * o[2]);
        }
        if constexpr (LAYER) l.subtract(d, o[3]);
      }
      if (!rest) continue;
      float v[8];
      Raw<L, T> ry;
      ry.load(at<const T>(p.y, b, tok), true, l);
      if (p.dx_out.p) {
        Raw<L, S> rd;
        rd.load(at<const S>(p.dx_out, b, tok), true, l);
        rd.get(x, l);
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] += x[e];
      }
      ry.get(v, l);
      if (LAYER && p.post) l.subtract(v, o[4]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] *= o[5];
        gg[e] = fmaf(d[e], fmaf(v[e], w_post[e], b_post[e]), gg[e]);
        d[e] *= w_gate[e];
        qg[e] = fmaf(d[e], v[e], qg[e]);
        if constexpr (LAYER) qb[e] += d[e];
      }
    }
    if (p.gate_unit) {
      put(gg, p.gate_part + (int64_t)unit * p.dim);
#pragma unroll
      for (int e = 0; e < 8; ++e) gg[e] = 0.0f;
    }
  }
  float* part = p.part + (int64_t)blockIdx.x * 4 * p.dim;
  if (p.wanted & 1) put(pg, part);
  if (p.wanted & 2) put(pb, part + p.dim);
  if (p.wanted & 4) put(qg, part + 2 * p.dim);
  if (p.wanted & 8) put(qb, part + 3 * p.dim);
  if ((p.wanted & 16) && !p.gate_unit) put(gg, p.gate_part + (int64_t)blockIdx.x * p.dim);
}

// Column sums of the parts, 64 columns a workgroup, 16 slices of the parts.
struct SumP {
  const float *part, *gate_part;
  float* out[kSums];
  int dim, parts;
  int gate_parts;  // of each gate
};
__global__ __launch_bounds__(1024) void block_sum_kernel(SumP p) {
  __shared__ float red[16][65];
  // The gates' gradients are further rows of the grid.
  const int sum = min((int)blockIdx.y, 4), gate = blockIdx.y - sum;
  float* out = p.out[sum];
  if (!out) return;
  const int n = sum == 4 ? p.gate_parts : p.parts;
  const int64_t ld = sum == 4 ? p.dim : 4 * (int64_t)p.dim;
  const float* from = sum == 4 ? p.gate_part + (int64_t)gate * n * p.dim : p.part + sum * (int64_t)p.dim;
  const int lane = threadIdx.x & 63, sl = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float s = 0.0f;
  if (c < p.dim)
#pragma unroll 8
    for (int i = sl; i < n; i += 16) s += from[i * ld + c];
  red[sl][lane] = s;
  __syncthreads();
  if (sl != 0 || c >= p.dim) return;
  s = 0.0f;
  for (int i = 0; i < 16; ++i) s += red[i][lane];
  out[(int64_t)gate * p.dim + c] = s;
}

// The gradients of a batch of no tokens.
__global__ __launch_bounds__(256) void block_zero_kernel(float* out, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) out[i] = 0.0f;
}

// ---------------------------------------------------------------- host

// Threads of a row and runs of eight a thread: as few as hold the row, so that short rows share a wave (281536
// rows of 40: a wave each 119 us, four a wave 32).
struct Width {
  int threads, runs;
};
// Forward: rows of up to 1024 in one wave, which needs no barrier.
Width forward_width(int dim) {
  if (dim <= 128) return {16, 1};
  if (dim <= 256) return {32, 1};
  if (dim <= 512) return {64, 1};
  if (dim <= 1024) return {64, 2};
  if (dim <= 2048) return {128, 2};
  if (dim <= 4096) return {256, 2};
  if (dim <= 8192) return {512, 2};
  return {1024, 2};
}
// Backward: eight values a thread, so that the sums, the weights and the next row's loads stay in
// registers.
Width backward_width(int dim) {
  if (dim <= 128) return {16, 1};
  if (dim <= 256) return {32, 1};
  if (dim <= 512) return {64, 1};
  if (dim <= 1024) return {128, 1};
  if (dim <= 2048) return {256, 1};
  if (dim <= 4096) return {512, 1};
  if (dim <= 8192) return {1024, 1};
  return {1024, 2};
}
// Workgroups of a forward launch: what the GPU holds, several times over for rows of one wave.
int forward_blocks(int dim) { return dim <= 4096 ? 256 * 8 : 256 * 4; }
// Backward: the workgroups that the GPU holds, three a CU of rows of up to 2048 (kept to a third of its
// registers: 243 -> 166 us where they took 190 and two ran; 50432 rows of 768, layer norm, 192 -> 109), and the
// units that they share out (below; with as many as workgroups 175 us, with four times as many 175).
int grad_blocks(Width w) { return w.threads <= 256 ? 768 : w.runs > 1 ? 128 : 256; }
int units_of(Width w) { return 2 * grad_blocks(w); }
int rows_of(Width w) { return workgroup(w.threads) / w.threads; }

template <typename T, typename S, bool LAYER, bool CUT>
void launch_forward(const BlockP& p, unsigned grid, hipStream_t s) {
  const Width w = forward_width(p.dim);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(workgroup(w.threads)), 0, s, p); };
  switch (w.threads * 2 + w.runs) {
    case 33: return go(block_norm_kernel<T, S, LAYER, CUT, 16, 1>);
    case 65: return go(block_norm_kernel<T, S, LAYER, CUT, 32, 1>);
    case 129: return go(block_norm_kernel<T, S, LAYER, CUT, 64, 1>);
    case 130: return go(block_norm_kernel<T, S, LAYER, CUT, 64, 2>);
    case 258: return go(block_norm_kernel<T, S, LAYER, CUT, 128, 2>);
    case 514: return go(block_norm_kernel<T, S, LAYER, CUT, 256, 2>);
    case 1026: return go(block_norm_kernel<T, S, LAYER, CUT, 512, 2>);
    default: return go(block_norm_kernel<T, S, LAYER, CUT, 1024, 2>);
  }
}
template <typename T, typename S, bool LAYER, bool CUT>
void launch_backward(const BlockP& p, unsigned grid, hipStream_t s) {
  const Width w = backward_width(p.dim);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(workgroup(w.threads)), 0, s, p); };
  switch (w.threads * 2 + w.runs) {
    case 33: return go(block_norm_bwd_kernel<T, S, LAYER, CUT, 16, 1>);
    case 65: return go(block_norm_bwd_kernel<T, S, LAYER, CUT, 32, 1>);
    case 129: return go(block_norm_bwd_kernel<T, S, LAYER, CUT, 64, 1>);
    case 257: return go(block_norm_bwd_kernel<T, S, LAYER, CUT, 128, 1>);
    case 513: return go(block_norm_bwd_kernel<T, S, LAYER, CUT, 256, 1>);
    case 1025: return go(block_norm_bwd_kernel<T, S, LAYER, CUT, 512, 1>);
    // A layer norm in fp32 runs with CUT in any case, which spills 10 registers instead of 43 (6000 rows of
    // 6144: 363 -> 277 us; bf16, where it spills none instead of 19, 176 -> 206).
    case 2049: return go(block_norm_bwd_kernel<T, S, LAYER, CUT || (LAYER && sizeof(T) == 4), 1024, 1>);
    default: return go(block_norm_bwd_kernel<T, S, LAYER, CUT, 1024, 2>);
  }
}

enum class Pass { kForward, kBackward, kColumns };
template <typename T, typename S>
void launch_kind(const BlockP& p, Pass pass, unsigned grid, hipStream_t s) {
  auto kind = [&](auto layer, auto cut) {
    constexpr bool LAYER = decltype(layer)::value, CUT = decltype(cut)::value;
    if (pass == Pass::kForward) return launch_forward<T, S, LAYER, CUT>(p, grid, s);
    if (pass == Pass::kBackward) return launch_backward<T, S, LAYER, CUT>(p, grid, s);
    hipLaunchKernelGGL((block_columns_kernel<T, S, LAYER, CUT>), dim3(grid, (unsigned)((p.dim + 511) / 512)), dim3(64),
                       0, s, p);
  };
  auto dims = [&](auto layer) { p.dim % 8 ? kind(layer, std::true_type()) : kind(layer, std::false_type()); };
  p.layer ? dims(std::true_type()) : dims(std::false_type());
}
void launch_types(const BlockP& p, bool bf16, bool stream_bf16, Pass pass, unsigned grid, hipStream_t s) {
  if (!bf16) return launch_kind<float, float>(p, pass, grid, s);
  if (stream_bf16) return launch_kind<uint16_t, uint16_t>(p, pass, grid, s);
  launch_kind<uint16_t, float>(p, pass, grid, s);
}

bool check_sizes(const elasto_block_norm_t* d) {
  if (!d) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: NULL description"), false;
  const bool types = (d->dtype == ELASTO_BF16 && (d->stream_dtype == ELASTO_BF16 || d->stream_dtype == ELASTO_FP32)) ||
                     (d->dtype == ELASTO_FP32 && d->stream_dtype == ELASTO_FP32);
  if (!types) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: bad dtypes %d and %d", d->dtype, d->stream_dtype), false;
  if (d->batch < 0 || d->tokens < 0 || d->dim < 1 || d->dim > kMaxDim || (int64_t)d->batch * d->tokens > (1 << 25))
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: bad batch, tokens or dim"), false;
  return true;
}

// Every sequence is cut into as many runs of its own rows; a workgroup takes runs a grid apart, so runs
// of sequences of all lengths.
struct Slices {
  int per;    // of a sequence
  int units;  // of all
  int grid;
};
Slices slices_of(const elasto_block_norm_t& d) {
  const Width w = backward_width(d.dim);
  const int r = rows_of(w);
  const int blocks = grad_blocks(w);
  const int64_t rounds = (d.tokens + r - 1) / r;
  const int64_t per = std::max<int64_t>(1, std::min<int64_t>(rounds, units_of(w) / std::max(1, d.batch)));
  const int64_t units = (int64_t)d.batch * per;
  return {(int)per, (int)units, (int)std::min<int64_t>(units, blocks)};
}
// Bytes of the parts: of the weights' sums by workgroups, of the gate's by units or workgroups (a unit that
// has a whole sequence writes the gate's gradient itself).
int64_t part_bytes(const Slices& s, int dim) { return (int64_t)s.grid * 4 * dim * 4; }
int64_t stats_bytes(const elasto_block_norm_t& d) {
  return backward_width(d.dim).runs > 1 ? (int64_t)d.batch * d.tokens * kStats * 4 : 0;
}
int64_t gate_bytes(const Slices& s, int dim) { return s.per > 1 ? (int64_t)s.units * dim * 4 : (int64_t)s.grid * dim * 4; }

bool check_desc(const elasto_block_norm_t* d) {
  if (!check_sizes(d)) return false;
  if (d->kind != ELASTO_NORM_RMS && d->kind != ELASTO_NORM_LAYER)
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: bad kind %d", d->kind), false;
  if (!(d->eps >= 1.17549435e-38f) || !(d->eps < INFINITY) || !(fabsf(d->residual_scale) < INFINITY))
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: eps must be a positive normal number, residual_scale finite"), false;
  if (!d->post_norm && (d->post_gamma || d->post_beta))
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: weights without their norm"), false;
  if (d->kind == ELASTO_NORM_RMS && (d->pre_beta || d->post_beta))
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: the RMS norm has no beta"), false;
  for (const void* p : {(const void*)d->pre_gamma, (const void*)d->pre_beta, (const void*)d->post_gamma,
                        (const void*)d->post_beta, (const void*)d->gate, (const void*)d->lens})
    if (!aligned(p, 4)) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: misaligned pointer"), false;
  return true;
}

// *r from t (NULL or of no data: r->p stays NULL).
bool take(const char* name, const elasto_rows_t* t, const elasto_block_norm_t& d, int es, bool needed, bool written,
          Rows* r) {
  *r = Rows{nullptr, 0, 0};
  if (!t || !t->data) {
    if (needed) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: %s is NULL", name), false;
    return true;
  }
  if (!aligned(t->data, es)) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: %s is misaligned", name), false;
  if (t->batch_stride < 0 || t->token_stride < 0)
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: %s has a negative stride", name), false;
  if (written && ((d.batch > 1 && t->batch_stride < d.dim) || (d.tokens > 1 && t->token_stride < d.dim)))
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: rows of %s overlap", name), false;
  *r = Rows{static_cast<char*>(t->data), t->batch_stride * es, t->token_stride * es};
  return true;
}

BlockP params(const elasto_block_norm_t& d) {
  BlockP p = {};
  p.pre_gamma = d.pre_gamma;
  p.pre_beta = d.pre_beta;
  p.post_gamma = d.post_gamma;
  p.post_beta = d.post_beta;
  p.gate = d.gate;
  p.gate_ld = d.gate && d.gate_per_sequence ? d.dim : 0;  // no gate: no sequence's place behind NULL
  p.lens = d.lens;
  p.batch = d.batch;
  p.tokens = d.tokens;
  p.dim = d.dim;
  p.layer = d.kind == ELASTO_NORM_LAYER;
  p.post = d.post_norm != 0;
  p.a = d.residual_scale;
  p.eps = d.eps;
  p.inv_dim = 1.0f / (float)d.dim;
  return p;
}

}  // namespace
}  // namespace elasto

using namespace elasto;

extern "C" {

elasto_status_t elasto_op_block_norm(const elasto_block_norm_t* d, const elasto_rows_t* x, const elasto_rows_t* y,
                                     const elasto_rows_t* x_out, const elasto_rows_t* u, void* hip_stream) {
  if (!check_desc(d)) return ELASTO_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)d->batch * d->tokens;
  if (rows == 0) return ELASTO_OK;
  const int es = d->dtype == ELASTO_BF16 ? 2 : 4, ss = d->stream_dtype == ELASTO_BF16 ? 2 : 4;
  BlockP p = params(*d);
  if (!take("x", x, *d, ss, true, false, &p.x) || !take("y", y, *d, es, false, false, &p.y) ||
      !take("x_out", x_out, *d, ss, false, true, &p.x_out) || !take("u", u, *d, es, false, true, &p.u))
    return ELASTO_ERR_INVALID_ARG;
  p.has_y = p.y.p != nullptr;
  if (!p.x_out.p && !p.u.p) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: neither x_out nor u is asked for");
  if (!p.has_y && (p.post || p.gate)) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: a norm or gate of no y");
  const int per = rows_of(forward_width(d->dim));
  const unsigned grid = (unsigned)std::min<int64_t>((rows + per - 1) / per, forward_blocks(d->dim));
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  launch_types(p, es == 2, ss == 2, Pass::kForward, grid, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "block_norm: %s", hipGetErrorString(e));
  return ELASTO_OK;
}

elasto_status_t elasto_op_block_norm_bwd(const elasto_block_norm_t* d, const elasto_rows_t* x_out,
                                         const elasto_rows_t* y, const elasto_rows_t* dx_out,
                                         const elasto_rows_t* du, const elasto_rows_t* dx, const elasto_rows_t* dy,
                                         float* d_pre_gamma, float* d_pre_beta, float* d_post_gamma,
                                         float* d_post_beta, float* d_gate, void* workspace,
                                         int64_t workspace_bytes, void* hip_stream) {
  if (!check_desc(d)) return ELASTO_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)d->batch * d->tokens;
  const int es = d->dtype == ELASTO_BF16 ? 2 : 4, ss = d->stream_dtype == ELASTO_BF16 ? 2 : 4;
  BlockP p = params(*d);
  if (rows > 0) {
    if (!take("x_out", x_out, *d, ss, du && du->data, false, &p.x_out) || !take("y", y, *d, es, false, false, &p.y) ||
        !take("dx_out", dx_out, *d, ss, false, false, &p.dx_out) || !take("du", du, *d, es, false, false, &p.du) ||
        !take("dx", dx, *d, ss, false, true, &p.dx) || !take("dy", dy, *d, es, false, true, &p.dy))
      return ELASTO_ERR_INVALID_ARG;
    p.has_y = p.y.p != nullptr;
    if (!p.dx_out.p && !p.du.p) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: neither dx_out nor du is given");
    if (!p.has_y && (p.post || p.gate || p.dy.p))
      return fail(ELASTO_ERR_INVALID_ARG, "block_norm: a norm, gate or gradient of no y");
    if (!p.du.p && (d_pre_gamma || d_pre_beta))
      return fail(ELASTO_ERR_INVALID_ARG, "block_norm: gradients of pre_gamma and pre_beta need du");
  }
  if ((d_post_gamma || d_post_beta) && !d->post_norm)
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: gradients of weights without their norm");
  if ((d_pre_beta || d_post_beta) && d->kind == ELASTO_NORM_RMS)
    return fail(ELASTO_ERR_INVALID_ARG, "block_norm: the RMS norm has no beta");
  if (d_gate && !d->gate) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: the gradient of no gate");
  float* const out[kSums] = {d_pre_gamma, d_pre_beta, d_post_gamma, d_post_beta, d_gate};
  for (int i = 0; i < kSums; ++i) {
    if (!aligned(out[i], 4)) return fail(ELASTO_ERR_INVALID_ARG, "block_norm: misaligned pointer");
    if (out[i]) p.wanted |= 1 << i;
  }
  const bool per_sequence = d->gate_per_sequence != 0;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipSuccess;
  if (rows == 0) {
    for (int i = 0; i < kSums && e == hipSuccess; ++i) {
      const int64_t n = (i == 4 && per_sequence ? (int64_t)d->batch : 1) * d->dim;
      if (!out[i] || n == 0) continue;
      hipLaunchKernelGGL(block_zero_kernel, dim3((unsigned)std::min<int64_t>((n + 255) / 256, 4096)), dim3(256), 0, s,
                         out[i], n);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "block_norm: %s", hipGetErrorString(e));
    return ELASTO_OK;
  }
  const Slices sl = slices_of(*d);
  p.slices = sl.per;
  p.gate_unit = d_gate && per_sequence;
  const bool direct = p.gate_unit && sl.per == 1;
  const int sums = p.wanted & ~(direct ? 16 : 0);
  const bool columns = p.wanted && backward_width(d->dim).runs > 1;
  if (sums || columns) {
    const int64_t need = part_bytes(sl, d->dim) + gate_bytes(sl, d->dim) + stats_bytes(*d);
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < need)
      return fail(ELASTO_ERR_INVALID_ARG, "block_norm: the workspace holds %lld of %lld bytes",
                  (long long)(workspace ? workspace_bytes : 0), (long long)need);
    p.part = static_cast<float*>(workspace);
    p.gate_part = p.part + part_bytes(sl, d->dim) / 4;
    if (columns) p.stats = p.gate_part + gate_bytes(sl, d->dim) / 4;
  }
  if (direct) p.gate_part = d_gate;
  if (columns) {
    // The columns are summed from the rows as they were: where the gradients take their place, a pass that
    // writes none comes first.
    BlockP first = p;
    const bool over = (p.dx.p && (p.dx.p == p.x_out.p || p.dx.p == p.dx_out.p)) ||
                      (p.dy.p && (p.dy.p == p.du.p || p.dy.p == p.y.p));
    if (over) first.dx.p = first.dy.p = nullptr;
    const unsigned grid = (unsigned)std::min(sl.units, 256);
    launch_types(first, es == 2, ss == 2, Pass::kBackward, grid, s);
    launch_types(p, es == 2, ss == 2, Pass::kColumns, (unsigned)sl.grid, s);
    p.stats = nullptr;
    if (over) launch_types(p, es == 2, ss == 2, Pass::kBackward, grid, s);
  } else {
    launch_types(p, es == 2, ss == 2, Pass::kBackward, (unsigned)sl.grid, s);
  }
  e = hipGetLastError();
  if (e == hipSuccess && sums) {
    SumP q = {};
    q.part = p.part;
    q.gate_part = p.gate_part;
    for (int i = 0; i < kSums; ++i) q.out[i] = i == 4 && direct ? nullptr : out[i];
    q.dim = d->dim;
    q.parts = sl.grid;
    q.gate_parts = per_sequence ? sl.per : sl.grid;
    const unsigned gates = !q.out[4] ? 0 : per_sequence ? (unsigned)d->batch : 1;
    hipLaunchKernelGGL(block_sum_kernel, dim3((unsigned)((d->dim + 63) / 64), 4 + gates), dim3(1024), 0, s, q);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "block_norm: %s", hipGetErrorString(e));
  return ELASTO_OK;
}

elasto_status_t elasto_block_norm_workspace(const elasto_block_norm_t* d, int64_t* bytes) {
  if (!bytes) return fail(ELASTO_ERR_INVALID_ARG, "NULL argument");
  if (!check_sizes(d)) return ELASTO_ERR_INVALID_ARG;
  const Slices s = slices_of(*d);
  *bytes = part_bytes(s, d->dim) + gate_bytes(s, d->dim) + stats_bytes(*d);
  return ELASTO_OK;
}

}  // extern "C"
