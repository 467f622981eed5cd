// What lies between two blocks of a transformer, in one pass over the tokens: the norm behind a
// block, its gate, the residual addition and the norm ahead of the next block.
//   n = N_post(y)  (or y),  x' = a x + g (.) n,  u = N_pre(x'),
//   N(v) = (v - mean) r (.) gamma + beta,  r = 1 / sqrt(mean((v - mean)^2) + eps)
// (RMS: mean = 0).  Backward, with v^ = (v - mean) r and N'(d) = r (d gamma - v^ mean(d gamma v^)
// - mean(d gamma)) (RMS: without the last term):
//   dX = dx' + N_pre'(du),  dx = a dX,  dn = g (.) dX,  dy = N_post'(dn)  (or dn),
//   dgamma = sum d v^ and dbeta = sum d over the tokens, dg = sum dX (.) n over a gate's tokens.
//
// A row is held in the registers of one to sixteen waves and read once; its statistics are taken in
// the registers, about the row's mean (each wave about its own, joined by the pairwise update of
// Chan, Golub and LeVeque), so a large mean costs no digits.  Everything between the load and the
// store is fp32; u is taken from x' before x' is rounded.  Backward, a workgroup walks the rows of
// one gate (or a part of them) and sums the weights' gradients of its columns in registers; the
// parts are summed by a second kernel in a fixed order.
//
// Bound by memory: forward four passes over the tokens, backward six.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "heads.h"

namespace elasto {
namespace {

constexpr int kMaxDim = 16384;
constexpr int kSums = 5;                   // pre gamma, pre beta, post gamma, post beta, gate

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
};

// Values of a row in the registers of a thread: E of them, in runs of 8 where WIDE.
template <int W, int CH, bool WIDE>
struct Place {
  static constexpr int E = 8 * CH, T = 64 * W;
  // Column of value e of thread t of the row's.
  static __device__ __forceinline__ int column(int e, int t) {
    return WIDE ? ((e >> 3) * T + t) * 8 + (e & 7) : e * T + t;
  }
};

__device__ __forceinline__ void load_run(const float* p, float* v) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
__device__ __forceinline__ void store_run(uint16_t* p, const float* v) {
  *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                       pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void store_run(float* p, const float* v) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ float load_value(const uint16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ float load_value(const float* p) { return *p; }
__device__ __forceinline__ void store_value(uint16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }

template <typename L, bool WIDE, typename T>
__device__ __forceinline__ void load_row(const T* p, int dim, int t, float (&v)[L::E], float none = 0.0f) {
  if constexpr (WIDE) {
#pragma unroll
    for (int e = 0; e < L::E; e += 8) {
      const int c = L::column(e, t);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[e + i] = none;
      if (c < dim) load_run(p + c, v + e);
    }
  } else {
#pragma unroll
    for (int e = 0; e < L::E; ++e) {
      const int c = L::column(e, t);
      v[e] = c < dim ? load_value(p + c) : none;
    }
  }
}
template <typename L, bool WIDE, typename T>
__device__ __forceinline__ void store_row(T* p, int dim, int t, const float (&v)[L::E]) {
#pragma unroll
  for (int e = 0; e < L::E; e += WIDE ? 8 : 1) {
    const int c = L::column(e, t);
    if (c >= dim) continue;
    if constexpr (WIDE)
      store_run(p + c, v + e);
    else
      store_value(p + c, v[e]);
  }
}

// The sum over a wave, in all lanes: in rows of 16 by lane moves of the adder itself, then the four
// rows' sums in their order.
template <int CTRL>
__device__ __forceinline__ float add_moved(float v) {
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                 0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum_of_wave(float v) {
  v = add_moved<0xB1>(v);   // lane ^ 1
  v = add_moved<0x4E>(v);   // lane ^ 2
  v = add_moved<0x141>(v);  // the other quad of eight
  v = add_moved<0x140>(v);  // the other eight of a row
  auto row = [&](int r) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 16 * r)); };
  return (row(0) + row(1)) + (row(2) + row(3));
}

// Sums over a row's W waves, the waves' through LDS: two buffers in turn, so that one barrier does for
// each exchange (who writes a buffer again has passed the barrier behind which all have read it).
constexpr int kMost = 3;  // sums of an exchange
template <int W>
struct Exchange {
  float* buf;  // [2][W][kMost]
  int turn = 0;
  template <int N>
  __device__ __forceinline__ void operator()(float (&v)[N], int t) {
    static_assert(N <= kMost, "room");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum_of_wave(v[i]);
    if constexpr (W > 1) {
      float* b = buf + turn * W * kMost;
      turn ^= 1;
      if ((t & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) b[(t >> 6) * kMost + i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = b[i];
#pragma unroll
        for (int k = 1; k < W; ++k) v[i] += b[k * kMost + i];
      }
    }
  }
};

template <typename T>
__device__ __forceinline__ T* at(const Rows& r, int b, int t) {
  return reinterpret_cast<T*>(r.p + b * r.sb + t * r.st);
}

// A row as it was loaded.
template <typename L, bool WIDE, typename T>
struct Raw {
  static constexpr bool kPacked = WIDE && sizeof(T) == 2;
  u32x4 w[kPacked ? L::E / 8 : 1];
  float f[kPacked ? 1 : L::E];
  __device__ __forceinline__ void load(const T* p, bool there, int dim, int t) {
    if constexpr (kPacked) {
#pragma unroll
      for (int i = 0; i < L::E / 8; ++i) {
        const int c = L::column(8 * i, t);
        w[i] = u32x4{0, 0, 0, 0};
        if (there && c < dim) w[i] = *reinterpret_cast<const u32x4*>(p + c);
      }
    } else if (there) {
      load_row<L, WIDE>(p, dim, t, f);
    } else {
#pragma unroll
      for (int e = 0; e < L::E; ++e) f[e] = 0.0f;
    }
  }
  __device__ __forceinline__ void get(float (&v)[L::E]) const {
#pragma unroll
    for (int e = 0; e < L::E; ++e) {
      if constexpr (kPacked)
        v[e] = __uint_as_float((e & 1) ? (w[e >> 3][(e & 7) >> 1] & 0xffff0000u) : (w[e >> 3][(e & 7) >> 1] << 16));
      else
        v[e] = f[e];
    }
  }
};

template <typename L, bool WIDE>
__device__ __forceinline__ void load_weight(const float* w, float none, int dim, int t, float (&v)[L::E]) {
  if (w)
    load_row<L, WIDE>(w, dim, t, v, none);
  else
#pragma unroll
    for (int e = 0; e < L::E; ++e) v[e] = none;
}

// 1 where a thread's column is there, 0 where it is not (a run of eight is there or not: dim is a multiple
// of 8 where rows are read in runs).  What is loaded from columns that are not there is 0, so only what is
// added to a whole row needs it.
template <typename L, bool WIDE>
struct There {
  float m[WIDE ? L::E / 8 : L::E];
  __device__ __forceinline__ There(int dim, int t) {
#pragma unroll
    for (int i = 0; i < (WIDE ? L::E / 8 : L::E); ++i) m[i] = L::column(WIDE ? 8 * i : i, t) < dim ? 1.0f : 0.0f;
  }
  // less[e] where the column is there: computed once a run.
  __device__ __forceinline__ void from(float (&v)[L::E], float less) const {
#pragma unroll
    for (int i = 0; i < (WIDE ? L::E / 8 : L::E); ++i) {
      const float k = less * m[i];
#pragma unroll
      for (int e = 0; e < (WIDE ? 8 : 1); ++e) v[(WIDE ? 8 : 1) * i + e] -= k;
    }
  }
};

// Whether the weights and the next row's loads stay in registers: not forward for rows of 16 waves (which
// have 128 registers), nor backward.
template <int W>
constexpr bool kKeepForward = W < 16;
template <int CH>
constexpr bool kKeepBackward = CH == 1;

// T: of y and u.  S: of the stream.  W waves a row; a workgroup of 256 threads holds 4 / W rows.  A group of
// W waves takes rows in strides of the grid's, the next one's loads in flight, the weights in registers.
template <typename T, typename S, bool LAYER, int W, int CH, bool WIDE>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256) void block_norm_kernel(BlockP p) {
  typedef Place<W, CH, WIDE> L;
  constexpr int E = L::E, R = W > 4 ? 1 : 4 / W;
  constexpr bool KEEP = kKeepForward<W>;
  __shared__ float red[R][2 * W * kMost];
  const int t = threadIdx.x % L::T, mine = __builtin_amdgcn_readfirstlane(threadIdx.x / L::T);
  Exchange<W> exchange = {red[mine]};
  const There<L, WIDE> there(p.dim, t);
  const int rows = p.batch * p.tokens, stride = gridDim.x * R;
  float pg[E], pb[E], qg[E], qb[E], g[E];
  auto pre = [&] {
    load_weight<L, WIDE>(p.pre_gamma, 1.0f, p.dim, t, pg);
    if constexpr (LAYER) load_weight<L, WIDE>(p.pre_beta, 0.0f, p.dim, t, pb);
  };
  auto post = [&] {
    load_weight<L, WIDE>(p.post_gamma, 1.0f, p.dim, t, qg);
    if constexpr (LAYER) load_weight<L, WIDE>(p.post_beta, 0.0f, p.dim, t, qb);
  };
  if (KEEP && p.u.p) pre();
  if (KEEP && p.post) post();
  if (KEEP) load_weight<L, WIDE>(p.gate, 1.0f, p.dim, t, g);  // of the first sequence, or of all
  int gate_of = 0;
  Raw<L, WIDE, S> rx;
  Raw<L, WIDE, T> ry;
  int b = 0, tok = 0;
  bool live = false;
  auto fetch = [&](int row) {
    live = row < rows;
    const int r = live ? row : 0;
    b = (int)((unsigned)r / (unsigned)p.tokens);
    tok = r - b * p.tokens;
    if (live && p.lens) live = tok < p.lens[b];
    rx.load(at<const S>(p.x, b, tok), live, p.dim, t);
    if (p.has_y) ry.load(at<const T>(p.y, b, tok), live, p.dim, t);
  };
  // All rows of a workgroup take as many rounds: with W > 1 they meet at its barriers.
  int row = blockIdx.x * R;
  if (KEEP) fetch(row + mine);
  for (; row < rows; row += stride) {
    if (!KEEP) fetch(row + mine);
    float x[E], v[E];
    rx.get(x);
    const bool now = live;
    const int nb = b, nt = tok;
    if (p.has_y) {
      ry.get(v);
      if (KEEP && row + stride < rows) fetch(row + stride + mine);
      if (p.post) {
        if constexpr (LAYER) {
          float s[1] = {0.0f};
#pragma unroll
          for (int e = 0; e < E; ++e) s[0] += v[e];
          exchange(s, t);
          there.from(v, s[0] * p.inv_dim);
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
      if (!KEEP && !p.gate_ld) load_weight<L, WIDE>(p.gate, 1.0f, p.dim, t, g);
      if (p.gate_ld && (!KEEP || nb != gate_of)) {
        load_weight<L, WIDE>(p.gate + nb * p.gate_ld, 1.0f, p.dim, t, g);
        gate_of = nb;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = fmaf(p.a, x[e], g[e] * v[e]);
    } else {
      if (KEEP && row + stride < rows) fetch(row + stride + mine);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] *= p.a;
    }
    if (now && p.x_out.p) store_row<L, WIDE>(at<S>(p.x_out, nb, nt), p.dim, t, x);
    if (!p.u.p) continue;
    if constexpr (LAYER) {
      float s[1] = {0.0f};
#pragma unroll
      for (int e = 0; e < E; ++e) s[0] += x[e];
      exchange(s, t);
      there.from(x, s[0] * p.inv_dim);
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < E; ++e) q[0] = fmaf(x[e], x[e], q[0]);
    exchange(q, t);
    const float r = 1.0f / sqrtf(fmaf(q[0], p.inv_dim, p.eps));
    if (!KEEP) pre();
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = LAYER ? fmaf(x[e] * r, pg[e], pb[e]) : x[e] * r * pg[e];
    if (now) store_row<L, WIDE>(at<T>(p.u, nb, nt), p.dim, t, x);
  }
}

// Three exchanges a row (RMS: two): sums for the means; about them, with what both norms need that the
// gradient of x' does not wait for; and the norm behind the block's.
template <typename T, typename S, bool LAYER, int W, int CH, bool WIDE>
__global__ __launch_bounds__(W > 4 ? 64 * W : 256, W > 4 ? 1 : 3) void block_norm_bwd_kernel(BlockP p) {
  typedef Place<W, CH, WIDE> L;
  constexpr int E = L::E, R = W > 4 ? 1 : 4 / W;
  constexpr bool KEEP = kKeepBackward<CH>;
  __shared__ float red[R][2 * W * kMost];
  __shared__ float sums[R > 1 ? (R - 1) * L::T : 1];
  const int t = threadIdx.x % L::T, mine = __builtin_amdgcn_readfirstlane(threadIdx.x / L::T);
  Exchange<W> exchange = {red[mine]};
  const There<L, WIDE> there(p.dim, t);
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
        if (mine > 0) sums[(mine - 1) * L::T + t] = s;
        __syncthreads();
        if (mine == 0)
#pragma unroll
          for (int k = 0; k < R - 1; ++k) s += sums[k * L::T + t];
      }
      const int c = L::column(e, t);
      if (mine == 0 && c < p.dim) out[c] = s;
    }
  };
  float w_pre[E], w_post[E], b_post[E], w_gate[E];
  auto post = [&] {
    load_weight<L, WIDE>(p.post_gamma, 1.0f, p.dim, t, w_post);
    if constexpr (LAYER) load_weight<L, WIDE>(p.post_beta, 0.0f, p.dim, t, b_post);
  };
  if (KEEP) {
    load_weight<L, WIDE>(p.pre_gamma, 1.0f, p.dim, t, w_pre);
    if (p.post) post();
    load_weight<L, WIDE>(p.gate, 1.0f, p.dim, t, w_gate);
  }
  const int units = p.batch * p.slices;
  for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int b = unit / p.slices, slice = unit - b * p.slices;
    const int n = p.lens ? max(0, min(p.tokens, p.lens[b])) : p.tokens;
    const int share = (n + p.slices - 1) / p.slices, first = slice * share, last = min(n, first + share);
    if (KEEP && p.gate_ld) load_weight<L, WIDE>(p.gate + b * p.gate_ld, 0.0f, p.dim, t, w_gate);
    Raw<L, WIDE, S> rx, rd;
    Raw<L, WIDE, T> ru, ry;
    auto fetch = [&](int tok) {
      const bool live = tok < last;
      const int k = live ? tok : 0;
      if (p.du.p) {
        ru.load(at<const T>(p.du, b, k), live, p.dim, t);
        rx.load(at<const S>(p.x_out, b, k), live, p.dim, t);
      }
      if (p.has_y) ry.load(at<const T>(p.y, b, k), live, p.dim, t);
      if (p.dx_out.p) rd.load(at<const S>(p.dx_out, b, k), live, p.dim, t);
    };
    if (KEEP && first < last) fetch(first + mine);
    // Every row of a workgroup takes as many rounds: they meet at its barriers.
    for (int k = first; k < last; k += R) {
      const int tok = k + mine;
      const bool live = tok < last;
      if (!KEEP) {
        fetch(tok);
        load_weight<L, WIDE>(p.pre_gamma, 1.0f, p.dim, t, w_pre);
      }
      float d[E], x[E], v[E], s[3] = {0.0f, 0.0f, 0.0f};
      if (p.du.p) {
        ru.get(d);
        rx.get(x);
        if constexpr (LAYER)
#pragma unroll
          for (int e = 0; e < E; ++e) pb[e] += d[e];
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = x[e] = 0.0f;
      }
      if (p.has_y)
        ry.get(v);
      else
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = 0.0f;
      float c = 0.0f;
      if constexpr (LAYER) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          s[0] += x[e];
          s[1] += v[e];
          s[2] = fmaf(d[e], w_pre[e], s[2]);
        }
        exchange(s, t);
        if (p.du.p) there.from(x, s[0] * p.inv_dim);
        if (p.post) there.from(v, s[1] * p.inv_dim);
        c = s[2] * p.inv_dim;
        s[0] = s[1] = s[2] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s[0] = fmaf(x[e], x[e], s[0]);
        s[1] = fmaf(v[e], v[e], s[1]);
        s[2] = fmaf(d[e] * w_pre[e], x[e], s[2]);
      }
      exchange(s, t);
      const float r = 1.0f / sqrtf(fmaf(s[0], p.inv_dim, p.eps));
      const float ry1 = p.post ? 1.0f / sqrtf(fmaf(s[1], p.inv_dim, p.eps)) : 1.0f;
      if (p.du.p) {
        const float a = r * s[2] * p.inv_dim;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float xn = x[e] * r;
          pg[e] = fmaf(d[e], xn, pg[e]);
          d[e] = r * fmaf(d[e], w_pre[e], -xn * a);
        }
        if constexpr (LAYER) there.from(d, r * c);
      }
      if (p.dx_out.p) {
        rd.get(x);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] += x[e];
      }
      if (KEEP && k + R < last) fetch(tok + R);
      if (p.dx.p && live) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = p.a * d[e];
        store_row<L, WIDE>(at<S>(p.dx, b, tok), p.dim, t, x);
      }
      if (!p.has_y) continue;
      if (!KEEP) {
        if (p.post) post();
        load_weight<L, WIDE>(p.gate ? p.gate + b * p.gate_ld : nullptr, 1.0f, p.dim, t, w_gate);
      }
      float q[2] = {0.0f, 0.0f};
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[e] *= ry1;
        const float n = p.post ? (LAYER ? fmaf(v[e], w_post[e], b_post[e]) : v[e] * w_post[e]) : v[e];
        gg[e] = fmaf(d[e], n, gg[e]);
        if (p.gate) d[e] *= w_gate[e];
        if (p.post) {
          qg[e] = fmaf(d[e], v[e], qg[e]);
          if constexpr (LAYER) qb[e] += d[e];
          d[e] *= w_post[e];
          q[0] = fmaf(d[e], v[e], q[0]);
          if constexpr (LAYER) q[1] += d[e];
        }
      }
      if (p.post) {
        exchange(q, t);
        const float a = q[0] * p.inv_dim, m = LAYER ? q[1] * p.inv_dim : 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] = ry1 * (d[e] - fmaf(v[e], a, m));
      }
      if (p.dy.p && live) store_row<L, WIDE>(at<T>(p.dy, b, tok), p.dim, t, d);
    }
    if (p.gate_unit) {
      flush(gg, p.gate_part + (int64_t)unit * p.dim);
#pragma unroll
      for (int e = 0; e < E; ++e) gg[e] = 0.0f;
    }
  }
  if (!p.part) return;
  float* part = p.part + (int64_t)blockIdx.x * 4 * p.dim;
  if (p.wanted & 1) flush(pg, part);
  if (p.wanted & 2) flush(pb, part + p.dim);
  if (p.wanted & 4) flush(qg, part + 2 * p.dim);
  if (p.wanted & 8) flush(qb, part + 3 * p.dim);
  if ((p.wanted & 16) && !p.gate_unit) flush(gg, p.gate_part + (int64_t)blockIdx.x * p.dim);
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

// Waves of a row and runs of eight a thread.
struct Width {
  int waves, runs;
};
// Forward: rows of up to 1024 in one wave, which needs no barrier.
Width forward_width(int dim) {
  if (dim <= 512) return {1, 1};
  if (dim <= 1024) return {1, 2};
  if (dim <= 2048) return {2, 2};
  if (dim <= 4096) return {4, 2};
  if (dim <= 8192) return {8, 2};
  return {16, 2};
}
// Backward: eight values a thread, so that the sums, the weights and the next row's loads stay in
// registers.
Width backward_width(int dim) {
  if (dim <= 512) return {1, 1};
  if (dim <= 1024) return {2, 1};
  if (dim <= 2048) return {4, 1};
  if (dim <= 4096) return {8, 1};
  if (dim <= 8192) return {8, 2};
  return {8, 4};
}
// Workgroups of a forward launch: what the GPU holds, several times over for rows of one wave.
int forward_blocks(int dim) { return dim <= 4096 ? 256 * 8 : 256 * 4; }
// Backward: the workgroups that the GPU holds, three a CU of rows of up to 2048 (kept to a third of its
// registers: 243 -> 166 us where they took 190 and two ran; 12608 rows of 768, layer norm, 192 -> 109), and the
// units that they share out (below; with as many as workgroups 175 us, with four times as many 175).
int grad_blocks(Width w) { return w.waves <= 4 ? 768 : w.runs == 1 ? 256 : 512; }
int units_of(Width w) { return w.runs == 1 ? 2 * grad_blocks(w) : grad_blocks(w); }
int rows_of(Width w) { return w.waves > 4 ? 1 : 4 / w.waves; }

template <typename T, typename S, bool LAYER, bool WIDE>
void launch_forward(const BlockP& p, unsigned grid, hipStream_t s) {
  auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, s, p); };
  const Width w = forward_width(p.dim);
  switch (w.waves * 2 + w.runs) {
    case 3: return go(block_norm_kernel<T, S, LAYER, 1, 1, WIDE>, 256);
    case 4: return go(block_norm_kernel<T, S, LAYER, 1, 2, WIDE>, 256);
    case 6: return go(block_norm_kernel<T, S, LAYER, 2, 2, WIDE>, 256);
    case 10: return go(block_norm_kernel<T, S, LAYER, 4, 2, WIDE>, 256);
    case 18: return go(block_norm_kernel<T, S, LAYER, 8, 2, WIDE>, 512);
    default: return go(block_norm_kernel<T, S, LAYER, 16, 2, WIDE>, 1024);
  }
}
template <typename T, typename S, bool LAYER, bool WIDE>
void launch_backward(const BlockP& p, unsigned grid, hipStream_t s) {
  auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, s, p); };
  const Width w = backward_width(p.dim);
  switch (w.waves * 2 + w.runs) {
    case 3: return go(block_norm_bwd_kernel<T, S, LAYER, 1, 1, WIDE>, 256);
    case 5: return go(block_norm_bwd_kernel<T, S, LAYER, 2, 1, WIDE>, 256);
    case 9: return go(block_norm_bwd_kernel<T, S, LAYER, 4, 1, WIDE>, 256);
    case 17: return go(block_norm_bwd_kernel<T, S, LAYER, 8, 1, WIDE>, 512);
    case 18: return go(block_norm_bwd_kernel<T, S, LAYER, 8, 2, WIDE>, 512);
    default: return go(block_norm_bwd_kernel<T, S, LAYER, 8, 4, WIDE>, 512);
  }
}

template <typename T, typename S>
void launch_kind(const BlockP& p, bool wide, bool back, unsigned grid, hipStream_t s) {
  auto kind = [&](auto layer) {
    constexpr bool LAYER = decltype(layer)::value;
    if (back)
      wide ? launch_backward<T, S, LAYER, true>(p, grid, s) : launch_backward<T, S, LAYER, false>(p, grid, s);
    else
      wide ? launch_forward<T, S, LAYER, true>(p, grid, s) : launch_forward<T, S, LAYER, false>(p, grid, s);
  };
  p.layer ? kind(std::true_type()) : kind(std::false_type());
}
void launch_types(const BlockP& p, bool wide, bool bf16, bool stream_bf16, bool back, unsigned grid, hipStream_t s) {
  if (!bf16) return launch_kind<float, float>(p, wide, back, grid, s);
  if (stream_bf16) return launch_kind<uint16_t, uint16_t>(p, wide, back, grid, s);
  launch_kind<uint16_t, float>(p, wide, back, grid, s);
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
  p.gate_ld = d.gate_per_sequence ? d.dim : 0;
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

// Whether everything starts at, and goes in steps of, 16 bytes.
bool wide(const BlockP& p) {
  auto ok = [](const Rows& r) { return aligned(r.p, 16) && r.sb % 16 == 0 && r.st % 16 == 0; };
  for (const Rows* r : {&p.x, &p.y, &p.x_out, &p.u, &p.dx_out, &p.du, &p.dx, &p.dy})
    if (r->p && !ok(*r)) return false;
  for (const void* w : {(const void*)p.pre_gamma, (const void*)p.pre_beta, (const void*)p.post_gamma,
                        (const void*)p.post_beta, (const void*)p.gate})
    if (!aligned(w, 16)) return false;
  return p.dim % 8 == 0;
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
  launch_types(p, wide(p), es == 2, ss == 2, false, grid, s);
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
  if (sums) {
    const int64_t need = part_bytes(sl, d->dim) + gate_bytes(sl, d->dim);
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < need)
      return fail(ELASTO_ERR_INVALID_ARG, "block_norm: the workspace holds %lld of %lld bytes",
                  (long long)(workspace ? workspace_bytes : 0), (long long)need);
    p.part = static_cast<float*>(workspace);
    p.gate_part = p.part + part_bytes(sl, d->dim) / 4;
  }
  if (direct) p.gate_part = d_gate;
  launch_types(p, wide(p), es == 2, ss == 2, true, (unsigned)sl.grid, s);
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
  *bytes = part_bytes(s, d->dim) + gate_bytes(s, d->dim);
  return ELASTO_OK;
}

}  // extern "C"
