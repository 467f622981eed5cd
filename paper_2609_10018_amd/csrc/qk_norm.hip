// Norms of queries and keys for each head with the position rotation in the
// same pass, forward and backward.
//
// A head vector x of d features becomes
//   u = x r,  r = 1 / sqrt(mean(x^2) + eps),  y = gamma (.) u,  out = R y
// where R turns the first rot features in pairs (a, b) by the angle of the
// token's position: a' = a c - b s, b' = b c + a s.  Backward, with e = R^T
// dout and g = gamma (.) e:
//   dx = r (g - u mean(g (.) u)),  dgamma = sum over tokens and heads of e (.) u.
//
// A group of GW lanes takes a head vector in 16-byte pieces, one a lane, so a
// vector is read once, straight into registers, and the reductions stay inside
// the group.  A group walks the heads of a token (or a part of them, where the
// tokens alone would leave CUs idle), kHeads loads in flight at a time: the
// token's cosines and sines, which depend on neither the head nor q or k, are
// loaded once and multiplied with gamma once, and a head then costs a feature
// about eight instructions.  With halves paired, feature i turns with i + rot/2,
// which another lane of the group holds: its raw piece is exchanged (4
// registers), since the norm is the group's and gamma is known to both.
//
// Everything between the load and the store is fp32; the result is rounded
// once.
//
// AXES: a token has a position on each of up to four axes (time, height, width), and
// pair f turns by that of its axis: row position[axis of f] of the tables, column f.  A
// lane's pairs lie on one axis as a rule where the axes' sections follow one another, and
// are then loaded like those of one position.  Without the norm r = 1, and the backward
// pass is the forward one by the opposite angles (2 x 16384 tokens, 24 heads of 128 in bf16 on three
// axes: 87 us, 4.6 TB/s).
//
// Bound by memory, 2 (backward 3) passes over q and k: 256 x 197 tokens,
// 24 heads of 64 in bf16, 68 us (4.8 TB/s, a copy runs at 5.1; 56 us called again on
// the same tensors, part of which the caches keep); backward on 4 x 6001 padded
// tokens, 40 heads of 128, with both weights' gradients, 133 us (4.7).
#include <algorithm>

#include "common.h"
#include "heads.h"

namespace elasto {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 4;          // head vectors in flight
constexpr int kGradBlocks = 768;   // workgroups of the backward pass (3 a CU, as its registers allow)
constexpr int64_t kMaxTokens = 1 << 25;  // of a call, at 64 lanes each: a launch holds fewer than 2^32 threads

struct Side {  // q or k
  View x;      // the input
  View dout;   // backward: the gradient of the result
  View out;    // forward: the result; backward: dx
  const float* gamma;
  int heads;
};

struct QkP {
  Side q, k;
  const float *cos, *sin;
  const int32_t *positions, *lens;
  int tokens, dim, rot, table_rows;
  int rows, parts, part_heads;  // batch * tokens; parts of the heads, heads of each
  bool wide;  // the tables allow 16-byte loads
  float eps, inv_dim;
  float* part;  // backward: [workgroup][2][dim]
  // AXES: positions of a token; what the sine is multiplied with; whether pairs of one axis
  // follow one another; whether there is a norm; the axis of each pair.
  int axes;
  float sense;
  bool blocks, norm;
  uint8_t axis_of[128];
};

template <typename T>
struct Piece;
template <>
struct Piece<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const u32x4& w, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float* v) {
    return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                 pack_bf16x2(v[6], v[7])};
  }
};
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const u32x4& w, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
  }
  static __device__ __forceinline__ u32x4 pack(const float* v) {
    return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                 __float_as_uint(v[3])};
  }
};

// K values of a table.  wide: all tables start at multiples of 16 bytes, and with
// them every lane's piece (11 x 1322 tokens, 6 heads of 128: 34 us with single loads,
// which were most of what a group did, 11 with 16-byte ones).
template <int K>
__device__ __forceinline__ void load_table(const float* p, bool wide, float* v) {
  typedef float piece __attribute__((ext_vector_type(K < 4 ? K : 4)));
  if (wide) {
#pragma unroll
    for (int i = 0; i < K; i += 4) {
      const piece x = *reinterpret_cast<const piece*>(p + i);
#pragma unroll
      for (int e = 0; e < (K < 4 ? K : 4); ++e) v[i + e] = x[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < K; ++i) v[i] = p[i];
  }
}

// The sum over the group in each of its lanes: in quads, in eights and in rows
// of 16 by lane moves of the adder itself (each step's operands are the same in
// all lanes that it pairs up), beyond by exchanging halves.
template <int CTRL>
__device__ __forceinline__ float add_moved(float v) {
  return v + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                 0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int GW>
__device__ __forceinline__ float group_sum(float v) {
  v = add_moved<0xB1>(v);                       // lane ^ 1
  if constexpr (GW >= 4) v = add_moved<0x4E>(v);   // lane ^ 2
  if constexpr (GW >= 8) v = add_moved<0x141>(v);  // the other quad of eight
  if constexpr (GW >= 16) v = add_moved<0x140>(v); // the other eight of a row
  if constexpr (GW >= 32) v += __shfl_xor(v, 16, 64);
  if constexpr (GW >= 64) v += __shfl_xor(v, 32, 64);
  return v;
}

__device__ __forceinline__ u32x4 exchange(const u32x4& w, int lane4) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(lane4, (int)w[i]);
  return r;
}

// What a lane knows about its features: out = r (x (.) own + xp (.) other), with
// xp the features that x turns with.
template <typename T, bool PAIRS, bool AXES>
struct Lane {
  static constexpr int N = Piece<T>::N;
  int f0;        // first feature of the piece
  bool on;       // the piece lies inside the head
  bool turns;    // its features are rotated
  int partner4;  // 4 * the lane that holds the features these turn with
  int pf;        // their first
  float sign;    // of the sine in this piece's results (halves)
  uint32_t kept; // all bits where it turns, none where it does not

  __device__ __forceinline__ Lane(const QkP& p, int li, int lane) {
    f0 = li * N;
    on = f0 < p.dim;
    turns = f0 < p.rot;
    const int half = p.rot / 2;
    const bool low = f0 < half;
    partner4 = 4 * (PAIRS || !turns ? lane : low ? lane + half / N : lane - half / N);
    pf = PAIRS || !turns ? f0 : low ? f0 + half : f0 - half;
    sign = low ? -1.0f : 1.0f;
    kept = turns ? ~0u : 0u;
  }

  // Cosines and signed sines of the piece at token row `row` (1 and 0 where it
  // does not turn); NaN where the position has no row in the tables.
  __device__ __forceinline__ void angles(const QkP& p, int row, int t, float* c, float* s) const {
#pragma unroll
    for (int e = 0; e < N; ++e) c[e] = 1.0f, s[e] = AXES ? -0.0f : 0.0f;  // x + 0 * -0 keeps a zero's sign
    if (!turns) return;
    if constexpr (AXES) return angles_on_axes(p, row, c, s);
    const int pos = p.positions ? p.positions[row] : t;
    const bool ok = pos >= 0 && pos < p.table_rows;
    const int half = p.rot / 2;
    const int at = PAIRS ? f0 / 2 : (f0 < half ? f0 : f0 - half);
    const float* cp = p.cos + (int64_t)(ok ? pos : 0) * half + at;
    const float* sp = p.sin + (int64_t)(ok ? pos : 0) * half + at;
    constexpr int K = PAIRS ? N / 2 : N;
    float cv[K], sv[K];
    load_table<K>(cp, p.wide, cv);
    load_table<K>(sp, p.wide, sv);
#pragma unroll
    for (int e = 0; e < K; ++e) {
      const float ce = ok ? cv[e] : NAN, se = ok ? sv[e] : NAN;
      if constexpr (PAIRS) {
        c[2 * e] = c[2 * e + 1] = ce;
        s[2 * e] = -se;
        s[2 * e + 1] = se;
      } else {
        c[e] = ce;
        s[e] = sign * se;
      }
    }
  }
  // The same where each pair has an axis; pairs whose position has no row become NaN.
  __device__ __forceinline__ void angles_on_axes(const QkP& p, int row, float* c, float* s) const {
    const int half = p.rot / 2;
    const int at = PAIRS ? f0 / 2 : (f0 < half ? f0 : f0 - half);
    const int32_t* pos = p.positions + (int64_t)row * p.axes;
    constexpr int K = PAIRS ? N / 2 : N;
    float cv[K], sv[K];
    const int a0 = p.axis_of[at];
    if (p.blocks && a0 == p.axis_of[at + K - 1]) {
      const int ps = pos[a0];
      const bool ok = ps >= 0 && ps < p.table_rows;
      const int64_t from = (int64_t)(ok ? ps : 0) * half + at;
      load_table<K>(p.cos + from, p.wide, cv);
      load_table<K>(p.sin + from, p.wide, sv);
      if (!ok)
#pragma unroll
        for (int e = 0; e < K; ++e) cv[e] = sv[e] = NAN;
    } else {
#pragma unroll
      for (int e = 0; e < K; ++e) {
        const int ps = pos[p.axis_of[at + e]];
        const bool ok = ps >= 0 && ps < p.table_rows;
        const int64_t from = (int64_t)(ok ? ps : 0) * half + at + e;
        cv[e] = ok ? p.cos[from] : NAN;
        sv[e] = ok ? p.sin[from] : NAN;
      }
    }
#pragma unroll
    for (int e = 0; e < K; ++e) {
      const float se = sv[e] * p.sense;
      if constexpr (PAIRS) {
        c[2 * e] = c[2 * e + 1] = cv[e];
        s[2 * e] = -se;
        s[2 * e + 1] = se;
      } else {
        c[e] = cv[e];
        s[e] = sign * se;
      }
    }
  }
  // gamma of the lane's features, and of those that they turn with.
  __device__ __forceinline__ void weights(const float* gamma, bool wide, float* g) const {
#pragma unroll
    for (int e = 0; e < N; ++e) g[e] = 1.0f;
    if (on && gamma) load_table<N>(gamma + f0, wide, g);
  }
  __device__ __forceinline__ void weights(const float* gamma, bool wide, float* g, float* gp) const {
    weights(gamma, wide, g);
#pragma unroll
    for (int e = 0; e < N; ++e) gp[e] = PAIRS ? g[e ^ 1] : 1.0f;
    if constexpr (!PAIRS)
      if (on && gamma) load_table<N>(gamma + pf, wide, gp);
  }
  // The features that x turns with, from the group's raw pieces.  AXES: zeros where it does not turn, since
  // an infinity times a sine of 0 would spoil what the rotation alone passes on (a choice behind the
  // arithmetic instead: 15 registers more, 87 -> 90 us).
  __device__ __forceinline__ void partners(const u32x4& raw, const float* x, float* xp) const {
    if constexpr (PAIRS && !AXES) {
#pragma unroll
      for (int e = 0; e < N; ++e) xp[e] = x[e ^ 1];
    } else if constexpr (PAIRS) {
#pragma unroll
      for (int e = 0; e < N; ++e) xp[e] = __uint_as_float(__float_as_uint(x[e ^ 1]) & kept);
    } else if constexpr (AXES) {
      Piece<T>::unpack(exchange(raw, partner4) & kept, xp);
    } else {
      Piece<T>::unpack(exchange(raw, partner4), xp);
    }
  }
};

// A group's token and its share of the heads.
struct Unit {
  int row, b, t, h0, h1;
  bool live;
};
__device__ __forceinline__ Unit unit_of(const QkP& p, int64_t u) {
  Unit w;
  w.live = u < (int64_t)p.rows * p.parts;
  const unsigned v = w.live ? (unsigned)u : 0u;  // rows * parts < 2^31
  w.row = (int)(v / (unsigned)p.parts);
  w.h0 = (int)(v - (unsigned)w.row * p.parts) * p.part_heads;
  w.h1 = min(w.h0 + p.part_heads, p.q.heads + p.k.heads);
  w.b = (int)((unsigned)w.row / (unsigned)p.tokens);
  w.t = w.row - w.b * p.tokens;
  if (w.live && p.lens) w.live = w.t < p.lens[w.b];
  return w;
}

template <bool AXES>
__device__ __forceinline__ float inv_norm(float ss, const QkP& p) {
  if constexpr (AXES)
    if (!p.norm) return 1.0f;
  return __builtin_amdgcn_rsqf(fmaf(ss, p.inv_dim, p.eps));
}

template <typename T, int GW, bool PAIRS, bool AXES>
__device__ __forceinline__ void forward_heads(const QkP& p, const Side& s, const Lane<T, PAIRS, AXES>& L,
                                              const Unit& w, int h0, int h1, const float* c,
                                              const float* sn) {
  constexpr int N = Piece<T>::N;
  float own[N], other[N];
  L.weights(s.gamma, p.wide, own, other);
#pragma unroll
  for (int e = 0; e < N; ++e) own[e] *= c[e], other[e] *= sn[e];
  const bool on = w.live && L.on;
  const char* x = s.x.p + w.b * s.x.sb + w.t * s.x.st + h0 * s.x.sh + L.f0 * (int)sizeof(T);
  char* out = s.out.p + w.b * s.out.sb + w.t * s.out.st + h0 * s.out.sh + L.f0 * (int)sizeof(T);
  for (int h = h0; h < h1; h += kHeads) {
    u32x4 raw[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      raw[i] = u32x4{0u, 0u, 0u, 0u};
      if (on && h + i < h1) raw[i] = *reinterpret_cast<const u32x4*>(x + i * s.x.sh);
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      float v[N], vp[N];
      Piece<T>::unpack(raw[i], v);
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) ss = fmaf(v[e], v[e], ss);
      const float r = inv_norm<AXES>(group_sum<GW>(ss), p);
      L.partners(raw[i], v, vp);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = r * fmaf(v[e], own[e], vp[e] * other[e]);
      if (on && h + i < h1) *reinterpret_cast<u32x4*>(out + i * s.out.sh) = Piece<T>::pack(v);
    }
    x += kHeads * s.x.sh;
    out += kHeads * s.out.sh;
  }
}

template <typename T, int GW, bool PAIRS, bool AXES>
__global__ __launch_bounds__(kThreads) void qk_norm_kernel(QkP p) {
  constexpr int N = Piece<T>::N;
  const int lane = threadIdx.x & 63;
  const Lane<T, PAIRS, AXES> L(p, lane % GW, lane);
  const Unit w = unit_of(p, (int64_t)blockIdx.x * (kThreads / GW) + threadIdx.x / GW);
  float c[N], sn[N];
  L.angles(p, w.row, w.t, c, sn);
  // Every group of a wave takes as many rounds: those of the longest share.
  const int q1 = min(w.h1, p.q.heads);
  if (__any(w.h0 < q1)) forward_heads<T, GW, PAIRS, AXES>(p, p.q, L, w, w.h0, q1, c, sn);
  const int k0 = max(w.h0 - p.q.heads, 0), k1 = w.h1 - p.q.heads;
  if (__any(k0 < k1)) forward_heads<T, GW, PAIRS, AXES>(p, p.k, L, w, k0, k1, c, sn);
}

template <typename T, int GW, bool PAIRS, bool AXES>
__device__ __forceinline__ void backward_heads(const QkP& p, const Side& s, const Lane<T, PAIRS, AXES>& L,
                                               const Unit& w, int h0, int h1, const float* c,
                                               const float* sn, const float* gamma, float* dgamma) {
  constexpr int N = Piece<T>::N;
  const bool on = w.live && L.on;
  const int f = L.f0 * (int)sizeof(T);
  const char* x = s.x.p + w.b * s.x.sb + w.t * s.x.st + h0 * s.x.sh + f;
  const char* d = s.dout.p + w.b * s.dout.sb + w.t * s.dout.st + h0 * s.dout.sh + f;
  char* out = s.out.p + w.b * s.out.sb + w.t * s.out.st + h0 * s.out.sh + f;
  for (int h = h0; h < h1; h += kHeads) {
    u32x4 raw[kHeads], draw[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      raw[i] = draw[i] = u32x4{0u, 0u, 0u, 0u};
      if (on && h + i < h1) {
        raw[i] = *reinterpret_cast<const u32x4*>(x + i * s.x.sh);
        draw[i] = *reinterpret_cast<const u32x4*>(d + i * s.dout.sh);
      }
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      float u[N], e[N], ep[N];
      Piece<T>::unpack(raw[i], u);
      float ss = 0.0f;
#pragma unroll
      for (int j = 0; j < N; ++j) ss = fmaf(u[j], u[j], ss);
      const float r = inv_norm<AXES>(group_sum<GW>(ss), p);
      Piece<T>::unpack(draw[i], e);
      L.partners(draw[i], e, ep);
      float gu = 0.0f;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        // The transposed rotation turns the other way.
        e[j] = fmaf(e[j], c[j], -ep[j] * sn[j]);
        u[j] *= r;
        const float a = e[j] * u[j];
        dgamma[j] += a;  // heads and lanes that are not there hold zeros
        gu = fmaf(gamma[j], a, gu);
      }
      gu = group_sum<GW>(gu) * p.inv_dim;
#pragma unroll
      for (int j = 0; j < N; ++j) e[j] = r * fmaf(gamma[j], e[j], -u[j] * gu);
      if (on && h + i < h1) *reinterpret_cast<u32x4*>(out + i * s.out.sh) = Piece<T>::pack(e);
    }
    x += kHeads * s.x.sh;
    d += kHeads * s.dout.sh;
    out += kHeads * s.out.sh;
  }
}

// Backward: a fixed grid walks the units, so that a lane sums its features'
// part of dgamma in registers; the workgroup's groups are summed in LDS and its
// row goes to part, which qk_gamma_kernel sums in a fixed order.
template <typename T, int GW, bool PAIRS, bool AXES>
__global__ __launch_bounds__(kThreads, 3) void qk_norm_bwd_kernel(QkP p) {
  constexpr int N = Piece<T>::N, G = kThreads / GW;
  __shared__ float red[2][G][GW * N];
  const int lane = threadIdx.x & 63, li = lane % GW, grp = threadIdx.x / GW;
  const Lane<T, PAIRS, AXES> L(p, li, lane);
  float dgq[N], dgk[N], gq[N], gk[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    dgq[e] = dgk[e] = 0.0f;
  }
  L.weights(p.q.gamma, p.wide, gq);
  L.weights(p.k.gamma, p.wide, gk);
  const int64_t units = (int64_t)p.rows * p.parts;
  for (int64_t u0 = (int64_t)blockIdx.x * G; u0 < units; u0 += (int64_t)gridDim.x * G) {
    const Unit w = unit_of(p, u0 + grp);
    float c[N], sn[N];
    L.angles(p, w.row, w.t, c, sn);
    if (!w.live)  // no position of a token that is not there spoils the sums
#pragma unroll
      for (int e = 0; e < N; ++e) c[e] = sn[e] = 0.0f;
    const int q1 = min(w.h1, p.q.heads);
    if (__any(w.h0 < q1)) backward_heads<T, GW, PAIRS, AXES>(p, p.q, L, w, w.h0, q1, c, sn, gq, dgq);
    const int k0 = max(w.h0 - p.q.heads, 0), k1 = w.h1 - p.q.heads;
    if (__any(k0 < k1)) backward_heads<T, GW, PAIRS, AXES>(p, p.k, L, w, k0, k1, c, sn, gk, dgk);
  }
  if (!p.part) return;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    red[0][grp][li * N + e] = dgq[e];
    red[1][grp][li * N + e] = dgk[e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * p.dim; i += kThreads) {
    const int side = i >= p.dim, f = side ? i - p.dim : i;
    float sum = 0.0f;
    for (int g = 0; g < G; ++g) sum += red[side][g][f];
    p.part[(int64_t)blockIdx.x * 2 * p.dim + i] = sum;
  }
}

// dgamma: column i of part summed over its rows, 16 columns a workgroup, its
// 1024 threads 64 slices of the rows.
__global__ __launch_bounds__(1024) void qk_gamma_kernel(const float* part, int rows, int dim,
                                                        float* dq, float* dk) {
  __shared__ float red[64][17];
  const int c = threadIdx.x & 15, sl = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float s = 0.0f;
#pragma unroll 16
  for (int r = sl; r < rows; r += 64) s += part[(int64_t)r * 2 * dim + col];
  red[sl][c] = s;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  s = 0.0f;
  for (int i = 0; i < 64; ++i) s += red[i][threadIdx.x];
  float* out = col < dim ? dq : dk;
  if (out) out[col < dim ? col : col - dim] = s;
}

template <typename T, int GW, bool PAIRS, bool AXES>
void launch(const QkP& p, bool back, int grid, hipStream_t s) {
  if (back)
    hipLaunchKernelGGL((qk_norm_bwd_kernel<T, GW, PAIRS, AXES>), dim3((unsigned)grid), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((qk_norm_kernel<T, GW, PAIRS, AXES>), dim3((unsigned)grid), dim3(kThreads), 0, s, p);
}

template <typename T, bool PAIRS, bool AXES>
void launch_width(const QkP& p, int gw, bool back, int grid, hipStream_t s) {
  switch (gw) {
    case 2: return launch<T, 2, PAIRS, AXES>(p, back, grid, s);
    case 4: return launch<T, 4, PAIRS, AXES>(p, back, grid, s);
    case 8: return launch<T, 8, PAIRS, AXES>(p, back, grid, s);
    case 16: return launch<T, 16, PAIRS, AXES>(p, back, grid, s);
    case 32: return launch<T, 32, PAIRS, AXES>(p, back, grid, s);
    default: return launch<T, 64, PAIRS, AXES>(p, back, grid, s);
  }
}

bool check_desc(const elasto_qk_norm_t* a) {
  if (!a) return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: NULL description"), false;
  if (a->dtype != ELASTO_BF16 && a->dtype != ELASTO_FP32)
    return fail(ELASTO_ERR_INVALID_ARG, "bad dtype %d", a->dtype), false;
  if (a->batch < 0 || a->tokens < 0 || a->q_heads < 0 || a->kv_heads < 0 ||
      (int64_t)a->q_heads + a->kv_heads < 1 || (int64_t)a->q_heads + a->kv_heads > 65536 ||
      (int64_t)a->batch * a->tokens > kMaxTokens)
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: bad batch, tokens or heads"), false;
  if (a->head_dim < 16 || a->head_dim > 256 || a->head_dim % 16)
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: head_dim %d is not a multiple of 16 in [16, 256]", a->head_dim), false;
  return true;
}

// Forward: x is the input, out the result.  Backward: x is the input, dout the
// gradient of the result, out dx.
bool set_side(Side* s, const elasto_qk_norm_t& a, const char* name, int heads, const elasto_heads_t* x,
              const elasto_heads_t* dout, const elasto_heads_t* out, const float* gamma, bool back) {
  *s = Side();
  s->heads = heads;
  s->gamma = gamma;
  if (gamma && !aligned(gamma, 4)) return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: misaligned gamma"), false;
  auto take = [&](const elasto_heads_t* t, bool written, View* v) {
    return take_view("qk_norm", name, t, a.batch, a.tokens, heads, a.head_dim,
                     a.dtype == ELASTO_BF16 ? 2 : 4, written, v);
  };
  return take(x, false, &s->x) && (!back || take(dout, false, &s->dout)) && take(out, true, &s->out);
}

// The axis of each pair: the axes' sections one after another, or dealt out in turn.
bool set_axes(const elasto_qk_axes_t& x, QkP* p) {
  if (x.axes < 1 || x.axes > 4) return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: %d axes, not 1 to 4", x.axes), false;
  int left[4] = {}, sum = 0;
  for (int a = 0; a < x.axes; ++a) {
    if (x.sections[a] < 0 || x.sections[a] > 128)
      return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: section %d of %d pairs", a, x.sections[a]), false;
    sum += left[a] = x.sections[a];
  }
  if (2 * sum != x.base.rot_dim)
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: the sections hold %d pairs, rot_dim %d", sum, x.base.rot_dim), false;
  for (int f = 0, a = 0; f < sum;) {
    if (left[a] > 0) {
      p->axis_of[f++] = (uint8_t)a;
      --left[a];
      if (!x.in_turn) continue;
    }
    a = (a + 1) % x.axes;
  }
  p->axes = x.axes;
  p->blocks = !x.in_turn;
  p->norm = x.norm != 0;
  p->sense = 1.0f;
  if (!p->norm && (x.base.q_gamma || x.base.k_gamma))
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: weights without the norm"), false;
  if (!x.base.positions && x.base.rot_dim > 0 && (int64_t)x.base.batch * x.base.tokens > 0)
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: positions is NULL"), false;
  return true;
}

template <bool AXES>
void launch_types(const QkP& p, bool bf16, bool pairs, int gw, bool back, int grid, hipStream_t s) {
  if (bf16)
    pairs ? launch_width<uint16_t, true, AXES>(p, gw, back, grid, s) : launch_width<uint16_t, false, AXES>(p, gw, back, grid, s);
  else
    pairs ? launch_width<float, true, AXES>(p, gw, back, grid, s) : launch_width<float, false, AXES>(p, gw, back, grid, s);
}

// axes: NULL where tokens have one position.
elasto_status_t run(const elasto_qk_norm_t* a, const elasto_qk_axes_t* axes, const elasto_heads_t* q, const elasto_heads_t* k,
                    const elasto_heads_t* dq_out, const elasto_heads_t* dk_out,
                    const elasto_heads_t* q_res, const elasto_heads_t* k_res, float* dq_gamma,
                    float* dk_gamma, void* ws, int64_t ws_bytes, bool back, void* hip_stream) {
  if (!check_desc(a)) return ELASTO_ERR_INVALID_ARG;
  if ((!axes || axes->norm) && (!(a->eps >= 1.17549435e-38f) || !(a->eps < INFINITY)))
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: eps must be a positive normal number");
  if (a->rot_dim < 0 || a->rot_dim > a->head_dim || a->rot_dim % 16)
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: rot_dim %d is not a multiple of 16 in [0, head_dim]", a->rot_dim);
  const int64_t rows = (int64_t)a->batch * a->tokens;
  if (a->rot_dim > 0 && rows > 0) {
    if (!a->cos || !a->sin || !aligned(a->cos, 4) || !aligned(a->sin, 4) || a->table_rows < 1)
      return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: a rotation needs cos, sin and table_rows >= 1");
    if (!axes && !a->positions && a->table_rows < a->tokens)
      return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: the tables hold %d rows for %d tokens", a->table_rows, a->tokens);
  }
  if (!aligned(a->positions, 4) || !aligned(a->lens, 4) || !aligned(dq_gamma, 4) || !aligned(dk_gamma, 4))
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: misaligned pointer");
  const int es = a->dtype == ELASTO_BF16 ? 2 : 4, n = 16 / es;
  QkP p = {};
  if (axes && !set_axes(*axes, &p)) return ELASTO_ERR_INVALID_ARG;
  if (back && axes && !p.norm) {
    if (dq_gamma || dk_gamma) return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: weights without the norm");
    back = false;
    p.sense = -1.0f;
    q = dq_out;
    k = dk_out;
  }
  if (!set_side(&p.q, *a, "q, its result or a gradient", a->q_heads, q, dq_out, q_res, a->q_gamma, back) ||
      !set_side(&p.k, *a, "k, its result or a gradient", a->kv_heads, k, dk_out, k_res, a->k_gamma, back))
    return ELASTO_ERR_INVALID_ARG;
  p.cos = a->cos;
  p.sin = a->sin;
  p.wide = aligned(a->cos, 16) && aligned(a->sin, 16) && aligned(a->q_gamma, 16) && aligned(a->k_gamma, 16);
  p.positions = a->positions;
  p.lens = a->lens;
  p.tokens = a->tokens;
  p.dim = a->head_dim;
  p.rot = a->rot_dim;
  p.table_rows = a->table_rows;
  p.eps = a->eps;
  p.inv_dim = 1.0f / (float)a->head_dim;
  int gw = 2;
  while (gw * n < a->head_dim) gw *= 2;
  const int groups = kThreads / gw;
  // Parts of the heads, whole rounds of kHeads each, where the tokens leave CUs
  // idle: as many as 512 workgroups take (backward: the fixed grid).  Each part
  // loads the cosines again.
  const int heads = a->q_heads + a->kv_heads, rounds = (heads + kHeads - 1) / kHeads;
  const int64_t want = (int64_t)(back ? kGradBlocks : 512) * groups;
  const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(rounds, want / std::max<int64_t>(rows, 1)));
  p.part_heads = (rounds + parts - 1) / parts * kHeads;
  p.parts = (heads + p.part_heads - 1) / p.part_heads;
  p.rows = (int)rows;
  int64_t grid = (rows * p.parts + groups - 1) / groups;
  const bool weights = back && (dq_gamma || dk_gamma);
  if (back) {
    grid = std::min<int64_t>(grid, kGradBlocks);
    if (weights) {
      const int64_t need = grid * 2 * a->head_dim * 4;
      if (need > 0 && (!ws || !aligned(ws, 16) || ws_bytes < need))
        return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: the workspace holds %lld of %lld bytes",
                    (long long)(ws ? ws_bytes : 0), (long long)need);
      p.part = static_cast<float*>(ws);
    }
  }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipSuccess;
  if (grid > 0) {
    if (axes)
      launch_types<true>(p, a->dtype == ELASTO_BF16, a->interleaved, gw, back, (int)grid, s);
    else
      launch_types<false>(p, a->dtype == ELASTO_BF16, a->interleaved, gw, back, (int)grid, s);
    e = hipGetLastError();
  }
  if (e == hipSuccess && weights) {
    hipLaunchKernelGGL(qk_gamma_kernel, dim3((unsigned)(2 * a->head_dim / 16)), dim3(1024), 0, s,
                       p.part, (int)grid, a->head_dim, dq_gamma, dk_gamma);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "qk_norm: %s", hipGetErrorString(e));
  return ELASTO_OK;
}

}  // namespace
}  // namespace elasto

using namespace elasto;

extern "C" {

elasto_status_t elasto_op_qk_norm_rotate(const elasto_qk_norm_t* desc, const elasto_heads_t* q,
                                  const elasto_heads_t* k, const elasto_heads_t* q_out,
                                  const elasto_heads_t* k_out, void* hip_stream) {
  return run(desc, nullptr, q, k, nullptr, nullptr, q_out, k_out, nullptr, nullptr, nullptr, 0, false,
             hip_stream);
}

elasto_status_t elasto_op_qk_norm_rotate_bwd(const elasto_qk_norm_t* desc, const elasto_heads_t* q,
                                      const elasto_heads_t* k, const elasto_heads_t* dq_out,
                                      const elasto_heads_t* dk_out, const elasto_heads_t* dq,
                                      const elasto_heads_t* dk, float* dq_gamma, float* dk_gamma,
                                      void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return run(desc, nullptr, q, k, dq_out, dk_out, dq, dk, dq_gamma, dk_gamma, workspace, workspace_bytes,
             true, hip_stream);
}

elasto_status_t elasto_op_qk_norm_rotate_axes(const elasto_qk_axes_t* desc, const elasto_heads_t* q,
                                              const elasto_heads_t* k, const elasto_heads_t* q_out,
                                              const elasto_heads_t* k_out, void* hip_stream) {
  return run(desc ? &desc->base : nullptr, desc, q, k, nullptr, nullptr, q_out, k_out, nullptr, nullptr,
             nullptr, 0, false, hip_stream);
}

elasto_status_t elasto_op_qk_norm_rotate_axes_bwd(const elasto_qk_axes_t* desc, const elasto_heads_t* q,
                                                  const elasto_heads_t* k, const elasto_heads_t* dq_out,
                                                  const elasto_heads_t* dk_out, const elasto_heads_t* dq,
                                                  const elasto_heads_t* dk, float* dq_gamma,
                                                  float* dk_gamma, void* workspace,
                                                  int64_t workspace_bytes, void* hip_stream) {
  return run(desc ? &desc->base : nullptr, desc, q, k, dq_out, dk_out, dq, dk, dq_gamma, dk_gamma, workspace,
             workspace_bytes, true, hip_stream);
}

elasto_status_t elasto_qk_norm_rotate_workspace(const elasto_qk_norm_t* desc, int64_t* bytes) {
  if (!bytes) return fail(ELASTO_ERR_INVALID_ARG, "NULL argument");
  if (!check_desc(desc)) return ELASTO_ERR_INVALID_ARG;
  // A row of 2 * head_dim sums for each workgroup of the largest launch.
  *bytes = (int64_t)kGradBlocks * 2 * desc->head_dim * 4;
  return ELASTO_OK;
}

}  // extern "C"
