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
// vector is read once, straight into registers, and the reductions are xor
// shuffles inside the group.  A unit of work is kHeads vectors of one token:
// their loads are all in flight together, and the token's cosines and sines
// (which depend on neither the head nor q or k) are loaded once for them.  With
// halves paired, feature i turns with i + rot/2, which another lane of the
// group holds: its raw piece is exchanged (4 registers) before the norm, since
// r is the group's and gamma is known to both.
//
// Everything between the load and the store is fp32; the result is rounded
// once.  Bound by memory: 2 (backward 3) passes over q and k.
#include <algorithm>

#include "common.h"
#include "heads.h"

namespace elasto {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 4;        // head vectors of a unit
constexpr int kGradBlocks = 1024;  // workgroups of the backward pass (4 a CU)

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
  int tokens, dim, rot, table_rows, chunks;
  int64_t units;  // batch * tokens * chunks
  float eps, inv_dim;
  float* part;  // backward: [workgroup][2][dim]
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

template <int GW>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = GW / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// What a lane knows about its features for the whole launch.
template <typename T, bool PAIRS>
struct Lane {
  static constexpr int N = Piece<T>::N;
  int f0;       // first feature of the piece
  bool on;      // the piece lies inside the head
  bool turns;   // its features are rotated
  int partner;  // lane that holds the features these turn with
  float sign;   // of the sine in this piece's results (halves)
  float gq[N], gk[N], pq[N], pk[N];  // gamma of the piece, and of the partner's

  __device__ __forceinline__ Lane(const QkP& p, int li, int lane) {
    f0 = li * N;
    on = f0 < p.dim;
    turns = f0 < p.rot;
    const int half = p.rot / 2;
    const bool low = f0 < half;
    const int shift = half / N;
    partner = PAIRS || !turns ? lane : low ? lane + shift : lane - shift;
    sign = low ? -1.0f : 1.0f;
    const int pf = PAIRS || !turns ? f0 : low ? f0 + half : f0 - half;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      gq[e] = on && p.q.gamma ? p.q.gamma[f0 + e] : 1.0f;
      gk[e] = on && p.k.gamma ? p.k.gamma[f0 + e] : 1.0f;
      pq[e] = on && p.q.gamma ? p.q.gamma[pf + e] : 1.0f;
      pk[e] = on && p.k.gamma ? p.k.gamma[pf + e] : 1.0f;
    }
  }

  // Cosines and sines of the piece at token row `row`; NaN where the position
  // has no row in the tables.
  __device__ __forceinline__ void angles(const QkP& p, int64_t row, int t, float* c,
                                         float* s) const {
    if (!turns) return;
    const int pos = p.positions ? p.positions[row] : t;
    const bool ok = pos >= 0 && pos < p.table_rows;
    const int half = p.rot / 2;
    const int at = PAIRS ? f0 / 2 : (f0 < half ? f0 : f0 - half);
    const float* cp = p.cos + (int64_t)(ok ? pos : 0) * half + at;
    const float* sp = p.sin + (int64_t)(ok ? pos : 0) * half + at;
    constexpr int M = PAIRS ? N / 2 : N;
#pragma unroll
    for (int e = 0; e < M; ++e) {
      c[e] = ok ? cp[e] : NAN;
      s[e] = ok ? sp[e] : NAN;
    }
  }
};

struct Unit {
  int64_t b;
  int t, h0;
};

__device__ __forceinline__ Unit unit_of(const QkP& p, int64_t u, int64_t* row) {
  Unit w;
  *row = u / p.chunks;
  w.h0 = (int)(u - *row * p.chunks) * kHeads;
  w.b = *row / p.tokens;
  w.t = (int)(*row - w.b * p.tokens);
  return w;
}

// y turned; yp: the partner's y (halves only).
template <typename T, bool PAIRS>
__device__ __forceinline__ void turn(const Lane<T, PAIRS>& L, const float* c, const float* s,
                                     float* y, const float* yp) {
  constexpr int N = Piece<T>::N;
  if (!L.turns) return;
  if constexpr (PAIRS) {
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float a = y[e], b = y[e + 1];
      y[e] = fmaf(a, c[e / 2], -b * s[e / 2]);
      y[e + 1] = fmaf(b, c[e / 2], a * s[e / 2]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = fmaf(y[e], c[e], L.sign * yp[e] * s[e]);
  }
}

__device__ __forceinline__ u32x4 from_lane(const u32x4& w, int lane) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)__shfl((int)w[i], lane, 64);
  return r;
}

template <typename T, int GW, bool PAIRS>
__global__ __launch_bounds__(kThreads) void qk_norm_kernel(QkP p) {
  constexpr int N = Piece<T>::N;
  const int lane = threadIdx.x & 63, li = lane % GW;
  const int64_t u = (int64_t)blockIdx.x * (kThreads / GW) + threadIdx.x / GW;
  const Lane<T, PAIRS> L(p, li, lane);
  int64_t row = 0;
  Unit w = {0, 0, 0};
  bool live = u < p.units;
  if (live) {
    w = unit_of(p, u, &row);
    live = !p.lens || w.t < p.lens[w.b];
  }
  const int heads = p.q.heads + p.k.heads;
  u32x4 raw[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = w.h0 + i;
    raw[i] = u32x4{0u, 0u, 0u, 0u};
    if (live && L.on && h < heads) {
      const Side& s = h < p.q.heads ? p.q : p.k;
      const int hh = h < p.q.heads ? h : h - p.q.heads;
      raw[i] = *reinterpret_cast<const u32x4*>(s.x.p + w.b * s.x.sb + w.t * s.x.st + hh * s.x.sh + L.f0 * (int)sizeof(T));
    }
  }
  float c[N], sn[N];
#pragma unroll
  for (int e = 0; e < N; ++e) c[e] = sn[e] = 0.0f;
  if (live) L.angles(p, row, w.t, c, sn);
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    const int h = w.h0 + i;
    const bool isq = h < p.q.heads;
    float x[N], xp[N];
    Piece<T>::unpack(raw[i], x);
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) ss = fmaf(x[e], x[e], ss);
    const float r = 1.0f / sqrtf(fmaf(group_sum<GW>(ss), p.inv_dim, p.eps));
    if constexpr (!PAIRS) Piece<T>::unpack(from_lane(raw[i], L.partner), xp);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      x[e] *= r * (isq ? L.gq[e] : L.gk[e]);
      if constexpr (!PAIRS) xp[e] *= r * (isq ? L.pq[e] : L.pk[e]);
    }
    turn<T, PAIRS>(L, c, sn, x, xp);
    if (live && L.on && h < heads) {
      const Side& s = isq ? p.q : p.k;
      const int hh = isq ? h : h - p.q.heads;
      *reinterpret_cast<u32x4*>(s.out.p + w.b * s.out.sb + w.t * s.out.st + hh * s.out.sh + L.f0 * (int)sizeof(T)) =
          Piece<T>::pack(x);
    }
  }
}

// Backward: a fixed grid walks the units, so that a lane sums its features'
// part of dgamma in registers; the workgroup's groups are summed in LDS and its
// row goes to part, which qk_gamma_kernel sums in a fixed order.
template <typename T, int GW, bool PAIRS>
__global__ __launch_bounds__(kThreads) void qk_norm_bwd_kernel(QkP p) {
  constexpr int N = Piece<T>::N, G = kThreads / GW;
  __shared__ float red[2][G][GW * N];
  const int lane = threadIdx.x & 63, li = lane % GW, grp = threadIdx.x / GW;
  const Lane<T, PAIRS> L(p, li, lane);
  const int heads = p.q.heads + p.k.heads;
  float dgq[N], dgk[N];
#pragma unroll
  for (int e = 0; e < N; ++e) dgq[e] = dgk[e] = 0.0f;
  // Every group of a workgroup takes the same number of rounds: the shuffles
  // stay uniform.
  for (int64_t u0 = (int64_t)blockIdx.x * G; u0 < p.units; u0 += (int64_t)gridDim.x * G) {
    const int64_t u = u0 + grp;
    int64_t row = 0;
    Unit w = {0, 0, 0};
    bool live = u < p.units;
    if (live) {
      w = unit_of(p, u, &row);
      live = !p.lens || w.t < p.lens[w.b];
    }
    u32x4 raw[kHeads], draw[kHeads];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      const int h = w.h0 + i;
      raw[i] = draw[i] = u32x4{0u, 0u, 0u, 0u};
      if (live && L.on && h < heads) {
        const Side& s = h < p.q.heads ? p.q : p.k;
        const int hh = h < p.q.heads ? h : h - p.q.heads;
        raw[i] = *reinterpret_cast<const u32x4*>(s.x.p + w.b * s.x.sb + w.t * s.x.st + hh * s.x.sh + L.f0 * (int)sizeof(T));
        draw[i] = *reinterpret_cast<const u32x4*>(s.dout.p + w.b * s.dout.sb + w.t * s.dout.st + hh * s.dout.sh + L.f0 * (int)sizeof(T));
      }
    }
    float c[N], sn[N];
#pragma unroll
    for (int e = 0; e < N; ++e) c[e] = sn[e] = 0.0f;
    if (live) {
      L.angles(p, row, w.t, c, sn);
      // The transposed rotation turns the other way.
#pragma unroll
      for (int e = 0; e < N; ++e) sn[e] = -sn[e];
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      const int h = w.h0 + i;
      const bool isq = h < p.q.heads, some = live && h < heads;
      float x[N], d[N], dp[N];
      Piece<T>::unpack(raw[i], x);
      Piece<T>::unpack(draw[i], d);
      if constexpr (!PAIRS) Piece<T>::unpack(from_lane(draw[i], L.partner), dp);
      turn<T, PAIRS>(L, c, sn, d, dp);
      float ss = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) ss = fmaf(x[e], x[e], ss);
      const float r = 1.0f / sqrtf(fmaf(group_sum<GW>(ss), p.inv_dim, p.eps));
      float gu = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        x[e] *= r;
        const float a = d[e] * x[e];
        if (some && isq) dgq[e] += a;
        if (some && !isq) dgk[e] += a;
        d[e] *= isq ? L.gq[e] : L.gk[e];
        gu = fmaf(d[e], x[e], gu);
      }
      gu = group_sum<GW>(gu) * p.inv_dim;
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = r * fmaf(-x[e], gu, d[e]);
      if (some && L.on) {
        const Side& s = isq ? p.q : p.k;
        const int hh = isq ? h : h - p.q.heads;
        *reinterpret_cast<u32x4*>(s.out.p + w.b * s.out.sb + w.t * s.out.st + hh * s.out.sh + L.f0 * (int)sizeof(T)) =
            Piece<T>::pack(d);
      }
    }
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

// dgamma: column i of part summed over its rows, 16 columns a workgroup.
__global__ __launch_bounds__(kThreads) void qk_gamma_kernel(const float* part, int rows, int dim,
                                                            float* dq, float* dk) {
  __shared__ float red[16][16];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), sl = threadIdx.x >> 4;
  float s = 0.0f;
  for (int r = sl; r < rows; r += 16) s += part[(int64_t)r * 2 * dim + col];
  red[sl][threadIdx.x & 15] = s;
  __syncthreads();
  if (threadIdx.x >= 16) return;
  s = 0.0f;
  for (int i = 0; i < 16; ++i) s += red[i][threadIdx.x];
  float* out = col < dim ? dq : dk;
  if (out) out[col < dim ? col : col - dim] = s;
}

template <typename T, int GW, bool PAIRS>
void launch(const QkP& p, bool back, int grid, hipStream_t s) {
  if (back)
    hipLaunchKernelGGL((qk_norm_bwd_kernel<T, GW, PAIRS>), dim3((unsigned)grid), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((qk_norm_kernel<T, GW, PAIRS>), dim3((unsigned)grid), dim3(kThreads), 0, s, p);
}

template <typename T, bool PAIRS>
void launch_width(const QkP& p, int gw, bool back, int grid, hipStream_t s) {
  switch (gw) {
    case 2: return launch<T, 2, PAIRS>(p, back, grid, s);
    case 4: return launch<T, 4, PAIRS>(p, back, grid, s);
    case 8: return launch<T, 8, PAIRS>(p, back, grid, s);
    case 16: return launch<T, 16, PAIRS>(p, back, grid, s);
    case 32: return launch<T, 32, PAIRS>(p, back, grid, s);
    default: return launch<T, 64, PAIRS>(p, back, grid, s);
  }
}

bool check_desc(const elasto_qk_norm_t* a) {
  if (!a) return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: NULL description"), false;
  if (a->dtype != ELASTO_BF16 && a->dtype != ELASTO_FP32)
    return fail(ELASTO_ERR_INVALID_ARG, "bad dtype %d", a->dtype), false;
  if (a->batch < 0 || a->tokens < 0 || a->q_heads < 0 || a->kv_heads < 0 ||
      (int64_t)a->q_heads + a->kv_heads < 1 || (int64_t)a->q_heads + a->kv_heads > 65536 ||
      (int64_t)a->batch * a->tokens >= ((int64_t)1 << 31))
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

elasto_status_t run(const elasto_qk_norm_t* a, const elasto_heads_t* q, const elasto_heads_t* k,
                    const elasto_heads_t* dq_out, const elasto_heads_t* dk_out,
                    const elasto_heads_t* q_res, const elasto_heads_t* k_res, float* dq_gamma,
                    float* dk_gamma, void* ws, int64_t ws_bytes, bool back, void* hip_stream) {
  if (!check_desc(a)) return ELASTO_ERR_INVALID_ARG;
  if (!(a->eps > 0.0f) || !(a->eps < INFINITY))
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: eps must be positive and finite");
  if (a->rot_dim < 0 || a->rot_dim > a->head_dim || a->rot_dim % 16)
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: rot_dim %d is not a multiple of 16 in [0, head_dim]", a->rot_dim);
  const int64_t rows = (int64_t)a->batch * a->tokens;
  if (a->rot_dim > 0 && rows > 0) {
    if (!a->cos || !a->sin || !aligned(a->cos, 4) || !aligned(a->sin, 4) || a->table_rows < 1)
      return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: a rotation needs cos, sin and table_rows >= 1");
    if (!a->positions && a->table_rows < a->tokens)
      return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: the tables hold %d rows for %d tokens", a->table_rows, a->tokens);
  }
  if (!aligned(a->positions, 4) || !aligned(a->lens, 4) || !aligned(dq_gamma, 4) || !aligned(dk_gamma, 4))
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: misaligned pointer");
  const int es = a->dtype == ELASTO_BF16 ? 2 : 4, n = 16 / es;
  QkP p = {};
  if (!set_side(&p.q, *a, "q, its result or a gradient", a->q_heads, q, dq_out, q_res, a->q_gamma, back) ||
      !set_side(&p.k, *a, "k, its result or a gradient", a->kv_heads, k, dk_out, k_res, a->k_gamma, back))
    return ELASTO_ERR_INVALID_ARG;
  p.cos = a->cos;
  p.sin = a->sin;
  p.positions = a->positions;
  p.lens = a->lens;
  p.tokens = a->tokens;
  p.dim = a->head_dim;
  p.rot = a->rot_dim;
  p.table_rows = a->table_rows;
  p.chunks = (a->q_heads + a->kv_heads + kHeads - 1) / kHeads;
  p.units = rows * p.chunks;
  p.eps = a->eps;
  p.inv_dim = 1.0f / (float)a->head_dim;
  int gw = 2;
  while (gw * n < a->head_dim) gw *= 2;
  const int groups = kThreads / gw;
  int64_t grid = (p.units + groups - 1) / groups;
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
  } else if (grid > 0x7fffffff) {
    return fail(ELASTO_ERR_INVALID_ARG, "qk_norm: too many head vectors");
  }
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipSuccess;
  if (grid > 0) {
    if (a->dtype == ELASTO_BF16)
      a->interleaved ? launch_width<uint16_t, true>(p, gw, back, (int)grid, s)
                     : launch_width<uint16_t, false>(p, gw, back, (int)grid, s);
    else
      a->interleaved ? launch_width<float, true>(p, gw, back, (int)grid, s)
                     : launch_width<float, false>(p, gw, back, (int)grid, s);
    e = hipGetLastError();
  }
  if (e == hipSuccess && weights) {
    hipLaunchKernelGGL(qk_gamma_kernel, dim3((unsigned)(2 * a->head_dim / 16)), dim3(kThreads), 0, s,
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
  return run(desc, q, k, nullptr, nullptr, q_out, k_out, nullptr, nullptr, nullptr, 0, false,
             hip_stream);
}

elasto_status_t elasto_op_qk_norm_rotate_bwd(const elasto_qk_norm_t* desc, const elasto_heads_t* q,
                                      const elasto_heads_t* k, const elasto_heads_t* dq_out,
                                      const elasto_heads_t* dk_out, const elasto_heads_t* dq,
                                      const elasto_heads_t* dk, float* dq_gamma, float* dk_gamma,
                                      void* workspace, int64_t workspace_bytes, void* hip_stream) {
  return run(desc, q, k, dq_out, dk_out, dq, dk, dq_gamma, dk_gamma, workspace, workspace_bytes,
             true, hip_stream);
}

elasto_status_t elasto_qk_norm_rotate_workspace(const elasto_qk_norm_t* desc, int64_t* bytes) {
  if (!bytes) return fail(ELASTO_ERR_INVALID_ARG, "NULL argument");
  if (!check_desc(desc)) return ELASTO_ERR_INVALID_ARG;
  // A row of 2 * head_dim sums for each workgroup of the largest launch.
  *bytes = (int64_t)kGradBlocks * 2 * desc->head_dim * 4;
  return ELASTO_OK;
}

}  // extern "C"
