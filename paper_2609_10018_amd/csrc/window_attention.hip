// Attention in a sliding window with first tokens that stay visible (sinks):
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j over the keys that query i sees,
//   lse_i = log sum_j exp(scale q_i . k_j)
// (the mask and the packed rows: window.h).  One pass over the visible tiles of
// keys with the running maximum and sum of each row; tiles that no row of the
// workgroup sees are not read, so the cost goes with tokens x window.
//
// Scores are taken transposed, S^T = K Q^T: a lane holds one row's scores, so
// the softmax needs one exchange between the half-waves a tile, and the
// probabilities are the operand of O^T = V^T P^T without moving.  On the bf16
// path they are rounded to bf16 for it, since an fp32 product runs at a ninth of
// the rate (155 and 1400 TFLOP/s): against 64 bits o is off by 0.0023 of itself, root
// mean square, of which rounding o alone makes 0.0017.  Their sum is taken before, in
// fp32, since lse is an fp32 result.
//
// Two shapes of a workgroup of four waves:
// * rows: 128 rows, 32 a wave, which share each tile of keys;
// * keys: 32 rows, the tiles shared out over the waves, joined in LDS at the
//   end: single tokens, and launches that would leave CUs idle.
// Where the workgroups are still few, each row block's tiles are split over
// several, whose unnormalised results a second kernel joins (the running
// maximum and sum of each part go with it).
//
// Every product takes one operand from LDS (1 KB an instruction, at the full rate
// half of what the LDS gives: 16-byte reads alone ran at 229 bytes a cycle of 2.4 GHz
// and CU) and one from registers, where q, the probabilities and the sums stay.
// What bounds it, and measured times (of several cards):
// * heads of 64: the vector ALU most (64 keys x 32 rows: 16 matrix instructions of 32
//   cycles, ~155 vector ones, 32 of them exponentials): it is busy 60% of the
//   launch's cycles, the matrix cores 31%, the LDS 16%, and a SIMD holds three waves on
//   average.  8 x 4097 tokens, 12 heads, 511 keys to either side: 150-155 us, 640
//   TFLOP/s;
// * heads of 128: no unit alone, with two waves a SIMD, as 204 registers allow (vector
//   ALU 41%, matrix cores 37%).  Causal, 16/4 heads: 2 x 8192 tokens, 1024 keys: 176-188
//   us, 690-730 TFLOP/s; 2 x 4096, all keys: 158, 870;
// * single tokens: the cache's bytes.  32 sequences, 16/4 heads of 128, 2048 of
//   8192 keys each: 32 us with other tensors at each call, 4.2 TB/s (a copy: 5.1),
//   28 with two sets of them in turn; fp32 70 us, 3.9 TB/s;
// * fp32: matrix instructions of 64 cycles, and at small sizes the latency of a
//   wave's two or three tiles.  5 x 777 padded tokens, 6 heads of 64, 200 keys:
//   25 us; 2 x 2048 x 8 heads of 128, 512 keys: 117-120 us.
#include <math.h>

#include <algorithm>

#include "layout.h"
#include "window.h"
#include "window_args.h"

namespace elasto {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

struct FwdP {
  View q, k, v, o;
  float* lse;              // [batch][heads][q_tokens] or NULL
  const int32_t *q_lens, *k_lens;
  int q_tokens, k_tokens, heads, kv_heads, group;
  Mask mask;
  float c2;                // scale * log2(e)
  int row_blocks, splits;
  int64_t blocks;
  float *part_o, *part_ml;  // splits > 1: [batch * kv_heads][split][row][HD], [...][2]
};

template <typename T, int HD, bool KEYS>
struct Shape {
  static constexpr int kSub = !KEYS && sizeof(T) == 2 ? 2 : 1;  // 32-key blocks of a tile
  static constexpr int kKeys = 32 * kSub;
  static constexpr int kTile = Tile<T, HD>::template bytes<kKeys>();  // of K (and of V)
  static constexpr int kPrivate = KEYS ? kWaves : 1;            // tiles held at once
  // fp32 waves with tiles of their own: one, which leaves room for two
  // workgroups on a CU (2 x 1024 tokens x 6 heads of 64: 21 us, with two 26 us).
  static constexpr int kBuffers = KEYS && sizeof(T) == 4 ? 1 : 2;
  // Of 64 features even that one holds K and V in turns, V on its way during the
  // softmax: three workgroups on a CU (5 x 777 tokens x 6 heads, 200 keys: 29 us
  // with both at once, 22 in turns, though 4 of its registers are spilled; 2 x 2048
  // x 8, 512 keys, two whole rounds otherwise: 56 and 60).  Heads of 128 have no registers for more workgroups.
  static constexpr bool kTurns = KEYS && sizeof(T) == 4 && HD == 64;
  static constexpr int kStaged = (kTurns ? 1 : 2) * kTile;  // of a tile
  static constexpr int kPerSimd = kTurns ? 3 : sizeof(T) == 2 || HD == 64 ? 2 : 1;  // waves
  static constexpr int kOs = HD + 4;  // floats of a row of the join
  static constexpr int kJoin = KEYS ? kWaves * 32 * kOs * 4 + kWaves * 64 * 4 : 0;
  static constexpr int kLds = std::max(kPrivate * kBuffers * kStaged, kJoin);
  static constexpr int kRows = KEYS ? 32 : 32 * kWaves;
};

// The running state of 32 rows: a lane's row is column l % 32 of S^T.
template <typename T, int HD>
struct State {
  f32x16 o[HD / 32];
  static constexpr float kRise = 8.0f;
  float m, l;  // reference of the exponentials (a raw score), this half-wave's part of the sum

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < HD / 32; ++n) zero(o[n]);
    m = -INFINITY;
    l = 0.0f;
  }

  __device__ __forceinline__ void hold() {
#pragma unroll
    for (int n = 0; n < HD / 32; ++n) stay<sizeof(T) == 2 || HD == 64>(o[n]);
  }

  // One tile of SUB * 32 keys from j0 on; low, high, sinks: as for hidden().
  // scored: called when the keys have been read; values: before the values are.
  template <int SUB, typename F, typename W>
  __device__ __forceinline__ void tile(const char* kt, const char* vt, int j0, const Frag<T>* q,
                                       float c2, bool low, bool high, bool sinks, const Keys& ks, int h,
                                       const typename Tile<T, HD>::Reader& rd, F&& scored, W&& values) {
    f32x16 s[SUB];
#pragma unroll
    for (int b = 0; b < SUB; ++b) {
      Frag<T> a;
      rd.operand(kt, b * 32, 0, a);
      if (!low && !high) {
        zero(s[b]);
        s[b] = mma(a, q[0], s[b]);
      } else {
        s[b] = mma(a, q[0], hidden(j0 + b * 32 + 4 * h, ks, low, high, sinks));
      }
    }
#pragma unroll
    for (int b = 0; b < SUB; ++b)
#pragma unroll
      for (int kk = 1; kk < HD / 16; ++kk) {
        Frag<T> a;
        rd.operand(kt, b * 32, kk, a);
        s[b] = mma(a, q[kk], s[b]);
      }
    scored();
    float t = s[0][0];
#pragma unroll
    for (int b = 0; b < SUB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) t = fmaxf(t, s[b][i]);
    t = half_max(t);
    // The reference of the exponentials follows the maximum only where that has
    // risen by more than 2^kRise since: terms of up to 2^kRise are as exact, and
    // a wave of 32 rows would rescale its sums in most tiles otherwise.
    if (__any((t - m) * c2 > kRise)) {
      const float to = fmaxf(m, t);
      const float f = to > m ? __builtin_amdgcn_exp2f((m - to) * c2) : 1.0f;
      l *= f;
#pragma unroll
      for (int n = 0; n < HD / 32; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[n][i] *= f;
      m = to;
    }
    const float off = m == -INFINITY ? 0.0f : -m * c2;  // nothing seen so far: all terms are 0
#pragma unroll
    for (int b = 0; b < SUB; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c2, off));
        l += s[b][i];
      }
      if (b == 0) values();
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        Frag<T> pf;
        as_operand(s[b], u, pf);
#pragma unroll
        for (int n = 0; n < HD / 32; ++n) {
          Frag<T> a;
          rd.transposed(vt, b * 32 + u * 16, n, a);
          o[n] = mma(a, pf, o[n]);
        }
      }
    }
  }
};

template <typename T, int HD, bool KEYS>
__global__ __launch_bounds__(kThreads, (Shape<T, HD, KEYS>::kPerSimd)) void window_fwd_kernel(FwdP p) {
  using S = Shape<T, HD, KEYS>;
  using Tl = Tile<T, HD>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = xcd_order(blockIdx.x, p.blocks);
  const int z = (int)(id % p.splits);
  const int64_t rest = id / p.splits;
  const int64_t bk = rest / p.row_blocks;
  const int turn = (int)(rest - bk * p.row_blocks);
  const int rb = p.mask.causal ? p.row_blocks - 1 - turn : turn;  // late rows, which have the most keys, first
  const int b = (int)(bk / p.kv_heads), hk = (int)(bk - (int64_t)b * p.kv_heads);
  const int ql = clamp_len(p.q_lens, b, p.q_tokens), kl = clamp_len(p.k_lens, b, p.k_tokens);
  const int G = p.group, rows = ql * G;
  const int first = rb * S::kRows;
  if (first >= rows) return;

  // This lane's row, this wave's and the workgroup's positions.
  const int wfirst = first + (KEYS ? 0 : 32 * wave);
  const int row = wfirst + (lane & 31), rc = min(row, rows - 1);
  const int i = rc / G, g = rc - i * G, shift = kl - ql;
  const Keys mine = keys_of(p.mask, i + shift, kl);
  const Keys a0 = keys_of(p.mask, first / G + shift, kl);
  const Keys a1 = keys_of(p.mask, (min(first + S::kRows, rows) - 1) / G + shift, kl);
  const int wl = min(wfirst, rows - 1);
  const Keys w0 = keys_of(p.mask, wl / G + shift, kl);
  const Keys w1 = keys_of(p.mask, (min(wl + 32, rows) - 1) / G + shift, kl);
  const bool idle = wfirst >= rows;

  // Tiles: those of the sinks, then those of the window.
  const int sink_tiles = a1.hs >= 0 ? a1.hs / S::kKeys + 1 : 0;
  const int t0 = max(a0.lo / S::kKeys, sink_tiles);
  const int tiles = sink_tiles + (a1.hi >= a0.lo ? max(a1.hi / S::kKeys + 1 - t0, 0) : 0);
  const int zs = (int)((int64_t)tiles * z / p.splits), ze = (int)((int64_t)tiles * (z + 1) / p.splits);
  auto key0 = [&](int n) { return (n < sink_tiles ? n : t0 + n - sink_tiles) * S::kKeys; };

  const SeenKeys seen(a0, a1);
  const KeyRows kr(p.k.p + b * p.k.sb + hk * p.k.sh, p.k.st, seen, Tl::kRow);
  const KeyRows vr(p.v.p + b * p.v.sb + hk * p.v.sh, p.v.st, seen, Tl::kRow);
  using Ld = typename Tl::template Loads<S::kKeys, KEYS ? 1 : kWaves>;
  const int lw = KEYS ? 0 : wave;
  auto stage = [&](int n, char* dst) {
    kr.template issue<Ld>(dst, lw, lane, key0(n), Tl::kRow);
    if constexpr (!S::kTurns) vr.template issue<Ld>(dst + S::kTile, lw, lane, key0(n), Tl::kRow);
  };

  const typename Tl::Reader rd(lane);
  State<T, HD> st;
  st.clear();
  Frag<T> q[HD / 16];
  const char* qrow = p.q.p + b * p.q.sb + (int64_t)i * p.q.st + (int64_t)(hk * G + g) * p.q.sh;
#pragma unroll
  for (int kk = 0; kk < HD / 16; ++kk) load_operand(qrow, kk, h, q[kk]);

  auto compute = [&](int n, char* buf) __attribute__((always_inline)) {
    const int j0 = key0(n), j1 = j0 + S::kKeys - 1;
    st.hold();
    // Unless this wave's rows see nothing of the tile.
    if (!idle && (j0 <= w1.hs || (j1 >= w0.lo && j0 <= w1.hi)))
      st.template tile<S::kSub>(
          buf, buf + S::kStaged - S::kTile, j0, q, p.c2, j0 < w1.lo, j1 > w0.hi, j0 <= w1.hs, mine, h, rd,
          [&]() __attribute__((always_inline)) {
            if constexpr (S::kTurns) {
              asm volatile("" ::: "memory");
              wait_lds();
              vr.template issue<Ld>(buf, lw, lane, j0, Tl::kRow);
              asm volatile("" ::: "memory");
            }
          },
          [&]() __attribute__((always_inline)) {
            if constexpr (S::kTurns) settle();
          });
    st.hold();
  };
  constexpr int kLoads = (S::kTurns ? 1 : 2) * Ld::kLoads;
  char* mem = smem + (KEYS ? wave * S::kBuffers * S::kStaged : 0);
  const int step = KEYS ? kWaves : 1;
  int n = zs + (KEYS ? wave : 0);
  if constexpr (S::kBuffers == 2) {
    // cur and next never overlap: without that word the compiler waits for the
    // next tile's loads before it reads this one.
    auto body = [&](char* __restrict__ cur, char* __restrict__ next) __attribute__((always_inline)) {
      const bool more = n + step < ze;
      if (more) stage(n + step, next);
      asm volatile("" ::: "memory");
      if (more) wait_vm_lds<kLoads>();
      else wait_vm_lds<0>();
      if (!KEYS) __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      compute(n, cur);
      // Every read of this tile is done before the next but one overwrites it.
      asm volatile("" ::: "memory");
      wait_lds();
      if (!KEYS) __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    if (n < ze) stage(n, mem);
    settle();
    for (int cur = 0; n < ze; n += step, cur ^= 1)
      body(mem + cur * 2 * S::kTile, mem + (cur ^ 1) * 2 * S::kTile);
  } else {
    for (; n < ze; n += step) {
      stage(n, mem);
      asm volatile("" ::: "memory");
      wait_vm_lds<0>();
      if (!KEYS) __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      compute(n, mem);
      asm volatile("" ::: "memory");
      wait_lds();
      if (!KEYS) __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
  }
  st.l = half_sum(st.l);

  const int head = hk * G + g;
  const int64_t prow = (bk * p.splits + z) * ((int64_t)p.q_tokens * G) + row;
  if constexpr (!KEYS) {
    if (row >= rows) return;
    if (p.splits > 1) {
      float* po = p.part_o + prow * HD;
#pragma unroll
      for (int n = 0; n < HD / 32; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          store4(po + n * 32 + 8 * e + 4 * h, st.o[n][4 * e], st.o[n][4 * e + 1], st.o[n][4 * e + 2], st.o[n][4 * e + 3]);
      if (h == 0) {
        p.part_ml[prow * 2] = st.m;
        p.part_ml[prow * 2 + 1] = st.l;
      }
      return;
    }
    const float inv = st.l > 0.0f ? 1.0f / st.l : st.l == 0.0f ? 0.0f : NAN;
    T* orow = reinterpret_cast<T*>(p.o.p + b * p.o.sb + (int64_t)i * p.o.st + (int64_t)head * p.o.sh);
#pragma unroll
    for (int n = 0; n < HD / 32; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        store4(orow + n * 32 + 8 * e + 4 * h, st.o[n][4 * e] * inv, st.o[n][4 * e + 1] * inv,
               st.o[n][4 * e + 2] * inv, st.o[n][4 * e + 3] * inv);
    if (p.lse && h == 0)
      p.lse[((int64_t)b * p.heads + head) * p.q_tokens + i] =
          st.l == 0.0f ? -INFINITY : fmaf(st.m, p.c2, log2f(st.l)) * kLn2;
  } else {
    // Join the waves: their maxima and sums first, then their rows at the
    // common maximum.
    float* ml = reinterpret_cast<float*>(smem + kWaves * 32 * S::kOs * 4);
    float* jo = reinterpret_cast<float*>(smem);
    __syncthreads();  // every wave is done with its tiles
    if (h == 0) {
      ml[wave * 64 + lane] = st.m;
      ml[wave * 64 + 32 + lane] = st.l;
    }
    __syncthreads();
    float M = -INFINITY, L = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, ml[w * 64 + (lane & 31)]);
    const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      L += ml[w * 64 + 32 + (lane & 31)] * __builtin_amdgcn_exp2f((ml[w * 64 + (lane & 31)] - base) * p.c2);
    const float f = __builtin_amdgcn_exp2f((st.m - base) * p.c2);
    float* jr = jo + (wave * 32 + (lane & 31)) * S::kOs;
#pragma unroll
    for (int n = 0; n < HD / 32; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        store4(jr + n * 32 + 8 * e + 4 * h, st.o[n][4 * e] * f, st.o[n][4 * e + 1] * f,
               st.o[n][4 * e + 2] * f, st.o[n][4 * e + 3] * f);
    // The joined maximum and sum of row r, for the threads that write it.
    __syncthreads();
    if (wave == 0 && h == 0) {
      ml[lane] = M;
      ml[32 + lane] = L;
    }
    __syncthreads();
    for (int u = threadIdx.x; u < 32 * (HD / 4); u += kThreads) {
      const int r = u / (HD / 4), c = (u - r * (HD / 4)) * 4, gr = first + r;
      if (gr >= rows) break;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(jo + (w * 32 + r) * S::kOs + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += x[e];
      }
      const float Lr = ml[32 + r];
      if (p.splits > 1) {
        const int64_t pr = (bk * p.splits + z) * ((int64_t)p.q_tokens * G) + gr;
        store4(p.part_o + pr * HD + c, v[0], v[1], v[2], v[3]);
        if (c == 0) {
          p.part_ml[pr * 2] = ml[r];
          p.part_ml[pr * 2 + 1] = Lr;
        }
      } else {
        const float inv = Lr > 0.0f ? 1.0f / Lr : Lr == 0.0f ? 0.0f : NAN;
        const int qi = gr / G, hd = hk * G + gr - qi * G;
        T* orow = reinterpret_cast<T*>(p.o.p + b * p.o.sb + (int64_t)qi * p.o.st + (int64_t)hd * p.o.sh);
        store4(orow + c, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        if (p.lse && c == 0)
          p.lse[((int64_t)b * p.heads + hd) * p.q_tokens + qi] =
              Lr == 0.0f ? -INFINITY : fmaf(ml[r], p.c2, log2f(Lr)) * kLn2;
      }
    }
  }
}

// Joins the splits of a row: HD / 4 threads a row.
template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void window_join_kernel(FwdP p) {
  constexpr int kPer = HD / 4;
  const int64_t at = (int64_t)blockIdx.x * (kThreads / kPer) + threadIdx.x / kPer;
  const int c = (threadIdx.x % kPer) * 4;
  const int64_t rmax = (int64_t)p.q_tokens * p.group, bk = at / rmax;
  const int row = (int)(at - bk * rmax);
  const int b = (int)(bk / p.kv_heads), hk = (int)(bk - (int64_t)b * p.kv_heads);
  const int64_t total = p.blocks / p.splits / p.row_blocks * rmax;
  if (at >= total || row >= clamp_len(p.q_lens, b, p.q_tokens) * p.group) return;
  float M = -INFINITY, L = 0.0f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int z = 0; z < p.splits; ++z) M = fmaxf(M, p.part_ml[((bk * p.splits + z) * rmax + row) * 2]);
  const float base = M == -INFINITY ? 0.0f : M;
#pragma unroll 4
  for (int z = 0; z < p.splits; ++z) {
    const int64_t pr = (bk * p.splits + z) * rmax + row;
    const float f = __builtin_amdgcn_exp2f((p.part_ml[pr * 2] - base) * p.c2);
    const f32x4 x = *reinterpret_cast<const f32x4*>(p.part_o + pr * HD + c);
    L = fmaf(p.part_ml[pr * 2 + 1], f, L);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(x[e], f, v[e]);
  }
  const float inv = L > 0.0f ? 1.0f / L : L == 0.0f ? 0.0f : NAN;
  const int i = row / p.group, head = hk * p.group + row - i * p.group;
  T* orow = reinterpret_cast<T*>(p.o.p + b * p.o.sb + (int64_t)i * p.o.st + (int64_t)head * p.o.sh);
  store4(orow + c, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  if (p.lse && c == 0)
    p.lse[((int64_t)b * p.heads + head) * p.q_tokens + i] =
        L == 0.0f ? -INFINITY : fmaf(M, p.c2, log2f(L)) * kLn2;
}

// How a launch is cut: workgroup shape, row blocks, splits.
struct Cut {
  bool keys;
  int row_blocks, splits;
};
Cut cut_of(const elasto_window_t& a) {
  constexpr int kCUs = 256;
  const int64_t pairs = (int64_t)a.batch * a.kv_heads, rows = (int64_t)a.q_tokens * (a.heads / a.kv_heads);
  Cut c;
  // fp32 products take 16 times as long a tile, so a launch of few workgroups
  // wants its tiles shared out over waves: 2 x 1024 tokens x 6 heads of 64 (96
  // workgroups of rows) 44 us by rows, 21 by keys; 2 x 4096 x 16 of 128 (1024)
  // 643 and 714 us.  In bf16 the two are within 3 us of each other there, and by
  // rows K and V are read a quarter as often.
  c.keys = rows <= 32 || (a.dtype == ELASTO_FP32 && pairs * ((rows + 127) / 128) < 512);
  const int per = c.keys ? 32 : 128;
  c.row_blocks = (int)((rows + per - 1) / per);
  const int64_t blocks = pairs * c.row_blocks;
  // Keys that a row block can see, in shares of at least 256 a workgroup.
  const int64_t reach = (a.causal ? (int64_t)a.window : 2 * (int64_t)a.window - 1) + per / (a.heads / a.kv_heads);
  const int64_t keys = std::min<int64_t>(a.k_tokens, reach + a.sinks);
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(keys / 256, 128));
  if (!c.keys) {
    // Two workgroups a CU, if whole shares make them (a CU holds two of heads of 128,
    // four of 64 in bf16, but two keep it busy): 5 x 1023 tokens x 12 heads of 64 (480 of
    // them) in 1 share 33 us, in 2 42; 2 x 2048 x 8, causal (256), in 1 41, in 2 37.
    c.splits = (int)std::max<int64_t>(1, std::min(2 * kCUs / std::max<int64_t>(blocks, 1), most));
    return c;
  }
  // By keys, a CU holds one workgroup of heads of 128, two of 64 (fp32 three), and
  // what counts is how many rounds of them there are: rounds times a share's length,
  // with 160 keys' worth (of 64 features twice that) for starting it, and 128 for
  // the join.
  // 32 x 16/4 heads of 128 on 2048 keys in 2 shares (one round) 28.4 us, in 4
  // (two) 30.4, in 8 36; 32 x 12 of 64 in 1 share 34.6, in 2 37.6; 40 x 32/8 of
  // 128 on 4096 in 1 146 (a round and a quarter takes two), in 4 121.
  const int64_t slots = kCUs * (a.head_dim == 128 ? 1 : a.dtype == ELASTO_FP32 ? 3 : 2);
  const double start = 160.0 * 128 / a.head_dim, join = 128.0 * 128 / a.head_dim;
  double best = INFINITY;
  c.splits = 1;
  for (int64_t n = 1; n <= most && blocks * n <= 4 * slots + blocks; ++n) {
    const double cost =
        (double)((blocks * n + slots - 1) / slots) * ((double)keys / n + start) + (n > 1 ? join : 0.0);
    if (cost < best) best = cost, c.splits = (int)n;
  }
  return c;
}

template <typename T, int HD, bool KEYS>
hipError_t launch(const FwdP& p, hipStream_t s) {
  constexpr int lds = Shape<T, HD, KEYS>::kLds;
  static_assert(lds <= 160 * 1024, "LDS");
  hipLaunchKernelGGL((window_fwd_kernel<T, HD, KEYS>), dim3((unsigned)p.blocks), dim3(kThreads), lds, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  const int64_t rows = p.blocks / p.splits / p.row_blocks * p.q_tokens * p.group;
  constexpr int kRows = kThreads / (HD / 4);
  hipLaunchKernelGGL((window_join_kernel<T, HD>), dim3((unsigned)((rows + kRows - 1) / kRows)),
                     dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_dim(const FwdP& p, int dim, bool keys, hipStream_t s) {
  if (dim == 64) return keys ? launch<T, 64, true>(p, s) : launch<T, 64, false>(p, s);
  return keys ? launch<T, 128, true>(p, s) : launch<T, 128, false>(p, s);
}

int64_t split_floats(const elasto_window_t& a, const Cut& c) {
  return c.splits == 1 ? 0 : (int64_t)a.batch * a.heads * a.q_tokens * c.splits * (a.head_dim + 2);
}

}  // namespace

int64_t window_fwd_workspace(const elasto_window_t& a) { return split_floats(a, cut_of(a)) * 4; }

hipError_t launch_window_fwd(const elasto_window_t& a, const WindowTensors& t, void* ws, hipStream_t s) {
  const Cut c = cut_of(a);
  FwdP p = {};
  p.q = t.q; p.k = t.k; p.v = t.v; p.o = t.o;
  p.lse = t.lse;
  p.q_lens = a.q_lens;
  p.k_lens = a.k_lens;
  p.q_tokens = a.q_tokens;
  p.k_tokens = a.k_tokens;
  p.heads = a.heads;
  p.kv_heads = a.kv_heads;
  p.group = a.heads / a.kv_heads;
  p.mask = Mask{a.causal, a.window, a.sinks};
  p.c2 = a.scale * kLog2e;
  p.row_blocks = c.row_blocks;
  p.splits = c.splits;
  p.blocks = (int64_t)a.batch * a.kv_heads * c.row_blocks * c.splits;
  p.part_o = static_cast<float*>(ws);
  p.part_ml = p.part_o + (int64_t)a.batch * a.heads * a.q_tokens * c.splits * a.head_dim;
  if (p.blocks >= kMaxBlocks) return hipErrorInvalidConfiguration;
  return a.dtype == ELASTO_BF16 ? launch_dim<uint16_t>(p, a.head_dim, c.keys, s)
                                : launch_dim<float>(p, a.head_dim, c.keys, s);
}

}  // namespace elasto
