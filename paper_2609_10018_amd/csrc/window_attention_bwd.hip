// Backward of the windowed attention (window_attention.hip).  With
// P = exp(scale S - lse) inside the mask, 0 outside, and D_i = do_i . o_i:
//   dv_j = sum_i P_ij do_i,  dS = P (.) (do v^T - D),
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i.
// The scores are formed again from q, k and lse rather than kept.  Two kernels,
// each of which sums in one order in registers, so there are no atomics and the
// gradients are the same bits every time:
// * rows: 32 packed rows a wave, over the tiles of keys that they see: dq, and
//   the row's lse (base 2) and D for the second kernel;
// * keys: 32 keys a wave, over the tiles of packed rows that see them: dk and
//   dv, summed over the heads of the group.
// Seven products of the size of S where five would do: what the two extra ones
// cost is less than adding dq up in memory would.
//
// P and dS are rounded to bf16 (bf16 path) as operands of the products that
// sum them, for the same reason and price as in the forward pass (root mean square
// 0.0024 of the gradients against 64 bits, 0.0017 for rounding the results alone);
// all sums are fp32.
//
// Bound by no unit alone: of the launches' cycles the matrix cores are busy 43%
// (rows) and 40% (keys), the vector ALU 33% and 27%, the LDS 22% and 25%.  Registers
// allow two waves a SIMD, each of which takes a sub-block's products, exponentials
// and products in turn, with two barriers a tile.  2 x 8192 tokens, 16/4 heads of
// 128, 1024 keys and 4 sinks: 514-529 us by the card (rows ~220, keys ~280, sinks 25,
// join 6 under a profiler); counted as five products 610-630 TFLOP/s, as the seven
// that run 850-880.  Without its exponentials and masks the row kernel ran at 1.24
// PFLOP/s, a library product of 8192^3 runs at 1.4.  fp32, 2 x 2048 x 8 heads of 128,
// 512 keys: 350 us.
//
// A key among the sinks is seen by every later row.  The key kernel takes the
// rows that see the first tile's keys through their windows, as for any tile;
// the rows behind them, which see the sinks alone, are a kernel of their own,
// where a workgroup's waves take different rows for the same 32 keys, and whose
// parts are added up in order.
#include <algorithm>

#include "layout.h"
#include "window.h"
#include "window_args.h"

namespace elasto {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kKeys = 32 * kWaves;  // keys of a workgroup of the key kernel
static_assert(kMaxSinks <= kKeys, "the sinks lie in the first tile of keys");

struct BwdP {
  View q, k, v, o, dout, dq, dk, dv;
  const float* lse;
  const int32_t *q_lens, *k_lens;
  int q_tokens, k_tokens, heads, kv_heads, group;
  Mask mask;
  float scale, c2;
  int64_t blocks;
  unsigned div_mul, div_shift;  // r / group = umulhi(8 r, div_mul) >> div_shift, r < 2^29
  int row_blocks;          // row kernel
  int key_tiles;           // key kernel
  int parts, sink_groups;  // sink kernel (parts 0: none): parts of the rows, 32s of sinks
  float2* stat;            // [batch * kv_heads][row]: lse in base 2, D
  float* part;             // [batch * kv_heads][key kernel, parts][dk, dv][kMaxSinks][HD]
  int row_parts;           // key kernel: parts of a tile's rows; more than one: their sums go to
  float* row_part;         // [batch * kv_heads][row part][dk, dv][k_tokens][HD]
};

template <typename T, int HD>
struct Shape {
  static constexpr int kSub = sizeof(T) == 2 ? 2 : 1;
  static constexpr int kRows = 32 * kSub;                    // of a staged tile
  static constexpr int kTile = Tile<T, HD>::template bytes<kRows>();
  static constexpr int kStat = 64 * 8 * 2;                   // a tile's lse and D, and a spare
  static constexpr int kLdsRow = 2 * 2 * kTile;
  static constexpr int kLdsKey = 2 * (2 * kTile + kStat);
};

template <typename T, int HD>
struct SinkShape {
  static constexpr int kTile = Tile<T, HD>::template bytes<32>();
  static constexpr int kBuf = 2 * kTile + 256;
  static constexpr int kBuffers = kWaves * 2 * kBuf <= 144 * 1024 ? 2 : 1;
  static constexpr int kOs = HD + 4;
  static constexpr int kLds = std::max(kWaves * kBuffers * kBuf, kWaves * 32 * kOs * 4);
  static_assert(kLds <= 160 * 1024, "LDS");
};

template <typename T, int HD>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 || HD == 64 ? 2 : 1)) void window_dq_kernel(BwdP p) {
  using S = Shape<T, HD>;
  using Tl = Tile<T, HD>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = xcd_order(blockIdx.x, p.blocks);
  const int64_t bk = id / p.row_blocks;
  const int turn = (int)(id - bk * p.row_blocks);
  const int rb = p.mask.causal ? p.row_blocks - 1 - turn : turn;  // late rows, which have the most keys, first
  const int b = (int)(bk / p.kv_heads), hk = (int)(bk - (int64_t)b * p.kv_heads);
  const int ql = clamp_len(p.q_lens, b, p.q_tokens), kl = clamp_len(p.k_lens, b, p.k_tokens);
  const int G = p.group, rows = ql * G, shift = kl - ql;
  const int first = rb * 32 * kWaves;
  if (first >= rows) return;
  const int wfirst = first + 32 * wave;
  const int row = wfirst + l32, rc = min(row, rows - 1);
  const int i = rc / G, head = hk * G + rc - i * G;
  const Keys mine = keys_of(p.mask, i + shift, kl);
  const Keys a0 = keys_of(p.mask, first / G + shift, kl);
  const Keys a1 = keys_of(p.mask, (min(first + 32 * kWaves, rows) - 1) / G + shift, kl);
  const int wl = min(wfirst, rows - 1);
  const Keys w0 = keys_of(p.mask, wl / G + shift, kl);
  const Keys w1 = keys_of(p.mask, (min(wl + 32, rows) - 1) / G + shift, kl);
  const bool idle = wfirst >= rows;
  const int sink_tiles = a1.hs >= 0 ? a1.hs / S::kRows + 1 : 0;
  const int t0 = max(a0.lo / S::kRows, sink_tiles);
  const int tiles = sink_tiles + (a1.hi >= a0.lo ? max(a1.hi / S::kRows + 1 - t0, 0) : 0);
  auto key0 = [&](int n) { return (n < sink_tiles ? n : t0 + n - sink_tiles) * S::kRows; };
  const SeenKeys seen(a0, a1);
  const KeyRows kr(p.k.p + b * p.k.sb + hk * p.k.sh, p.k.st, seen, Tl::kRow);
  const KeyRows vr(p.v.p + b * p.v.sb + hk * p.v.sh, p.v.st, seen, Tl::kRow);
  using Ld = typename Tl::template Loads<S::kRows, kWaves>;
  auto stage = [&](int n, char* dst) {
    kr.template issue<Ld>(dst, wave, lane, key0(n), Tl::kRow);
    vr.template issue<Ld>(dst + S::kTile, wave, lane, key0(n), Tl::kRow);
  };
  const typename Tl::Reader rd(lane);

  Frag<T> q[HD / 16], d[HD / 16];
  const char* qrow = p.q.p + b * p.q.sb + (int64_t)i * p.q.st + (int64_t)head * p.q.sh;
  const char* drow = p.dout.p + b * p.dout.sb + (int64_t)i * p.dout.st + (int64_t)head * p.dout.sh;
  const char* orow = p.o.p + b * p.o.sb + (int64_t)i * p.o.st + (int64_t)head * p.o.sh;
  float D = 0.0f;
#pragma unroll
  for (int kk = 0; kk < HD / 16; ++kk) {
    Frag<T> of;
    load_operand(qrow, kk, h, q[kk]);
    load_operand(drow, kk, h, d[kk]);
    load_operand(orow, kk, h, of);
    D = dot(d[kk], of, D);
  }
  D = half_sum(D);
  float l2 = p.lse[((int64_t)b * p.heads + head) * p.q_tokens + i] * kLog2e;
  if (l2 == -INFINITY) l2 = 0.0f;  // a row that sees nothing: every term is masked
  if (h == 0 && row < rows) p.stat[bk * ((int64_t)p.q_tokens * G) + row] = make_float2(l2, D);

  constexpr bool kStay = sizeof(T) == 2 || HD == 64;
  f32x16 dq[HD / 32];
#pragma unroll
  for (int n = 0; n < HD / 32; ++n) zero(dq[n]);
  constexpr int kLoads = 2 * Ld::kLoads;
  // cur and next never overlap: without that word the compiler waits for the
  // next tile's loads before it reads this one.
  auto body = [&](int n, const char* __restrict__ kt, char* __restrict__ next) __attribute__((always_inline)) {
    const char* vt = kt + S::kTile;
    if (n + 1 < tiles) {
      stage(n + 1, next);
      wait_and_meet<kLoads>();
    } else {
      wait_and_meet<0>();
    }
    const int j0 = key0(n), j1 = j0 + S::kRows - 1;
#pragma unroll
    for (int f = 0; f < HD / 32; ++f) stay<kStay>(dq[f]);
    // Unless this wave's rows see nothing of the tile.
    if (!idle && (j0 <= w1.hs || (j1 >= w0.lo && j0 <= w1.hi))) {
      const bool low = j0 < w1.lo, high = j1 > w0.hi;
#pragma unroll
      for (int s = 0; s < S::kSub; ++s) {
        f32x16 sc, dp;
        Frag<T> a;
        rd.operand(kt, s * 32, 0, a);
        if (!low && !high) {
          zero(sc);
          sc = mma(a, q[0], sc);
        } else {
          sc = mma(a, q[0], hidden(j0 + s * 32 + 4 * h, mine, low, high, j0 <= w1.hs));
        }
        zero(dp);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          if (kk > 0) {
            rd.operand(kt, s * 32, kk, a);
            sc = mma(a, q[kk], sc);
          }
          rd.operand(vt, s * 32, kk, a);
          dp = mma(a, d[kk], dp);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sc[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], p.c2, -l2)) * (dp[e] - D);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          Frag<T> df;
          as_operand(sc, u, df);
#pragma unroll
          for (int f = 0; f < HD / 32; ++f) {
            Frag<T> a;
            rd.transposed(kt, s * 32 + u * 16, f, a);
            dq[f] = mma(a, df, dq[f]);
          }
        }
      }
    }
#pragma unroll
    for (int f = 0; f < HD / 32; ++f) stay<kStay>(dq[f]);
    asm volatile("" ::: "memory");
    wait_lds();  // every read of this tile is done before the next but one overwrites it
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  if (tiles > 0) stage(0, smem);
  settle();
  for (int n = 0; n < tiles; ++n) body(n, smem + (n & 1) * 2 * S::kTile, smem + ((n + 1) & 1) * 2 * S::kTile);
  if (row >= rows) return;
  T* out = reinterpret_cast<T*>(p.dq.p + b * p.dq.sb + (int64_t)i * p.dq.st + (int64_t)head * p.dq.sh);
#pragma unroll
  for (int n = 0; n < HD / 32; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      store4(out + n * 32 + 8 * e + 4 * h, dq[n][4 * e] * p.scale, dq[n][4 * e + 1] * p.scale,
             dq[n][4 * e + 2] * p.scale, dq[n][4 * e + 3] * p.scale);
}

// Packed rows that see key j: [lo, hi]; sink: as one of the sinks, if it is one.
struct Rows {
  int lo, hi;
};
__device__ __forceinline__ Rows rows_of(const Mask& m, int j, int shift, int rows, int G, bool sink) {
  const int plo = m.causal ? j : sink && j < m.sinks ? 0 : j - m.window + 1;
  const int64_t phi = sink && j < m.sinks ? (int64_t)1 << 31 : (int64_t)j + m.window - 1;
  Rows r;
  r.lo = (int)min((int64_t)rows, max((int64_t)0, (int64_t)(plo - shift) * G));
  if (!m.causal && sink && j < m.sinks) r.lo = 0;
  r.hi = (int)min((int64_t)rows - 1, max((int64_t)-1, (phi - shift + 1) * G - 1));
  return r;
}

// 32 keys' side of the products: a lane's key is column l % 32.
template <typename T, int HD>
struct KeySide {
  static constexpr bool kStay = sizeof(T) == 2 || HD == 64;
  Frag<T> k[HD / 16], v[HD / 16];
  f32x16 dk[HD / 32], dv[HD / 32];

  // seen: by any row (what the memory of another key holds meets no product).
  __device__ __forceinline__ void load(const char* krow, const char* vrow, int h, bool seen) {
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk) {
      if (seen) {
        load_operand(krow, kk, h, k[kk]);
        load_operand(vrow, kk, h, v[kk]);
      } else {
        k[kk] = Frag<T>{};
        v[kk] = Frag<T>{};
      }
    }
#pragma unroll
    for (int n = 0; n < HD / 32; ++n) {
      zero(dk[n]);
      zero(dv[n]);
    }
  }
  __device__ __forceinline__ void hold() {
#pragma unroll
    for (int n = 0; n < HD / 32; ++n) stay<kStay>(dk[n]), stay<kStay>(dv[n]);
  }

  // SUB * 32 rows of q and dout, and their lse and D (st: two rows each); from
  // and len: which of them see the lane's key.
  template <int SUB>
  __device__ __forceinline__ void rows(const char* qt, const char* dt, const f32x4* st, bool inside,
                                       int from, unsigned len, float c2, int h,
                                       const typename Tile<T, HD>::Reader& rd) {
#pragma unroll 1
    for (int s = 0; s < SUB; ++s) {
      f32x16 sc, dp;
      Frag<T> a;
      rd.operand(qt, s * 32, 0, a);
      if (inside) {
        zero(sc);
        sc = mma(a, k[0], sc);
      } else {
        sc = mma(a, k[0], hidden(from + s * 32 + 4 * h, len));
      }
      zero(dp);
#pragma unroll
      for (int kk = 0; kk < HD / 16; ++kk) {
        if (kk > 0) {
          rd.operand(qt, s * 32, kk, a);
          sc = mma(a, k[kk], sc);
        }
        rd.operand(dt, s * 32, kk, a);
        dp = mma(a, v[kk], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const f32x4 x = st[(s * 32 + 8 * (e >> 2) + 4 * h + (e & 3)) >> 1];
        sc[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], c2, -x[0]));
        sc[e + 1] = __builtin_amdgcn_exp2f(fmaf(sc[e + 1], c2, -x[2]));
        dp[e] = sc[e] * (dp[e] - x[1]);
        dp[e + 1] = sc[e + 1] * (dp[e + 1] - x[3]);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        Frag<T> pf, df;
        as_operand(sc, u, pf);
        as_operand(dp, u, df);
#pragma unroll
        for (int f = 0; f < HD / 32; ++f) {
          rd.transposed(dt, s * 32 + u * 16, f, a);
          dv[f] = mma(a, pf, dv[f]);
          rd.transposed(qt, s * 32 + u * 16, f, a);
          dk[f] = mma(a, df, dk[f]);
        }
      }
    }
  }

  // fp32 rows of the parts, HD floats a key and then kMaxSinks keys on.
  __device__ __forceinline__ void store_part(float* ok, float* ov, int h) const {
#pragma unroll
    for (int n = 0; n < HD / 32; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = n * 32 + 8 * e + 4 * h;
        store4(ok + c, dk[n][4 * e], dk[n][4 * e + 1], dk[n][4 * e + 2], dk[n][4 * e + 3]);
        store4(ov + c, dv[n][4 * e], dv[n][4 * e + 1], dv[n][4 * e + 2], dv[n][4 * e + 3]);
      }
  }
};

// Loads of packed rows [r0, r0 + ROWS) of q or dout (base: its first query of
// the group) to LDS; rows past the last are that one again.
template <typename T, int HD, int ROWS, int WAVES>
__device__ __forceinline__ void stage_rows(const BwdP& p, char* dst, const char* base, const View& t,
                                           int r0, int rows, int wave, int lane) {
  using Tl = Tile<T, HD>;
  using Ld = typename Tl::template Loads<ROWS, WAVES>;
  const int G = p.group, i0 = r0 / G;
  const __amdgpu_buffer_rsrc_t from = buffer_of(base + i0 * t.st, 0xffffffffll);
  const uint32_t st = (uint32_t)t.st, sh = (uint32_t)t.sh;
  // Where the rows of two loads are whole queries apart, one offset serves all
  // loads of every tile.
  int ln = lane;  // nothing of this is to be kept in registers over the loop
  asm volatile("" : "+v"(ln));
  auto query = [&](unsigned r) { return __umulhi(r << 3, p.div_mul) >> p.div_shift; };
  if (WAVES == 4 && 4 * Tl::kBlockRows % G == 0 && r0 + ROWS <= rows) {
    const unsigned r = (unsigned)Ld::row(0, wave, ln), i = query(r);
    const uint32_t first = i * st + (r - i * (unsigned)G) * sh;
    const uint32_t next = query(4 * Tl::kBlockRows) * st;
    Ld::issue(dst, wave, ln, from, [&](int l) { return first + (uint32_t)l * next; });
  } else {
    Ld::issue(dst, wave, ln, from, [&](int l) {
      const unsigned r = (unsigned)min(r0 + Ld::row(l, wave, ln), rows - 1), i = query(r);
      return (i - (uint32_t)i0) * st + (r - i * (unsigned)G) * sh;
    });
  }
}

// 32 rows' lse and D, 4 bytes a lane.
__device__ __forceinline__ void stage_stat(char* dst, const float2* stat, int r0, int rows, int lane) {
  const char* src = reinterpret_cast<const char*>(stat + min(r0 + (lane >> 1), rows - 1)) + (lane & 1) * 4;
  __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)src, (lds_void*)dst, 4, 0, 0);
}

template <typename T, int HD>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 || HD == 64 ? 2 : 1)) void window_dkv_kernel(BwdP p) {
  using S = Shape<T, HD>;
  using Tl = Tile<T, HD>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = xcd_order(blockIdx.x, p.blocks);
  const int z = (int)(id % p.row_parts);
  const int64_t rest = id / p.row_parts, bk = rest / p.key_tiles;
  // Causal: early keys have the most rows.  Every other sequence the other way
  // round, so that a CU's two workgroups are not both of early ones.
  const int turn = (int)(rest - bk * p.key_tiles);
  const int first = ((bk & 1) ? p.key_tiles - 1 - turn : turn) * kKeys;
  const int b = (int)(bk / p.kv_heads), hk = (int)(bk - (int64_t)b * p.kv_heads);
  const int ql = clamp_len(p.q_lens, b, p.q_tokens), kl = clamp_len(p.k_lens, b, p.k_tokens);
  const int G = p.group, rows = ql * G, shift = kl - ql;
  if (first >= kl) return;
  const int wfirst = first + 32 * wave, key = wfirst + l32, kc = min(key, kl - 1);
  // Rows that see this lane's key, some key and every key of the wave, some key
  // of the workgroup.  The earliest row is that of the first key; the last that
  // of the last key or, with a sink among the keys, the last of all: those
  // behind every key's window are left to the sink kernel where there is one.
  const int wlast = min(wfirst + 31, kl - 1);
  const Rows last = rows_of(p.mask, min(first + kKeys, kl) - 1, shift, rows, G, false);
  Rows mine = rows_of(p.mask, kc, shift, rows, G, true);
  if (key >= kl) mine = Rows{0, -1};
  const Rows w0 = rows_of(p.mask, wfirst, shift, rows, G, true);
  const Rows w1 = rows_of(p.mask, wlast, shift, rows, G, true);
  const Rows n0 = rows_of(p.mask, first, shift, rows, G, true);
  const int lo = n0.lo, hi = p.parts ? last.hi : max(n0.hi, last.hi);
  const bool idle = wfirst >= kl;
  const int wlo = w0.lo, whi = max(w0.hi, w1.hi);
  const int ilo = w1.lo, ihi = rows_of(p.mask, wfirst, shift, rows, G, false).hi;
  const bool whole = wfirst + 31 < kl;
  mine.hi = min(mine.hi, hi);
  const unsigned len = (unsigned)max(mine.hi - mine.lo + 1, 0);
  const int t_lo = lo / S::kRows, tiles = hi >= lo ? hi / S::kRows + 1 - t_lo : 0;
  // The tiles are taken from the one whose number is a multiple of how many there
  // are, and round: workgroups of neighbouring keys, whose rows are mostly the
  // same, then read the same tile at the same time, out of the L2 that they share.
  const int t_first = tiles > 0 ? (tiles - t_lo % tiles) % tiles : 0;
  auto row0 = [&](int n) {
    const int t = t_first + n;
    return (t_lo + (t < tiles ? t : t - tiles)) * S::kRows;
  };

  const char* qp = p.q.p + b * p.q.sb + (int64_t)hk * G * p.q.sh;
  const char* dp = p.dout.p + b * p.dout.sb + (int64_t)hk * G * p.dout.sh;
  const float2* stat = p.stat + bk * ((int64_t)p.q_tokens * G);
  constexpr int kBuf = 2 * S::kTile + S::kStat;
  auto stage = [&](int n, char* dst) {
    const int r0 = row0(n);
    stage_rows<T, HD, S::kRows, kWaves>(p, dst, qp, p.q, r0, rows, wave, lane);
    stage_rows<T, HD, S::kRows, kWaves>(p, dst + S::kTile, dp, p.dout, r0, rows, wave, lane);
    // Every wave issues one, so that all count the same (waves 2 and 3 to the spare).
    stage_stat(dst + 2 * S::kTile + wave * 256, stat, r0 + (wave & 1) * 32, rows, lane);
  };
  constexpr int kLoads = 2 * Tl::template Loads<S::kRows, kWaves>::kLoads + 1;

  const typename Tl::Reader rd(lane);
  KeySide<T, HD> ks;
  ks.load(p.k.p + b * p.k.sb + (int64_t)kc * p.k.st + hk * p.k.sh,
          p.v.p + b * p.v.sb + (int64_t)kc * p.v.st + hk * p.v.sh, h, len > 0);
  // cur and next never overlap (as in window_dq_kernel).
  const int zs = (int)((int64_t)tiles * z / p.row_parts), ze = (int)((int64_t)tiles * (z + 1) / p.row_parts);
  auto body = [&](int n, const char* __restrict__ cur, char* __restrict__ next) __attribute__((always_inline)) {
    if (n + 1 < ze) {
      stage(n + 1, next);
      wait_and_meet<kLoads>();
    } else {
      wait_and_meet<0>();
    }
    const int r0 = row0(n), r1 = r0 + S::kRows - 1;
    ks.hold();
    if (!idle && r1 >= wlo && r0 <= whi)
      ks.template rows<S::kSub>(cur, cur + S::kTile, reinterpret_cast<const f32x4*>(cur + 2 * S::kTile),
                                whole && r0 >= ilo && r1 <= ihi, r0 - mine.lo, len, p.c2, h, rd);
    ks.hold();
    asm volatile("" ::: "memory");
    wait_lds();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  if (zs < ze) stage(zs, smem);
  settle();
  for (int n = zs; n < ze; ++n) body(n, smem + ((n - zs) & 1) * kBuf, smem + ((n + 1 - zs) & 1) * kBuf);
  if (key >= kl) return;
  if (p.row_parts > 1) {
    float* out = p.row_part + ((bk * p.row_parts + z) * 2 * p.k_tokens + key) * (int64_t)HD;
    ks.store_part(out, out + (int64_t)p.k_tokens * HD, h);
    return;
  }
  if (p.parts && key < p.mask.sinks) {  // the sink kernel's sums come to these
    float* out = p.part + ((bk * (p.parts + 1)) * 2 * kMaxSinks + key) * (int64_t)HD;
    ks.store_part(out, out + kMaxSinks * HD, h);
    return;
  }
  T* ok = reinterpret_cast<T*>(p.dk.p + b * p.dk.sb + (int64_t)key * p.dk.st + hk * p.dk.sh);
  T* ov = reinterpret_cast<T*>(p.dv.p + b * p.dv.sb + (int64_t)key * p.dv.st + hk * p.dv.sh);
#pragma unroll
  for (int n = 0; n < HD / 32; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = n * 32 + 8 * e + 4 * h;
      store4(ok + c, ks.dk[n][4 * e] * p.scale, ks.dk[n][4 * e + 1] * p.scale,
             ks.dk[n][4 * e + 2] * p.scale, ks.dk[n][4 * e + 3] * p.scale);
      store4(ov + c, ks.dv[n][4 * e], ks.dv[n][4 * e + 1], ks.dv[n][4 * e + 2], ks.dv[n][4 * e + 3]);
    }
}

// The sinks' rows behind every window of the first tile of keys: one part of
// them and 32 of the sinks a workgroup, the rows shared out over its waves (no
// barrier until they join).
template <typename T, int HD>
__global__ __launch_bounds__(kThreads, 1) void window_sink_kernel(BwdP p) {
  using S = SinkShape<T, HD>;
  using Tl = Tile<T, HD>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t id = xcd_order(blockIdx.x, p.blocks);
  const int part = (int)(id % p.parts);
  const int64_t rest = id / p.parts;
  const int group = (int)(rest % p.sink_groups);
  const int64_t bk = rest / p.sink_groups;
  const int b = (int)(bk / p.kv_heads), hk = (int)(bk - (int64_t)b * p.kv_heads);
  const int ql = clamp_len(p.q_lens, b, p.q_tokens), kl = clamp_len(p.k_lens, b, p.k_tokens);
  const int G = p.group, rows = ql * G, shift = kl - ql;
  const int wfirst = 32 * group, key = wfirst + l32, sinks = min(p.mask.sinks, kl);
  if (wfirst >= sinks) return;
  const int kc = min(key, kl - 1);
  // All rows from `from` on see all of the sinks: they stand behind the windows
  // of keys no earlier.
  const int from = rows_of(p.mask, min(kKeys, kl) - 1, shift, rows, G, false).hi + 1;
  const int far = rows - from, all = (far + 31) / 32;
  const int ts = (int)((int64_t)all * part / p.parts), te = (int)((int64_t)all * (part + 1) / p.parts);
  const char* qp = p.q.p + b * p.q.sb + (int64_t)hk * G * p.q.sh;
  const char* dp = p.dout.p + b * p.dout.sb + (int64_t)hk * G * p.dout.sh;
  const float2* stat = p.stat + bk * ((int64_t)p.q_tokens * G);
  char* mem = smem + wave * S::kBuffers * S::kBuf;
  auto stage = [&](int n, char* dst) {
    const int r0 = from + n * 32;
    stage_rows<T, HD, 32, 1>(p, dst, qp, p.q, r0, rows, 0, lane);
    stage_rows<T, HD, 32, 1>(p, dst + S::kTile, dp, p.dout, r0, rows, 0, lane);
    stage_stat(dst + 2 * S::kTile, stat, r0, rows, lane);
  };
  constexpr int kLoads = 2 * Tl::template Loads<32, 1>::kLoads + 1;
  const typename Tl::Reader rd(lane);
  const bool seen = key < sinks;
  KeySide<T, HD> ks;
  ks.load(p.k.p + b * p.k.sb + (int64_t)kc * p.k.st + hk * p.k.sh,
          p.v.p + b * p.v.sb + (int64_t)kc * p.v.st + hk * p.v.sh, h, seen);
  auto compute = [&](int n, const char* cur) {
    ks.hold();
    const int left = far - n * 32;
    ks.template rows<1>(cur, cur + S::kTile, reinterpret_cast<const f32x4*>(cur + 2 * S::kTile),
                        left >= 32 && wfirst + 32 <= sinks, 0, seen ? (unsigned)min(left, 32) : 0u, p.c2,
                        h, rd);
    ks.hold();
    asm volatile("" ::: "memory");
    wait_lds();
    asm volatile("" ::: "memory");
  };
  int n = ts + wave;
  if constexpr (S::kBuffers == 2) {
    auto body = [&](const char* __restrict__ cur, char* __restrict__ next) __attribute__((always_inline)) {
      const bool more = n + kWaves < te;
      if (more) stage(n + kWaves, next);
      asm volatile("" ::: "memory");
      if (more) wait_vm_lds<kLoads>();
      else wait_vm_lds<0>();
      asm volatile("" ::: "memory");
      compute(n, cur);
    };
    if (n < te) stage(n, mem);
    settle();
    for (int cur = 0; n < te; n += kWaves, cur ^= 1) body(mem + cur * S::kBuf, mem + (cur ^ 1) * S::kBuf);
  } else {
    for (; n < te; n += kWaves) {
      stage(n, mem);
      settle();
      compute(n, mem);
    }
  }
  // Join the waves, dk and then dv.
  float* jo = reinterpret_cast<float*>(smem);
  float* out = p.part + ((bk * (p.parts + 1) + 1 + part) * 2 * kMaxSinks + wfirst) * (int64_t)HD;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const f32x16* x = side ? ks.dv : ks.dk;
    __syncthreads();
    float* jr = jo + (wave * 32 + l32) * S::kOs;
#pragma unroll
    for (int n = 0; n < HD / 32; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        store4(jr + n * 32 + 8 * e + 4 * h, x[n][4 * e], x[n][4 * e + 1], x[n][4 * e + 2], x[n][4 * e + 3]);
    __syncthreads();
    for (int u = threadIdx.x; u < 32 * (HD / 4); u += kThreads) {
      const int r = u / (HD / 4), c = (u - r * (HD / 4)) * 4;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v += *reinterpret_cast<const f32x4*>(jo + (w * 32 + r) * S::kOs + c);
      *reinterpret_cast<f32x4*>(out + (side * kMaxSinks + r) * (int64_t)HD + c) = v;
    }
  }
}

// The gradients of keys whose sums are in parts (all keys, or with a single
// part of the rows the sinks): the parts added up in order, four features a
// thread.
template <typename T, int HD>
__global__ __launch_bounds__(kThreads) void window_key_join_kernel(BwdP p, int keys) {
  constexpr int kPer = HD / 4, kBlockKeys = kThreads / kPer;
  const int blocks = (keys + kBlockKeys - 1) / kBlockKeys;
  const int64_t bk = blockIdx.x / blocks;
  const int key = (int)(blockIdx.x - bk * blocks) * kBlockKeys + threadIdx.x / kPer;
  const int c = (threadIdx.x % kPer) * 4;
  const int b = (int)(bk / p.kv_heads), hk = (int)(bk - (int64_t)b * p.kv_heads);
  if (key >= min(keys, clamp_len(p.k_lens, b, p.k_tokens))) return;
  f32x4 dk = {0.f, 0.f, 0.f, 0.f}, dv = dk;
  auto add = [&](const float* in, int n, int64_t side) {
#pragma unroll 4
    for (int i = 0; i < n; ++i, in += 2 * side) {
      dk += *reinterpret_cast<const f32x4*>(in);
      dv += *reinterpret_cast<const f32x4*>(in + side);
    }
  };
  const int64_t all = (int64_t)p.k_tokens * HD, few = (int64_t)kMaxSinks * HD, at = (int64_t)key * HD + c;
  if (p.row_parts > 1) add(p.row_part + bk * p.row_parts * 2 * all + at, p.row_parts, all);
  if (p.parts > 0 && key < p.mask.sinks) {
    const int skip = p.row_parts > 1;  // the key kernel's own sums are then among the row parts
    add(p.part + (bk * (p.parts + 1) + skip) * 2 * few + at, p.parts + 1 - skip, few);
  }
  T* ok = reinterpret_cast<T*>(p.dk.p + b * p.dk.sb + (int64_t)key * p.dk.st + hk * p.dk.sh);
  T* ov = reinterpret_cast<T*>(p.dv.p + b * p.dv.sb + (int64_t)key * p.dv.st + hk * p.dv.sh);
  store4(ok + c, dk[0] * p.scale, dk[1] * p.scale, dk[2] * p.scale, dk[3] * p.scale);
  store4(ov + c, dv[0], dv[1], dv[2], dv[3]);
}

// Rows that see some key of a tile through its window, at most.
int64_t near_rows(const elasto_window_t& a) {
  const int64_t G = a.heads / a.kv_heads, reach = a.causal ? (int64_t)a.window : 2 * (int64_t)a.window;
  return std::min<int64_t>((int64_t)a.q_tokens * G, (kKeys + reach) * G);
}

// Parts of the rows that only the sinks are seen by, for launches in which they
// are more than a tile of keys has otherwise (0: the first tile's workgroup
// takes them along): about 256 workgroups, 128 rows or more each.
int parts_of(const elasto_window_t& a) {
  const int64_t G = a.heads / a.kv_heads, rows = (int64_t)a.q_tokens * G;
  const int64_t near = (kKeys + (int64_t)a.window) * G;
  if (a.sinks == 0 || rows - near <= std::max<int64_t>(near / 2, 512)) return 0;
  const int64_t groups = (int64_t)a.batch * a.kv_heads * ((a.sinks + 31) / 32);
  return (int)std::max<int64_t>(1, std::min<int64_t>({(rows - near) / 128, 256 / groups, 256}));
}

// Parts of a tile's rows, where the tiles of keys would leave CUs idle (few
// key heads): as many workgroups as run at once (2 a CU, fp32 of 128 features 1) or
// fewer, four tiles of rows or more each (fp32, of tiles half as long that take 8
// times as long: 3 x 481 tokens x 6 heads of 128, 54 keys, in 1 part 198 us, in 2
// 140; bf16 62 x 256 x 3, 184 keys, in 1 part 52 us, in 2 80).
int row_parts_of(const elasto_window_t& a) {
  const int64_t blocks = (int64_t)a.batch * a.kv_heads * ((a.k_tokens + kKeys - 1) / kKeys);
  const int64_t near = near_rows(a), most = a.dtype == ELASTO_FP32 ? (near + 127) / 128 : near / 256;
  const int64_t places = a.dtype == ELASTO_FP32 && a.head_dim == 128 ? 256 : 512;
  return (int)std::max<int64_t>(1, std::min<int64_t>({places / std::max<int64_t>(blocks, 1), most, 16}));
}
int64_t row_part_bytes(const elasto_window_t& a) {
  const int n = row_parts_of(a);
  return n > 1 ? (int64_t)a.batch * a.kv_heads * n * 2 * a.k_tokens * a.head_dim * 4 : 0;
}
int64_t part_bytes(const elasto_window_t& a) {
  const int n = parts_of(a);
  return n > 0 ? (int64_t)a.batch * a.kv_heads * (n + 1) * 2 * kMaxSinks * a.head_dim * 4 : 0;
}
int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

int64_t stat_bytes(const elasto_window_t& a) { return (int64_t)a.batch * a.heads * a.q_tokens * 8; }

// Keys whose gradients are joined from parts.
int64_t join_keys(const BwdP& p) { return p.row_parts > 1 ? p.k_tokens : p.parts > 0 ? p.mask.sinks : 0; }

template <typename T, int HD>
hipError_t launch(BwdP p, int64_t pairs, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (p.row_blocks > 0) {
    p.blocks = pairs * p.row_blocks;
    hipLaunchKernelGGL((window_dq_kernel<T, HD>), dim3((unsigned)p.blocks), dim3(kThreads),
                       (Shape<T, HD>::kLdsRow), s, p);
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.key_tiles == 0) return e;
  if (p.parts > 0) {
    p.blocks = pairs * p.sink_groups * p.parts;
    hipLaunchKernelGGL((window_sink_kernel<T, HD>), dim3((unsigned)p.blocks), dim3(kThreads),
                       (SinkShape<T, HD>::kLds), s, p);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  p.blocks = pairs * p.key_tiles * p.row_parts;
  hipLaunchKernelGGL((window_dkv_kernel<T, HD>), dim3((unsigned)p.blocks), dim3(kThreads),
                     (Shape<T, HD>::kLdsKey), s, p);
  e = hipGetLastError();
  const int keys = (int)join_keys(p), per = 1024 / HD;
  if (e != hipSuccess || keys == 0) return e;
  hipLaunchKernelGGL((window_key_join_kernel<T, HD>), dim3((unsigned)(pairs * ((keys + per - 1) / per))),
                     dim3(kThreads), 0, s, p, keys);
  return hipGetLastError();
}

}  // namespace

int64_t window_bwd_workspace(const elasto_window_t& a) {
  return up256(stat_bytes(a)) + up256(part_bytes(a)) + row_part_bytes(a);
}

hipError_t launch_window_bwd(const elasto_window_t& a, const WindowTensors& t, void* ws, hipStream_t s) {
  BwdP p = {};
  p.q = t.q; p.k = t.k; p.v = t.v; p.o = t.o; p.dout = t.dout; p.dq = t.dq; p.dk = t.dk; p.dv = t.dv;
  p.lse = t.lse;
  p.q_lens = a.q_lens;
  p.k_lens = a.k_lens;
  p.q_tokens = a.q_tokens;
  p.k_tokens = a.k_tokens;
  p.heads = a.heads;
  p.kv_heads = a.kv_heads;
  p.group = a.heads / a.kv_heads;
  // With 2^(s - 1) < group <= 2^s and m = ceil(2^(29 + s) / group), r m / 2^(29 + s)
  // exceeds r / group by less than r / 2^29 / group, under 1 / group.
  while ((1u << p.div_shift) < (unsigned)p.group) ++p.div_shift;
  p.div_mul = (unsigned)((((uint64_t)1 << (29 + p.div_shift)) + p.group - 1) / p.group);
  p.mask = Mask{a.causal, a.window, a.sinks};
  p.scale = a.scale;
  p.c2 = a.scale * kLog2e;
  const int64_t pairs = (int64_t)a.batch * a.kv_heads;
  p.row_blocks = (int)(((int64_t)a.q_tokens * p.group + 32 * kWaves - 1) / (32 * kWaves));
  p.key_tiles = (a.k_tokens + kKeys - 1) / kKeys;
  p.parts = parts_of(a);
  p.stat = static_cast<float2*>(ws);
  p.part = reinterpret_cast<float*>(static_cast<char*>(ws) + up256(stat_bytes(a)));
  p.row_parts = row_parts_of(a);
  p.row_part = reinterpret_cast<float*>(static_cast<char*>(ws) + up256(stat_bytes(a)) + up256(part_bytes(a)));
  p.sink_groups = (a.sinks + 31) / 32;
  const int64_t join = join_keys(p) * a.head_dim / 1024 + 1;
  if (pairs * std::max({(int64_t)p.row_blocks, (int64_t)p.key_tiles * p.row_parts,
                        (int64_t)p.sink_groups * p.parts, join}) >= kMaxBlocks)
    return hipErrorInvalidConfiguration;
  if (a.dtype == ELASTO_BF16)
    return a.head_dim == 64 ? launch<uint16_t, 64>(p, pairs, s) : launch<uint16_t, 128>(p, pairs, s);
  return a.head_dim == 64 ? launch<float, 64>(p, pairs, s) : launch<float, 128>(p, pairs, s);
}

}  // namespace elasto
