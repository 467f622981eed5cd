// Softmax cross-entropy of a linear layer, z = x W^T + b, without keeping z:
//   lse_r = log sum_c exp(z_rc),  loss_r = lse_r - z_r,label,
// and with dz = w_r (softmax(z)_rc - [c = label]), w the row's weight,
//   dx = s dz W,  dW = s dz^T x,  db = s sum_r dz.
//
// Forward: each tile of z stays in the accumulators of its workgroup; what leaves it is,
// for each row, the largest logit of the tile and the sum of exponentials about it.  A
// second kernel joins the tiles of a row.
// Backward: z is formed again, in pieces of the classes.  A piece's dz goes to the
// workspace, rounded to the operands' type (bf16: the two products that sum it would run
// at a ninth of the rate in fp32), and is the left operand of dx (straight) and of dW
// (turned).  dx is summed over the pieces, and over parts of a piece where its tiles leave
// CUs idle, in fp32; everything in a fixed order.
//
// Bound by the matrix cores, where rows are few by reading W: forward, 4096 rows of 2048 and 50021 classes
// 744 us (1.13 PFLOP/s, where a large product reaches 1.28), 16 rows of 4096 and 100003 classes 158 us (5.2
// TB/s); gradients, 3277 rows of 2048 that count and 131072 classes 4.72 ms (1.12 PFLOP/s); fp32, 1000 rows of
// 384 and 10007 classes 226 us (102 TFLOP/s of 154).
#include <math.h>

#include <algorithm>

#include "heads.h"
#include "tile_product.h"

namespace elasto {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct CeP {
  Matrix x, w, dz;  // dz: the piece's gradient of the logits, [rows][piece]
  int64_t rows, dim;
  int64_t c0;  // first class of the piece
  int64_t classes;  // of the piece (forward: all)
  const float* bias;
  const int32_t* labels;
  const float* weight;
  const float* lse;
  float2* part;   // forward: [tiles of classes][rows]
  float* picked;  // forward: the label's logit
  const int32_t *count, *index;  // rows that are there and where they come from, or NULL: `rows`
  float* db_part;  // [tiles of rows][ld_db], or NULL
  float* db;       // of the piece, where one tile has all rows (then no db_part), or NULL
  float scale;     // of db
  uint32_t* live;  // one bit a row: whether it gives the gradients anything; or NULL
  int64_t ld_db;
  int tiles_n, group;
  int label_classes;  // all classes
};

// Rows that are there, and a launch's tile of them: false for a workgroup that has none.
__device__ __forceinline__ int64_t rows_there(const int32_t* count, int64_t rows) { return count ? *count : rows; }

// The tile of workgroup v: each XCD (workgroup v runs on XCD v % 8) takes a run of tiles, in
// groups of `group` row tiles that share the other operand's panels in its L2.
__device__ __forceinline__ void tile_of(int v, int tiles_m, int tiles_n, int group, int& tm, int& tn) {
  const int total = tiles_m * tiles_n, q = total >> 3, r8 = total & 7, xcd = v & 7, idx = v >> 3;
  const int logical = xcd < r8 ? xcd * (q + 1) + idx : r8 * (q + 1) + (xcd - r8) * q + idx;
  const int gsz = group * tiles_n, g = logical / gsz, in_group = logical - g * gsz;
  const int gm = min(group, tiles_m - g * group);
  tn = in_group / gm;
  tm = g * group + (in_group - tn * gm);
}

template <typename S>
__device__ __forceinline__ bool find_tile(const CeP& p, int64_t rows, int64_t& m0, int64_t& n0, int& tm, int& tn) {
  const int tiles_m = (int)((rows + S::BM - 1) / S::BM);
  if ((int64_t)blockIdx.x >= (int64_t)tiles_m * p.tiles_n) return false;
  tile_of(blockIdx.x, tiles_m, p.tiles_n, p.group, tm, tn);
  m0 = (int64_t)tm * S::BM;
  n0 = (int64_t)tn * S::BN;
  return true;
}

// Logits of a tile: the accumulators start from the bias, -infinity behind the last class.
template <typename S>
__device__ __forceinline__ void logits(char* smem, const CeP& p, int64_t rows, int64_t m0, int64_t n0,
                                       f32x16 (&acc)[S::TM][S::TN]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c0 = (int)n0 + wave % S::WN * S::WTN + 4 * (lane >> 5);
#pragma unroll
  for (int j = 0; j < S::TN; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int c = c0 + j * 32 + 8 * (e >> 2) + (e & 3);
      float b = c < p.classes ? (p.bias ? p.bias[p.c0 + c] : 0.0f) : -INFINITY;
      if (!leads<S>()) b = 0.0f;
#pragma unroll
      for (int i = 0; i < S::TM; ++i) acc[i][j][e] = b;
    }
  const Matrix w = {p.w.p + p.c0 * p.w.ld, p.w.ld};
  tile_product<S, false, false, false>(smem, p.x, w, rows, p.classes, m0, n0, 0, p.dim, nullptr, acc);
}

// A reference for the exponentials of values up to m.
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.0f : m; }

// exp(z - ref) for many z as one multiply-add and 2^: the product ref log2(e) is rounded once, and what
// that leaves out is the same factor for all of them (`left`).  Where ref lies so far out that the
// rounding would leave the exponents' range, only what equals ref counts, and a smaller factor says so.
struct Power {
  float c, off, left;
  __device__ __forceinline__ explicit Power(float ref) {
#pragma clang fp contract(off)
    constexpr float kFar = 1073741824.0f;
    c = fabsf(ref * kLog2e) > kFar ? kFar / fabsf(ref) : kLog2e;
    const float r = -ref * c;
    off = r;
    left = __builtin_amdgcn_exp2f(-fmaf(ref, c, r));
  }
  __device__ __forceinline__ float operator()(float z) const { return __builtin_amdgcn_exp2f(fmaf(z, c, off)); }
};

template <typename S>
__global__ __launch_bounds__(S::kThreads, S::kWaves) void ce_forward_kernel(CeP p) {
  __shared__ __attribute__((aligned(1024))) char smem[S::STAGES * S::kStage];
  const int64_t rows = rows_there(p.count, p.rows);
  int64_t m0, n0;
  int tm, tn;
  if (!find_tile<S>(p, rows, m0, n0, tm, tn)) return;
  f32x16 acc[S::TM][S::TN];
  logits<S>(smem, p, rows, m0, n0, acc);
  __syncthreads();
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % S::kTeam / S::WN, wn = wave % S::WN, lr = lane & 31, lg = lane >> 5;
  float2* red = reinterpret_cast<float2*>(smem);  // [WN][BM]
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
    float m = acc[i][0][0];
#pragma unroll
    for (int j = 0; j < S::TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) m = fmaxf(m, acc[i][j][e]);
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    const Power power(reference(m));
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < S::TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) s += power(acc[i][j][e]);
    s += __shfl_xor(s, 32, 64);
    s *= power.left;
    const int r = wm * S::WTM + i * 32 + lr;
    if (lg == 0) red[wn * S::BM + r] = make_float2(m, s);
    // The label's logit, by the one lane that holds it.
    const int64_t row = m0 + r;
    const int first = (int)n0 + wn * S::WTN;
    const int y = row < rows ? p.labels[row] : -1;
    if (y >= first && y < first + S::WTN && y < p.classes)
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (y == first + j * 32 + 8 * (e >> 2) + 4 * lg + (e & 3)) p.picked[row] = acc[i][j][e];
  }
  __syncthreads();
  for (int r = tid; r < S::BM && m0 + r < rows; r += S::kThreads) {
    float2 t = red[r];
    float m = t.x;
#pragma unroll
    for (int k = 1; k < S::WN; ++k) m = fmaxf(m, red[k * S::BM + r].x);
    const float ref = reference(m);
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < S::WN; ++k) {
      const float2 o = red[k * S::BM + r];
      s += o.y * __builtin_amdgcn_exp2f((o.x - ref) * kLog2e);
    }
    p.part[(int64_t)tn * p.rows + m0 + r] = make_float2(m, s);
  }
}

// Joins the tiles of R rows: 1024 / R threads of a row take them in turn.  64 rows where that leaves no CU
// without a workgroup, otherwise 8 (16 rows of 1563 tiles: 21 us with 64, 6 with 8).
struct JoinP {
  const float2* part;
  const float *picked, *weight;
  const int32_t* labels;
  float *loss, *lse;
  const int32_t *count, *index;  // rows that are there and where their results go, or NULL
  int64_t rows;
  int tiles, classes;
};
// (m, s) and (n, u): largest logits and sums of exponentials about them.
__device__ __forceinline__ void join(float& m, float& s, float n, float u) {
  const float top = fmaxf(m, n), ref = reference(top);
  s = s * __builtin_amdgcn_exp2f((m - ref) * kLog2e) + u * __builtin_amdgcn_exp2f((n - ref) * kLog2e);
  m = top;
}
template <int R>
__global__ __launch_bounds__(1024) void ce_join_kernel(JoinP p) {
  __shared__ float2 red[16][R];
  const int lane = threadIdx.x % R, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * R + lane;
  const bool there = row < rows_there(p.count, p.rows);
  float m = -INFINITY, s = 0.0f;
  if (there)
#pragma unroll 4
    for (int t = threadIdx.x / R; t < p.tiles; t += 1024 / R) {
      const float2 o = p.part[(int64_t)t * p.rows + row];
      join(m, s, o.x, o.y);
    }
#pragma unroll
  for (int k = R; k < 64; k *= 2) join(m, s, __shfl_xor(m, k), __shfl_xor(s, k));
  if ((threadIdx.x & 63) < R) red[wave][lane] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x >= R || !there) return;
  float top = m;
  for (int k = 1; k < 16; ++k) top = fmaxf(top, red[k][lane].x);
  const float ref = reference(top);
  s = 0.0f;
  for (int k = 0; k < 16; ++k) s += red[k][lane].y * __builtin_amdgcn_exp2f((red[k][lane].x - ref) * kLog2e);
  const float above = log2f(s) * kLn2;
  const bool out = p.weight && p.weight[row] == 0.0f;
  const int y = p.labels[row];
  const bool ok = y >= 0 && y < p.classes;
  const int64_t to = p.index ? p.index[row] : row;
  p.loss[to] = out ? 0.0f : ok ? above + (ref - p.picked[row]) : NAN;
  if (p.lse) p.lse[to] = out ? 0.0f : above + ref;
}

// Rows that count, one after another: what rows of weight 0 would cost is not spent.  A backward pass
// leaves out rows with bad labels too.
struct GatherP {
  Matrix x;
  const float *weight, *lse;
  const int32_t* labels;
  int64_t rows;
  int bytes, classes;    // of a row
  bool back;
  int32_t *count, *first;  // first[b]: place of the first row of rows 64 b ..
  int32_t* index;        // rows that count, in order; then what they hold:
  char* xs;
  int32_t* ys;
  float *ws, *ls;
  char* dx;              // (or NULL) zeros where a row does not count
  int64_t lddx;
  float *loss, *lse_out;  // forward: zeros likewise
};
__device__ __forceinline__ bool counts(const GatherP& p, int64_t r) {
  if (r >= p.rows || p.weight[r] == 0.0f) return false;
  return !p.back || (p.labels[r] >= 0 && p.labels[r] < p.classes);
}
constexpr int kGatherRows = 1 << 18;
// One workgroup: a wave counts 64 rows at a time, then all counts are added up.
__global__ __launch_bounds__(1024) void ce_count_kernel(GatherP p) {
  constexpr int kBlocks = kGatherRows / 64, kEach = kBlocks / 1024;
  __shared__ int32_t n[kBlocks];
  __shared__ int32_t sums[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, blocks = (int)((p.rows + 63) / 64);
  for (int b = wave; b < blocks; b += 64) {
    bool on[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) on[i] = counts(p, (int64_t)(b + 16 * i) * 64 + lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t m = __ballot(on[i]);
      if (lane == 0 && b + 16 * i < blocks) n[b + 16 * i] = __popcll(m);
    }
  }
  __syncthreads();
  int32_t mine = 0;
  for (int i = 0; i < kEach; ++i)
    if (tid * kEach + i < blocks) mine += n[tid * kEach + i];
  int32_t upto = mine;  // of this wave's threads up to this one
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int32_t at = upto - mine;
  for (int w = 0; w < wave; ++w) at += sums[w];
  for (int i = 0; i < kEach; ++i)
    if (tid * kEach + i < blocks) {
      p.first[tid * kEach + i] = at;
      at += n[tid * kEach + i];
    }
  if (tid == 1023) *p.count = at;
}
// 16 rows a workgroup, four a wave.
__global__ __launch_bounds__(256) void ce_gather_kernel(GatherP p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t block = blockIdx.x >> 2;
  const uint64_t m = __ballot(counts(p, block * 64 + lane));
  const int first = p.first[block];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int in = (blockIdx.x & 3) * 16 + wave * 4 + i;
    const int64_t r = block * 64 + in;
    if (r >= p.rows) return;
    if ((m >> in) & 1) {
      const int64_t to = first + __popcll(m & ((1ull << in) - 1));
      if (lane == 0) {
        p.index[to] = (int32_t)r;
        p.ys[to] = p.labels[r];
        p.ws[to] = p.weight[r];
        if (p.back) p.ls[to] = p.lse[r];
      }
      const char* from = p.x.p + r * p.x.ld;
      for (int c = lane * 16; c < p.bytes; c += 1024)
        *reinterpret_cast<u32x4*>(p.xs + to * p.bytes + c) = *reinterpret_cast<const u32x4*>(from + c);
    } else {
      if (p.dx)
        for (int c = lane * 16; c < p.bytes; c += 1024)
          *reinterpret_cast<u32x4*>(p.dx + r * p.lddx + c) = u32x4{0, 0, 0, 0};
      if (!p.back && lane == 0) {
        p.loss[r] = 0.0f;
        if (p.lse_out) p.lse_out[r] = 0.0f;
      }
    }
  }
}

__device__ __forceinline__ void store4(float* p, const float* v) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void store4(uint16_t* p, const float* v) {
  *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// A wave's block of 32 rows x S::WTN columns as rows: through the wave's part of LDS, from which each
// lane takes 16 bytes of a row.  each(row, first column, the 16 bytes) for the block's pieces.
template <typename S, typename O>
struct RowsOut {
  static constexpr int kRow = S::WTN * (int)sizeof(O) + 16;
  static constexpr int kPieces = S::WTN * (int)sizeof(O) / 16, kPer = 16 / (int)sizeof(O);
  static constexpr int kWave = 32 * kRow;
  static_assert(kWave * S::kThreads / 64 <= S::STAGES * S::kStage, "the tiles' LDS holds it");
  template <typename F>
  static __device__ __forceinline__ void go(char* mine, const f32x16 (&acc)[S::TN], int lane, F&& each) {
    O* to = reinterpret_cast<O*>(mine + (lane & 31) * kRow) + 4 * (lane >> 5);
#pragma unroll
    for (int j = 0; j < S::TN; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float v[4] = {acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]};
        store4(to + j * 32 + 8 * g, v);
      }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < kPieces / 2; ++i) {
      const int r = (i * 64 + lane) / kPieces, c = (i * 64 + lane) % kPieces;
      each(r, c * kPer, *reinterpret_cast<const u32x4*>(mine + r * kRow + c * 16));
    }
    asm volatile("" ::: "memory");
  }
};

// dz of one tile of the piece.  The first column of tiles also says which rows count, and a tile of all rows
// sums dbias itself: launches that small calls would wait for (8 rows of 768,
// 1000 classes: 24.7 -> 20.2 us).
template <typename S>
__global__ __launch_bounds__(S::kThreads, S::kWaves) void ce_dz_kernel(CeP p) {
  typedef typename S::T T;
  __shared__ __attribute__((aligned(1024))) char smem[S::STAGES * S::kStage];
  const int64_t rows = rows_there(p.count, p.rows);
  int64_t m0, n0;
  int tm, tn;
  if (!find_tile<S>(p, rows, m0, n0, tm, tn)) return;
  f32x16 acc[S::TM][S::TN];
  logits<S>(smem, p, rows, m0, n0, acc);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % S::kTeam / S::WN, wn = wave % S::WN, lr = lane & 31, lg = lane >> 5;
  const int first = (int)n0 + wn * S::WTN;  // of the wave's classes in the piece
  typedef RowsOut<S, T> Out;
  char* mine = smem + wave * Out::kWave;
  __syncthreads();  // the tiles have been read
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
    const int64_t block = m0 + wm * S::WTM + i * 32, row = block + lr;
    float w = 0.0f, lse = 0.0f;
    int y = -1;
    if (row < rows) {
      y = p.labels[row];
      w = y >= 0 && y < p.label_classes ? (p.weight ? p.weight[row] : 1.0f) : 0.0f;
      lse = p.lse[row];
    }
    const uint32_t on = (uint32_t)__ballot(w != 0.0f);  // lanes 32 on have the same rows
    if (p.live && tn == 0 && wn == 0 && lane == 0 && leads<S>()) p.live[block / 32] = on;
    const Power power(lse);
    const float f = w * power.left;
#pragma unroll
    for (int j = 0; j < S::TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float v = f * power(acc[i][j][e]);
        acc[i][j][e] = w != 0.0f ? v : 0.0f;
      }
    const int64_t at = y - p.c0 - first;
    if (w != 0.0f && at >= 0 && at < S::WTN)
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (at == j * 32 + 8 * (e >> 2) + 4 * lg + (e & 3)) acc[i][j][e] -= w;
    Out::go(mine, acc[i], lane, [&](int r, int c, const u32x4& v) {
      if (block + r < rows && leads<S>())
        *reinterpret_cast<u32x4*>(const_cast<char*>(p.dz.p) + (block + r) * p.dz.ld +
                                  (int64_t)(first + c) * (int)sizeof(T)) = v;
    });
  }
  if (!p.db_part && !p.db) return;
  // Sums over the tile's rows: over the wave's blocks, its lanes, then the waves.
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem);  // [WM][BN]
#pragma unroll
  for (int j = 0; j < S::TN; ++j)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float s = acc[0][j][e];
#pragma unroll
      for (int i = 1; i < S::TM; ++i) s += acc[i][j][e];
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
      if (lr == 0) red[wm * S::BN + wn * S::WTN + j * 32 + 8 * (e >> 2) + 4 * lg + (e & 3)] = s;
    }
  __syncthreads();
  for (int c = tid; c < S::BN; c += S::kThreads) {
    float s = red[c];
#pragma unroll
    for (int k = 1; k < S::WM; ++k) s += red[k * S::BN + c];
    if (p.db) {
      if (n0 + c < p.classes) p.db[n0 + c] = s * p.scale;
    } else if (n0 + c < p.ld_db) {
      p.db_part[tm * p.ld_db + n0 + c] = s;
    }
  }
}

__global__ __launch_bounds__(256) void ce_db_kernel(const float* part, const int32_t* count, int64_t rows, int side,
                                                    int64_t ld, int64_t n, float scale, float* db) {
  const int tiles = (int)((rows_there(count, rows) + side - 1) / side);
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < n; c += (int64_t)gridDim.x * 256) {
    float s = 0.0f;
#pragma unroll 8
    for (int t = 0; t < tiles; ++t) s += part[t * ld + c];
    db[c] = s * scale;
  }
}

// C = s A B^T of one tile: dx (A = dz, B = W turned) and dW (A = dz turned, B = x turned).
struct ProductP {
  Matrix a, b;
  int64_t M, N, K;
  char* out;        // the result, of T
  int64_t ldo;      // bytes
  float* sum;       // or fp32 sums [split][M][N], N's stride ld_sum
  int64_t ld_sum;
  bool add;         // to what sum holds
  float scale;
  const uint32_t* live;
  const int32_t *count, *index;  // rows that are there and where their results go, or NULL
  bool rows_of_k;   // which are rows of K (else of the result)
  int tiles_n, group, split;
};
// Workgroup `block` of the product.
template <typename S, bool TA, bool LIVE>
__device__ __forceinline__ void product_tile(const ProductP& p, int block, char* smem) {
  typedef typename S::T T;
  const int64_t M = p.rows_of_k ? p.M : rows_there(p.count, p.M), K = p.rows_of_k ? rows_there(p.count, p.K) : p.K;
  const int tiles_m = (int)((M + S::BM - 1) / S::BM), tiles = tiles_m * p.tiles_n;
  if ((int64_t)block >= (int64_t)tiles * p.split) return;
  const int part = block / tiles;
  int tm, tn;
  tile_of(block - part * tiles, tiles_m, p.tiles_n, p.group, tm, tn);
  const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
  // Parts of whole steps; the last ones may have fewer, or none.
  const int64_t chunk = (K + (int64_t)p.split * S::kK - 1) / ((int64_t)p.split * S::kK) * S::kK;
  const int64_t k0 = part * chunk, k1 = min(K, k0 + chunk);
  f32x16 acc[S::TM][S::TN];
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  tile_product<S, TA, true, LIVE>(smem, p.a, p.b, M, p.N, m0, n0, k0, k1, p.live, acc);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r0 = m0 + wave % S::kTeam / S::WN * S::WTM, c0 = n0 + wave % S::WN * S::WTN;
  __syncthreads();  // the tiles have been read
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
    const int64_t block = r0 + i * 32;
    if (p.sum) {
      typedef RowsOut<S, float> Out;
      Out::go(smem + wave * Out::kWave, acc[i], lane, [&](int r, int c, const u32x4& v) {
        if (block + r >= M || c0 + c >= p.N || !leads<S>()) return;
        f32x4* at = reinterpret_cast<f32x4*>(p.sum + (part * p.M + block + r) * p.ld_sum + c0 + c);
        f32x4 f = __builtin_bit_cast(f32x4, v);
        if (p.add) f += *at;
        *at = f;
      });
    } else {
      typedef RowsOut<S, T> Out;
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] *= p.scale;
      Out::go(smem + wave * Out::kWave, acc[i], lane, [&](int r, int c, const u32x4& v) {
        if (block + r >= M || c0 + c >= p.N || !leads<S>()) return;
        const int64_t to = p.index ? p.index[block + r] : block + r;
        *reinterpret_cast<u32x4*>(p.out + to * p.ldo + (c0 + c) * (int)sizeof(T)) = v;
      });
    }
  }
}

template <typename S, bool TA, bool LIVE>
__global__ __launch_bounds__(S::kThreads, S::kWaves) void ce_product_kernel(ProductP p) {
  __shared__ __attribute__((aligned(1024))) char smem[S::STAGES * S::kStage];
  product_tile<S, TA, LIVE>(p, blockIdx.x, smem);
}
// dx and dW of a piece in one launch: where dx has not a whole round of workgroups, dW's take the CUs
// that are left.  dx has the first x_blocks, a multiple of 8 (each XCD keeps its run of tiles).
template <typename S, bool LIVE>
__global__ __launch_bounds__(S::kThreads, S::kWaves) void ce_products_kernel(ProductP x, ProductP w, int x_blocks) {
  __shared__ __attribute__((aligned(1024))) char smem[S::STAGES * S::kStage];
  if ((int)blockIdx.x < x_blocks)
    product_tile<S, false, false>(x, blockIdx.x, smem);
  else
    product_tile<S, true, LIVE>(w, blockIdx.x - x_blocks, smem);
}

// dx = s times the sum of the parts.
template <typename T>
__global__ __launch_bounds__(256) void ce_sum_kernel(const float* sum, int split, int64_t M, int64_t N, float scale,
                                                     char* out, int64_t ldo, const int32_t* count,
                                                     const int32_t* index) {
  const int64_t quads = N / 4, rows = rows_there(count, M);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * quads; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / quads, c = (i - r * quads) * 4;
    float v[4] = {};
    // Eight parts' loads in flight (19 x 504 values, 64 parts: 16 us one after another, 6).
    for (int s = 0; s < split; s += 8) {
      f32x4 o[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        o[k] = s + k < split ? *reinterpret_cast<const f32x4*>(sum + ((s + k) * M + r) * N + c) : f32x4{0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += o[k][e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= scale;
    store4(reinterpret_cast<T*>(out + (index ? index[r] : r) * ldo) + c, v);
  }
}

// The gradients of a batch of no rows.
template <typename T>
__global__ __launch_bounds__(256) void ce_zero_kernel(char* out, int64_t ldo, int64_t M, int64_t N) {
  const int64_t quads = N / 4;
  const float v[4] = {};
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * quads; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / quads;
    store4(reinterpret_cast<T*>(out + r * ldo) + (i - r * quads) * 4, v);
  }
}
__global__ __launch_bounds__(256) void ce_zero_db_kernel(float* db, int64_t n) {
  for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < n; c += (int64_t)gridDim.x * 256) db[c] = 0.0f;
}

// ---------------------------------------------------------------- host

constexpr int64_t kMaxRows = 1 << 24, kMaxClasses = 1 << 30, kMaxDim = 1 << 20;
constexpr int64_t kMaxTiles = 1 << 22;  // of 128 x 128: two products of 256 threads a tile; a launch holds fewer than 2^32

// Row tiles that an XCD walks together: 13 by 128 of dW's and 13 by 8 of dx's tiles, 4.72 ms of gradients with 4 (2:
// 4.71), 4.96 with 8; 16 row tiles and other shapes lie within 1% of each other.
constexpr int kGroup = 4;

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
int64_t tiles(int64_t n, int64_t b) { return (n + b - 1) / b; }

// Tile shapes.  Large (bf16): one workgroup of eight waves a CU.  Middle: two workgroups.  Deep: one,
// with three steps of loads in flight, where there are not two for each CU.  Small: two, for few tiles.
enum class Kind { Large, Middle, Deep, Narrow, Small, Tiny };
template <typename T, Kind K>
struct ShapeOf;
template <typename T>
struct ShapeOf<T, Kind::Middle> {
  typedef Shape<T, 128, 128, 2, 2, 2, 2> S;
};
template <typename T>
struct ShapeOf<T, Kind::Deep> {
  typedef Shape<T, 128, 128, 2, 2, 4, 1> S;
};
template <typename T>
struct ShapeOf<T, Kind::Small> {
  typedef Shape<T, 64, 64, 2, 2, 4, 2> S;
};
template <typename T>
struct ShapeOf<T, Kind::Tiny> {
  typedef Shape<T, 32, 32, 1, 1, 4, 4, 4> S;
};
template <typename T>
struct ShapeOf<T, Kind::Narrow> {
  typedef Shape<T, 128, 64, 2, 2, 2, 3> S;
};
template <typename T>
struct ShapeOf<T, Kind::Large> {
  typedef Shape<T, 256, 256, 2, 4, 2, 1> S;
};

// f(Shape()) for the shape of kind k, one of the type's (kRounds).
template <typename T, typename F>
void with_shape(Kind k, F&& f) {
  if constexpr (sizeof(T) == 2) {
    if (k == Kind::Large) return f(typename ShapeOf<T, Kind::Large>::S());
    if (k == Kind::Deep) return f(typename ShapeOf<T, Kind::Deep>::S());
  } else {
    if (k == Kind::Narrow) return f(typename ShapeOf<T, Kind::Narrow>::S());
  }
  if (k == Kind::Middle) return f(typename ShapeOf<T, Kind::Middle>::S());
  if (k == Kind::Small) return f(typename ShapeOf<T, Kind::Small>::S());
  return f(typename ShapeOf<T, Kind::Tiny>::S());
}

// What a round of workgroups takes, in us: `step` a step of 128 bytes of K where a CU holds all its workgroups,
// `alone` where it holds one, and `end` for the first loads and the results.  Measured: bf16 4096 x 131072 x
// 2048 58 us a round of Large tiles, 8192 x 1000 x 4096 67 of Middle ones (Large, which fill half of the
// CUs: 82), 300 x 10007 x 1024 15 of Middle, alone (Large 28, two rounds of Small 21), 256 x 1000 x 768 7
// of Small, alone (Middle 12); 128 x 32000 x 4096 54 of Deep (Middle 67); fp32 2048 x 20000 x 1024 131 of
// Middle (four rounds of Small 160), 256 x 1000 x 768 19 of Small, alone (Middle 56).
struct Round {
  Kind kind;
  int rows, cols, groups;  // tile, workgroups of a CU
  float step, alone, end;
};
constexpr Round kRounds[2][5] = {{{Kind::Large, 256, 256, 1, 1.6f, 1.6f, 8.0f},
                                  {Kind::Middle, 128, 128, 2, 1.0f, 0.75f, 3.5f},
                                  {Kind::Deep, 128, 128, 1, 0.7f, 0.7f, 4.5f},
                                  {Kind::Small, 64, 64, 2, 0.45f, 0.35f, 3.0f},
                                  {Kind::Tiny, 32, 32, 4, 0.5f, 0.25f, 3.0f}},
                                 {{Kind::Middle, 128, 128, 2, 3.9f, 2.2f, 4.0f},
                                  {Kind::Narrow, 128, 64, 3, 2.8f, 1.3f, 3.5f},
                                  {Kind::Small, 64, 64, 2, 1.18f, 0.68f, 3.0f},
                                  {Kind::Tiny, 32, 32, 4, 0.6f, 0.3f, 3.0f},
                                  {Kind::Tiny, 32, 32, 4, 0.6f, 0.3f, 3.0f}}};

// How a product of M x N over K runs: in tiles of a kind, and in parts of K that are summed afterwards.
struct Way {
  Kind kind;
  int cols, parts;
};
Way way_of(int64_t M, int64_t N, int64_t K, int es, bool may_split) {
  Way best = {Kind::Small, 64, 1};
  float least = INFINITY;
  const int64_t steps = (K * es + 127) / 128;
  for (const Round& r : kRounds[es == 4]) {
    const int64_t t = tiles(M, r.rows) * tiles(N, r.cols), slots = 256 * r.groups;
    // As many parts as fill the GPU once, of at least eight steps; or one.
    const int64_t most = may_split ? std::max<int64_t>(1, std::min<int64_t>({slots / t, steps / 8, 64})) : 1;
    for (int64_t parts : {most, (int64_t)1}) {
      const int64_t full = t * parts / slots, left = t * parts - full * slots;
      const float each = (float)tiles(steps, parts);
      float us = (float)full * (r.step * each + r.end);
      if (left > 0) {  // the last round: some CUs hold fewer workgroups than they could
        const int64_t held = tiles(left, 256);
        us += (r.groups == 1 ? r.step : r.alone + (r.step - r.alone) * (float)(held - 1) / (float)(r.groups - 1)) * each + r.end;
      }
      if (parts > 1) us += 3.0f + (float)(parts * M * N) * 8e-6f / 4.5f;
      if (us < least) {
        least = us;
        best = {r.kind, r.cols, (int)parts};
      }
    }
  }
  return best;
}

// Classes of a piece of the backward pass: a piece's dz takes about 256 MB (the cache
// behind L2), but at least 2048 classes.
int64_t piece_of(const elasto_linear_ce_t& d, int es) {
  const int64_t fit = ((int64_t)256 << 20) / (std::max<int64_t>(1, d.rows) * es) / 256 * 256;
  return std::min(up(d.classes, 256), std::max<int64_t>(2048, fit));
}

// Rows that count are taken together where that costs little against what it may save (two launches and a
// copy of x: 11 us for 4096 x 2048, against 5.8 ms of gradients at 131072 classes, of which a fifth of
// the rows left out now saves a fifth).  Below some 40 us of products the launches alone cost as much.
bool gathers(const elasto_linear_ce_t& d) {
  const double flops = 2.0 * (double)d.rows * d.dim * d.classes * (d.dtype == ELASTO_BF16 ? 1.0 : 8.0);
  return d.rows >= 64 && d.rows <= kGatherRows && flops > 4e10;
}
struct GatherLayout {
  int64_t count, first, index, ys, ws, ls, xs, bytes;
};
GatherLayout gather_layout(const elasto_linear_ce_t& d) {
  GatherLayout l = {};
  if (!gathers(d)) return l;
  auto take = [&](int64_t bytes) {
    const int64_t at = l.bytes;
    l.bytes += up(bytes, 256);
    return at;
  };
  l.count = take(4);
  l.first = take((d.rows + 63) / 64 * 4);
  l.index = take(d.rows * 4);
  l.ys = take(d.rows * 4);
  l.ws = take(d.rows * 4);
  l.ls = take(d.rows * 4);
  l.xs = take(d.rows * d.dim * (d.dtype == ELASTO_BF16 ? 2 : 4));
  return l;
}

struct BackLayout {
  int64_t gather = 0, live = 0, dz = 0, db = 0, sum = 0, wsum = 0, total = 0;
  int64_t piece = 0;
  Way x = {}, w = {};     // of dx and of dW
  bool x_summed = false;         // dx goes through fp32 sums
};
BackLayout backward_layout(const elasto_linear_ce_t& d) {
  const int es = d.dtype == ELASTO_BF16 ? 2 : 4;
  BackLayout l;
  if (d.rows == 0) return l;
  l.piece = piece_of(d, es);
  l.x = way_of(d.rows, d.dim, l.piece, es, true);
  l.w = way_of(l.piece, d.dim, d.rows, es, true);
  l.x_summed = l.x.parts > 1 || l.piece < d.classes;
  auto take = [&](int64_t bytes) {
    const int64_t at = l.total;
    l.total += up(bytes, 256);
    return at;
  };
  l.gather = take(gather_layout(d).bytes);
  l.live = take(up(d.rows, 256) / 8);
  l.dz = take(d.rows * l.piece * es);
  l.db = take(tiles(d.rows, 32) * l.piece * 4);
  // dx's sums live through all pieces, dW's through one.
  l.sum = take(l.x_summed ? (int64_t)l.x.parts * d.rows * d.dim * 4 : 0);
  l.wsum = take(l.w.parts > 1 ? (int64_t)l.w.parts * l.piece * d.dim * 4 : 0);
  return l;
}
Way forward_way(const elasto_linear_ce_t& d) {
  return way_of(d.rows, d.classes, d.dim, d.dtype == ELASTO_BF16 ? 2 : 4, false);
}
int64_t forward_bytes(const elasto_linear_ce_t& d) {
  return up(tiles(d.classes, forward_way(d).cols) * d.rows * 8, 256) + up(d.rows * 4, 256) + gather_layout(d).bytes;
}

struct Args {
  elasto_linear_ce_t d;
  Matrix x, w;
  int es = 0;
};

bool check_desc(const elasto_linear_ce_t* d) {
  if (!d) return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: NULL description"), false;
  if (d->dtype != ELASTO_BF16 && d->dtype != ELASTO_FP32)
    return fail(ELASTO_ERR_INVALID_ARG, "bad dtype %d", d->dtype), false;
  const int n = d->dtype == ELASTO_BF16 ? 8 : 4;
  if (d->rows < 0 || d->rows > kMaxRows || d->classes < 1 || d->classes > kMaxClasses || d->dim < n ||
      d->dim > kMaxDim || d->dim % n)
    return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: bad rows or classes, or dim %d is not a multiple of %d", d->dim, n),
           false;
  const int64_t tr = tiles(d->rows, 128), tc = tiles(d->classes, 128), td = tiles(d->dim, 128);
  if (tr * tc >= kMaxTiles || tr * td >= kMaxTiles || tc * td >= kMaxTiles)
    return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: too many tiles for a launch"), false;
  return true;
}

bool check_matrix(const char* name, const void* p, int64_t ld, int dim, int es) {
  if (!p) return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: %s is NULL", name), false;
  if (!aligned(p, 16) || ld * es % 16 || ld < dim || ld > kMaxDim)
    return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: %s and its row stride must be multiples of 16 bytes, the stride in [dim, 2^20]", name),
           false;
  return true;
}

bool check_common(const elasto_linear_ce_t* d, Args* a) {
  if (!check_desc(d)) return false;
  a->d = *d;
  a->es = d->dtype == ELASTO_BF16 ? 2 : 4;
  if (d->rows > 0 && !check_matrix("x", d->x, d->ldx, d->dim, a->es)) return false;
  if (!check_matrix("weight", d->weight, d->ldw, d->dim, a->es)) return false;
  if (d->rows > 0 && !d->labels) return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: labels is NULL"), false;
  if (!aligned(d->labels, 4) || !aligned(d->bias, 4) || !aligned(d->row_weight, 4))
    return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: misaligned pointer"), false;
  a->x = Matrix{static_cast<const char*>(d->x), d->ldx * a->es};
  a->w = Matrix{static_cast<const char*>(d->weight), d->ldw * a->es};
  return true;
}

bool check_workspace(const void* ws, int64_t have, int64_t need) {
  if (need > 0 && (!ws || !aligned(ws, 256) || have < need))
    return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: the workspace holds %lld of %lld bytes (256-byte aligned)",
                (long long)(ws ? have : 0), (long long)need),
           false;
  return true;
}

CeP params(const Args& a) {
  CeP p = {};
  p.x = a.x;
  p.w = a.w;
  p.rows = a.d.rows;
  p.dim = a.d.dim;
  p.bias = a.d.bias;
  p.labels = a.d.labels;
  p.weight = a.d.row_weight;
  p.classes = a.d.classes;
  p.label_classes = a.d.classes;
  p.group = kGroup;
  return p;
}

// Takes the rows that count together in ws; p then stands for them.  False: the call's own rows are used.
bool gather(const Args& a, CeP* p, GatherP g, char* ws, hipStream_t s) {
  if (!a.d.row_weight || !gathers(a.d)) return false;
  const GatherLayout l = gather_layout(a.d);
  g.x = a.x;
  g.weight = a.d.row_weight;
  g.labels = a.d.labels;
  g.rows = a.d.rows;
  g.bytes = a.d.dim * a.es;
  g.classes = a.d.classes;
  g.count = reinterpret_cast<int32_t*>(ws + l.count);
  g.first = reinterpret_cast<int32_t*>(ws + l.first);
  g.index = reinterpret_cast<int32_t*>(ws + l.index);
  g.ys = reinterpret_cast<int32_t*>(ws + l.ys);
  g.ws = reinterpret_cast<float*>(ws + l.ws);
  g.ls = reinterpret_cast<float*>(ws + l.ls);
  g.xs = ws + l.xs;
  hipLaunchKernelGGL(ce_count_kernel, dim3(1), dim3(1024), 0, s, g);
  hipLaunchKernelGGL(ce_gather_kernel, dim3((unsigned)((g.rows + 63) / 64 * 4)), dim3(256), 0, s, g);
  p->x = Matrix{g.xs, g.bytes};
  p->labels = g.ys;
  p->weight = g.ws;
  p->lse = g.ls;
  p->count = g.count;
  p->index = g.index;
  return true;
}

template <typename T>
hipError_t forward(const Args& a, float* loss, float* lse, char* ws, hipStream_t s) {
  CeP p = params(a);
  const Way way = forward_way(a.d);
  p.tiles_n = (int)tiles(a.d.classes, way.cols);
  const int64_t parts = up((int64_t)p.tiles_n * a.d.rows * 8, 256);
  p.part = reinterpret_cast<float2*>(ws);
  p.picked = reinterpret_cast<float*>(ws + parts);
  GatherP g = {};
  g.loss = loss;
  g.lse_out = lse;
  (void)gather(a, &p, g, ws + parts + up(a.d.rows * 4, 256), s);
  with_shape<T>(way.kind, [&](auto shape) {
    typedef decltype(shape) S;
    hipLaunchKernelGGL((ce_forward_kernel<S>), dim3((unsigned)(tiles(p.rows, S::BM) * p.tiles_n)), dim3(S::kThreads),
                       0, s, p);
  });
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const JoinP j = {p.part, p.picked, p.weight, p.labels, loss, lse, p.count, p.index, a.d.rows, p.tiles_n, a.d.classes};
  if (a.d.rows > 64 * 256)
    hipLaunchKernelGGL((ce_join_kernel<64>), dim3((unsigned)((a.d.rows + 63) / 64)), dim3(1024), 0, s, j);
  else
    hipLaunchKernelGGL((ce_join_kernel<8>), dim3((unsigned)((a.d.rows + 7) / 8)), dim3(1024), 0, s, j);
  return hipGetLastError();
}

struct Grads {
  const float* lse;
  char* dx;
  int64_t lddx;
  char* dw;
  int64_t lddw;
  float* db;
  float scale;
};

unsigned blocks(int64_t n) { return (unsigned)std::min<int64_t>((n + 255) / 256, 1 << 16); }

// q.out = q.scale q.a q.b^T, in `split` parts of K where sums are given.
template <typename T, bool TA, bool LIVE>
hipError_t product(ProductP q, Kind kind, hipStream_t s) {
  with_shape<T>(kind, [&](auto shape) {
    typedef decltype(shape) S;
    q.tiles_n = (int)tiles(q.N, S::BN);
    hipLaunchKernelGGL((ce_product_kernel<S, TA, LIVE>), dim3((unsigned)(tiles(q.M, S::BM) * q.tiles_n * q.split)),
                       dim3(S::kThreads), 0, s, q);
  });
  return hipGetLastError();
}
// dx and dW (or one of them) of a piece.  In one launch where both run in large tiles (3277 rows, 131072
// classes of 2048: 5051 us in two, 4945) or in the smallest, whose launches count; fp32 in tiles of 128x64
// loses by it (1000 rows, 10007 classes of 384: 220 us in two, 235).
template <typename T, bool LIVE>
hipError_t products(const ProductP* px, Kind kx, const ProductP* pw, Kind kw, hipStream_t s) {
  const bool large = kx == Kind::Large && sizeof(T) == 2;
  if (px && pw && kx == kw && (large || kx == Kind::Tiny)) {
    ProductP x = *px, w = *pw;
    auto go = [&](auto shape) {
      typedef decltype(shape) S;
      x.tiles_n = (int)tiles(x.N, S::BN);
      w.tiles_n = (int)tiles(w.N, S::BN);
      const int64_t nx = up(tiles(x.M, S::BM) * x.tiles_n * x.split, 8);
      hipLaunchKernelGGL((ce_products_kernel<S, LIVE>), dim3((unsigned)(nx + tiles(w.M, S::BM) * w.tiles_n * w.split)),
                         dim3(S::kThreads), 0, s, x, w, (int)nx);
    };
    if constexpr (sizeof(T) == 2)
      if (large) go(typename ShapeOf<T, Kind::Large>::S());
    if (!large) go(typename ShapeOf<T, Kind::Tiny>::S());
    return hipGetLastError();
  }
  hipError_t e = hipSuccess;
  if (px) e = product<T, false, false>(*px, kx, s);
  if (pw && e == hipSuccess) e = product<T, true, LIVE>(*pw, kw, s);
  return e;
}
template <typename T>
hipError_t sum_parts(const ProductP& q, hipStream_t s) {
  hipLaunchKernelGGL((ce_sum_kernel<T>), dim3(blocks(q.M * q.N / 4)), dim3(256), 0, s, q.sum, q.split, q.M, q.N,
                     q.scale, q.out, q.ldo, q.rows_of_k ? nullptr : q.count, q.index);
  return hipGetLastError();
}

template <typename T>
hipError_t backward(const Args& a, const Grads& g, char* ws, hipStream_t s) {
  const elasto_linear_ce_t& d = a.d;
  const int es = a.es;
  if (d.rows == 0) {
    if (g.dw)
      hipLaunchKernelGGL((ce_zero_kernel<T>), dim3(blocks((int64_t)d.classes * d.dim / 4)), dim3(256), 0, s, g.dw,
                         g.lddw * es, d.classes, d.dim);
    if (g.db) hipLaunchKernelGGL(ce_zero_db_kernel, dim3(blocks(d.classes)), dim3(256), 0, s, g.db, d.classes);
    return hipGetLastError();
  }
  const BackLayout l = backward_layout(d);
  uint32_t* live = reinterpret_cast<uint32_t*>(ws + l.live);
  CeP p = params(a);
  p.lse = g.lse;
  p.scale = g.scale;
  GatherP take = {};
  take.back = true;
  take.lse = g.lse;
  take.dx = g.dx;
  take.lddx = g.lddx * es;
  const bool gathered = gather(a, &p, take, ws + l.gather, s);
  hipError_t e = hipGetLastError();
  ProductP x = {};
  x.scale = g.scale;
  x.M = d.rows;
  x.N = d.dim;
  x.out = g.dx;
  x.ldo = g.lddx * es;
  x.ld_sum = d.dim;
  x.count = p.count;
  x.index = p.index;
  x.group = kGroup;
  x.split = l.x.parts;
  if (l.x_summed) x.sum = reinterpret_cast<float*>(ws + l.sum);
  ProductP w = {};
  w.scale = g.scale;
  w.N = d.dim;
  w.K = d.rows;
  w.ldo = g.lddw * es;
  w.ld_sum = d.dim;
  w.group = kGroup;
  w.split = l.w.parts;
  if (l.w.parts > 1) w.sum = reinterpret_cast<float*>(ws + l.wsum);
  w.live = live;
  w.count = p.count;
  w.rows_of_k = true;
  for (int64_t c0 = 0; c0 < d.classes && e == hipSuccess; c0 += l.piece) {
    const int64_t n = std::min<int64_t>(l.piece, d.classes - c0);
    p.c0 = c0;
    p.classes = n;
    p.dz = Matrix{ws + l.dz, l.piece * es};
    p.ld_db = l.piece;
    p.live = !gathered && g.dw && c0 == 0 ? live : nullptr;
    int side = 0;
    with_shape<T>(way_of(d.rows, n, d.dim, es, false).kind, [&](auto shape) {
      typedef decltype(shape) S;
      side = S::BM;
      p.tiles_n = (int)tiles(n, S::BN);
      const bool direct = !gathered && p.rows <= side;
      p.db = g.db && direct ? g.db + c0 : nullptr;
      p.db_part = g.db && !direct ? reinterpret_cast<float*>(ws + l.db) : nullptr;
      hipLaunchKernelGGL((ce_dz_kernel<S>), dim3((unsigned)(tiles(p.rows, S::BM) * p.tiles_n)), dim3(S::kThreads), 0,
                         s, p);
    });
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (p.db_part) {
      hipLaunchKernelGGL(ce_db_kernel, dim3(blocks(n)), dim3(256), 0, s, p.db_part, p.count, d.rows, side, l.piece, n,
                         g.scale, g.db + c0);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    x.a = p.dz;
    x.b = Matrix{a.w.p + c0 * a.w.ld, a.w.ld};
    x.K = n;
    x.add = c0 > 0;
    w.a = p.dz;
    w.b = p.x;
    w.M = n;
    w.out = g.dw + c0 * g.lddw * es;
    const ProductP *px = g.dx ? &x : nullptr, *pw = g.dw ? &w : nullptr;
    e = gathered ? products<T, false>(px, l.x.kind, pw, l.w.kind, s) : products<T, true>(px, l.x.kind, pw, l.w.kind, s);
    if (e != hipSuccess) return e;
    if (g.dw && l.w.parts > 1) e = sum_parts<T>(w, s);
  }
  if (e == hipSuccess && g.dx && l.x_summed) e = sum_parts<T>(x, s);
  return e;
}

}  // namespace
}  // namespace elasto

using namespace elasto;

extern "C" {

elasto_status_t elasto_op_linear_ce(const elasto_linear_ce_t* desc, float* loss, float* lse, void* workspace,
                                    int64_t workspace_bytes, void* hip_stream) {
  Args a;
  if (!check_common(desc, &a)) return ELASTO_ERR_INVALID_ARG;
  if (a.d.rows == 0) return ELASTO_OK;
  if (!loss) return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: loss is NULL");
  if (!aligned(loss, 4) || !aligned(lse, 4)) return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: misaligned pointer");
  if (!check_workspace(workspace, workspace_bytes, forward_bytes(a.d))) return ELASTO_ERR_INVALID_ARG;
  char* ws = static_cast<char*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = a.d.dtype == ELASTO_BF16 ? forward<uint16_t>(a, loss, lse, ws, s)
                                                : forward<float>(a, loss, lse, ws, s);
  if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "linear_ce: %s", hipGetErrorString(e));
  return ELASTO_OK;
}

elasto_status_t elasto_op_linear_ce_bwd(const elasto_linear_ce_t* desc, const float* lse, float scale, void* dx,
                                        int64_t lddx, void* dweight, int64_t lddw, float* dbias, void* workspace,
                                        int64_t workspace_bytes, void* hip_stream) {
  Args a;
  if (!check_common(desc, &a)) return ELASTO_ERR_INVALID_ARG;
  if (!(fabsf(scale) < INFINITY)) return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: scale must be finite");
  if (a.d.rows > 0 && !lse) return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: lse is NULL");
  if (!aligned(lse, 4) || !aligned(dbias, 4)) return fail(ELASTO_ERR_INVALID_ARG, "linear_ce: misaligned pointer");
  if ((dx && a.d.rows > 0 && !check_matrix("dx", dx, lddx, a.d.dim, a.es)) ||
      (dweight && !check_matrix("dweight", dweight, lddw, a.d.dim, a.es)))
    return ELASTO_ERR_INVALID_ARG;
  if (!check_workspace(workspace, workspace_bytes, backward_layout(a.d).total)) return ELASTO_ERR_INVALID_ARG;
  const Grads g = {lse, static_cast<char*>(dx), lddx, static_cast<char*>(dweight), lddw, dbias, scale};
  char* ws = static_cast<char*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const hipError_t e = a.d.dtype == ELASTO_BF16 ? backward<uint16_t>(a, g, ws, s) : backward<float>(a, g, ws, s);
  if (e != hipSuccess) return fail(ELASTO_ERR_HIP, "linear_ce: %s", hipGetErrorString(e));
  return ELASTO_OK;
}

elasto_status_t elasto_linear_ce_workspace(const elasto_linear_ce_t* desc, int32_t backward, int64_t* bytes) {
  if (!bytes) return fail(ELASTO_ERR_INVALID_ARG, "NULL argument");
  if (!check_desc(desc)) return ELASTO_ERR_INVALID_ARG;
  *bytes = backward ? backward_layout(*desc).total : forward_bytes(*desc);
  return ELASTO_OK;
}

}  // extern "C"
