// Dense layers of the output head and their gradients:
//   u = x W^T + b,  y = act(u) + r                       (forward)
//   dz = dy * act'(u),  dx = dz W,  dW = dz^T x,  db = sum of dz's rows
// with one weight for all rows, or one for each contiguous group of rows
// (ragged: group g holds rows offsets[g] .. offsets[g + 1] - 1, read on the
// device; empty groups allowed).
//
// The three products run on the same tile cores (ring_device.h where rows are whole
// 16-byte vectors, else product_device.h): the forward's operands are both
// k-contiguous, dx reads W by columns, dW reads dz and x by columns. dz is formed once, in the storage dtype (the products then read
// 16-bit values; bf16 rounds it to 2^-9, which adds in quadrature to the same
// rounding of dx and dW), by the kernel that also sums db, in fp32, from the
// values before that rounding.
#include <algorithm>

#include "kernels.h"
#include "ring_device.h"

namespace pinsage {
namespace {

// ---- activations -----------------------------------------------------------
// gelu in its tanh form, 0.5 u (1 + tanh t) = u sigmoid(2 t),
// t = sqrt(2 / pi) (u + 0.044715 u^3).
constexpr float kGelu2 = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kGeluCube = 0.044715f;

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + __expf(-x)); }

__device__ __forceinline__ float activate(float u, int act) {
  if (act == kActRelu) return u < 0.0f ? 0.0f : u;  // NaN stays
  if (act == kActGelu) return u * sigmoid(kGelu2 * (u + kGeluCube * u * u * u));
  if (act == kActSilu) return u * sigmoid(u);
  return u;
}

__device__ __forceinline__ float grad_through(float dy, float u, int act) {
  if (act == kActRelu) return u > 0.0f ? dy : 0.0f;
  if (act == kActGelu) {
    const float s = sigmoid(kGelu2 * (u + kGeluCube * u * u * u));
    return dy * (s + u * s * (1.0f - s) * kGelu2 * (1.0f + 3.0f * kGeluCube * u * u));
  }
  if (act == kActSilu) {
    const float s = sigmoid(u);
    return dy * (s * (1.0f + u * (1.0f - s)));
  }
  return dy;
}

// ---- groups of rows ----------------------------------------------------------
// Pieces of `unit` rows, group after group; in `at_least_one` mode an empty
// group has one (empty) piece. Offsets are clamped to [0, n] and to ascending
// order, so that no row outside the operands is ever read or written; the rows
// past the last group are group G's, the one without a weight (`tail` mode).
struct Piece {
  int group = -1;
  int64_t lo = 0, hi = 0;  // the group's rows
  int64_t index = 0;       // the piece within the group
  int pieces = 0;          // of the group
  int64_t slot = 0;        // pieces of groups that have several, before this group
};

__device__ __forceinline__ int xcd_tile(int b, int nt) {
  const int per = nt / 8, rem = nt % 8;
  const int xcd = b % 8, slot = b / 8;
  return xcd < rem ? xcd * (per + 1) + slot : rem * (per + 1) + (xcd - rem) * per + slot;
}

struct Groups {
  const int64_t* offsets;
  int G;
  int64_t n;
  int unit;
  bool at_least_one, tail;

  __device__ __forceinline__ int count() const { return tail ? G + 1 : G; }
  __device__ __forceinline__ void bounds(int g, int64_t& lo, int64_t& hi) const {
    lo = offsets[g];
    lo = lo < 0 ? 0 : (lo > n ? n : lo);
    hi = g < G ? offsets[g + 1] : n;
    hi = hi < lo ? lo : (hi > n ? n : hi);
  }
  __device__ __forceinline__ int pieces(int g) const {
    int64_t lo, hi;
    bounds(g, lo, hi);
    const int p = (int)((hi - lo + unit - 1) / unit);
    return at_least_one && p == 0 ? 1 : p;
  }
  // All lanes of a wave take part in these two; the results are wave-uniform.
  __device__ __forceinline__ int total(int lane) const {
    int sum = 0;
    for (int g0 = 0; g0 < count(); g0 += 64)
      sum += g0 + lane < count() ? pieces(g0 + lane) : 0;
    return wave_sum_i32(sum);
  }
  __device__ __forceinline__ Piece find(int t, int lane) const {
    Piece out;
    int before = 0, slots = 0;
    for (int g0 = 0; g0 < count(); g0 += 64) {
      const int p = g0 + lane < count() ? pieces(g0 + lane) : 0;
      const int incl = wave_inclusive_sum(p, lane) + before;
      const int slot_incl = wave_inclusive_sum(p > 1 ? p : 0, lane) + slots;
      const unsigned long long past = __ballot(incl > t);
      if (past) {
        const int l = __builtin_ctzll(past);
        out.group = g0 + l;
        out.pieces = __builtin_amdgcn_readlane(p, l);
        out.index = t - (__builtin_amdgcn_readlane(incl, l) - out.pieces);
        out.slot = __builtin_amdgcn_readlane(slot_incl, l) - (out.pieces > 1 ? out.pieces : 0);
        bounds(out.group, out.lo, out.hi);
        return out;
      }
      before = __builtin_amdgcn_readlane(incl, 63);
      slots = __builtin_amdgcn_readlane(slot_incl, 63);
    }
    return out;
  }
};

// ---- products over rows: the forward pass, and dx -----------------------------
// C[r][c] = act(sum_k A[r][k] B(c, k) + bias[c]) + residual[r][c], U[r][c] the
// value before act. B(c, k) = B[c * ldb + k] (B_COL: B[k * ldb + c]) of r's group.
template <class C>
__global__ __launch_bounds__(C::THREADS, C::WPE) void dense_rows_kernel(DenseLaunch a) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::LDS_BYTES];
  constexpr bool BF16 = C::MODE == kBf16;
  const int lane = threadIdx.x & 63;
  const int tiles_n = (a.N + C::BN - 1) / C::BN;
  int tile;
  int64_t lo = 0, hi = a.M, m0;
  int group = 0;
  if (a.offsets) {
    const Groups gr{a.offsets, a.G, a.M, C::BM, false, true};
    const int total = gr.total(lane) * tiles_n;
    if ((int)blockIdx.x >= total) return;
    tile = xcd_tile(blockIdx.x, total);
    const Piece p = gr.find(tile / tiles_n, lane);
    if (p.group < 0) return;
    group = p.group;
    lo = p.lo;
    hi = p.hi;
    m0 = lo + p.index * C::BM;
  } else {
    tile = xcd_tile(blockIdx.x, gridDim.x);
    m0 = (int64_t)(tile / tiles_n) * C::BM;
  }
  const int n0 = (tile % tiles_n) * C::BN;
  const int valid = (int)(hi - m0 < C::BM ? hi - m0 : C::BM);
  const unsigned char* const Ap = static_cast<const unsigned char*>(a.A) + m0 * a.lda * C::ESZ;
  const unsigned char* const Bg =
      static_cast<const unsigned char*>(a.B) + (int64_t)group * a.group_stride * C::ESZ;
  const bool orphans = a.offsets && group == a.G;  // rows of no group: zeros

  TileSums<C> sums;
  const Operand A{Ap, a.lda, valid, 0};
  const Operand B{Bg + (C::B_COL ? (int64_t)n0 : n0 * a.ldb) * C::ESZ, a.ldb,
                  a.N - n0 < C::BN ? a.N - n0 : C::BN, 0};
  tile_sums(A, B, 0, orphans ? 0 : a.K, smem, sums);
  const float* const bias = a.bias && !orphans ? a.bias + (int64_t)group * a.N : nullptr;
  product_rows(sums, smem, [&](int m, int nn, float (&v)[4]) __attribute__((always_inline)) {
    const int n = n0 + nn;
    const int cols = a.N - n;
    if (m >= valid || cols <= 0) return;
    const int64_t r = m0 + m;
    if constexpr (!BF16) {
      const float* const b = reinterpret_cast<const float*>(Bg);
      redo_not_finite(v, cols < 4 ? cols : 4, reinterpret_cast<const float*>(Ap) + m * a.lda, 1,
                      C::B_COL ? b + n : b + n * a.ldb, C::B_COL ? a.ldb : 1,
                      C::B_COL ? 1 : a.ldb, a.K);
    }
    if (bias) {
      float w[4];
      read4<false>(bias, n, cols, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += w[e];
    }
    if (a.U) write4<BF16>(static_cast<unsigned char*>(a.U) + r * a.ldu * C::ESZ, n, cols, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = activate(v[e], a.act);
    if (a.residual && !orphans) {
      float w[4];
      read4<BF16>(static_cast<const unsigned char*>(a.residual) + r * a.ldr * C::ESZ, n, cols, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += w[e];
    }
    write4<BF16>(static_cast<unsigned char*>(a.C) + r * a.ldc * C::ESZ, n, cols, v);
  });
}

// ---- the forward pass of few rows ---------------------------------------------
// What bounds it is the weight: every element is read once for at most 64 rows,
// so a block takes 16 of its rows (output columns) and its eight waves split k,
// each with its loads straight from global memory into MFMA operands, 16 rows of x
// beside them. The eight partial sums meet in LDS, in order.
constexpr int kFewWaves = 8;

template <bool BF16, int MT>
__device__ __forceinline__ void few_rows(const DenseLaunch& a, const unsigned char* Bg,
                                         int group, int64_t r0, int valid, int n0, bool orphans,
                                         float (*part)[16 * MT][16]) {
  constexpr int ESZ = BF16 ? 2 : 4, VE = 16 / ESZ, STEP = 4 * VE;  // k columns per load
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int row = lane & 15, q = lane >> 4;
  f32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = f32x4{0, 0, 0, 0};
  if (!orphans) {
    const int wn = n0 + row < a.N ? n0 + row : a.N - 1;
    const unsigned char* const pw = Bg + (int64_t)wn * a.ldb * ESZ;
    const unsigned char* px[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const int m = 16 * t + row;
      px[t] = static_cast<const unsigned char*>(a.A) + (r0 + (m < valid ? m : valid - 1)) * a.lda * ESZ;
    }
    auto multiply = [&](const u32x4& w, const u32x4 (&x)[MT]) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        if constexpr (BF16) {
          acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x[t]), acc[t], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[e]),
                                                          __uint_as_float(x[t][e]), acc[t], 0, 0, 0);
        }
      }
    };
    const int steps = a.K / STEP;
    int s = wave;
    constexpr int DEEP = MT == 1 ? 8 : 2;
    for (; s + (DEEP - 1) * kFewWaves < steps; s += DEEP * kFewWaves) {
      u32x4 w[DEEP], x[DEEP][MT];
#pragma unroll
      for (int d = 0; d < DEEP; ++d) {
        const uint32_t at = (uint32_t)(((s + d * kFewWaves) * STEP + q * VE) * ESZ);
        w[d] = load_any<u32x4>(pw + at);
#pragma unroll
        for (int t = 0; t < MT; ++t) x[d][t] = load_any<u32x4>(px[t] + at);
      }
#pragma unroll
      for (int d = 0; d < DEEP; ++d) multiply(w[d], x[d]);
    }
    for (; s <= steps; s += kFewWaves) {  // the rest, and the part past the last whole step
      const int at = s * STEP + q * VE, have = a.K - at;
      u32x4 w = {0, 0, 0, 0}, x[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) x[t] = w;
      if (have >= VE) {
        w = load_any<u32x4>(pw + at * ESZ);
#pragma unroll
        for (int t = 0; t < MT; ++t) x[t] = load_any<u32x4>(px[t] + at * ESZ);
      } else if (have > 0) {
        w = load_part<ESZ>(pw + at * ESZ, have);
#pragma unroll
        for (int t = 0; t < MT; ++t) x[t] = load_part<ESZ>(px[t] + at * ESZ, have);
      }
      multiply(w, x);
    }
  }
  // A lane holds x row lane % 16 and weight rows 4 (lane / 16) + e.
#pragma unroll
  for (int t = 0; t < MT; ++t)
    *reinterpret_cast<float4*>(&part[wave][16 * t + row][4 * q]) =
        make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
  __syncthreads();
  const int tid = threadIdx.x;
  if (tid < 64 * MT) {
    const int m = tid / 4, nn = tid % 4 * 4, n = n0 + nn, cols = a.N - n;
    float v[4] = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float4 p = *reinterpret_cast<const float4*>(&part[w][m][nn]);
      v[0] += p.x;
      v[1] += p.y;
      v[2] += p.z;
      v[3] += p.w;
    }
    if (m < valid && cols > 0) {
      const int64_t r = r0 + m;
      if (a.bias && !orphans) {
        float w[4];
        read4<false>(a.bias + (int64_t)group * a.N, n, cols, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
      }
      if (a.U) write4<BF16>(static_cast<unsigned char*>(a.U) + r * a.ldu * ESZ, n, cols, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = activate(v[e], a.act);
      if (a.residual && !orphans) {
        float w[4];
        read4<BF16>(static_cast<const unsigned char*>(a.residual) + r * a.ldr * ESZ, n, cols, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
      }
      write4<BF16>(static_cast<unsigned char*>(a.C) + r * a.ldc * ESZ, n, cols, v);
    }
  }
  __syncthreads();
}

template <bool BF16>
__global__ __launch_bounds__(64 * kFewWaves) void dense_few_kernel(DenseLaunch a) {
  __shared__ __attribute__((aligned(16))) float part[kFewWaves][64][16];
  const int group = blockIdx.y, n0 = blockIdx.x * 16;
  int64_t lo = 0, hi = a.M;
  if (a.offsets) Groups{a.offsets, a.G, a.M, 1, false, true}.bounds(group, lo, hi);
  const bool orphans = a.offsets && group == a.G;
  const unsigned char* const Bg =
      static_cast<const unsigned char*>(a.B) + (int64_t)group * a.group_stride * (BF16 ? 2 : 4);
  for (int64_t r = lo; r < hi;) {
    if (hi - r <= 16) {
      few_rows<BF16, 1>(a, Bg, group, r, (int)(hi - r), n0, orphans,
                        reinterpret_cast<float (*)[16][16]>(part));
      r = hi;
    } else {
      const int rows = (int)(hi - r < 64 ? hi - r : 64);
      few_rows<BF16, 4>(a, Bg, group, r, rows, n0, orphans, part);
      r += rows;
    }
  }
}

// ---- dz and db -----------------------------------------------------------------
// A block takes a piece of a.bias_rows rows of one group and up to 256 columns, a
// thread 4 columns of every (256 / lanes)-th row, lanes the smallest power of two
// of threads that covers the columns.
template <bool BF16>
__global__ __launch_bounds__(256) void dense_dz_kernel(DenseGradLaunch a, int lanes) {
  __shared__ float4 sums[256];
  constexpr int ESZ = BF16 ? 2 : 4;
  const int tid = threadIdx.x;
  Piece p;
  if (a.offsets) {
    p = Groups{a.offsets, a.G, a.n, a.bias_rows, true, true}.find(blockIdx.x, tid & 63);
    if (p.group < 0) return;
  } else {
    p.group = 0;
    p.lo = 0;
    p.hi = a.n;
    p.index = blockIdx.x;
  }
  const int64_t r0 = p.lo + p.index * a.bias_rows;
  const int64_t r1 = p.hi - r0 < a.bias_rows ? p.hi : r0 + a.bias_rows;
  const int n = (blockIdx.y * lanes + tid % lanes) * 4, cols = a.N - n;
  float s[4] = {0, 0, 0, 0};
  if (cols > 0) {
    const int step = 256 / lanes;
#pragma unroll 4
    for (int64_t r = r0 + tid / lanes; r < r1; r += step) {
      float d[4];
      read4<BF16>(static_cast<const unsigned char*>(a.dy) + r * a.lddy * ESZ, n, cols, d);
      if (a.act != kActNone) {
        float u[4];
        read4<BF16>(static_cast<const unsigned char*>(a.U) + r * a.ldu * ESZ, n, cols, u);
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] = grad_through(d[e], u[e], a.act);
      }
      if (a.dz) write4<BF16>(static_cast<unsigned char*>(a.dz) + r * a.lddz * ESZ, n, cols, d);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += d[e];
    }
  }
  if (!a.db_parts) return;
  sums[tid] = make_float4(s[0], s[1], s[2], s[3]);
  __syncthreads();
  if (tid < lanes && cols > 0) {
    for (int t = tid + lanes; t < 256; t += lanes) {
      const float4 x = sums[t];
      s[0] += x.x;
      s[1] += x.y;
      s[2] += x.z;
      s[3] += x.w;
    }
    write4<false>(a.db_parts + (int64_t)blockIdx.x * a.N, n, cols, s);
  }
}

// db[g] = the sum of the group's pieces, in order within each of the four
// threads that share a column.
__global__ __launch_bounds__(256) void dense_db_kernel(DenseGradLaunch a) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int g = blockIdx.y, n = blockIdx.x * 64 + lane;
  int64_t first = 0, pieces = (a.n + a.bias_rows - 1) / a.bias_rows;
  if (a.offsets) {
    const Groups gr{a.offsets, a.G, a.n, a.bias_rows, true, true};
    int before = 0;
    for (int q = lane; q < g; q += 64) before += gr.pieces(q);
    first = wave_sum_i32(before);
    pieces = gr.pieces(g);
  }
  // Offsets that overlap could count more pieces than there are.
  const int64_t all = dense_bias_pieces(a.n, a.offsets ? a.G : 0, a.bias_rows);
  if (first + pieces > all) pieces = first < all ? all - first : 0;
  const int64_t per = (pieces + 3) / 4;
  const int64_t q1 = per * (w + 1) < pieces ? per * (w + 1) : pieces;
  float s = 0.0f;
  if (n < a.N)
#pragma unroll 8
    for (int64_t q = per * w; q < q1; ++q) s += a.db_parts[(first + q) * a.N + n];
  part[w][lane] = s;
  __syncthreads();
  if (w == 0 && n < a.N)
    a.db[(int64_t)g * a.N + n] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
}

// ---- dW ------------------------------------------------------------------------
// dW[g][n][k] = sum over the group's rows of dz[r][n] x[r][k]. Where the tiles of
// dW alone leave CUs idle, a group's rows are cut into pieces of a.piece rows; a
// group of several leaves fp32 partial sums in the workspace, which
// dense_dw_join_kernel adds in order.
template <class C>
__global__ __launch_bounds__(C::THREADS, C::WPE) void dense_dw_kernel(DenseGradLaunch a) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::LDS_BYTES];
  constexpr bool BF16 = C::MODE == kBf16;
  const int lane = threadIdx.x & 63;
  const int tiles_k = (a.K + C::BN - 1) / C::BN, tiles = tiles_k * ((a.N + C::BM - 1) / C::BM);
  Piece p;
  int tile;
  if (a.offsets) {
    const Groups gr{a.offsets, a.G, a.n, a.piece, true, false};
    const int total = gr.total(lane) * tiles;
    if ((int)blockIdx.x >= total) return;
    tile = xcd_tile(blockIdx.x, total);
    p = gr.find(tile / tiles, lane);
    if (p.group < 0) return;
  } else {
    tile = xcd_tile(blockIdx.x, gridDim.x);
    p.group = 0;
    p.lo = 0;
    p.hi = a.n;
    p.index = tile / tiles;
    p.pieces = (int)((a.n + a.piece - 1) / a.piece);
  }
  tile %= tiles;
  const int n0 = tile / tiles_k * C::BM, k0 = tile % tiles_k * C::BN;
  const int64_t r0 = p.lo + p.index * a.piece;
  const int64_t rows = p.hi - r0 < a.piece ? p.hi - r0 : a.piece;
  const int vn = a.N - n0 < C::BM ? a.N - n0 : C::BM, vk = a.K - k0 < C::BN ? a.K - k0 : C::BN;
  const unsigned char* const Z =
      static_cast<const unsigned char*>(a.dz) + (r0 * a.lddz + n0) * C::ESZ;
  const unsigned char* const X =
      static_cast<const unsigned char*>(a.x) + (r0 * a.ldx + k0) * C::ESZ;
  TileSums<C> sums;
  tile_sums(Operand{Z, a.lddz, vn, 0}, Operand{X, a.ldx, vk, 0}, 0, rows, smem, sums);
  // Offsets that overlap could count more pieces than the workspace holds.
  if (p.pieces > 1 && p.slot + p.index >= dense_dw_parts(a.n, a.piece, a.offsets ? a.G : 0)) return;
  float* const part = p.pieces > 1 ? a.dw_parts + (p.slot + p.index) * (int64_t)a.N * a.K : nullptr;
  unsigned char* const out =
      static_cast<unsigned char*>(a.dW) + (int64_t)p.group * a.N * a.K * C::ESZ;
  product_rows(sums, smem, [&](int m, int nn, float (&v)[4]) __attribute__((always_inline)) {
    const int cols = vk - nn;
    if (m >= vn || cols <= 0) return;
    if constexpr (!BF16)
      redo_not_finite(v, cols < 4 ? cols : 4, reinterpret_cast<const float*>(Z) + m, a.lddz,
                      reinterpret_cast<const float*>(X) + nn, a.ldx, 1, rows);
    const int64_t at = (int64_t)(n0 + m) * a.K + k0 + nn;
    if (part) write4<false>(part, at, cols, v);
    else write4<BF16>(out, at, cols, v);
  });
}

template <bool BF16>
__global__ __launch_bounds__(256) void dense_dw_join_kernel(DenseGradLaunch a) {
  const int64_t size = (int64_t)a.N * a.K;
  Piece p;
  if (a.offsets) {
    // The group's first piece: pieces before it, then its own.
    const Groups gr{a.offsets, a.G, a.n, a.piece, true, false};
    const int lane = threadIdx.x & 63, g = blockIdx.y;
    p.pieces = gr.pieces(g);
    if (p.pieces < 2) return;
    int before = 0;
    for (int q = lane; q < g; q += 64) {
      const int c = gr.pieces(q);
      before += c > 1 ? c : 0;
    }
    p.group = g;
    p.slot = wave_sum_i32(before);
    const int64_t all = dense_dw_parts(a.n, a.piece, a.G);
    if (p.slot + p.pieces > all) p.pieces = p.slot < all ? (int)(all - p.slot) : 0;
  } else {
    p.group = 0;
    p.pieces = (int)((a.n + a.piece - 1) / a.piece);
  }
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (at >= size) return;
  const int cols = (int)(size - at < 4 ? size - at : 4);
  const float* src = a.dw_parts + p.slot * size;
  float s[4] = {0, 0, 0, 0};
#pragma unroll 4
  for (int q = 0; q < p.pieces; ++q, src += size) {
    float v[4];
    read4<false>(src, at, cols, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += v[e];
  }
  write4<BF16>(static_cast<unsigned char*>(a.dW) + p.group * size * (BF16 ? 2 : 4), at, cols, s);
}

// ---- tile shapes -----------------------------------------------------------------
// Ring: rows of whole 16-byte vectors; else the register core, which has no
// 256 x 256 tile.
template <bool BF16, bool A_COL, bool B_COL>
struct Tiles;
template <bool A_COL, bool B_COL>
struct Tiles<true, A_COL, B_COL> {
  using RingBig = RingCfg<kBf16, 256, 256, 64, 2, 4, A_COL, B_COL, 2>;
  using RingMid = RingCfg<kBf16, 128, 128, 64, 2, 2, A_COL, B_COL, 2>;
  using RingSmall = RingCfg<kBf16, 64, 64, 64, 2, 2, A_COL, B_COL, 4>;
  using Mid = ProductCfg<kBf16, 128, 128, 64, 2, 2, A_COL, B_COL, 2>;
  using Small = ProductCfg<kBf16, 64, 64, 128, 2, 2, A_COL, B_COL, 2>;
};
template <bool A_COL, bool B_COL>
struct Tiles<false, A_COL, B_COL> {
  using RingMid = RingCfg<kF32, 128, 128, 16, 2, 2, A_COL, B_COL, 4, 2>;
  using RingSmall = RingCfg<kF32, 64, 64, 16, 2, 2, A_COL, B_COL, 4>;
  using RingBig = RingMid;
  using Mid = ProductCfg<kF32, 128, 128, 32, 2, 2, A_COL, B_COL, 1>;
  using Small = ProductCfg<kF32, 64, 64, 64, 2, 2, A_COL, B_COL, 1>;
};

enum Shape { kSmall, kMid, kBig };
constexpr int side(Shape s) { return s == kSmall ? 64 : (s == kMid ? 128 : 256); }

inline int64_t tiles_of(int64_t m, int64_t n, int b) { return ((m + b - 1) / b) * ((n + b - 1) / b); }

inline Shape rows_shape(int64_t m, int64_t n, bool bf16) {
  if (!bf16) return tiles_of(m, n, 128) < 512 ? kSmall : kMid;
  if (tiles_of(m, n, 64) <= 512) return kSmall;
  return tiles_of(m, n, 256) < 256 ? kMid : kBig;
}

inline bool vectors(const void* p, int64_t ld, int64_t width, bool bf16) {
  const int64_t ve = bf16 ? 8 : 4;
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % ve == 0 && width % ve == 0;
}

template <class C>
hipError_t rows_cfg(const DenseLaunch& a, hipStream_t s) {
  const int64_t tiles_n = (a.N + C::BN - 1) / C::BN;
  const int64_t tiles = ((a.M + C::BM - 1) / C::BM + (a.offsets ? a.G + 1 : 0)) * tiles_n;
  if (tiles > 0x7FFFFFFFll) return hipErrorInvalidValue;
  hipLaunchKernelGGL(dense_rows_kernel<C>, dim3((unsigned)tiles), dim3(C::THREADS), 0, s, a);
  return hipGetLastError();
}

template <bool BF16, bool B_COL>
hipError_t rows_dtype(const DenseLaunch& a, hipStream_t s) {
  using T = Tiles<BF16, false, B_COL>;
  const Shape shape = rows_shape(a.M, a.N, BF16);
  if (vectors(a.A, a.lda, a.K, BF16) && vectors(a.B, a.ldb, B_COL ? a.N : a.K, BF16)) {
    if (shape == kSmall) return rows_cfg<typename T::RingSmall>(a, s);
    if (shape == kMid) return rows_cfg<typename T::RingMid>(a, s);
    return rows_cfg<typename T::RingBig>(a, s);
  }
  return shape == kSmall ? rows_cfg<typename T::Small>(a, s) : rows_cfg<typename T::Mid>(a, s);
}

// Tiles of dW: the largest of which enough pieces of 512 rows or more (1,024 under
// 256 x 256) fill the chip.
inline Shape dw_shape(int64_t n, int N, int K, bool bf16) {
  if (bf16 && tiles_of(N, K, 256) * (n / 1024) >= 256 && N > 128 && K > 128) return kBig;
  return tiles_of(N, K, 128) * (n / 512) >= 256 && N > 64 && K > 64 ? kMid : kSmall;
}

template <class C>
hipError_t dw_cfg(const DenseGradLaunch& a, hipStream_t s) {
  const int64_t pieces = (a.n + a.piece - 1) / a.piece + (a.offsets ? a.G : 0);
  const int64_t blocks = (pieces > 0 ? pieces : 1) * tiles_of(a.N, a.K, C::BM);
  if (blocks > 0x7FFFFFFFll) return hipErrorInvalidValue;
  hipLaunchKernelGGL(dense_dw_kernel<C>, dim3((unsigned)blocks), dim3(C::THREADS), 0, s, a);
  return hipGetLastError();
}

template <bool BF16>
hipError_t dw_tiles(const DenseGradLaunch& a, hipStream_t s) {
  using T = Tiles<BF16, true, true>;
  const Shape shape = dw_shape(a.n, a.N, a.K, BF16);
  if (vectors(a.dz, a.lddz, a.N, BF16) && vectors(a.x, a.ldx, a.K, BF16)) {
    if (shape == kSmall) return dw_cfg<typename T::RingSmall>(a, s);
    if (shape == kMid) return dw_cfg<typename T::RingMid>(a, s);
    return dw_cfg<typename T::RingBig>(a, s);
  }
  return shape == kSmall ? dw_cfg<typename T::Small>(a, s) : dw_cfg<typename T::Mid>(a, s);
}

template <bool BF16>
hipError_t dw_dtype(const DenseGradLaunch& a, hipStream_t s) {
  const hipError_t e = dw_tiles<BF16>(a, s);
  if (e != hipSuccess || !a.dw_parts) return e;
  const int64_t blocks = ((int64_t)a.N * a.K + 1023) / 1024;
  hipLaunchKernelGGL(dense_dw_join_kernel<BF16>, dim3((unsigned)blocks, a.offsets ? a.G : 1),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

bool few_rows_wanted(const DenseLaunch& a) {
  return !a.b_col && a.M <= 16 * (int64_t)(a.offsets ? a.G : 4);
}

}  // namespace

hipError_t launch_dense_rows(const DenseLaunch& a, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  ProfileScope prof(a.b_col ? kKDenseGrad : kKDense, s);
  if (few_rows_wanted(a)) {
    const dim3 grid((unsigned)((a.N + 15) / 16), a.offsets ? a.G + 1 : 1);
    if (a.bf16) hipLaunchKernelGGL(dense_few_kernel<true>, grid, dim3(64 * kFewWaves), 0, s, a);
    else hipLaunchKernelGGL(dense_few_kernel<false>, grid, dim3(64 * kFewWaves), 0, s, a);
    return hipGetLastError();
  }
  if (a.b_col) return a.bf16 ? rows_dtype<true, true>(a, s) : rows_dtype<false, true>(a, s);
  return a.bf16 ? rows_dtype<true, false>(a, s) : rows_dtype<false, false>(a, s);
}

// Rows per piece of dW's sums: as many pieces as give the chip 512 blocks, of 256
// rows at least.
int64_t dense_dw_piece(int64_t n, int N, int K, bool bf16) {
  const int64_t tiles = tiles_of(N, K, side(dw_shape(n, N, K, bf16)));
  const int64_t want = (512 + tiles - 1) / tiles;
  const int64_t rows = ((n + want - 1) / want + 63) / 64 * 64;
  return rows < 256 ? 256 : rows;
}

hipError_t launch_dense_dz(const DenseGradLaunch& a, hipStream_t s) {
  ProfileScope prof(kKDenseGrad, s);
  int lanes = 1;
  while (lanes < 64 && lanes * 4 < a.N) lanes *= 2;
  const int64_t pieces = dense_bias_pieces(a.n, a.offsets ? a.G : 0, a.bias_rows);
  const dim3 grid((unsigned)(pieces > 0 ? pieces : 1), (unsigned)((a.N + 4 * lanes - 1) / (4 * lanes)));
  if (pieces > 0) {
    if (a.bf16) hipLaunchKernelGGL(dense_dz_kernel<true>, grid, dim3(256), 0, s, a, lanes);
    else hipLaunchKernelGGL(dense_dz_kernel<false>, grid, dim3(256), 0, s, a, lanes);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.db) return hipSuccess;
  hipLaunchKernelGGL(dense_db_kernel, dim3((unsigned)((a.N + 63) / 64), a.offsets ? a.G : 1),
                     dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_dense_dw(const DenseGradLaunch& a, hipStream_t s) {
  ProfileScope prof(kKDenseGrad, s);
  return a.bf16 ? dw_dtype<true>(a, s) : dw_dtype<false>(a, s);
}

}  // namespace pinsage
