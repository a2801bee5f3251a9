// Dense layers of the output head and their gradients:
//   u = x W^T + b,  y = act(u) + r                       (forward)
//   dz = dy * act'(u),  dx = dz W,  dW = dz^T x,  db = sum of dz's rows
// with one weight for all rows, or one for each contiguous group of rows
// (ragged: group g holds rows offsets[g] .. offsets[g + 1] - 1, read on the
// device; empty groups allowed).
//
// The three products run on the same tiles (ring_device.h): the forward's operands are
// both k-contiguous, dx reads W by columns, dW reads dz and x by columns. dz is formed
// once, by the kernel that also sums db, in fp32, from the values before any rounding.
// fp32 storage keeps it in fp32, bf16 storage in two bf16 parts (2^-17) that the products
// take one after the other: in one, dz's rounding adds in quadrature to the same one
// of dx and dW (2-norm error 2.3e-3 against 1.7e-3). Where dz is dy or 0 (ReLU, no
// activation) it needs no second part.
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

// For bf16 results the exponential whose relative error grows with |x| (2^-20 at 10)
// and the reciprocal instruction (1 unit in the last place) are near enough; fp32 takes
// the exact forms.
template <bool BF16>
__device__ __forceinline__ float sigmoid(float x) {
  if constexpr (BF16) return __builtin_amdgcn_rcpf(1.0f + __expf(-x));
  else return 1.0f / (1.0f + expf(-x));
}

// One branch for all values, not one for each.
template <bool BF16, int N>
__device__ __forceinline__ void activate(float (&u)[N], int act) {
  if (act == kActRelu) {
#pragma unroll
    for (int e = 0; e < N; ++e) u[e] = u[e] < 0.0f ? 0.0f : u[e];  // NaN stays
  } else if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < N; ++e)
      u[e] *= sigmoid<BF16>(kGelu2 * (u[e] + kGeluCube * u[e] * u[e] * u[e]));
  } else if (act == kActSilu) {
#pragma unroll
    for (int e = 0; e < N; ++e) u[e] *= sigmoid<BF16>(u[e]);
  }
}

// dy becomes dy * act'(u).
template <bool BF16, int N>
__device__ __forceinline__ void grad_through(float (&dy)[N], const float (&u)[N], int act) {
  if (act == kActRelu) {
#pragma unroll
    for (int e = 0; e < N; ++e) dy[e] = u[e] > 0.0f ? dy[e] : 0.0f;
  } else if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      // 0 and 1 long before 64, where u^2 could overflow beside a factor that is 0. NaN stays.
      const float x = fabsf(u[e]) > 64.0f ? copysignf(64.0f, u[e]) : u[e];
      const float q = kGeluCube * x * x, s = sigmoid<BF16>(kGelu2 * x * (1.0f + q));
      dy[e] *= s + x * s * (1.0f - s) * kGelu2 * (1.0f + 3.0f * q);
    }
  } else if (act == kActSilu) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float s = sigmoid<BF16>(u[e]);
      dy[e] *= s * (1.0f + u[e] * (1.0f - s));
    }
  }
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

struct Groups {
  const int64_t* offsets;
  int G;
  int64_t n;
  int unit;
  bool at_least_one, tail;
  // Blocks take whole pieces before the groups' shorter last ones, and those (up to 64
  // groups) by descending length: dW's pieces differ by what they sum over.
  bool longest_first = false;

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
  // Piece t, or, given `tiles` per piece, the piece and tile (in t) of block
  // `block`, neighbouring tiles on one XCD. All lanes of a wave
  // take part; the results are wave-uniform. Up to 64 groups the offsets are read once.
  __device__ __forceinline__ Piece find(int lane, int& t, int block, int tiles) const {
    Piece out;
    const int all = count();
    int64_t lo = 0, hi = 0;
    int p = 0, whole = 0;
    auto load = [&](int g) __attribute__((always_inline)) {
      lo = hi = 0;
      if (g < all) bounds(g, lo, hi);
      const int q = (int)((hi - lo + unit - 1) / unit);
      p = g < all ? (at_least_one && q == 0 ? 1 : q) : 0;
      whole = longest_first ? (int)((hi - lo) / unit) : 0;
    };
    load(lane);
    int at = t;
    int first_whole = 0;  // whole pieces of all groups
    if (tiles > 0) {
      int total = wave_sum_i32(p);
      if (longest_first) first_whole = wave_sum_i32(whole);
      for (int g0 = 64; g0 < all; g0 += 64) {
        load(g0 + lane);
        total += wave_sum_i32(p);
        if (longest_first) first_whole += wave_sum_i32(whole);
      }
      if (all > 64) load(lane);
      if (longest_first) {
        // Block b runs on XCD b % 8: a piece's tiles on one of them, the pieces there and
        // back, so that each XCD has its share of the long ones.
        const int row = block / 8 / tiles, xcd = block % 8;
        at = row * 8 + (row & 1 ? 7 - xcd : xcd);
        t = block / 8 % tiles;
        if (at >= total) return out;
      } else {
        total *= tiles;
        if (block >= total) return out;
        at = xcd_tile(block, total);
        t = at % tiles;
        at /= tiles;
      }
    }
    // Counted among the whole pieces, or among the others.
    const bool of_whole = at < first_whole;
    if (!of_whole) at -= first_whole;
    if (longest_first && !of_whole && all <= 64) {
      // The group whose last piece is the at-th longest (ties: the first group).
      const int rest = p > whole ? (int)((hi - lo) % unit) : -1;
      int rank = 0;
      for (int l = 0; l < all; ++l) {
        const int other = __builtin_amdgcn_readlane(rest, l);
        rank += other > rest || (other == rest && l < lane);
      }
      const unsigned long long hit = __ballot(rest >= 0 && rank == at);
      const int found = hit ? __builtin_ctzll(hit) : 0;
      // Its place among the last pieces in group order, which is looked up below.
      const int order = wave_inclusive_sum(p - whole, lane) - (p - whole);
      at = __builtin_amdgcn_readlane(order, found);
    }
    int before = 0, slots = 0;
    for (int g0 = 0;;) {
      const int mine = of_whole ? whole : p - whole;
      const int incl = wave_inclusive_sum(mine, lane) + before;
      const int slot_incl = wave_inclusive_sum(p > 1 ? p : 0, lane) + slots;
      const unsigned long long past = __ballot(incl > at);
      if (past) {
        const int l = __builtin_ctzll(past);
        out.group = g0 + l;
        out.pieces = __builtin_amdgcn_readlane(p, l);
        out.index = at - (__builtin_amdgcn_readlane(incl, l) - __builtin_amdgcn_readlane(mine, l)) +
                    (of_whole ? 0 : __builtin_amdgcn_readlane(whole, l));
        out.slot = __builtin_amdgcn_readlane(slot_incl, l) - (out.pieces > 1 ? out.pieces : 0);
        out.lo = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(lo >> 32), l) << 32) |
                           (uint32_t)__builtin_amdgcn_readlane((int)lo, l));
        out.hi = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(hi >> 32), l) << 32) |
                           (uint32_t)__builtin_amdgcn_readlane((int)hi, l));
        return out;
      }
      before = __builtin_amdgcn_readlane(incl, 63);
      slots = __builtin_amdgcn_readlane(slot_incl, 63);
      g0 += 64;
      if (g0 >= all) return out;
      load(g0 + lane);
    }
  }
};

// ---- products over rows: the forward pass, and dx -----------------------------
// C[r][c] = act(sum_k A[r][k] B(c, k) + bias[c]) + residual[r][c], U[r][c] the
// value before act. B(c, k) = B[c * ldb + k] (B_COL: B[k * ldb + c]) of r's group.
// Large layers are bound by their MFMAs at the clock that power leaves and by the tiles'
// edges, middling ones by the edges (loads until the first chunk is there, the epilogue's
// reads and writes), small ones by the launch. bf16: 300,000 rows of 1,024 -> 2,048
// 1.28-1.33 ms (945-985 TFLOP/s; 48% of the cycles have MFMAs, at 1.88 GHz of 2.4); 60,000 of
// 1,024 -> 512 in 64 groups with residual and pre-activations 125-130 us (2.9 TB/s); its
// dx with dz in two parts 178 us (33% of the cycles have MFMAs). fp32: 4,596 of 512 -> 512
// 39 us; dx and dW of 100,003 rows of 256 -> 512 in one launch 400 us (131 TFLOP/s, 53%).
template <class C>
__device__ __forceinline__ void rows_block(const DenseLaunch& a, int block, int blocks,
                                           unsigned char* smem) {
  constexpr bool BF16 = C::ESZ == 2;
  const int lane = threadIdx.x & 63;
  const int tiles_n = (a.N + C::BN - 1) / C::BN;
  int64_t hi = a.M, m0;
  int group = 0, tile_n = 0;
  if (a.offsets) {
    const Piece p = Groups{a.offsets, a.G, a.M, C::BM, false, true}.find(lane, tile_n, block, tiles_n);
    if (p.group < 0) return;
    group = p.group;
    hi = p.hi;
    m0 = p.lo + p.index * C::BM;
  } else {
    const int tile = xcd_tile(block, blocks);
    m0 = (int64_t)(tile / tiles_n) * C::BM;
    tile_n = tile % tiles_n;
  }
  const int n0 = tile_n * C::BN;
  const int valid = (int)(hi - m0 < C::BM ? hi - m0 : C::BM);
  const unsigned char* const Ap = static_cast<const unsigned char*>(a.A) + m0 * a.lda * C::ESZ;
  const unsigned char* const Bg =
      static_cast<const unsigned char*>(a.B) + (int64_t)group * a.group_stride * C::ESZ;
  const bool orphans = a.offsets && group == a.G;  // rows of no group: zeros

  // A lane keeps its columns through the epilogue: the bias is read once, ahead.
  constexpr int V = BF16 ? 8 : 4;
  float bias[V] = {};
  const int lane_n = n0 + product_column<C, V>();
  if (a.bias && !orphans && lane_n < a.N)
    read_row<false>(a.bias + (int64_t)group * a.N, lane_n, a.N - lane_n, bias);

  TileSums<C> sums;
  const Operand A{Ap, a.lda, valid, a.a_plane};
  const Operand B{Bg + (C::B_COL ? (int64_t)n0 : n0 * a.ldb) * C::ESZ, a.ldb,
                  a.N - n0 < C::BN ? a.N - n0 : C::BN, 0, n0};
  // The residual's tile is touched, a value per 128 bytes, so that it lies in L2 when the
  // epilogue reads it (60,000 x 1,024 -> 512 bf16: 24 us on top of 73 without).
  const unsigned char* const res =
      a.residual && !orphans ? static_cast<const unsigned char*>(a.residual) : nullptr;
  constexpr int LINES = C::BN * C::ESZ / 128;
  constexpr int TOUCHES = (C::BM * LINES + C::THREADS - 1) / C::THREADS;
  uint32_t touched[TOUCHES] = {};
  if (res)
#pragma unroll
    for (int t = 0; t < TOUCHES; ++t) {
      const int i = t * C::THREADS + threadIdx.x, m = i / LINES, n = n0 + i % LINES * (128 / C::ESZ);
      if (m < valid && n < a.N)  // valid <= BM
        touched[t] = load_any<uint16_t>(res + ((m0 + m) * a.ldr + n) * C::ESZ);
    }
  tile_sums(A, B, 0, orphans ? 0 : a.K, smem, sums);
#pragma unroll
  for (int t = 0; t < TOUCHES; ++t) asm volatile("" : : "v"(touched[t]));
  struct Row {
    float v[V];
  };
  product_rows_cols<V>(
      sums, smem,
      [&](int m, int nn) __attribute__((always_inline)) {
        Row x = {};
        if (res && m < valid && n0 + nn < a.N)
          read_row<BF16>(res + (m0 + m) * a.ldr * C::ESZ, n0 + nn, a.N - n0 - nn, x.v);
        return x;
      },
      [&](int m, int nn, float (&v)[V], const Row& x) __attribute__((always_inline)) {
        const int n = n0 + nn;
        const int cols = a.N - n;
        if (m >= valid || cols <= 0) return;
        const int64_t r = m0 + m;
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += bias[e];
        if (a.U)
          write_row<BF16>(static_cast<unsigned char*>(a.U) + r * a.ldu * C::ESZ, n, cols, v);
        activate<BF16>(v, a.act);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += x.v[e];
        write_row<BF16>(static_cast<unsigned char*>(a.C) + r * a.ldc * C::ESZ, n, cols, v);
      },
      [](int, int, const float (&)[8]) {}, false);
}

template <class C>
__global__ __launch_bounds__(C::THREADS, C::WPE) void dense_rows_kernel(DenseLaunch a) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::LDS_BYTES];
  rows_block<C>(a, blockIdx.x, gridDim.x, smem);
}

// ---- the forward pass of few rows ---------------------------------------------
// What bounds it is the weight: every element is read once for at most 64 rows,
// so a block takes 16 of its rows (output columns) and its eight waves split k,
// each with its loads straight from global memory into MFMA operands, 16 rows of x
// beside them. The eight partial sums meet in LDS, in order. One row of 1,024 -> 2,048
// in bf16 6-8 us, an empty launch's 5 among them; in fp32 (8 MB of weight) 6.1 us.
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
        read_row<false>(a.bias + (int64_t)group * a.N, n, cols, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
      }
      if (a.U) write_row<BF16>(static_cast<unsigned char*>(a.U) + r * a.ldu * ESZ, n, cols, v);
      activate<BF16>(v, a.act);
      if (a.residual && !orphans) {
        float w[4];
        read_row<BF16>(static_cast<const unsigned char*>(a.residual) + r * a.ldr * ESZ, n, cols, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e];
      }
      write_row<BF16>(static_cast<unsigned char*>(a.C) + r * a.ldc * ESZ, n, cols, v);
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
// A block takes a piece of a.bias_rows rows of one group; `lanes` threads (the
// smallest power of two that covers the columns, 64 at most) lie side by side along a
// row, 16 bytes each, over (256 / lanes) rows at once, four such in flight. Bound by
// memory: it reads dy and u and writes dz once (100,003 x 512 fp32 118 us, 5.2 TB/s;
// 60,000 x 512 bf16, dz in two parts, 54 us, 4.6 TB/s).
template <bool BF16>
__global__ __launch_bounds__(256) void dense_dz_kernel(DenseGradLaunch a, int lanes) {
  constexpr int ESZ = BF16 ? 2 : 4, V = 16 / ESZ, DEEP = 4;
  __shared__ float sums[256][V];
  const int tid = threadIdx.x;
  Piece p;
  if (a.offsets) {
    int t = blockIdx.x;
    p = Groups{a.offsets, a.G, a.n, a.bias_rows, true, true}.find(tid & 63, t, 0, 0);
    if (p.group < 0) return;
  } else {
    p.group = 0;
    p.lo = 0;
    p.hi = a.n;
    p.index = blockIdx.x;
  }
  const int64_t r0 = p.lo + p.index * a.bias_rows;
  const int rows = (int)(p.hi - r0 < a.bias_rows ? p.hi - r0 : a.bias_rows);
  const int n = (blockIdx.y * lanes + tid % lanes) * V, cols = a.N - n;
  const unsigned char* const dy = static_cast<const unsigned char*>(a.dy) + r0 * a.lddy * ESZ;
  const unsigned char* const u =
      a.act != kActNone ? static_cast<const unsigned char*>(a.U) + r0 * a.ldu * ESZ : nullptr;
  unsigned char* const dz = static_cast<unsigned char*>(a.dz) + r0 * a.lddz * ESZ;
  float s[V] = {};
  // `have` is a constant where all V columns exist: no branch between the loads.
  auto walk = [&](int have) __attribute__((always_inline)) {
    const int step = 256 / lanes;
    for (int r = tid / lanes; r < rows; r += DEEP * step) {
      float d[DEEP][V], x[DEEP][V];
#pragma unroll
      for (int k = 0; k < DEEP; ++k) {
        const int64_t q = r + k * step < rows ? r + k * step : r;
        read_row<BF16>(dy + q * a.lddy * ESZ, n, have, d[k]);
        if (u) read_row<BF16>(u + q * a.ldu * ESZ, n, have, x[k]);
      }
#pragma unroll
      for (int k = 0; k < DEEP; ++k) {
        const int64_t q = r + k * step;
        if (q >= rows) break;
        if (u) grad_through<BF16>(d[k], x[k], a.act);
        if (a.dz) {
          write_row<BF16>(dz + q * a.lddz * ESZ, n, have, d[k]);
          if constexpr (BF16)
            if (a.dz_plane) {
              float lo[V];
#pragma unroll
              for (int e = 0; e < V; e += 2) {
                const uint32_t w = pack_bf16x2(d[k][e], d[k][e + 1]);
                const float h0 = __uint_as_float(w << 16), h1 = __uint_as_float(w & 0xFFFF0000u);
                lo[e] = fabsf(h0) < INFINITY ? d[k][e] - h0 : 0.0f;
                lo[e + 1] = fabsf(h1) < INFINITY ? d[k][e + 1] - h1 : 0.0f;
              }
              write_row<BF16>(dz + a.dz_plane + q * a.lddz * ESZ, n, have, lo);
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) s[e] += d[k][e];
      }
    }
  };
  if (cols >= V) walk(V);
  else if (cols > 0) walk(cols);
  if (!a.db_parts) return;
#pragma unroll
  for (int e = 0; e < V; ++e) sums[tid][e] = s[e];
  __syncthreads();
  if (tid < lanes && cols > 0) {
    for (int t = tid + lanes; t < 256; t += lanes)
#pragma unroll
      for (int e = 0; e < V; ++e) s[e] += sums[t][e];
    write_row<false>(a.db_parts + (int64_t)blockIdx.x * a.N, n, cols, s);
  }
}

// ---- dW ------------------------------------------------------------------------
// dW[g][n][k] = sum over the group's rows of dz[r][n] x[r][k]. Where the tiles of
// dW alone leave CUs idle, a group's rows are cut into pieces of a.piece rows; a
// group of several leaves fp32 partial sums in the workspace, which
// dense_join_kernel adds in order. 60,000 rows of 1,024 -> 512 bf16 in 64 uneven groups
// 94 us (670 TFLOP/s), with dz in two parts 137 us (42% of the cycles have MFMAs).
template <class C>
__device__ __forceinline__ void dw_block(const DenseGradLaunch& a, int block, int blocks,
                                         unsigned char* smem) {
  constexpr bool BF16 = C::ESZ == 2;
  const int lane = threadIdx.x & 63;
  const int tiles_k = (a.K + C::BN - 1) / C::BN, tiles = tiles_k * ((a.N + C::BM - 1) / C::BM);
  Piece p;
  int tile = 0;
  if (a.offsets) {
    p = Groups{a.offsets, a.G, a.n, a.piece, true, false, true}.find(lane, tile, block, tiles);
    if (p.group < 0) return;
  } else {
    tile = xcd_tile(block, blocks);
    p.group = 0;
    p.lo = 0;
    p.hi = a.n;
    p.index = tile / tiles;
    p.pieces = (int)((a.n + a.piece - 1) / a.piece);
    tile %= tiles;
  }
  const int n0 = tile / tiles_k * C::BM, k0 = tile % tiles_k * C::BN;
  const int64_t r0 = p.lo + p.index * a.piece;
  const int64_t rows = p.hi - r0 < a.piece ? p.hi - r0 : a.piece;
  const int vn = a.N - n0 < C::BM ? a.N - n0 : C::BM, vk = a.K - k0 < C::BN ? a.K - k0 : C::BN;
  const unsigned char* const Z =
      static_cast<const unsigned char*>(a.dz) + (r0 * a.lddz + n0) * C::ESZ;
  const unsigned char* const X =
      static_cast<const unsigned char*>(a.x) + (r0 * a.ldx + k0) * C::ESZ;
  TileSums<C> sums;
  tile_sums(Operand{Z, a.lddz, vn, a.dz_plane, n0}, Operand{X, a.ldx, vk, 0, k0}, 0, rows, smem, sums);
  // Offsets that overlap could count more pieces than the workspace holds.
  if (p.pieces > 1 && p.slot + p.index >= dense_dw_parts(a.n, a.piece, a.offsets ? a.G : 0)) return;
  float* const part = p.pieces > 1 ? a.dw_parts + (p.slot + p.index) * (int64_t)a.N * a.K : nullptr;
  unsigned char* const out =
      static_cast<unsigned char*>(a.dW) + (int64_t)p.group * a.N * a.K * C::ESZ;
  constexpr int V = BF16 ? 8 : 4;
  product_rows_cols<V>(
      sums, smem, [](int, int) { return Nothing{}; },
      [&](int m, int nn, float (&v)[V], Nothing) __attribute__((always_inline)) {
        const int cols = vk - nn;
        if (m >= vn || cols <= 0) return;
        const int64_t at = (int64_t)(n0 + m) * a.K + k0 + nn;
        if (part) write_row<false>(part, at, cols, v);
        else write_row<BF16>(out, at, cols, v);
      },
      [](int, int, const float (&)[8]) {}, false);
}

template <class C>
__global__ __launch_bounds__(C::THREADS, C::WPE) void dense_dw_kernel(DenseGradLaunch a) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::LDS_BYTES];
  dw_block<C>(a, blockIdx.x, gridDim.x, smem);
}

// dx and dW in one launch, dW's blocks first: for few rows a launch costs as much as
// either (about 5 us), for many dx's first blocks run beside dW's last. A whole backward
// pass, together and apart, us: 1,000 rows of 256 -> 256 19.4, 22.1 (bf16, no activation),
// 19.3, 22.0 (SiLU), 21.3, 31.1 (fp32); 4,596 of 512 -> 512 25.8, 28.7; 37.1, 40.5; 71.2,
// 79.2; 30,000 of 512 -> 512 77.9, 80.9; 112.8, 121.5; 284, 293; 300,000 of 256 -> 512
// fp32 1,502, 1,550. It loses nowhere by more than 2% (100,000 of 1,024 -> 512 fp32 in 32
// uneven groups 1,675, 1,645).
template <class CX, class CW>
__global__ __launch_bounds__(CX::THREADS, CX::WPE) void dense_grads_kernel(DenseLaunch x,
                                                                           DenseGradLaunch w,
                                                                           int w_blocks) {
  static_assert(CX::THREADS == CW::THREADS, "one block size");
  __shared__ __attribute__((aligned(16))) unsigned char
      smem[CX::LDS_BYTES > CW::LDS_BYTES ? CX::LDS_BYTES : CW::LDS_BYTES];
  if ((int)blockIdx.x < w_blocks) dw_block<CW>(w, blockIdx.x, w_blocks, smem);
  else rows_block<CX>(x, blockIdx.x - w_blocks, gridDim.x - w_blocks, smem);
}

// The partial sums, added in order: of dW (blocks below dw_blocks) and of db. An item
// is 256 elements of a group that has partial sums; `shares` (1, 4 or 16) of a
// block's 16 waves add its pieces, in order within each and then over the shares.
// Bound by the latency of few reads each: 33 MB of 100,003 rows of 256 -> 512 fp32 23 us.
constexpr int kJoinWaves = 16;
template <bool BF16>
__global__ __launch_bounds__(64 * kJoinWaves) void dense_join_kernel(DenseGradLaunch a,
                                                                     int dw_blocks, int dw_shares,
                                                                     int db_shares) {
  __shared__ float4 part[kJoinWaves][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const bool of_dw = (int)blockIdx.x < dw_blocks;
  const int shares = of_dw ? dw_shares : db_shares, per_block = kJoinWaves / shares;
  const int unit = of_dw ? a.piece : a.bias_rows, groups = a.offsets ? a.G : 0;
  const int64_t size = of_dw ? (int64_t)a.N * a.K : a.N;
  const uint32_t chunks = (uint32_t)((size + 255) / 256);
  const Groups gr{a.offsets, a.G, a.n, unit, true, !of_dw};
  uint32_t items = chunks;
  if (groups) {
    uint32_t several = of_dw ? 0 : groups;
    if (of_dw)
      for (int g0 = 0; g0 < groups; g0 += 64)
        several += __popcll(__ballot(g0 + lane < groups && gr.pieces(g0 + lane) > 1));
    items *= several;
  }
  const uint32_t blocks = of_dw ? dw_blocks : gridDim.x - dw_blocks;
  // Offsets that overlap could count more pieces than there are.
  const int64_t all = of_dw ? dense_dw_parts(a.n, a.piece, groups)
                            : dense_bias_pieces(a.n, groups, a.bias_rows);
  const float* const parts = of_dw ? a.dw_parts : a.db_parts;
  for (uint32_t item0 = (of_dw ? blockIdx.x : blockIdx.x - dw_blocks) * per_block; item0 < items;
       item0 += blocks * per_block) {
    const uint32_t item = item0 + w / shares;
    const int share = w % shares;
    int g = (int)(item / chunks), cols = 0;
    const int64_t at = (int64_t)(item % chunks) * 256 + lane * 4;
    float s[4] = {0, 0, 0, 0};
    if (item < items) {
      int64_t first = 0, pieces = (a.n + unit - 1) / unit;
      if (groups) {
        // The g-th group that counts, its pieces and those before it.
        int seen = 0, before = 0;
        for (int g0 = 0; g0 < groups; g0 += 64) {
          const int p = g0 + lane < groups ? gr.pieces(g0 + lane) : 0;
          const bool counts = p > (of_dw ? 1 : 0);
          const int rank = seen + wave_inclusive_sum(counts, lane);
          const int end = before + wave_inclusive_sum(counts ? p : 0, lane);
          const unsigned long long hit = __ballot(counts && rank == g + 1);
          if (hit) {
            const int l = __builtin_ctzll(hit);
            pieces = __builtin_amdgcn_readlane(p, l);
            first = __builtin_amdgcn_readlane(end, l) - pieces;
            g = g0 + l;
            break;
          }
          seen = __builtin_amdgcn_readlane(rank, 63);
          before = __builtin_amdgcn_readlane(end, 63);
        }
      }
      if (first + pieces > all) pieces = first < all ? all - first : 0;
      const int per = (int)((pieces + shares - 1) / shares);
      const int64_t q0 = (int64_t)per * share;
      const int count = (int)(q0 >= pieces ? 0 : (pieces - q0 < per ? pieces - q0 : per));
      cols = (int)(size - at < 4 ? size - at : 4);
      const float* src = parts + (first + q0) * size + at;
      auto add = [&](int have) __attribute__((always_inline)) {
#pragma unroll 16
        for (int q = 0; q < count; ++q, src += size) {
          float v[4];
          read_row<false>(src, 0, have, v);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] += v[e];
        }
      };
      if (cols >= 4) add(4);  // no branch between the loads
      else if (cols > 0) add(cols);
    }
    if (shares > 1) {
      part[w][lane] = make_float4(s[0], s[1], s[2], s[3]);
      __syncthreads();
      if (share == 0)
        for (int q = 1; q < shares; ++q) {
          const float4 v = part[w + q][lane];
          s[0] += v.x;
          s[1] += v.y;
          s[2] += v.z;
          s[3] += v.w;
        }
      __syncthreads();
    }
    if (share == 0 && cols > 0) {
      if (of_dw)
        write_row<BF16>(static_cast<unsigned char*>(a.dW) + g * size * (BF16 ? 2 : 4), at, cols, s);
      else
        write_row<false>(a.db + (int64_t)g * a.N, at, cols, s);
    }
  }
}

// ---- tile shapes -----------------------------------------------------------------
// Ring: rows of whole 16-byte vectors; else through registers, of which 256 x 256
// leaves none, nor 128 x 128 in fp32 (by 64 and by 128 x 64, the largest without scratch:
// 120,011 rows of 255 -> 257 224 us, 215, gradients 655, 724; 60,003 of 511 -> 259 217,
// 206 and 589, 570).
template <int MODE, bool A_COL, bool B_COL>
struct Tiles;
template <bool A_COL, bool B_COL>
struct Tiles<kBf16, A_COL, B_COL> {
  using RingBig = RingCfg<kBf16, 256, 256, 64, 2, 4, A_COL, B_COL, 2, 1, 1>;
  using RingMid = RingCfg<kBf16, 128, 128, 64, 2, 2, A_COL, B_COL, 2, 1, 1>;
  using RingSmall = RingCfg<kBf16, 64, 64, 64, 2, 2, A_COL, B_COL, 4>;
  using RingMany = RingCfg<kBf16, 64, 64, 64, 2, 2, A_COL, B_COL, 2>;
  using Mid = RingCfg<kBf16, 128, 128, 64, 2, 2, A_COL, B_COL, 2, 1, 0, true>;
  using Small = RingCfg<kBf16, 64, 64, 64, 2, 2, A_COL, B_COL, 2, 4, 0, true>;
};
template <bool A_COL, bool B_COL>
struct Tiles<kBf16A2, A_COL, B_COL> {
  using RingBig = RingCfg<kBf16A2, 256, 256, 32, 2, 4, A_COL, B_COL, 2, 1, 1>;
  using RingMid = RingCfg<kBf16A2, 128, 128, 32, 2, 2, A_COL, B_COL, 2, 1, 1>;
  using RingSmall = RingCfg<kBf16A2, 64, 64, 64, 2, 2, A_COL, B_COL, 3>;
  using RingMany = RingCfg<kBf16A2, 64, 64, 64, 2, 2, A_COL, B_COL, 2>;
  using Mid = RingCfg<kBf16A2, 128, 128, 32, 2, 2, A_COL, B_COL, 2, 1, 0, true>;
  using Small = RingCfg<kBf16A2, 64, 64, 64, 2, 2, A_COL, B_COL, 2, 2, 0, true>;
};
template <bool A_COL, bool B_COL>
struct Tiles<kF32, A_COL, B_COL> {
  using RingMid = RingCfg<kF32, 128, 128, 16, 2, 2, A_COL, B_COL, 4, 2>;
  using RingSmall = RingCfg<kF32, 64, 64, 16, 2, 2, A_COL, B_COL, 4>;
  using RingMany = RingSmall;
  using RingBig = RingMid;
  using Small = RingCfg<kF32, 64, 64, 32, 2, 2, A_COL, B_COL, 2, 3, 0, true>;
  using Mid = Small;
};

enum Shape { kSmall, kMid, kBig };
constexpr int side(Shape s) { return s == kSmall ? 64 : (s == kMid ? 128 : 256); }

inline int64_t tiles_of(int64_t m, int64_t n, int b) { return ((m + b - 1) / b) * ((n + b - 1) / b); }

// The larger the tile, the fewer bytes a product passes through LDS; the smaller, the
// sooner the chip is full. Each limit with the forward's time on both sides, in us:
//   bf16 64, 128:  576 tiles of 64: 7.9, 10.5 (512 -> 512); 1,024 tiles: 10.9, 10.9;
//     through registers 752 tiles: 9.8, 12.2 (300 -> 500).
//   bf16 128, 256: 128 tiles of 256: 16.4, 21.5; 256 tiles: 29.1, 25.1 (512 -> 512),
//     44.6, 38.5 (1,024 -> 2,048). Up to 128 columns half of a 256-wide tile is empty:
//     26.9, 39.0 (65,536 rows of 1,024 -> 128).
//   bf16 groups, forward and dx of 60,000 rows by 128, 256: 48 uneven groups (1,250 rows
//     on average) 88, 75 (1,024 -> 512), 113, 94 (512 -> 1,024), with residual and
//     pre-activations 124, 102 and 177, 158; 64 (937 rows) 88, 99 and 116, 111; 126, 135
//     and 184, 179; dx 110, 103 and 86, 94, through SiLU 213, 206 and 255, 254.
//   dx, bf16, 64, 128: 576 tiles of 64: 10.3, 11.1, through SiLU 20.8, 23.0 (dz with it);
//     1,024 tiles: 11.1, 11.7 and 30.2, 28.7. 128, 256: 128 tiles of 256: 16.5, 21.0 and
//     40.1, 47.3; 256 tiles: 31.1, 24.4 and 67.2, 61.4 (all 512 -> 512).
//   fp32 64, 128:  188 tiles of 128: 22.1, 23.7 (256 -> 256); 256 tiles: 27.1, 25.4, 46.0,
//     40.6 (512 -> 512); dx with dz, 144 tiles: 44.7, 49.7, 256 tiles: 57.0, 55.0.
inline Shape rows_shape(const DenseLaunch& a, bool bf16) {
  const int64_t m = a.M, n = a.N;
  if (!bf16) return tiles_of(m, n, 128) < 256 ? kSmall : kMid;
  if (tiles_of(m, n, 64) <= 768) return kSmall;
  if (n <= 128 || (a.offsets && m < 1024 * (int64_t)a.G)) return kMid;
  return tiles_of(m, n, 256) < 256 ? kMid : kBig;
}

// Tiles of 64 in bf16 have four stages of 16 KB, which two blocks a CU hold; where
// there are more blocks than that, two stages, so that they run together: 576 tiles of
// depth 512 8.5 us with two, 11.4 with four; 256 tiles of depth 2,048 18.5 and 11.4. With A
// in two parts three stages of 24 KB or two: 576 tiles of depth 256 (dx and dW in one
// launch, dz) 28.5 with two, 30.2 with three; 128 of depth 2,048 28.2 and 23.0.
inline bool many(int64_t blocks) { return blocks > 512; }

inline bool vectors(const void* p, int64_t ld, int64_t width, bool bf16) {
  const int64_t ve = bf16 ? 8 : 4;
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % ve == 0 && width % ve == 0;
}

template <class C>
int64_t rows_blocks(const DenseLaunch& a) {
  const int64_t tiles_n = (a.N + C::BN - 1) / C::BN;
  return ((a.M + C::BM - 1) / C::BM + (a.offsets ? a.G + 1 : 0)) * tiles_n;
}
template <class C>
int64_t dw_blocks(const DenseGradLaunch& a) {
  int64_t pieces = (a.n + a.piece - 1) / a.piece;
  if (a.offsets) pieces = (pieces + a.G + 7) / 8 * 8;  // as Groups::find hands them out
  return (pieces > 0 ? pieces : 1) * tiles_of(a.N, a.K, C::BM);
}

template <class C>
hipError_t rows_cfg(const DenseLaunch& a, hipStream_t s) {
  const int64_t blocks = rows_blocks<C>(a);
  if (blocks > 0x7FFFFFFFll) return hipErrorInvalidValue;
  hipLaunchKernelGGL(dense_rows_kernel<C>, dim3((unsigned)blocks), dim3(C::THREADS), 0, s, a);
  return hipGetLastError();
}
template <class C>
hipError_t dw_cfg(const DenseGradLaunch& a, hipStream_t s) {
  const int64_t blocks = dw_blocks<C>(a);
  if (blocks > 0x7FFFFFFFll) return hipErrorInvalidValue;
  hipLaunchKernelGGL(dense_dw_kernel<C>, dim3((unsigned)blocks), dim3(C::THREADS), 0, s, a);
  return hipGetLastError();
}
template <class CX, class CW>
bool grads_cfg(const DenseLaunch& x, const DenseGradLaunch& w, hipStream_t s, hipError_t* e) {
  const int64_t bw = dw_blocks<CW>(w), bx = rows_blocks<CX>(x);
  if (bw + bx > 0x7FFFFFFFll) return false;
  ProfileScope prof(kKDenseGrad, s);
  hipLaunchKernelGGL((dense_grads_kernel<CX, CW>), dim3((unsigned)(bw + bx)), dim3(CX::THREADS), 0, s,
                     x, w, (int)bw);
  *e = hipGetLastError();
  return true;
}

template <bool B_COL>
bool rows_vectors(const DenseLaunch& a) {
  return vectors(a.A, a.lda, a.K, a.bf16) && vectors(a.B, a.ldb, B_COL ? a.N : a.K, a.bf16);
}
bool dw_vectors(const DenseGradLaunch& a) {
  return vectors(a.dz, a.lddz, a.N, a.bf16) && vectors(a.x, a.ldx, a.K, a.bf16);
}

template <int MODE, bool B_COL>
hipError_t rows_mode(const DenseLaunch& a, hipStream_t s) {
  using T = Tiles<MODE, false, B_COL>;
  const bool ring = rows_vectors<B_COL>(a);
  const Shape shape = rows_shape(a, MODE != kF32);
  if (ring) {
    if (shape == kSmall)
      return many(rows_blocks<typename T::RingSmall>(a)) ? rows_cfg<typename T::RingMany>(a, s)
                                                         : rows_cfg<typename T::RingSmall>(a, s);
    if (shape == kMid) return rows_cfg<typename T::RingMid>(a, s);
    return rows_cfg<typename T::RingBig>(a, s);
  }
  return shape == kSmall ? rows_cfg<typename T::Small>(a, s) : rows_cfg<typename T::Mid>(a, s);
}

// Tiles of dW. 256 x 256 (bf16) where there are 8 of them or more and one round of
// blocks takes 1,536 rows each or more: with fewer of either, the partial sums cost
// what the tile gains. Times of dW and the sums' join in us, by 128 and by 256, and the
// same with dz through SiLU: 300,000 rows of 1,024 -> 512 364, 289 and 807, 753; 60,000
// 81, 82 and 181, 176, in 64 groups 97, 81 and 205, 175, in uneven ones 107, 99 and 212,
// 190; 4,096 of 2,048 -> 2,048 (1,024 rows a block) 54, 57 and 95, 96; 100,000 of
// 256 -> 512 (2 tiles) 47, 53 and 157, 163. 128 x 128 where pieces of 512 rows fill the
// chip; by 64 and by 128: 60,000 of 1,024 -> 512 135, 81 and, fp32 with dz, 712, 506;
// 20,000 of 256 -> 256 19, 23, through SiLU 30, 33, fp32 52, 54.
inline Shape dw_shape(int64_t n, int N, int K, int G, bool bf16) {
  const int64_t tiles = tiles_of(N, K, 256);
  if (bf16 && tiles >= 8 && n >= 512 * (int64_t)G && n * tiles >= 1536 * 256 && N > 128 && K > 128)
    return kBig;
  return tiles_of(N, K, 128) * (n / 512) >= 256 && N > 64 && K > 64 ? kMid : kSmall;
}

template <int MODE>
hipError_t dw_mode(const DenseGradLaunch& a, hipStream_t s) {
  using T = Tiles<MODE, true, true>;
  const Shape shape = dw_shape(a.n, a.N, a.K, a.G, MODE != kF32);
  if (dw_vectors(a)) {
    if (shape == kSmall)
      return many(dw_blocks<typename T::RingSmall>(a)) ? dw_cfg<typename T::RingMany>(a, s)
                                                       : dw_cfg<typename T::RingSmall>(a, s);
    if (shape == kMid) return dw_cfg<typename T::RingMid>(a, s);
    return dw_cfg<typename T::RingBig>(a, s);
  }
  return shape == kSmall ? dw_cfg<typename T::Small>(a, s) : dw_cfg<typename T::Mid>(a, s);
}

// Both in one launch where both take ring tiles of four waves; false: apart.
template <int MODE>
bool grads_mode(const DenseLaunch& x, const DenseGradLaunch& w, hipStream_t s, hipError_t* e) {
  using X = Tiles<MODE, false, true>;
  using W = Tiles<MODE, true, true>;
  if (!rows_vectors<true>(x) || !dw_vectors(w)) return false;
  const Shape sx = rows_shape(x, MODE != kF32), sw = dw_shape(w.n, w.N, w.K, w.G, MODE != kF32);
  if (sx == kBig || sw == kBig) return false;
  if (sx == kSmall && sw == kSmall) {
    if (many(rows_blocks<typename X::RingSmall>(x) + dw_blocks<typename W::RingSmall>(w)))
      return grads_cfg<typename X::RingMany, typename W::RingMany>(x, w, s, e);
    return grads_cfg<typename X::RingSmall, typename W::RingSmall>(x, w, s, e);
  }
  if (sx == kSmall) return grads_cfg<typename X::RingSmall, typename W::RingMid>(x, w, s, e);
  if (sw == kSmall) return grads_cfg<typename X::RingMid, typename W::RingSmall>(x, w, s, e);
  return grads_cfg<typename X::RingMid, typename W::RingMid>(x, w, s, e);
}

// Few rows: the weight goes through registers once, without LDS tiles. Times in us, by
// this kernel and by tiles of 64. fp32, whose tiles split each weight first: up to 128
// rows (512 -> 512 16 rows 6.3, 15.8, 128 rows 12.3, 16.2, 192 rows 17.6, 16.3), or 16
// a group on average (64 groups, 1,024 rows 20.4, 25.9, 2,048 rows 32.7, 26.1). bf16:
// up to 32 rows (2,048 -> 4,096 8 rows 6.1, 9.7, 64 rows 11.6, 9.9), or 16 a group
// in one round of blocks (8 groups, 1,024 -> 1,024, 128 rows 6.5, 7.1; 16 groups,
// 2,048 -> 1,024, two rounds, 16.4, 12.5). A group that has most of the rows takes
// them 64 at a time, hence the limits on the sum.
bool few_rows_wanted(const DenseLaunch& a) {
  if (a.b_col) return false;
  if (!a.offsets) return a.M <= (a.bf16 ? 32 : 128);
  const int64_t blocks = (a.N + 15) / 16 * (a.G + 1), per_group = 16 * (int64_t)a.G;
  return a.bf16 ? blocks <= 1024 && a.M <= std::min<int64_t>(per_group, 256)
                : a.M <= std::min<int64_t>(per_group, 1024);
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
  if (!a.b_col) return a.bf16 ? rows_mode<kBf16, false>(a, s) : rows_mode<kF32, false>(a, s);
  if (!a.bf16) return rows_mode<kF32, true>(a, s);
  return a.a_plane ? rows_mode<kBf16A2, true>(a, s) : rows_mode<kBf16, true>(a, s);
}

// Rows per piece of dW's sums: pieces that give every CU one round of blocks (one
// block of 256 x 256, two of the others), of 256 rows at least. More and smaller ones
// even out uneven groups but cost partial sums: whole, half and a quarter as long, us:
// 200,000 rows of 512 -> 512 bf16 in 32 uneven groups through SiLU 384, 400, 426; 60,000
// of 512 -> 256 fp32 in 64 183, 186, 217.
int64_t dense_dw_piece(int64_t n, int N, int K, int G, bool bf16) {
  const Shape shape = dw_shape(n, N, K, G, bf16);
  const int64_t tiles = tiles_of(N, K, side(shape));
  const int64_t want = ((shape == kBig ? 256 : 512) + tiles - 1) / tiles;
  const int64_t rows = ((n + want - 1) / want + 63) / 64 * 64;
  return rows < 256 ? 256 : rows;
}

hipError_t launch_dense_dz(const DenseGradLaunch& a, hipStream_t s) {
  const int64_t pieces = dense_bias_pieces(a.n, a.offsets ? a.G : 0, a.bias_rows);
  if (pieces <= 0) return hipSuccess;
  ProfileScope prof(kKDenseGrad, s);
  const int v = a.bf16 ? 8 : 4;
  int lanes = 1;
  while (lanes < 64 && lanes * v < a.N) lanes *= 2;
  const dim3 grid((unsigned)pieces, (unsigned)((a.N + v * lanes - 1) / (v * lanes)));
  if (a.bf16) hipLaunchKernelGGL(dense_dz_kernel<true>, grid, dim3(256), 0, s, a, lanes);
  else hipLaunchKernelGGL(dense_dz_kernel<false>, grid, dim3(256), 0, s, a, lanes);
  return hipGetLastError();
}

hipError_t launch_dense_dw(const DenseGradLaunch& a, hipStream_t s) {
  ProfileScope prof(kKDenseGrad, s);
  if (!a.bf16) return dw_mode<kF32>(a, s);
  return a.dz_plane ? dw_mode<kBf16A2>(a, s) : dw_mode<kBf16>(a, s);
}

hipError_t launch_dense_dx_dw(const DenseLaunch& x, const DenseGradLaunch& w, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (!w.bf16 ? grads_mode<kF32>(x, w, s, &e)
              : (w.dz_plane ? grads_mode<kBf16A2>(x, w, s, &e) : grads_mode<kBf16>(x, w, s, &e)))
    return e;
  e = launch_dense_rows(x, s);
  return e != hipSuccess ? e : launch_dense_dw(w, s);
}

hipError_t launch_dense_join(const DenseGradLaunch& a, hipStream_t s) {
  const int64_t groups = a.offsets ? a.G : 1;
  // Waves per item for a group's usual count of pieces: each then adds about eight.
  auto shares = [&](int64_t unit) {
    const int64_t pieces = a.n / groups / unit;
    return pieces > 32 ? 16 : (pieces > 8 ? 4 : 1);
  };
  const int dw_shares = shares(a.piece), db_shares = shares(a.bias_rows);
  // Groups of more than one piece at most, and two blocks per CU.
  const int64_t several = std::min(groups, a.n / (a.piece + 1));
  auto blocks = [](int64_t size, int64_t count, int share) {
    const int64_t items = (size + 255) / 256 * count, per_block = kJoinWaves / share;
    return std::min<int64_t>((items + per_block - 1) / per_block, 512);
  };
  const int64_t dw = a.dW && a.dw_parts ? blocks((int64_t)a.N * a.K, several, dw_shares) : 0;
  const int64_t db = a.db ? blocks(a.N, groups, db_shares) : 0;
  if (dw + db == 0) return hipSuccess;
  ProfileScope prof(kKDenseGrad, s);
  const dim3 grid((unsigned)(dw + db)), block(64 * kJoinWaves);
  if (a.bf16)
    hipLaunchKernelGGL(dense_join_kernel<true>, grid, block, 0, s, a, (int)dw, dw_shares, db_shares);
  else
    hipLaunchKernelGGL(dense_join_kernel<false>, grid, block, 0, s, a, (int)dw, dw_shares, db_shares);
  return hipGetLastError();
}

}  // namespace pinsage
