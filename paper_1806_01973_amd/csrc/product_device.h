// One output tile of C[m][n] = sum_k A(m, k) B(n, k) on the matrix cores, for
// operands of any alignment, size and orientation: the products of the dense
// layers' forward and backward passes and of the Newton-Schulz iteration.
//
// An operand is "row" (k contiguous: A[m * ld + k]) or "column" (m contiguous:
// A[k * ld + m]). Chunks of BK columns of k go global -> registers -> LDS ->
// MFMA: half of the block's waves carry A, half B, eight 16-byte loads per
// thread and chunk, issued one chunk ahead. The registers let one layout in LDS
// serve every operand: k-contiguous rows of BK 16-bit values in 16-byte slots,
// slot v of row r at v ^ swizzle(r), which spreads the 32 rows of a fragment
// read, and the 4 or 8 rows a transposing store writes, over distinct banks.
// A column operand is transposed on the way: a thread loads 8 k by 4 (fp32) or
// 8 (16-bit) m and stores whole slots.
//
// Modes:
//   kBf16   bf16 in memory, one MFMA per product
//   kF16    fp16 in memory, the same
//   kF16x2  two fp16 parts in memory (x = hi + lo, planes apart by `plane`
//           bytes): 22 significand bits, three MFMAs (hi lo, lo hi, hi hi); for
//           operands the caller keeps inside fp16's range
//   kF32    fp32 in memory, split on the way to LDS into three bf16 parts (24
//           significand bits), six MFMAs: all products of parts down to 2^-17 of
//           the leading one. Left out is at most 2^-25 of a product, as fp32's own
//           rounding. Infinities and NaN, and values that round to a bf16
//           infinity, make an element that is not finite; the caller takes such
//           elements from redo_not_finite.
// Sums run in fp32, chunks in order, so an element's bits follow from its row,
// its column and the k range alone, whatever tile it lies in.
#pragma once

#include "device_util.h"
#include "split_device.h"

namespace pinsage {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

enum ProductMode { kBf16 = 0, kF16 = 1, kF16x2 = 2, kF32 = 3 };

// A tile's operand: `p` at the tile's first row (row operand, k = 0) or first
// column (column operand, k = 0); `valid` rows exist from there (at least 1).
struct Operand {
  const void* p;
  int64_t ld;     // elements
  int valid;
  int64_t plane;  // kF16x2: bytes from the hi plane to the lo plane
};

template <int MODE_, int BM_, int BN_, int BK_, int WAVES_M_, int WAVES_N_, bool A_COL_,
          bool B_COL_, int NBUF_, int WPE_ = 1>
struct ProductCfg {
  static constexpr int MODE = MODE_, BM = BM_, BN = BN_, BK = BK_;
  static constexpr int WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, NBUF = NBUF_, WPE = WPE_;
  static constexpr bool A_COL = A_COL_, B_COL = B_COL_;
  static constexpr int NWAVES = WAVES_M * WAVES_N, THREADS = 64 * NWAVES;
  static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 32, TN = WN / 32;
  static constexpr int ESZ = MODE == kF32 ? 4 : 2;             // bytes in memory
  static constexpr int MEM_PLANES = MODE == kF16x2 ? 2 : 1;
  static constexpr int PLANES = MODE == kF32 ? 3 : MEM_PLANES;  // in LDS
  static constexpr int ROW_BYTES = BK * 2;
  static constexpr int A_PLANE = BM * ROW_BYTES, B_PLANE = BN * ROW_BYTES;
  static constexpr int BUF_BYTES = (A_PLANE + B_PLANE) * PLANES;
  // Epilogue: a wave's 32 rows of WN fp32 columns, padded by four.
  static constexpr int STAGE_LD = WN + 4;
  static constexpr int STAGE_BYTES = 32 * STAGE_LD * 4;
  static constexpr int RING = NBUF * BUF_BYTES;
  static constexpr int LDS_BYTES =
      RING > NWAVES * STAGE_BYTES ? RING : NWAVES * STAGE_BYTES;
  static constexpr int VE = 16 / ESZ;               // elements of a 16-byte vector
  static constexpr int LOADERS = THREADS / 2;       // threads per operand
  static constexpr int VECS = BM * BK * ESZ * MEM_PLANES / 16 / LOADERS;
  static_assert(BM == BN, "both operands have the same share of the block's threads");
  static_assert(WM % 32 == 0 && WN % 32 == 0 && (NWAVES % 2) == 0, "");
  static_assert(VECS == 8, "eight vectors per thread and chunk");
  static_assert(BK == 32 || BK == 64 || BK == 128, "");
};

// Block b of nt to a tile: the hardware hands block b to XCD b % 8, this gives each
// XCD a contiguous run of tiles, whose operands its L2 then shares.
__device__ __forceinline__ int xcd_tile(int b, int nt) {
  const int per = nt / 8, rem = nt % 8;
  const int xcd = b % 8, slot = b / 8;
  return xcd < rem ? xcd * (per + 1) + slot : rem * (per + 1) + (xcd - rem) * per + slot;
}

// Reads of any alignment: one wide load each on gfx950.
template <typename T>
__device__ __forceinline__ T load_any(const void* p) {
  T v;
  __builtin_memcpy(&v, p, sizeof(T));
  return v;
}
template <typename T>
__device__ __forceinline__ void store_any(void* p, const T& v) {
  __builtin_memcpy(p, &v, sizeof(T));
}

// N (4 or 8) elements of a row from column n on, `cols` of which exist; any alignment.
template <bool BF16, int N>
__device__ __forceinline__ void read_row(const void* row, int64_t n, int cols, float (&v)[N]) {
  if constexpr (BF16) {
    const uint16_t* const p = static_cast<const uint16_t*>(row) + n;
    if (cols >= N) {
      typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
      const words w = load_any<words>(p);
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        v[2 * e] = __uint_as_float(w[e] << 16);
        v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = e < cols ? bf16_to_f32(p[e]) : 0.0f;
    }
  } else {
    const float* const p = static_cast<const float*>(row) + n;
    if (cols >= N) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q) {
        const float4 w = load_any<float4>(p + 4 * q);
        v[4 * q] = w.x;
        v[4 * q + 1] = w.y;
        v[4 * q + 2] = w.z;
        v[4 * q + 3] = w.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = e < cols ? p[e] : 0.0f;
    }
  }
}

template <bool BF16, int N>
__device__ __forceinline__ void write_row(void* row, int64_t n, int cols, const float (&v)[N]) {
  if constexpr (BF16) {
    uint16_t* const p = static_cast<uint16_t*>(row) + n;
    typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
    words w;
#pragma unroll
    for (int e = 0; e < N / 2; ++e) w[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
    if (cols >= N) {
      store_any(p, w);
    } else {
#pragma unroll
      for (int e = 0; e < N - 1; ++e)
        if (e < cols) p[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    }
  } else {
    float* const p = static_cast<float*>(row) + n;
    if (cols >= N) {
#pragma unroll
      for (int q = 0; q < N / 4; ++q)
        store_any(p + 4 * q, make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]));
    } else {
#pragma unroll
      for (int e = 0; e < N - 1; ++e)
        if (e < cols) p[e] = v[e];
    }
  }
}

template <int BK>
__device__ __forceinline__ int product_swizzle(int row) {
  return BK == 32 ? ((row >> 1) ^ (row >> 3)) & 3 : (row ^ (row >> 3)) & 7;
}

template <int MODE>
__device__ __forceinline__ f32x16 product_mfma(const u32x4& b, const u32x4& a, const f32x16& c) {
  if constexpr (MODE == kF16 || MODE == kF16x2)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, b),
                                                  __builtin_bit_cast(f16x8, a), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, b),
                                                   __builtin_bit_cast(bf16x8, a), c, 0, 0, 0);
}

// The first `count` elements (at least 1, fewer than a vector's) at p, zeros after.
template <int ESZ>
__device__ __forceinline__ u32x4 load_part(const unsigned char* p, int count) {
  u32x4 v = {0, 0, 0, 0};
  if constexpr (ESZ == 4) {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < count) v[e] = load_any<uint32_t>(p + 4 * e);
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < count) v[e >> 1] |= (uint32_t)load_any<uint16_t>(p + 2 * e) << (16 * (e & 1));
  }
  return v;
}

// A wave's blocks of 32 x 32 sums: block i, j has its rows from
// row0 + 32 i and its columns from col0 + 32 j of the tile, of which a lane holds
// row lane % 32 and columns 8 (e / 4) + 4 (lane / 32) + e % 4.
template <class C>
struct TileSums {
  f32x16 v[C::TM][C::TN];
  int row0, col0;
};

__device__ __forceinline__ void clear_block(f32x16& v) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = 0.0f;
}

// The tile's products over k in [k0, k1). All of the block's threads call it; smem
// holds C::LDS_BYTES and is free again when it returns (after a barrier).
template <class C>
__device__ __forceinline__ void product_tile(const Operand& A, const Operand& B, int64_t k0,
                                             int64_t k1, unsigned char* smem, TileSums<C>& sums) {
  auto& acc = sums.v;
#pragma unroll
  for (int i = 0; i < C::TM; ++i)
#pragma unroll
    for (int j = 0; j < C::TN; ++j) clear_block(acc[i][j]);
  constexpr int BK = C::BK, ESZ = C::ESZ, VE = C::VE, T = C::LOADERS, PL = C::PLANES;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
  sums.row0 = wm * C::WM;
  sums.col0 = wn * C::WN;
  const bool is_a = wave < C::NWAVES / 2;
  const int t = is_a ? tid : tid - T;
  const unsigned char* const src = static_cast<const unsigned char*>(is_a ? A.p : B.p);
  const int64_t ld_bytes = (is_a ? A.ld : B.ld) * ESZ;
  const uint32_t ld32 = (uint32_t)ld_bytes;  // the host keeps 256 ld below 2^31 bytes
  const int valid = is_a ? A.valid : B.valid;
  const int64_t plane = is_a ? A.plane : B.plane;
  const int nchunks = (int)((k1 - k0 + BK - 1) / BK);
  if (nchunks <= 0) return;

  // Row operand: thread t takes slot t % (BK / 8) of rows t / (BK / 8) + i * (T BK / 8 ...).
  constexpr int SLOTS = BK / 8;
  constexpr int ROW_UNITS = C::VECS / (ESZ / 2);        // slots per thread, both planes
  constexpr int ROWS_STEP = T / SLOTS;
  // Column operand: thread t takes k rows 8 kb .. 8 kb + 7, columns VE mb .. .
  constexpr int MBLOCKS = C::BM / VE;
  const int row_t = t / SLOTS, slot_t = t % SLOTS;
  const int mb = t % MBLOCKS, kb = t / MBLOCKS % SLOTS, col_plane = t / MBLOCKS / SLOTS;

  u32x4 v[8];
  auto load_row = [&](int c) __attribute__((always_inline)) {
    const int64_t kc = k0 + (int64_t)c * BK;
    const unsigned char* const base = src + kc * ESZ;
    const int left = (int)(k1 - kc < BK ? k1 - kc : BK) - slot_t * 8;
    const bool full = k1 - kc >= BK;
#pragma unroll
    for (int i = 0; i < ROW_UNITS; ++i) {
      constexpr int PER_PLANE = ROW_UNITS / C::MEM_PLANES;
      int r = row_t + (i % PER_PLANE) * ROWS_STEP;
      r = r < valid ? r : valid - 1;
      const unsigned char* const from = base + (i >= PER_PLANE ? plane : 0);
      const uint32_t off = (uint32_t)r * ld32 + (uint32_t)(slot_t * 8 * ESZ);
#pragma unroll
      for (int h = 0; h < ESZ / 2; ++h) {
        u32x4& x = v[i * (ESZ / 2) + h];
        if (full) {
          x = load_any<u32x4>(from + (off + 16u * h));
        } else {
          x = u32x4{0, 0, 0, 0};
          const int have = left - h * VE;
          if (have >= VE) x = load_any<u32x4>(from + (off + 16u * h));
          else if (have > 0) x = load_part<ESZ>(from + (off + 16u * h), have);
        }
      }
    }
  };
  auto load_col = [&](int c) __attribute__((always_inline)) {
    const int64_t kc = k0 + (int64_t)c * BK;
    const unsigned char* const base = src + kc * ld_bytes + (C::MEM_PLANES > 1 && col_plane ? plane : 0);
    const int have = valid - mb * VE;
    const int left = (int)(k1 - kc < BK ? k1 - kc : BK) - kb * 8;
    const bool full = k1 - kc >= BK && valid >= C::BM;
    const uint32_t off = (uint32_t)(kb * 8) * ld32 + (uint32_t)(mb * 16);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (full) {
        v[j] = load_any<u32x4>(base + (off + j * ld32));
      } else {
        v[j] = u32x4{0, 0, 0, 0};
        if (j < left && have > 0)
          v[j] = have >= VE ? load_any<u32x4>(base + (off + j * ld32))
                            : load_part<ESZ>(base + (off + j * ld32), have);
      }
    }
  };
  auto load = [&](int c) __attribute__((always_inline)) {
    if (is_a) {
      if constexpr (C::A_COL) load_col(c);
      else load_row(c);
    } else {
      if constexpr (C::B_COL) load_col(c);
      else load_row(c);
    }
  };

  // Slot `slot` of row r of a plane.
  auto at = [](int r, int slot) __attribute__((always_inline)) {
    return r * C::ROW_BYTES + ((slot ^ product_swizzle<BK>(r)) * 16);
  };
  auto put = [&](unsigned char* to, int plane_bytes, int r, int slot, const u32x4& lo,
                 const u32x4& hi) __attribute__((always_inline)) {
    if constexpr (C::MODE == kF32) {
      uint32_t key = 0;
      const Split3 s = split3(lo, hi, key);
#pragma unroll
      for (int q = 0; q < 3; ++q)
        *reinterpret_cast<u32x4*>(to + q * plane_bytes + at(r, slot)) = s.p[q];
    } else {
      *reinterpret_cast<u32x4*>(to + at(r, slot)) = lo;
    }
  };
  auto store_row = [&](unsigned char* to, int plane_bytes) __attribute__((always_inline)) {
    constexpr int PER_PLANE = ROW_UNITS / C::MEM_PLANES;
#pragma unroll
    for (int i = 0; i < ROW_UNITS; ++i) {
      unsigned char* const q = to + (i >= PER_PLANE ? plane_bytes : 0);
      const int r = row_t + (i % PER_PLANE) * ROWS_STEP;
      if constexpr (ESZ == 4) put(q, plane_bytes, r, slot_t, v[2 * i], v[2 * i + 1]);
      else put(q, plane_bytes, r, slot_t, v[i], v[i]);
    }
  };
  auto store_col = [&](unsigned char* to, int plane_bytes) __attribute__((always_inline)) {
    if constexpr (ESZ == 4) {
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const u32x4 lo = {v[0][m], v[1][m], v[2][m], v[3][m]};
        const u32x4 hi = {v[4][m], v[5][m], v[6][m], v[7][m]};
        put(to, plane_bytes, mb * 4 + m, kb, lo, hi);
      }
    } else {
      unsigned char* const q = to + (C::MEM_PLANES > 1 ? col_plane * plane_bytes : 0);
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        u32x4 w;
#pragma unroll
        for (int d = 0; d < 4; ++d)
          w[d] = __builtin_amdgcn_perm(v[2 * d + 1][m >> 1], v[2 * d][m >> 1],
                                       (m & 1) ? 0x07060302u : 0x05040100u);
        put(q, plane_bytes, mb * 8 + m, kb, w, w);
      }
    }
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
    unsigned char* const b0 = smem + buf * C::BUF_BYTES;
    if (is_a) {
      if constexpr (C::A_COL) store_col(b0, C::A_PLANE);
      else store_row(b0, C::A_PLANE);
    } else {
      if constexpr (C::B_COL) store_col(b0 + PL * C::A_PLANE, C::B_PLANE);
      else store_row(b0 + PL * C::A_PLANE, C::B_PLANE);
    }
  };

  const int frag_row = lane & 31, half = lane >> 5;
  auto compute = [&](int buf) __attribute__((always_inline)) {
    const unsigned char* const a0 = smem + buf * C::BUF_BYTES;
    const unsigned char* const b0 = a0 + PL * C::A_PLANE;
#pragma unroll
    for (int ks = 0; ks < BK / 16; ++ks) {
      u32x4 fa[C::TM][PL], fb[C::TN][PL];
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int p = 0; p < PL; ++p)
          fa[i][p] = *reinterpret_cast<const u32x4*>(
              a0 + p * C::A_PLANE + at(wm * C::WM + 32 * i + frag_row, 2 * ks + half));
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
#pragma unroll
        for (int p = 0; p < PL; ++p)
          fb[j][p] = *reinterpret_cast<const u32x4*>(
              b0 + p * C::B_PLANE + at(wn * C::WN + 32 * j + frag_row, 2 * ks + half));
      constexpr int PRODUCTS = PL * (PL + 1) / 2;  // parts (pb, pa) with pb + pa < PL
#pragma unroll
      for (int q = 0; q < PRODUCTS; ++q) {
        // Smallest first: (2,0) (0,2) (1,1) (1,0) (0,1) (0,0).
        constexpr int kB3[6] = {2, 0, 1, 1, 0, 0}, kA3[6] = {0, 2, 1, 0, 1, 0};
        const int pb = kB3[6 - PRODUCTS + q], pa = kA3[6 - PRODUCTS + q];
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
          for (int j = 0; j < C::TN; ++j)
            acc[i][j] = product_mfma<C::MODE>(fb[j][pb], fa[i][pa], acc[i][j]);
      }
    }
  };

  load(0);
  if constexpr (C::NBUF == 2) {
    store(0);
    if (nchunks > 1) load(1);
    __syncthreads();
    for (int c = 0; c < nchunks; ++c) {
      compute(c & 1);
      if (c + 1 < nchunks) {
        store((c + 1) & 1);
        if (c + 2 < nchunks) load(c + 2);
      }
      __syncthreads();
    }
  } else {
    for (int c = 0; c < nchunks; ++c) {
      store(0);
      if (c + 1 < nchunks) load(c + 1);
      __syncthreads();
      compute(0);
      __syncthreads();
    }
  }
}

// The column within the tile from which this lane gets its V values of every row.
template <class C, int V>
__device__ __forceinline__ int product_column() {
  const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
  return wave % C::WAVES_N * C::WN + lane % (C::WN / V) * V;
}

// Hands the tile out in whole rows, V columns a lane, a wave's lanes side by side
// along them: f(m, n, v, x) with the tile's row m, columns n .. n + V - 1 and
// x = fetch(m, n), called for a band of 32 rows ahead of it (what the epilogue
// reads is then in flight together); then, when `turned`, by columns: g(m, n, v)
// with rows m .. m + 7 of column n, of the values that f left in v. A wave's bands
// pass through LDS of its own.
template <int V, class C, class P, class F, class G>
__device__ __forceinline__ void product_rows_cols(const TileSums<C>& sums, unsigned char* smem,
                                                  P fetch, F f, G g, bool turned) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  float* const stage = reinterpret_cast<float*>(smem + wave * C::STAGE_BYTES);
  constexpr int WIDTH = C::WN, LANES = WIDTH / V;      // lanes per row
  constexpr int ROWS = 64 / LANES, PASSES = 32 / ROWS;  // rows at once
  const int r_lane = lane / LANES, col = lane % LANES * V;
#pragma unroll
  for (int i = 0; i < C::TM; ++i) {
    const int m0 = sums.row0 + 32 * i;
    decltype(fetch(0, 0)) ahead[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) ahead[p] = fetch(m0 + ROWS * p + r_lane, sums.col0 + col);
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(stage + (lane & 31) * C::STAGE_LD + 32 * j + 8 * q +
                                   4 * (lane >> 5)) =
            make_float4(sums.v[i][j][4 * q], sums.v[i][j][4 * q + 1], sums.v[i][j][4 * q + 2],
                        sums.v[i][j][4 * q + 3]);
    wave_lds_sync();
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      float* const at = stage + (ROWS * p + r_lane) * C::STAGE_LD + col;
      float v[V];
#pragma unroll
      for (int q = 0; q < V; q += 4) {
        const float4 x = *reinterpret_cast<const float4*>(at + q);
        v[q] = x.x;
        v[q + 1] = x.y;
        v[q + 2] = x.z;
        v[q + 3] = x.w;
      }
      f(m0 + ROWS * p + r_lane, sums.col0 + col, v, ahead[p]);
      if (turned)
#pragma unroll
        for (int q = 0; q < V; q += 4)
          *reinterpret_cast<float4*>(at + q) = make_float4(v[q], v[q + 1], v[q + 2], v[q + 3]);
    }
    wave_lds_sync();
    if (turned) {
      constexpr int COLS = WIDTH < 64 ? WIDTH : 64;  // columns at once, 64 / COLS row groups
#pragma unroll
      for (int c0 = 0; c0 < WIDTH; c0 += 64)
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += 8 * (64 / COLS)) {
          const int n = c0 + lane % COLS, r = r0 + 8 * (lane / COLS);
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = stage[(r + e) * C::STAGE_LD + n];
          g(m0 + r, sums.col0 + n, v);
        }
      wave_lds_sync();
    }
  }
}

struct Nothing {};

// Of four elements of a row, `cols` of which exist, those that a split product left
// without a finite value, again as fp32 dot products over `count` columns of k (a:
// the row, b: the first of the four columns, b_next apart).
__device__ __forceinline__ void redo_not_finite(float (&v)[4], int cols, const float* a,
                                                int64_t a_step, const float* b, int64_t b_step,
                                                int64_t b_next, int64_t count) {
  const float probe = fmaf(v[0], 0.0f, fmaf(v[1], 0.0f, fmaf(v[2], 0.0f, v[3] * 0.0f)));
  if (probe == 0.0f) return;
#pragma unroll 1
  for (int e = 0; e < cols; ++e) {
    const float old = e == 0 ? v[0] : (e == 1 ? v[1] : (e == 2 ? v[2] : v[3]));
    if (fabsf(old) < INFINITY) continue;
    float s = 0.0f;
#pragma unroll 1
    for (int64_t k = 0; k < count; ++k) s = fmaf(a[k * a_step], b[e * b_next + k * b_step], s);
    v[0] = e == 0 ? s : v[0];
    v[1] = e == 1 ? s : v[1];
    v[2] = e == 2 ? s : v[2];
    v[3] = e == 3 ? s : v[3];
  }
}

}  // namespace pinsage
