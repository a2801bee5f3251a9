// Parts of one output tile of C[m][n] = sum_k A(m, k) B(n, k) on the matrix cores
// (ring_device.h computes it): the products of the dense layers' forward and backward
// passes and of the Newton-Schulz iteration.
//
// An operand is "row" (k contiguous: A[m * ld + k]) or "column" (m contiguous:
// A[k * ld + m]).
//
// Modes:
//   kBf16   bf16 in memory, one MFMA per product
//   kBf16A2 the same, A in two bf16 parts (planes apart by `plane` bytes: 16
//           significand bits), two MFMAs (lo, hi)
//   kF16x2  two fp16 parts in memory (x = hi + lo, planes apart by `plane`
//           bytes): 22 significand bits, three MFMAs (hi lo, lo hi, hi hi, the last
//           in sums of its own); for operands the caller keeps inside fp16's range
//   kF32    fp32 in memory, split on the way to the MFMAs into three bf16 parts (24
//           significand bits), eight MFMAs, the leading products in sums of their
//           own: what is left out is below 2^-33 of a product (split_device.h).
//           Elements of rows and columns that the parts do not cover, and sums that
//           are not finite, come from fp32 MFMAs.
// Sums run in fp32, chunks in order, so an element's bits follow from its row,
// its column and the k range alone, whatever tile it lies in.
#pragma once

#include "device_util.h"
#include "split_device.h"

namespace pinsage {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

enum ProductMode { kBf16 = 0, kBf16A2 = 1, kF16x2 = 2, kF32 = 3 };

// A tile's operand: `p` at the tile's first row (row operand, k = 0) or first
// column (column operand, k = 0); `valid` rows exist from there (at least 1).
struct Operand {
  const void* p;
  int64_t ld;     // elements
  int valid;
  int64_t plane;  // two parts: bytes from the hi plane to the lo plane
  int before = 0;  // columns that exist before p
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
  if constexpr (MODE == kF16x2)
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

// The same, element by element in a loop: few registers, for rare cases.
template <int ESZ>
__device__ __forceinline__ u32x4 load_few(const unsigned char* p, int count) {
  u32x4 v = {0, 0, 0, 0};
#pragma unroll 1
  for (int e = count - 1; e >= 0; --e) {
    if constexpr (ESZ == 4) {
      v = u32x4{load_any<uint32_t>(p + 4 * e), v[0], v[1], v[2]};
    } else {
      const uint32_t x = load_any<uint16_t>(p + 2 * e);
      v = u32x4{(v[0] << 16) | x, (v[1] << 16) | (v[0] >> 16), (v[2] << 16) | (v[1] >> 16),
                (v[3] << 16) | (v[2] >> 16)};
    }
  }
  return v;
}

// Without the first `count` (fewer than a vector's) elements; zeros follow.
template <int ESZ>
__device__ __forceinline__ u32x4 drop_first(u32x4 v, int count) {
  if constexpr (ESZ == 2) {
    const bool odd = count & 1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t next = e < 3 ? v[e + 1] : 0;
      v[e] = odd ? (v[e] >> 16) | (next << 16) : v[e];
    }
    count >>= 1;
  }
#pragma unroll
  for (int step = 1; step < 4; step *= 2) {
    const bool shift = count & step;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t from = e + step < 4 ? v[e + step < 4 ? e + step : 3] : 0;
      v[e] = shift ? from : v[e];
    }
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

}  // namespace pinsage
