// Newton-Schulz orthogonalisation of a batch of matrices G [rows][cols] (the
// direction of an optimiser's update), in the orientation X [m][n] with m <= n:
//   X = G / (|G|_F + eps), then `steps` times
//   A = X X^T,  B = b A + c A A,  X = a X + B X,
// which moves every singular value of X towards 1.
//
// Every singular value of X stays near [0, 1.3], so all intermediates fit fp16
// around a fixed scale 2^12 (values to 16, the smallest normal 2^-26). They are kept as
// two fp16 parts (22 significand bits, three MFMAs a product, against six for bf16
// parts), whatever the storage type. Five steps enlarge small singular directions about
// 480 times, and what is rounded off X, A and B in their place with them: of a bf16
// matrix of rank 1 (16) one part's 2^-11 leaves an error of 9.5e-2 (3.8e-2), two parts
// 1.6e-3 as the formula in fp32 does, which is bf16's own rounding of the result. fp32
// 256 x 512 of rank 1: 6.3e-5, the formula in fp32 1.4e-4. Sums, and a X, run in fp32;
// |G|_F is summed in fp64, so no finite G overflows.
// Y = X^T, A and B live in the workspace, padded with zeros to whole tiles, so that
// no product has an edge: A = Y^T Y (both operands by columns), A A, and
// Y = a Y + Y B. A and A A are symmetric: only their tiles on and above the diagonal
// are computed, and stored twice.
#include "kernels.h"
#include "ring_device.h"

namespace pinsage {
namespace {

constexpr float kScale = 4096.0f;  // the stored values over the true ones
constexpr int kParts = 2;          // fp16 parts of a stored value
constexpr int kMaxNormBlocks = 1024;  // partial sums of a matrix's norm

struct NewtonWork {
  double* norms;     // [batch][kMaxNormBlocks]
  uint16_t* Y[2];    // [batch][kParts][np][mp]
  uint16_t* A;       // [batch][kParts][mp][mp]
  uint16_t* B;
  int m, n, mp, np;  // m <= n; padded
  int norm_blocks;
  bool flip;         // X is G^T
};

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, (f16x2){(_Float16)a, (_Float16)b});
}
__device__ __forceinline__ float unpack_f16(uint32_t w, int h) {
  return (float)__builtin_bit_cast(f16x2, w)[h];
}

// Stores N scaled values as two fp16 parts; p on 2 N bytes.
template <int N>
__device__ __forceinline__ void put(uint16_t* p, int64_t plane, const float (&v)[N]) {
  typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
  words hi, lo;
#pragma unroll
  for (int e = 0; e < N / 2; ++e) {
    hi[e] = pack_f16(v[2 * e], v[2 * e + 1]);
    lo[e] = pack_f16(v[2 * e] - unpack_f16(hi[e], 0), v[2 * e + 1] - unpack_f16(hi[e], 1));
  }
  *reinterpret_cast<words*>(p) = hi;
  *reinterpret_cast<words*>(p + plane) = lo;
}
struct Parts8 {
  u32x4 p[kParts];
};
__device__ __forceinline__ Parts8 get8(const uint16_t* p, int64_t plane) {
  Parts8 x;
  x.p[0] = *reinterpret_cast<const u32x4*>(p);
  x.p[1] = *reinterpret_cast<const u32x4*>(p + plane);
  return x;
}
__device__ __forceinline__ float value(const Parts8& x, int e) {
  return unpack_f16(x.p[0][e / 2], e & 1) + unpack_f16(x.p[1][e / 2], e & 1);
}

// ---- the norm, with the momentum's update ---------------------------------------
// What is orthogonalised, elements at .. at + 3 of the batch's storage: the input,
// or the step's combination of it with the already updated momentum. The norm of
// 2,048 x 2,048 bf16 with its momentum takes 9 us (42 MB, 4.7 TB/s), Y0 11 us.
template <bool BF16>
__device__ __forceinline__ void update4(const NewtonLaunch& a, int64_t at, int cols, float (&u)[4]) {
  read_row<BF16>(a.in, at, cols, u);
  if (!a.weight) return;
  float m[4];
  read_row<false>(a.momentum_out, at, cols, m);
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = a.nesterov ? fmaf(a.beta, m[e], u[e]) : m[e];
}

template <bool BF16>
__global__ __launch_bounds__(256) void newton_norm_kernel(NewtonLaunch a, NewtonWork w) {
  __shared__ double part[4];
  const int64_t size = (int64_t)a.rows * a.cols, base = blockIdx.y * size;
  double s = 0.0;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size;
       i += (int64_t)w.norm_blocks * 1024) {
    const int cols = (int)(size - i < 4 ? size - i : 4);
    float u[4];
    if (a.weight) {
      float m[4];
      read_row<BF16>(a.in, base + i, cols, u);
      read_row<false>(a.momentum, base + i, cols, m);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = fmaf(a.beta, m[e], u[e]);
        u[e] = a.nesterov ? fmaf(a.beta, m[e], u[e]) : m[e];
      }
      write_row<false>(a.momentum_out, base + i, cols, m);
    } else {
      read_row<BF16>(a.in, base + i, cols, u);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s = fma((double)u[e], (double)u[e], s);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    w.norms[blockIdx.y * kMaxNormBlocks + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// ---- Y0: scaled, in fp16 parts, padded ---------------------------------------------
template <bool BF16>
__global__ __launch_bounds__(256) void newton_start_kernel(NewtonLaunch a, NewtonWork w) {
  __shared__ float tile[64][65];
  __shared__ double part[4];
  const int tid = threadIdx.x;
  double s = 0.0;
  for (int q = tid; q < w.norm_blocks; q += 256)
    s += w.norms[(int64_t)blockIdx.z * kMaxNormBlocks + q];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
  if ((tid & 63) == 0) part[tid >> 6] = s;
  __syncthreads();
  s = (part[0] + part[1]) + (part[2] + part[3]);
  const double inv = (double)kScale / (sqrt(s) + (double)a.eps);
  const int64_t base = (int64_t)blockIdx.z * a.rows * a.cols;
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;              // of Y
  const int r0 = w.flip ? i0 : j0, c0 = w.flip ? j0 : i0;  // of G
#pragma unroll
  for (int q = tid; q < 64 * 16; q += 256) {
    const int r = q / 16, c = q % 16 * 4, cols = a.cols - c0 - c;
    float u[4] = {0, 0, 0, 0};
    if (r0 + r < a.rows && cols > 0)
      update4<BF16>(a, base + (int64_t)(r0 + r) * a.cols + c0 + c, cols, u);
#pragma unroll
    for (int e = 0; e < 4; ++e) tile[r][c + e] = (float)(u[e] * inv);
  }
  __syncthreads();
  const int64_t plane = (int64_t)w.mp * w.np;
  uint16_t* const Y = w.Y[0] + blockIdx.z * kParts * plane;
#pragma unroll
  for (int q = tid; q < 64 * 8; q += 256) {
    const int i = q / 8, j = q % 8 * 8;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = w.flip ? tile[i][j + e] : tile[j + e][i];
    put(Y + (int64_t)(i0 + i) * w.mp + j0 + j, plane, v);
  }
}

// ---- the three products -----------------------------------------------------------
enum NewtonProduct { kGram = 0, kSquare = 1, kApply = 2, kLast = 3 };

// P[i][j] = sum_k L(i, k) R(j, k): Y^T Y, A A, or Y B (A and B are symmetric). About 8 us
// of each are its launch, first loads and epilogue; the rest waits for the tiles' loads,
// the MFMAs have 20% of the cycles by 64 x 64 and 42% by 128 x 128. By the counters 64 x 64
// tiles take 10 to 12 TB/s out of the L2s, well below what those serve, so the latency of
// two stages bounds them; order of tiles and row pitch make no difference. 2,048 x 2,048
// 54, 54 (528 tiles of 64, 550 MB each) and 57 us (256 of 128, 545 MB), 2,048 x 1,024 20,
// 13 (136 tiles on 256 CUs, 134 and 69 MB) and 19 us (512 tiles, 225 MB).
template <class C, int KIND, bool BF16>
__global__ __launch_bounds__(C::THREADS, C::WPE) void newton_kernel(NewtonLaunch a, NewtonWork w,
                                                                    int from, int tiles) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[C::LDS_BYTES];
  static_assert(C::A_PLANES == kParts && C::B_PLANES == kParts, "");
  constexpr bool kSymmetric = KIND == kGram || KIND == kSquare;
  const int64_t px = (int64_t)w.mp * w.np, pa = (int64_t)w.mp * w.mp;
  // Neighbouring tiles, and whole matrices of a batch, on one XCD.
  const int id = xcd_tile(blockIdx.x, gridDim.x), tile = id % tiles;
  const int64_t z = id / tiles;
  const uint16_t* const Y = w.Y[from] + z * kParts * px;
  uint16_t* const A = w.A + z * kParts * pa;
  uint16_t* const B = w.B + z * kParts * pa;
  int ti, tj;
  if constexpr (kSymmetric) {
    // Tiles on and above the diagonal, row by row.
    const int T = w.mp / C::BM;
    int left = tile;
    ti = 0;
    while (left >= T - ti) left -= T - ti++;
    tj = ti + left;
  } else {
    const int T = w.mp / C::BN;
    ti = tile / T;
    tj = tile % T;
  }
  const int i0 = ti * C::BM, j0 = tj * C::BN;
  Operand L, R;
  int depth;
  if constexpr (KIND == kGram) {
    L = Operand{Y + i0, w.mp, C::BM, px * 2};
    R = Operand{Y + j0, w.mp, C::BN, px * 2};
    depth = w.np;
  } else {
    L = Operand{(KIND == kSquare ? A : Y) + (int64_t)i0 * w.mp, w.mp, C::BM,
                (KIND == kSquare ? pa : px) * 2};
    R = Operand{(KIND == kSquare ? A : B) + (int64_t)j0 * w.mp, w.mp, C::BN, pa * 2};
    depth = w.mp;
  }
  TileSums<C> sums;
  tile_sums(L, R, 0, depth, smem, sums);

  // Products carry the scale twice. What a product is added to is read a band ahead.
  const float back = 1.0f / kScale;
  if constexpr (kSymmetric) {
    uint16_t* const out = KIND == kGram ? A : B;
    product_rows_cols<8>(
        sums, smem,
        [&](int m, int n) __attribute__((always_inline)) {
          if constexpr (KIND == kGram) return Nothing{};
          else return get8(A + (int64_t)(i0 + m) * w.mp + j0 + n, pa);
        },
        [&](int m, int n, float (&v)[8], const auto& x) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if constexpr (KIND == kGram) v[e] *= back;
            else v[e] = fmaf(a.b, value(x, e), a.c * back * v[e]);
          }
          put(out + (int64_t)(i0 + m) * w.mp + j0 + n, pa, v);
        },
        [&](int m, int n, const float (&v)[8]) __attribute__((always_inline)) {
          put(out + (int64_t)(j0 + n) * w.mp + i0 + m, pa, v);
        },
        ti != tj);
  } else if constexpr (KIND == kApply) {
    uint16_t* const out = w.Y[1 - from] + z * kParts * px;
    product_rows_cols<8>(
        sums, smem,
        [&](int m, int n) __attribute__((always_inline)) {
          return get8(Y + (int64_t)(i0 + m) * w.mp + j0 + n, px);
        },
        [&](int m, int n, float (&v)[8], const auto& x) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fmaf(a.a, value(x, e), back * v[e]);
          put(out + (int64_t)(i0 + m) * w.mp + j0 + n, px, v);
        },
        [](int, int, const float (&)[8]) {}, false);
  } else {
    const int64_t base = z * a.rows * a.cols;
    // Up to eight results of one row of G, from `at` on.
    auto give = [&](int64_t at, int cols, float (&y)[8]) __attribute__((always_inline)) {
      if (a.weight) {
        float old[8];
        read_row<BF16>(a.weight, at, cols, old);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmaf(a.decay, old[e], -a.rate * y[e]);
      }
      write_row<BF16>(a.out, at, cols, y);
    };
    product_rows_cols<8>(
        sums, smem,
        [&](int m, int n) __attribute__((always_inline)) {
          return get8(Y + (int64_t)(i0 + m) * w.mp + j0 + n, px);
        },
        [&](int m, int n, float (&v)[8], const auto& x) __attribute__((always_inline)) {
          const int i = i0 + m, j = j0 + n;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fmaf(a.a, value(x, e), back * v[e]) * back;
          if (w.flip && i < w.n && j < w.m) give(base + (int64_t)i * a.cols + j, w.m - j, v);
        },
        [&](int m, int n, const float (&v)[8]) __attribute__((always_inline)) {
          const int i = i0 + m, j = j0 + n;
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = v[e];
          if (i < w.n && j < w.m) give(base + (int64_t)j * a.cols + i, w.n - i, y);
        },
        !w.flip);
  }
}

// ---- matrices in LDS -------------------------------------------------------------------
// Rows of 16-bit values in parts, 16-byte slot s of row r at s ^ lds_swizzle(r): a fragment
// read's 8 rows, and the 4 rows of a transposing read, fall on distinct banks.
__device__ __forceinline__ int lds_swizzle(int r) { return ((r & 3) << 1) | ((r >> 2) & 1); }

// Eight k of each of 32 rows from r0 on: step ks of 16.
__device__ __forceinline__ Parts8 lds_fragment(const unsigned char* M, int pitch, int plane,
                                                       int r0, int ks) {
  const int lane = threadIdx.x & 63, r = r0 + (lane & 31);
  Parts8 f;
#pragma unroll
  for (int p = 0; p < kParts; ++p)
    f.p[p] = *reinterpret_cast<const u32x4*>(M + p * plane + r * pitch +
                                             (((2 * ks + (lane >> 5)) ^ lds_swizzle(r)) * 16));
  return f;
}
// All products of the parts, lo lo too: the diagonal of A sums squares, so what is left
// out has one sign, which shows with few singular values (fp32, 16 x 100, 4 draws: mean
// error 1.3e-6, with lo lo 1.0e-6). hi hi has sums of its own.
struct PartSums {
  f32x16 large, small;
  __device__ __forceinline__ void clear() {
    clear_block(large);
    clear_block(small);
  }
};
__device__ __forceinline__ void multiply_parts(const Parts8& b, const Parts8& l, PartSums& acc) {
  acc.small = product_mfma<kF16x2>(b.p[1], l.p[1], acc.small);
  acc.small = product_mfma<kF16x2>(b.p[1], l.p[0], acc.small);
  acc.small = product_mfma<kF16x2>(b.p[0], l.p[1], acc.small);
  acc.large = product_mfma<kF16x2>(b.p[0], l.p[0], acc.large);
}

// ---- medium matrices: A's square and its product with Y in one launch -------------------
// Y (a I + b A + c A A) = a Y + b T + c T A with T = Y A: a block holds A and 32 rows of Y in
// LDS, forms T in Y's place (rounded as Y is) and Y's successor from it. Against the two
// launches (B, then Y B) it multiplies more, 4 m^2 n against m^3 + 2 m^2 n, but up to 128
// columns, where A fits beside Y, launches and loads are what costs. Whole calls in us,
// with it and without: 64 x 384 63, 79; 128 x 512 79, 95; 4 of 100 x 1,000 102, 119; 32 of
// 128 x 512 102, 113; 8 of 128 x 2,048 153, 163. The width is a compile-time constant: at
// run time its divisions alone took 3 us.
constexpr int kBandWaves = 8, kBandRows = 32;

template <int mp>
__global__ __launch_bounds__(64 * kBandWaves) void newton_band_kernel(NewtonLaunch a, NewtonWork w,
                                                                      int from) {
  constexpr int THREADS = 64 * kBandWaves, slots = mp / 8, pitch = mp * 2;
  constexpr int plane_a = mp * pitch, plane_y = kBandRows * pitch;
  __shared__ __attribute__((aligned(16))) unsigned char smem[kParts * (plane_a + plane_y)];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bands = w.np / kBandRows, id = xcd_tile(blockIdx.x, gridDim.x);
  const int64_t z = id / bands, i0 = (int64_t)(id % bands) * kBandRows;
  const int64_t px = (int64_t)mp * w.np, pa = (int64_t)mp * mp;
  const uint16_t* const Y = w.Y[from] + z * kParts * px + i0 * mp;
  uint16_t* const out = w.Y[1 - from] + z * kParts * px + i0 * mp;
  const uint16_t* const A = w.A + z * kParts * pa;
  unsigned char* const lds_a = smem;                          // planes of mp rows
  unsigned char* const lds_y = smem + kParts * plane_a;       // planes of 32 rows
  auto at = [&](unsigned char* M, int r, int slot) __attribute__((always_inline)) {
    return reinterpret_cast<u32x4*>(M + r * pitch + ((slot ^ lds_swizzle(r)) * 16));
  };
  constexpr int VECTORS = kParts * mp * slots, BATCH = (VECTORS + THREADS - 1) / THREADS;
  u32x4 v[BATCH];  // all of a thread's loads in flight
#pragma unroll
  for (int u = 0; u < BATCH; ++u) {
    const int q = tid + u * THREADS;
    if (VECTORS % THREADS == 0 || q < VECTORS) v[u] = *reinterpret_cast<const u32x4*>(A + q * 8);
  }
#pragma unroll
  for (int u = 0; u < BATCH; ++u) {
    const int q = tid + u * THREADS, row = q / slots;  // of all planes
    if (VECTORS % THREADS == 0 || q < VECTORS)
      *at(lds_a + row / mp * plane_a, row % mp, q % slots) = v[u];
  }
  for (int q = tid; q < kParts * kBandRows * slots; q += THREADS) {
    const int p = q / (kBandRows * slots), e = q % (kBandRows * slots);
    *at(lds_y + p * plane_y, e / slots, e % slots) =
        *reinterpret_cast<const u32x4*>(Y + p * px + e * 8);
  }
  __syncthreads();

  // A wave's 32 columns; waves past the last one only load and wait.
  const bool works = 32 * wave < mp;
  const int i = lane & 31;
  const float back = 1.0f / kScale;  // products carry the scale twice
  f32x16 acc;
  auto product = [&]() __attribute__((always_inline)) {
    PartSums sums;
    sums.clear();
#pragma unroll
    for (int ks = 0; ks < mp / 16; ++ks)
      multiply_parts(lds_fragment(lds_a, pitch, plane_a, 32 * wave, ks),
                     lds_fragment(lds_y, pitch, plane_y, 0, ks), sums);
    acc = sums.large + sums.small;
  };
  // The lane's columns 8 g + 4 (lane / 32) of the wave's, row i of the band.
  auto place = [&](int g) __attribute__((always_inline)) {
    const int j = 32 * wave + 8 * g + 4 * (lane >> 5);
    return reinterpret_cast<uint16_t*>(lds_y + i * pitch + (((j >> 3) ^ lds_swizzle(i)) * 16) +
                                       (j & 4) * 2);
  };
  float sum[16];
  if (works) {
    product();
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint2 hi = *reinterpret_cast<const uint2*>(place(g));
      const uint2 lo = *reinterpret_cast<const uint2*>(place(g) + plane_y / 2);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y =
            unpack_f16(e < 2 ? hi.x : hi.y, e & 1) + unpack_f16(e < 2 ? lo.x : lo.y, e & 1);
        sum[4 * g + e] = fmaf(a.a, y, a.b * back * acc[4 * g + e]);
      }
    }
  }
  __syncthreads();  // all have read Y
  if (works)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float t[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = back * acc[4 * g + e];
      put(place(g), plane_y / 2, t);
    }
  __syncthreads();
  if (works) product();
  __syncthreads();  // all have read T
  if (works)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(a.c * back, acc[4 * g + e], sum[4 * g + e]);
      put(place(g), plane_y / 2, y);
    }
  __syncthreads();
  for (int q = tid; q < kParts * kBandRows * slots; q += THREADS) {
    const int p = q / (kBandRows * slots), e = q % (kBandRows * slots);
    *reinterpret_cast<u32x4*>(out + p * px + e * 8) =
        *at(lds_y + p * plane_y, e / slots, e % slots);
  }
}

// ---- small matrices: everything in one block ------------------------------------------
// A block of eight waves takes a matrix from G to the result, X and one m x m matrix in
// its LDS: what bounds a small matrix else is that there are 13 launches, at 3 to 5 us
// each whatever they compute. Up to 64 x 320, us, one block and launches: 64 x 64 26, 50;
// 512 of them 55, 89; 300 x 40 51, 61; 64 x 320 59, 62; 64 x 384 67, 63; 128 x 128 72, 63.
// X [mp][np] and A [mp][mp] lie in LDS in fp16 parts; X's columns, for B X, come through
// transposing reads. A wave's blocks of 32 x 32 stay in its accumulators until all waves
// have read what they replace.
constexpr int kSmallWaves = 8, kSmallBlocks = 3;  // blocks per wave at most, of X or A
constexpr int kSmallSide = 64, kSmallLong = 320;
constexpr int kSmallLds = 2 * 2 * kSmallSide * (kSmallLong + kSmallSide);

inline bool fits_one_block(const NewtonWork& w) {
  return w.mp == kSmallSide && w.np <= kSmallLong;
}

template <bool BF16>
__global__ __launch_bounds__(64 * kSmallWaves) void newton_small_kernel(NewtonLaunch a,
                                                                        NewtonWork w) {
  constexpr int THREADS = 64 * kSmallWaves;
  __shared__ __attribute__((aligned(16))) unsigned char smem[kSmallLds];
  __shared__ double norms[kSmallWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mp = w.mp, np = w.np, mb = mp / 32, nb = np / 32;
  const int64_t size = (int64_t)a.rows * a.cols, base = blockIdx.x * size;
  unsigned char* const X = smem;                          // planes of mp rows of np
  unsigned char* const A = smem + kParts * mp * np * 2;   // planes of mp rows of mp
  const int px = mp * np * 2, pa = mp * mp * 2;

  // The norm, with the momentum's update.
  double s = 0.0;
  const int cells = (a.cols + 3) / 4;  // of four elements of a row
  for (int q = tid; q < a.rows * cells; q += THREADS) {
    const int r = q / cells, c = q % cells * 4, cols = a.cols - c;
    const int64_t at = base + (int64_t)r * a.cols + c;
    float u[4];
    read_row<BF16>(a.in, at, cols, u);
    if (a.weight) {
      float m[4];
      read_row<false>(a.momentum, at, cols, m);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = fmaf(a.beta, m[e], u[e]);
        u[e] = a.nesterov ? fmaf(a.beta, m[e], u[e]) : m[e];
      }
      write_row<false>(a.momentum_out, at, cols, m);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s = e < cols ? fma((double)u[e], (double)u[e], s) : s;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
  if (lane == 0) norms[wave] = s;
  // X's padding.
  for (int q = tid; q < kParts * mp * np / 8; q += THREADS)
    reinterpret_cast<u32x4*>(X)[q] = u32x4{0, 0, 0, 0};
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int q = 0; q < kSmallWaves; ++q) s += norms[q];
  const double inv = (double)kScale / (sqrt(s) + (double)a.eps);

  // X0; a thread reads what it wrote of the momentum.
  for (int q = tid; q < a.rows * cells; q += THREADS) {
    const int r = q / cells, c = q % cells * 4, cols = a.cols - c;
    float u[4];
    update4<BF16>(a, base + (int64_t)r * a.cols + c, cols, u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e >= cols) break;
      const int i = w.flip ? c + e : r, j = w.flip ? r : c + e;
      unsigned char* const to = X + i * np * 2 + (((j >> 3) ^ lds_swizzle(i)) * 16) + (j & 7) * 2;
      const float v = (float)(u[e] * inv);
      const _Float16 hi = (_Float16)v;
      *reinterpret_cast<_Float16*>(to) = hi;
      *reinterpret_cast<_Float16*>(to + px) = (_Float16)(v - (float)hi);
    }
  }
  __syncthreads();

  const int frag_row = lane & 31, half = lane >> 5;
  // Columns c0 .. c0 + 31 of X, k along its rows.
  auto col_frag = [&](int c0, int ks) __attribute__((always_inline)) {
    Parts8 f;
    const int c = c0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int p = 0; p < kParts; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = 16 * ks + 8 * half + 4 * h + ((lane >> 2) & 3);
        const unsigned char* const at =
            X + p * px + k * np * 2 + (((c >> 3) ^ lds_swizzle(k)) * 16) + (c & 4) * 2;
        const u32x2 x = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                       (__attribute__((address_space(3))) s16x4*)at));
        f.p[p][2 * h] = x[0];
        f.p[p][2 * h + 1] = x[1];
      }
    return f;
  };
  // Block (bi, bj) of M becomes p M + q sum.
  auto update = [&](unsigned char* M, int pitch, int plane, int bi, int bj, float p, float q,
                    const PartSums& parts) __attribute__((always_inline)) {
    const f32x16 sum = parts.large + parts.small;
    const int i = 32 * bi + frag_row;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int j = 32 * bj + 8 * g + 4 * half;
      uint16_t* const at = reinterpret_cast<uint16_t*>(
          M + i * pitch + (((j >> 3) ^ lds_swizzle(i)) * 16) + (j & 4) * 2);
      float v[4];
      if (p == 0.0f) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = q * sum[4 * g + e];
      } else {
        const uint2 hi = *reinterpret_cast<const uint2*>(at);
        const uint2 lo = *reinterpret_cast<const uint2*>(at + plane / 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t h = e < 2 ? hi.x : hi.y, l = e < 2 ? lo.x : lo.y;
          const float old = unpack_f16(h, e & 1) + unpack_f16(l, e & 1);
          v[e] = fmaf(p, old, q * sum[4 * g + e]);
        }
      }
      put(at, plane / 2, v);
    }
  };
  const float back = 1.0f / kScale;  // products carry the scale twice
  PartSums acc[kSmallBlocks];

  for (int step = 0; step < a.steps; ++step) {
    // A = X X^T, a wave's blocks in turn.
    for (int b = wave; b < mb * mb; b += kSmallWaves) {
      const int bi = b / mb, bj = b % mb;
      acc[0].clear();
      for (int ks = 0; ks < np / 16; ++ks)
        multiply_parts(lds_fragment(X, np * 2, px, 32 * bj, ks),
                       lds_fragment(X, np * 2, px, 32 * bi, ks), acc[0]);
      update(A, mp * 2, pa, bi, bj, 0.0f, back, acc[0]);
    }
    __syncthreads();
    // A becomes b A + c A A (A is symmetric: both operands are its rows).
#pragma unroll
    for (int t = 0; t < kSmallBlocks; ++t) acc[t].clear();
    for (int ks = 0; ks < mp / 16; ++ks)
#pragma unroll
      for (int t = 0; t < kSmallBlocks; ++t) {
        const int b = wave + t * kSmallWaves;
        if (b < mb * mb)
          multiply_parts(lds_fragment(A, mp * 2, pa, 32 * (b % mb), ks),
                         lds_fragment(A, mp * 2, pa, 32 * (b / mb), ks), acc[t]);
      }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kSmallBlocks; ++t) {
      const int b = wave + t * kSmallWaves;
      if (b < mb * mb) update(A, mp * 2, pa, b / mb, b % mb, a.b, a.c * back, acc[t]);
    }
    __syncthreads();
    // X becomes a X + A X.
#pragma unroll
    for (int t = 0; t < kSmallBlocks; ++t) acc[t].clear();
    for (int ks = 0; ks < mp / 16; ++ks)
#pragma unroll
      for (int t = 0; t < kSmallBlocks; ++t) {
        const int b = wave + t * kSmallWaves;
        if (b < mb * nb)
          multiply_parts(col_frag(32 * (b / mb), ks),
                         lds_fragment(A, mp * 2, pa, 32 * (b % mb), ks), acc[t]);
      }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kSmallBlocks; ++t) {
      const int b = wave + t * kSmallWaves;
      if (b < mb * nb) update(X, np * 2, px, b % mb, b / mb, a.a, back, acc[t]);
    }
    __syncthreads();
  }

  // The result, along G's rows.
  for (int q = tid; q < a.rows * cells; q += THREADS) {
    const int r = q / cells, c = q % cells * 4, cols = a.cols - c;
    const int64_t at = base + (int64_t)r * a.cols + c;
    float v[4], old[4] = {};
    if (a.weight) read_row<BF16>(a.weight, at, cols, old);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = w.flip ? c + e : r, j = w.flip ? r : c + e;
      v[e] = 0.0f;
      if (e < cols) {
        const unsigned char* const from =
            X + i * np * 2 + (((j >> 3) ^ lds_swizzle(i)) * 16) + (j & 7) * 2;
        v[e] = (float)*reinterpret_cast<const _Float16*>(from) +
               (float)*reinterpret_cast<const _Float16*>(from + px);
      }
      v[e] *= back;
      if (a.weight) v[e] = fmaf(a.decay, old[e], -a.rate * v[e]);
    }
    write_row<BF16>(a.out, at, cols, v);
  }
}

// ---- tile shapes --------------------------------------------------------------------
// 64 x 64 with four stages (128 KB, a block a CU) while the tiles are no more than CUs,
// with two stages, which more of them share, up to 600 tiles, else 128 x 128. Whole calls
// in us. Four stages, two: 1,024 x 1,024 (136 and 256 tiles) 200, 234; 1,024 x 2,048's 512
// tiles 296, 272. 64, 128 for the symmetric products: 435 tiles (1,800 x 1,800) 569, 690;
// 544 (4 of 1,024 x 1,024) 476, 479; 576 (16 of 512 x 512) 311, 330; 528 deep ones (2,048 x
// 2,048) 827, 785. For Y B: 484 tiles (1,408 x 1,408) 320, 356; 625 (1,600 x 1,600) 486,
// 459; 768 (3 of 1,024 x 1,024) 364, 352; 1,024 (2,048 x 2,048) 875, 827.
inline int64_t tiles_of(const NewtonWork& w, int64_t batch, bool symmetric, int side) {
  const int64_t tm = (w.mp + side - 1) / side, tn = (w.np + side - 1) / side;
  return (symmetric ? tm * (tm + 1) / 2 : tm * tn) * batch;
}
inline bool small_tiles(const NewtonWork& w, int64_t batch, bool symmetric) {
  return tiles_of(w, batch, symmetric, 64) <= 600;
}

template <class C, int KIND, bool BF16>
void launch_one(const NewtonLaunch& a, const NewtonWork& w, int from, hipStream_t s) {
  const int64_t tiles = tiles_of(w, 1, KIND == kGram || KIND == kSquare, C::BM);
  hipLaunchKernelGGL((newton_kernel<C, KIND, BF16>), dim3((unsigned)(tiles * a.batch)),
                     dim3(C::THREADS), 0, s, a, w, from, (int)tiles);
}

template <int KIND, bool BF16>
void launch_product(const NewtonLaunch& a, const NewtonWork& w, int from, hipStream_t s) {
  constexpr bool kSymmetric = KIND == kGram || KIND == kSquare, kCol = KIND == kGram;
  const bool small = small_tiles(w, a.batch, kSymmetric);
  if (small && tiles_of(w, a.batch, kSymmetric, 64) <= 256)
    launch_one<RingCfg<kF16x2, 64, 64, 64, 2, 2, kCol, kCol, 4>, KIND, BF16>(a, w, from, s);
  else if (small)
    launch_one<RingCfg<kF16x2, 64, 64, 64, 2, 2, kCol, kCol, 2>, KIND, BF16>(a, w, from, s);
  else
    launch_one<RingCfg<kF16x2, 128, 128, 32, 2, 2, kCol, kCol, 4>, KIND, BF16>(a, w, from, s);
}

inline size_t aligned(size_t v) { return (v + 255) / 256 * 256; }

size_t layout(int64_t batch, int rows, int cols, unsigned char* ws, NewtonWork* w) {
  w->flip = rows > cols;
  w->m = w->flip ? cols : rows;
  w->n = w->flip ? rows : cols;
  w->mp = (w->m + 63) / 64 * 64;
  w->np = (w->n + 63) / 64 * 64;
  if (!small_tiles(*w, batch, true) || !small_tiles(*w, batch, false)) {
    w->mp = (w->m + 127) / 128 * 128;
    w->np = (w->n + 127) / 128 * 128;
  }
  const int64_t blocks = ((int64_t)rows * cols + 4095) / 4096;
  w->norm_blocks = (int)(blocks < kMaxNormBlocks ? blocks : kMaxNormBlocks);
  const size_t x = aligned((size_t)batch * kParts * w->mp * w->np * 2);
  const size_t g = aligned((size_t)batch * kParts * w->mp * w->mp * 2);
  const size_t norms = aligned((size_t)batch * kMaxNormBlocks * sizeof(double));
  w->norms = reinterpret_cast<double*>(ws);
  uint16_t* const rest = reinterpret_cast<uint16_t*>(ws + norms);
  w->Y[0] = rest;
  w->Y[1] = rest + x / 2;
  w->A = rest + x;
  w->B = rest + x + g / 2;
  return norms + 2 * x + 2 * g;
}

// The padded sides of a small matrix, whatever its batch asks of the launches.
bool one_block(NewtonWork* w) {
  NewtonWork one = *w;
  one.mp = (w->m + 63) / 64 * 64;
  one.np = (w->n + 63) / 64 * 64;
  if (!fits_one_block(one)) return false;
  *w = one;
  return true;
}

template <int MP>
bool launch_band_of(const NewtonLaunch& a, const NewtonWork& w, int from, hipStream_t s) {
  if (w.mp != MP) return false;
  hipLaunchKernelGGL((newton_band_kernel<MP>),
                     dim3((unsigned)(w.np / kBandRows * a.batch)), dim3(64 * kBandWaves), 0, s, a, w,
                     from);
  return true;
}
bool launch_band(const NewtonLaunch& a, const NewtonWork& w, int from, hipStream_t s) {
  return launch_band_of<64>(a, w, from, s) || launch_band_of<128>(a, w, from, s);
}

template <bool BF16>
hipError_t launch_dtype(const NewtonLaunch& a, NewtonWork w, hipStream_t s) {
  const unsigned batch = (unsigned)a.batch;
  if (one_block(&w)) {
    hipLaunchKernelGGL(newton_small_kernel<BF16>, dim3(batch), dim3(64 * kSmallWaves), 0, s, a, w);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(newton_norm_kernel<BF16>, dim3((unsigned)w.norm_blocks, batch), dim3(256), 0, s,
                     a, w);
  hipLaunchKernelGGL(newton_start_kernel<BF16>,
                     dim3((unsigned)(w.mp / 64), (unsigned)(w.np / 64), batch), dim3(256), 0, s, a, w);
  for (int k = 0, from = 0; k < a.steps; ++k, from = 1 - from) {
    launch_product<kGram, BF16>(a, w, from, s);
    if (k + 1 < a.steps && launch_band(a, w, from, s)) continue;
    launch_product<kSquare, BF16>(a, w, from, s);
    if (k + 1 < a.steps) launch_product<kApply, BF16>(a, w, from, s);
    else launch_product<kLast, BF16>(a, w, from, s);
  }
  return hipGetLastError();
}

}  // namespace

size_t newton_workspace(int64_t batch, int rows, int cols) {
  NewtonWork w;
  return layout(batch, rows, cols, nullptr, &w);
}

hipError_t launch_newton(const NewtonLaunch& a, void* workspace, hipStream_t s) {
  if (a.batch <= 0) return hipSuccess;
  ProfileScope prof(kKNewtonSchulz, s);
  NewtonWork w;
  layout(a.batch, a.rows, a.cols, static_cast<unsigned char*>(workspace), &w);
  return a.bf16 ? launch_dtype<true>(a, w, s) : launch_dtype<false>(a, w, s);
}

}  // namespace pinsage
