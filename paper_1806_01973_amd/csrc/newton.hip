// Newton-Schulz orthogonalisation of a batch of matrices G [rows][cols] (the
// direction of an optimiser's update), in the orientation X [m][n] with m <= n:
//   X = G / (|G|_F + eps), then `steps` times
//   A = X X^T,  B = b A + c A A,  X = a X + B X,
// which moves every singular value of X towards 1.
//
// Every singular value of X stays near [0, 1.3], so all intermediates fit fp16
// around a fixed scale 2^12 (values to 16, the smallest normal 2^-26): bf16
// storage keeps them as one fp16 value each (2^-11 instead of bf16's 2^-8; the
// result rounds to bf16 once, at the end), fp32 storage as two (22 significand
// bits, three MFMAs a product, against six for bf16 parts). Sums, and a X, run in
// fp32; |G|_F is summed in fp64, so no finite G overflows.
// X, A and B live in the workspace, padded with zeros to multiples of 128, so no
// product has an edge. A and A A are symmetric: only their tiles on and above the
// diagonal are computed, and stored twice.
#include "kernels.h"
#include "product_device.h"

namespace pinsage {
namespace {

constexpr float kScale = 4096.0f;  // the stored values over the true ones
constexpr int kPad = 128;
constexpr int kNormBlocks = 64;    // partial sums of a matrix's norm

inline int padded(int v) { return (v + kPad - 1) / kPad * kPad; }

struct NewtonWork {
  double* norms;     // [batch][kNormBlocks]
  uint16_t* X[2];    // [batch][planes][mp][np]
  uint16_t* A;       // [batch][planes][mp][mp]
  uint16_t* B;
  int m, n, mp, np;  // m <= n; padded
  bool flip;         // X is G^T
};

// ---- four elements of the storage dtype, any alignment -------------------------
template <bool BF16>
__device__ __forceinline__ float read1(const void* p, int64_t at) {
  if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t*>(p)[at]);
  else return static_cast<const float*>(p)[at];
}
template <bool BF16>
__device__ __forceinline__ void write1(void* p, int64_t at, float v) {
  if constexpr (BF16) static_cast<uint16_t*>(p)[at] = f32_to_bf16(v);
  else static_cast<float*>(p)[at] = v;
}

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, (f16x2){(_Float16)a, (_Float16)b});
}
__device__ __forceinline__ float unpack_f16(uint32_t w, int h) {
  return (float)__builtin_bit_cast(f16x2, w)[h];
}

// Stores four scaled values as one or two fp16 parts; p on 8 bytes.
template <int PLANES>
__device__ __forceinline__ void put4(uint16_t* p, int64_t plane, const float (&v)[4]) {
  const uint2 hi = make_uint2(pack_f16(v[0], v[1]), pack_f16(v[2], v[3]));
  *reinterpret_cast<uint2*>(p) = hi;
  if constexpr (PLANES == 2) {
    const uint2 lo = make_uint2(pack_f16(v[0] - unpack_f16(hi.x, 0), v[1] - unpack_f16(hi.x, 1)),
                                pack_f16(v[2] - unpack_f16(hi.y, 0), v[3] - unpack_f16(hi.y, 1)));
    *reinterpret_cast<uint2*>(p + plane) = lo;
  }
}
template <int PLANES>
__device__ __forceinline__ void get4(const uint16_t* p, int64_t plane, float (&v)[4]) {
  const uint2 hi = *reinterpret_cast<const uint2*>(p);
  v[0] = unpack_f16(hi.x, 0);
  v[1] = unpack_f16(hi.x, 1);
  v[2] = unpack_f16(hi.y, 0);
  v[3] = unpack_f16(hi.y, 1);
  if constexpr (PLANES == 2) {
    const uint2 lo = *reinterpret_cast<const uint2*>(p + plane);
    v[0] += unpack_f16(lo.x, 0);
    v[1] += unpack_f16(lo.x, 1);
    v[2] += unpack_f16(lo.y, 0);
    v[3] += unpack_f16(lo.y, 1);
  }
}

// ---- the norm, with the momentum's update ---------------------------------------
// What is orthogonalised: the input, or the step's combination of it with the
// already updated momentum.
template <bool BF16>
__device__ __forceinline__ float update_at(const NewtonLaunch& a, int64_t at, float momentum) {
  const float g = read1<BF16>(a.in, at);
  if (!a.weight) return g;
  return a.nesterov ? fmaf(a.beta, momentum, g) : momentum;
}

template <bool BF16>
__global__ __launch_bounds__(256) void newton_norm_kernel(NewtonLaunch a, NewtonWork w) {
  __shared__ double part[4];
  const int64_t size = (int64_t)a.rows * a.cols, base = blockIdx.y * size;
  double s = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size; i += kNormBlocks * 256) {
    float mom = 0.0f;
    if (a.weight) {
      mom = fmaf(a.beta, a.momentum[base + i], read1<BF16>(a.in, base + i));
      a.momentum_out[base + i] = mom;
    }
    const double u = update_at<BF16>(a, base + i, mom);
    s = fma(u, u, s);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    w.norms[blockIdx.y * kNormBlocks + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// ---- X0: scaled, split into fp16 parts, transposed when flipped, padded ----------
template <bool BF16>
__global__ __launch_bounds__(256) void newton_start_kernel(NewtonLaunch a, NewtonWork w) {
  constexpr int PLANES = BF16 ? 1 : 2;
  __shared__ float tile[64][65];
  const int tid = threadIdx.x, lane = tid & 63;
  double s = w.norms[(int64_t)blockIdx.z * kNormBlocks + lane];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
  const double inv = (double)kScale / (sqrt(s) + (double)a.eps);
  const int64_t base = (int64_t)blockIdx.z * a.rows * a.cols;
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;  // in X
  for (int q = tid >> 6; q < 64; q += 4) {
    // Along G's rows, so that reads are contiguous either way.
    const int gr = w.flip ? j0 + q : i0 + q, gc = w.flip ? i0 + lane : j0 + lane;
    float v = 0.0f;
    if (gr < a.rows && gc < a.cols) {
      const int64_t at = base + (int64_t)gr * a.cols + gc;
      v = (float)(update_at<BF16>(a, at, a.weight ? a.momentum_out[at] : 0.0f) * inv);
    }
    if (w.flip) tile[lane][q] = v;
    else tile[q][lane] = v;
  }
  __syncthreads();
  const int64_t plane = (int64_t)w.mp * w.np;
  uint16_t* const X = w.X[0] + blockIdx.z * PLANES * plane;
  for (int q = tid; q < 64 * 16; q += 256) {
    const int i = q / 16, j = q % 16 * 4;
    const float v[4] = {tile[i][j], tile[i][j + 1], tile[i][j + 2], tile[i][j + 3]};
    put4<PLANES>(X + (int64_t)(i0 + i) * w.np + j0 + j, plane, v);
  }
}

// ---- the three products -----------------------------------------------------------
enum NewtonProduct { kGram = 0, kSquare = 1, kApply = 2, kLast = 3 };

// P[i][j] = sum_k L(i, k) R(j, k): X X^T, A A (A is symmetric), or B X.
template <class C, int KIND, bool BF16>
__global__ __launch_bounds__(C::THREADS, C::WPE) void newton_kernel(NewtonLaunch a, NewtonWork w,
                                                                    int from) {
  __shared__ __attribute__((aligned(16))) unsigned char smem[C::LDS_BYTES];
  constexpr int PLANES = C::MEM_PLANES;
  constexpr bool kSymmetric = KIND == kGram || KIND == kSquare;
  const int64_t px = (int64_t)w.mp * w.np, pa = (int64_t)w.mp * w.mp, z = blockIdx.y;
  const uint16_t* const X = w.X[from] + z * PLANES * px;
  uint16_t* const A = w.A + z * PLANES * pa;
  uint16_t* const B = w.B + z * PLANES * pa;
  int ti, tj;
  if constexpr (kSymmetric) {
    // Tiles on and above the diagonal, row by row.
    const int T = w.mp / C::BM;
    int left = blockIdx.x;
    ti = 0;
    while (left >= T - ti) left -= T - ti++;
    tj = ti + left;
  } else {
    const int T = w.np / C::BN;
    ti = blockIdx.x / T;
    tj = blockIdx.x % T;
  }
  const int i0 = ti * C::BM, j0 = tj * C::BN;
  f32x16 acc[C::TM][C::TN];
  product_clear<C>(acc);
  Operand L, R;
  int depth;
  if constexpr (KIND == kGram) {
    L = Operand{X + (int64_t)i0 * w.np, w.np, C::BM, px * 2};
    R = Operand{X + (int64_t)j0 * w.np, w.np, C::BN, px * 2};
    depth = w.np;
  } else if constexpr (KIND == kSquare) {
    L = Operand{A + (int64_t)i0 * w.mp, w.mp, C::BM, pa * 2};
    R = Operand{A + (int64_t)j0 * w.mp, w.mp, C::BN, pa * 2};
    depth = w.mp;
  } else {
    L = Operand{B + (int64_t)i0 * w.mp, w.mp, C::BM, pa * 2};
    R = Operand{X + j0, w.np, C::BN, px * 2};
    depth = w.mp;
  }
  product_tile<C>(L, R, 0, depth, smem, acc);

  // Products carry the scale twice.
  const float back = 1.0f / kScale;
  if constexpr (kSymmetric) {
    uint16_t* const out = KIND == kGram ? A : B;
    const bool mirror = ti != tj;
    product_rows<C>(acc, smem, [&](int m, int n, float (&v)[4]) __attribute__((always_inline)) {
      const int64_t at = (int64_t)(i0 + m) * w.mp + j0 + n;
      if constexpr (KIND == kGram) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] *= back;
      } else {
        float x[4];
        get4<PLANES>(A + at, pa, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(a.b, x[e], a.c * back * v[e]);
      }
      put4<PLANES>(out + at, pa, v);
      if (mirror) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t to = (int64_t)(j0 + n + e) * w.mp + i0 + m;
          const _Float16 hi = (_Float16)v[e];
          out[to] = __builtin_bit_cast(uint16_t, hi);
          if constexpr (PLANES == 2)
            out[pa + to] = __builtin_bit_cast(uint16_t, (_Float16)(v[e] - (float)hi));
        }
      }
    });
  } else if constexpr (KIND == kApply) {
    uint16_t* const out = w.X[1 - from] + z * PLANES * px;
    product_rows<C>(acc, smem, [&](int m, int n, float (&v)[4]) __attribute__((always_inline)) {
      const int64_t at = (int64_t)(i0 + m) * w.np + j0 + n;
      float x[4];
      get4<PLANES>(X + at, px, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(a.a, x[e], back * v[e]);
      put4<PLANES>(out + at, px, v);
    });
  } else {
    const int64_t base = z * a.rows * a.cols;
    product_rows<C>(acc, smem, [&](int m, int n, float (&v)[4]) __attribute__((always_inline)) {
      const int i = i0 + m, j = j0 + n;
      if (i >= w.m || j >= w.n) return;
      float x[4];
      get4<PLANES>(X + (int64_t)i * w.np + j, px, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (j + e >= w.n) break;
        const int64_t at = base + (w.flip ? (int64_t)(j + e) * a.cols + i : (int64_t)i * a.cols + j + e);
        float y = fmaf(a.a, x[e], back * v[e]) * back;
        if (a.weight) y = fmaf(a.decay, read1<BF16>(a.weight, at), -a.rate * y);
        write1<BF16>(a.out, at, y);
      }
    });
  }
}

template <class CR, class CC, bool BF16>
hipError_t iterate(const NewtonLaunch& a, const NewtonWork& w, hipStream_t s) {
  const int T = w.mp / CR::BM, TX = T * (w.np / CC::BN), batch = (int)a.batch;
  int from = 0;
  for (int k = 0; k < a.steps; ++k) {
    hipLaunchKernelGGL((newton_kernel<CR, kGram, BF16>), dim3(T * (T + 1) / 2, batch),
                       dim3(CR::THREADS), 0, s, a, w, from);
    hipLaunchKernelGGL((newton_kernel<CR, kSquare, BF16>), dim3(T * (T + 1) / 2, batch),
                       dim3(CR::THREADS), 0, s, a, w, from);
    if (k + 1 < a.steps)
      hipLaunchKernelGGL((newton_kernel<CC, kApply, BF16>), dim3(TX, batch), dim3(CC::THREADS), 0, s,
                         a, w, from);
    else
      hipLaunchKernelGGL((newton_kernel<CC, kLast, BF16>), dim3(TX, batch), dim3(CC::THREADS), 0, s,
                         a, w, from);
    from = 1 - from;
  }
  return hipGetLastError();
}

inline size_t aligned(size_t v) { return (v + 255) / 256 * 256; }

size_t layout(int64_t batch, int rows, int cols, bool bf16, unsigned char* ws, NewtonWork* w) {
  w->flip = rows > cols;
  w->m = w->flip ? cols : rows;
  w->n = w->flip ? rows : cols;
  w->mp = padded(w->m);
  w->np = padded(w->n);
  const size_t planes = bf16 ? 1 : 2;
  const size_t x = aligned((size_t)batch * planes * w->mp * w->np * 2);
  const size_t g = aligned((size_t)batch * planes * w->mp * w->mp * 2);
  const size_t norms = aligned((size_t)batch * kNormBlocks * sizeof(double));
  w->norms = reinterpret_cast<double*>(ws);
  w->X[0] = reinterpret_cast<uint16_t*>(ws + norms);
  w->X[1] = reinterpret_cast<uint16_t*>(ws + norms + x);
  w->A = reinterpret_cast<uint16_t*>(ws + norms + 2 * x);
  w->B = reinterpret_cast<uint16_t*>(ws + norms + 2 * x + g);
  return norms + 2 * x + 2 * g;
}

template <bool BF16>
hipError_t launch_dtype(const NewtonLaunch& a, const NewtonWork& w, hipStream_t s) {
  constexpr int MODE = BF16 ? kF16 : kF16x2;
  hipLaunchKernelGGL(newton_norm_kernel<BF16>, dim3(kNormBlocks, (unsigned)a.batch), dim3(256), 0, s,
                     a, w);
  hipLaunchKernelGGL(newton_start_kernel<BF16>,
                     dim3((unsigned)(w.np / 64), (unsigned)(w.mp / 64), (unsigned)a.batch), dim3(256),
                     0, s, a, w);
  constexpr int BK = BF16 ? 64 : 32;
  const int64_t tiles = (int64_t)(w.mp / 128) * (w.np / 128) * a.batch;
  if (tiles >= 256)
    return iterate<ProductCfg<MODE, 128, 128, BK, 2, 2, false, false, 2>,
                   ProductCfg<MODE, 128, 128, BK, 2, 2, false, true, 2>, BF16>(a, w, s);
  return iterate<ProductCfg<MODE, 64, 64, 2 * BK, 2, 2, false, false, 2>,
                 ProductCfg<MODE, 64, 64, 2 * BK, 2, 2, false, true, 2>, BF16>(a, w, s);
}

}  // namespace

size_t newton_workspace(int64_t batch, int rows, int cols, bool bf16) {
  NewtonWork w;
  return layout(batch, rows, cols, bf16, nullptr, &w);
}

hipError_t launch_newton(const NewtonLaunch& a, void* workspace, hipStream_t s) {
  if (a.batch <= 0) return hipSuccess;
  ProfileScope prof(kKNewtonSchulz, s);
  NewtonWork w;
  layout(a.batch, a.rows, a.cols, a.bf16, static_cast<unsigned char*>(workspace), &w);
  return a.bf16 ? launch_dtype<true>(a, w, s) : launch_dtype<false>(a, w, s);
}

}  // namespace pinsage
