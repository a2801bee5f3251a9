// One output tile of C[m][n] = sum_k A(m, k) B(n, k), its operands fed through a ring of
// stages in LDS.
//
// Chunks of BK columns of k travel global -> LDS by DMA (no registers, no VALU beside
// one scalar add per chunk), up to STAGES chunks ahead of the MFMAs, with one barrier
// per chunk: where a CU holds one tile a chunk's MFMAs (0.2 us at 128 x 128 x 64) are
// far shorter than a load's latency. AHEAD gives A, the operand that comes from HBM
// where B is a weight that L2 holds, a stage more than B: 8,192 cubed by 256 x 256
// 979 us, with it 900; by 128 x 128 1,425 and 1,217.
// DMAs take whole aligned 16-byte vectors. Operands whose rows are not (REGS) come
// through registers, a chunk held there beside the two in LDS, with loads of any
// alignment; a vector across the end of a row is the one that ends there, shifted.
// A row operand lies in LDS as rows of BK values, 16-byte slot v of row r at
// v ^ swizzle(r); a column operand as it lies in memory, BK rows of BM values. Of
// 16-bit values its fragments come through the transposing LDS read (16 lanes read
// four k rows of 16 m; lane i gets the four k of m = i), slot s of row k at
// s ^ ring_col_swizzle(k); of fp32 as eight 4-byte reads.
// fp32 values are split into their three bf16 parts after the LDS read, among the
// MFMAs of the step before: 7 VALU instructions a value, twice per value and tile
// with 64 x 64 wave tiles, under 8 MFMAs per product, and the least magnitudes are
// kept. A tile of which the parts do not cover some pair of rows (split_covers), or of
// which some sum is not finite, is formed again with fp32 MFMAs: twice a call's time
// when it is all of them (4,096 x 512 -> 512 28 and 49 us, gradients 61 and 92;
// gradients of 100,003 x 256 -> 512 448 and 821).
//
// What bounds large products are the MFMAs, in 63% of the cycles of 8,192 cubed by
// 256 x 256 (counted when it took 943 us; it takes 878), and the clock, which power holds
// at 1.76 GHz of 2.4; the LDS serves fragments in a quarter of the cycles. With every
// tile's operands in L2 the same product takes 11% less. Smaller tiles wait for their
// loads, 64 x 64 at 10 to 12 TB/s out of the L2s in Newton-Schulz. Waves that share a
// tile's k steps, so that smaller tiles keep larger wave tiles, gained 5% at most and are
// not here.
// Where rows end inside a tile, lanes read the last row or vector again (the
// results of those rows are never used); past the end of k they read zeros.
// bf16, 300,000 x 1,024 -> 2,048 by 256 x 256 1,332 us (945 TFLOP/s), the epilogue with
// it; 4,596 x 512 -> 512 by 64 x 64 7.9 us, 511 -> 511 (REGS) 11.9.
#pragma once

#include <type_traits>

#include "product_device.h"

namespace pinsage {

__device__ __attribute__((aligned(16))) const uint32_t g_ring_zero[4] = {0, 0, 0, 0};

template <int MODE_, int BM_, int BN_, int BK_, int WAVES_M_, int WAVES_N_, bool A_COL_,
          bool B_COL_, int STAGES_, int WPE_ = 1, int AHEAD_ = 0, bool REGS_ = false>
struct RingCfg {
  static constexpr int MODE = MODE_, BM = BM_, BN = BN_, BK = BK_, STAGES = STAGES_, WPE = WPE_;
  static constexpr int AHEAD = AHEAD_;  // stages that A has beyond STAGES
  static constexpr int WAVES_M = WAVES_M_, WAVES_N = WAVES_N_;
  static constexpr bool REGS = REGS_;  // chunks go through registers: any alignment
  static constexpr bool A_COL = A_COL_, B_COL = B_COL_;
  static constexpr int NWAVES = WAVES_M * WAVES_N, THREADS = 64 * NWAVES;
  static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, TM = WM / 32, TN = WN / 32;
  static constexpr int ESZ = MODE == kF32 ? 4 : 2;
  static constexpr int A_PLANES = MODE == kF16x2 || MODE == kBf16A2 ? 2 : 1;  // in memory
  static constexpr int B_PLANES = MODE == kF16x2 ? 2 : 1;
  static constexpr int A_PARTS = MODE == kF32 ? 3 : A_PLANES;  // of a fragment
  static constexpr int B_PARTS = MODE == kF32 ? 3 : B_PLANES;
  static constexpr int A_PLANE = BM * BK * ESZ, B_PLANE = BN * BK * ESZ;
  static constexpr int A_BYTES = A_PLANE * A_PLANES, B_BYTES = B_PLANE * B_PLANES;
  static constexpr int STEPS = BK / 16;  // k steps of a chunk
  // One DMA instruction of a wave fills a group of 1 KB.
  static constexpr int A_GROUPS = A_PLANE / 1024, B_GROUPS = B_PLANE / 1024;  // per plane
  static constexpr int DA = A_GROUPS * A_PLANES / NWAVES;  // of a wave, per chunk
  static constexpr int DB = B_GROUPS * B_PLANES / NWAVES;
  static constexpr int PENDING = (STAGES - 2) * (DA + DB) + AHEAD * DA;
  static constexpr int STAGE_LD = WN + 4;
  static constexpr int STAGE_BYTES = 32 * STAGE_LD * 4;
  static constexpr int RING = (STAGES + AHEAD) * A_BYTES + STAGES * B_BYTES;
  // kF32: behind the ring a word a wave, whether it wants the tile again.
  static constexpr int FLAGS = RING > NWAVES * STAGE_BYTES ? RING : NWAVES * STAGE_BYTES;
  static constexpr int LDS_BYTES = FLAGS + (MODE == kF32 ? 4 * NWAVES : 0);
  static_assert(A_GROUPS * A_PLANES % NWAVES == 0 && B_GROUPS * B_PLANES % NWAVES == 0 &&
                    A_GROUPS % DA == 0 && B_GROUPS % DB == 0,
                "every wave serves one plane of each operand");
  static_assert(STAGES >= 2 && PENDING <= 63 && LDS_BYTES <= 160 * 1024, "");
  static_assert((!REGS && MODE != kF32) || AHEAD == 0, "");
  static_assert(BK * ESZ == 64 || BK * ESZ == 128, "rows of 4 or 8 slots");
};

// Slot swizzle of a row operand of `SLOTS` 16-byte slots a row.
template <int SLOTS>
__device__ __forceinline__ int ring_row_swizzle(int r) {
  return product_swizzle<SLOTS * 8>(r);
}
__device__ __forceinline__ int ring_col_swizzle(int k) { return (k & 3) << 1; }

__device__ __forceinline__ void ring_dma(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory");
}
__device__ __forceinline__ void ring_dma_at(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(lds), "v"(p)
               : "memory");
}
template <int N>
__device__ __forceinline__ void ring_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void ring_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

// A pointer that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const unsigned char* ring_uniform(const unsigned char* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const unsigned char*>(((uint64_t)hi << 32) | lo);
}

// f(integral_constant) for FROM .. TO - 1.
template <int FROM, int TO, class F>
__device__ __forceinline__ void unroll(F&& f) {
  if constexpr (FROM < TO) {
    f(std::integral_constant<int, FROM>{});
    unroll<FROM + 1, TO>(f);
  }
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// The tile's products over k in [k0, k1). All of the block's threads call it; smem
// holds C::LDS_BYTES and is free again when it returns (after a barrier). Without
// C::REGS, operands' `p` and `ld` are multiples of 16 bytes, and so are the `valid`
// values of a column operand and the k1 - k0 of a row operand.
template <class C>
__device__ __forceinline__ void tile_sums(const Operand& A, const Operand& B, int64_t k0,
                                          int64_t k1, unsigned char* smem, TileSums<C>& sums) {
  constexpr int BK = C::BK, ESZ = C::ESZ, VE = 16 / ESZ, STAGES = C::STAGES;
  constexpr int STAGES_A = STAGES + C::AHEAD;
  constexpr int SLOTS = BK / VE;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
  sums.row0 = wm * C::WM;
  sums.col0 = wn * C::WN;
  auto& acc = sums.v;
#pragma unroll
  for (int i = 0; i < C::TM; ++i)
#pragma unroll
    for (int j = 0; j < C::TN; ++j) clear_block(acc[i][j]);
  // The products of parts beside the leading one have sums of their own, so that the large
  // ones round once a step (bf16 results need none).
  constexpr bool kApart = C::MODE == kF32 || C::MODE == kF16x2;
  f32x16 small[kApart ? C::TM : 1][C::TN];
  if constexpr (kApart)
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j) clear_block(small[i][j]);
  const int nchunks = __builtin_amdgcn_readfirstlane((int)((k1 - k0 + BK - 1) / BK));
  if (nchunks <= 0) return;
  const uint32_t smem_base =
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)smem;

  // ---- this wave's DMAs --------------------------------------------------------
  constexpr int DA = C::DA, DB = C::DB;
  const int first_a = wave * DA, first_b = wave * DB;  // its groups of a stage
  const unsigned char* base_a =
      static_cast<const unsigned char*>(A.p) + first_a / C::A_GROUPS * A.plane;
  const unsigned char* base_b =
      static_cast<const unsigned char*>(B.p) + first_b / C::B_GROUPS * B.plane;
  uint32_t off[DA + DB];  // from the chunk's base
  int kk[DA + DB];        // the vector's first k within the chunk
  auto place = [&](auto column, int d, int g, int width, const Operand& o)
      __attribute__((always_inline)) {
    if constexpr (decltype(column)::value) {
      const int spr = width / VE, k = g * 64 / spr + lane / spr;
      int m = ((lane % spr) ^ (ESZ == 2 ? ring_col_swizzle(k) : 0)) * VE;
      if constexpr (!C::REGS) m = m < o.valid ? m : o.valid - VE;
      off[d] = ((uint32_t)k * (uint32_t)o.ld + (uint32_t)m) * ESZ;
      kk[d] = k;
    } else {
      const int r = g * (64 / SLOTS) + lane / SLOTS;
      const int v = (lane % SLOTS) ^ ring_row_swizzle<SLOTS>(r);
      off[d] = ((uint32_t)(r < o.valid ? r : o.valid - 1) * (uint32_t)o.ld + (uint32_t)(v * VE)) * ESZ;
      kk[d] = v * VE;
    }
  };
#pragma unroll
  for (int d = 0; d < DA; ++d)
    place(std::bool_constant<C::A_COL>{}, d, first_a % C::A_GROUPS + d, C::BM, A);
#pragma unroll
  for (int d = 0; d < DB; ++d)
    place(std::bool_constant<C::B_COL>{}, DA + d, first_b % C::B_GROUPS + d, C::BN, B);
  const int64_t step_a = (C::A_COL ? A.ld * BK : BK) * ESZ;
  const int64_t step_b = (C::B_COL ? B.ld * BK : BK) * ESZ;
  base_a = ring_uniform(base_a + (C::A_COL ? k0 * A.ld : k0) * ESZ);
  base_b = ring_uniform(base_b + (C::B_COL ? k0 * B.ld : k0) * ESZ);
  const unsigned char* const first_base_a = base_a;
  const unsigned char* const first_base_b = base_b;
  const int whole = __builtin_amdgcn_readfirstlane((int)((k1 - k0) / BK));  // chunks inside k
  const int rest = (int)((k1 - k0) % BK);
  // DMA d of a turn: B's of chunk `turn` and A's of chunk turn + AHEAD, in this order.
  auto issue_one = [&](int turn, auto dma, auto inside) __attribute__((always_inline)) {
    constexpr int d = decltype(dma)::value;
    constexpr bool kOfA = d >= DB;
    constexpr int at = kOfA ? d - DB : DA + d;  // in off and kk
    const int c = kOfA ? turn + C::AHEAD : turn;
    const uint32_t dst = __builtin_amdgcn_readfirstlane(
        smem_base + (kOfA ? (uint32_t)(c % STAGES_A) * C::A_BYTES + (first_a + d - DB) * 1024
                          : STAGES_A * C::A_BYTES + (uint32_t)(c % STAGES) * C::B_BYTES +
                                (first_b + d) * 1024));
    const unsigned char*& base = kOfA ? base_a : base_b;
    if (decltype(inside)::value || c < whole) {
      ring_dma(base, off[at], dst);
      if constexpr (d == DB - 1) base_b += step_b;
      if constexpr (d == DA + DB - 1) base_a += step_a;
    } else {
      // The last part of k, or beyond it: groups of zeros keep the count of loads in
      // flight the same.
      const unsigned char* const zero = reinterpret_cast<const unsigned char*>(g_ring_zero);
      ring_dma_at(kk[at] < (c == whole ? rest : 0) ? base + off[at] : zero, dst);
    }
  };
  auto issue = [&](int turn, auto from, auto to) __attribute__((always_inline)) {
    constexpr int d0 = decltype(from)::value, d1 = decltype(to)::value;
    if constexpr (d0 < d1) {
      if (turn + C::AHEAD < whole)
        unroll<d0, d1>([&](auto d) __attribute__((always_inline)) {
          issue_one(turn, d, std::true_type{});
        });
      else
        unroll<d0, d1>([&](auto d) __attribute__((always_inline)) {
          issue_one(turn, d, std::false_type{});
        });
    }
  };

  // ---- the same through registers ---------------------------------------------------
  // The vector's first m of a column operand: one for all of the lane's.
  auto first_m = [&](int width) __attribute__((always_inline)) {
    const int spr = width / VE;
    return ((lane % spr) ^ (ESZ == 2 ? ring_col_swizzle(lane / spr) : 0)) * VE;
  };
  const int m_a = C::A_COL ? first_m(C::BM) : 0, m_b = C::B_COL ? first_m(C::BN) : 0;
  // Whether the tile has no edge, and a vector of existing elements fits each operand's rows.
  const bool inner = (!C::A_COL || A.valid >= C::BM) && (!C::B_COL || B.valid >= C::BN);
  const bool room = (C::A_COL ? A.before + A.valid : k1 - k0) >= VE &&
                    (C::B_COL ? B.before + B.valid : k1 - k0) >= VE;
  auto fetch = [&](int c, u32x4(&v)[DA + DB]) __attribute__((always_inline)) {
    if (c >= nchunks) return;
    const int left = c < whole ? BK : rest;
    // How many elements of a vector exist.
    auto count = [&](auto dma) __attribute__((always_inline)) {
      constexpr int d = decltype(dma)::value;
      constexpr bool kOfA = d < DA;
      const int have = (kOfA ? C::A_COL : C::B_COL)
                           ? (kk[d] < left ? (kOfA ? A.valid - m_a : B.valid - m_b) : 0)
                           : left - kk[d];
      return have < 0 ? 0 : (have < VE ? have : VE);
    };
    if (c < whole && inner) {
      unroll<0, DA + DB>([&](auto dma) __attribute__((always_inline)) {
        constexpr int d = decltype(dma)::value;
        v[d] = load_any<u32x4>((d < DA ? base_a : base_b) + off[d]);
      });
    } else if (room) {
      // The vector that ends where the elements do, shifted.
      unroll<0, DA + DB>([&](auto dma) __attribute__((always_inline)) {
        constexpr int d = decltype(dma)::value;
        const int have = count(dma);
        const unsigned char* const p = (d < DA ? base_a : base_b) + off[d] - (VE - have) * ESZ;
        const unsigned char* const zero = reinterpret_cast<const unsigned char*>(g_ring_zero);
        v[d] = drop_first<ESZ>(load_any<u32x4>(have ? p : zero), VE - have);
      });
    } else {
      unroll<0, DA + DB>([&](auto dma) __attribute__((always_inline)) {
        constexpr int d = decltype(dma)::value;
        v[d] = load_few<ESZ>((d < DA ? base_a : base_b) + off[d], count(dma));
      });
    }
    base_a += step_a;
    base_b += step_b;
  };
  auto store = [&](int c, const u32x4(&v)[DA + DB]) __attribute__((always_inline)) {
    if (c >= nchunks) return;
    unsigned char* const to_a = smem + (c % STAGES) * C::A_BYTES + first_a * 1024 + lane * 16;
    unsigned char* const to_b =
        smem + STAGES * C::A_BYTES + (c % STAGES) * C::B_BYTES + first_b * 1024 + lane * 16;
    unroll<0, DA + DB>([&](auto dma) __attribute__((always_inline)) {
      constexpr int d = decltype(dma)::value;
      *reinterpret_cast<u32x4*>(d < DA ? to_a + d * 1024 : to_b + (d - DA) * 1024) = v[d];
    });
  };

  // ---- fragments ------------------------------------------------------------------
  const int frag_row = lane & 31, half = lane >> 5;
  struct Frags {
    u32x4 a[C::TM][C::A_PARTS], b[C::TN][C::B_PARTS];
  };
  // Eight k of one row: a vector of 16-bit values, or two of fp32 (in parts 0 and 1).
  auto read_row = [&](const unsigned char* tile, int r, int ks, auto& out)
      __attribute__((always_inline)) {
    const unsigned char* const row = tile + r * (BK * ESZ);
    const int s0 = (2 * ks + half) * (8 / VE), sw = ring_row_swizzle<SLOTS>(r);
    out[0] = *reinterpret_cast<const u32x4*>(row + (s0 ^ sw) * 16);
    if constexpr (ESZ == 4) out[1] = *reinterpret_cast<const u32x4*>(row + ((s0 + 1) ^ sw) * 16);
  };
  // The same of a column operand: with 16-bit values a lane (j, c) of 16 reads k row
  // j's values 4 c .. 4 c + 3, twice for k and k + 4.
  auto read_col = [&](const unsigned char* tile, int m0, int ks, int width, auto& out)
      __attribute__((always_inline)) {
    if constexpr (ESZ == 4) {
      const unsigned char* const at =
          tile + ((16 * ks + 8 * half) * width + m0 + frag_row) * 4;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        out[k >> 2][k & 3] = *reinterpret_cast<const uint32_t*>(at + k * width * 4);
    } else {
      const int m = m0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = 16 * ks + 8 * half + 4 * h + ((lane >> 2) & 3);
        const unsigned char* const at =
            tile + k * (width * 2) + (((m >> 3) ^ ring_col_swizzle(k)) * 16) + (m & 4) * 2;
        const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)at);
        const u32x2 x = __builtin_bit_cast(u32x2, w);
        out[0][2 * h] = x[0];
        out[0][2 * h + 1] = x[1];
      }
    }
  };
  // Fragment q of step ks of chunk c, of A's TM and B's TN.
  auto read_one = [&](int c, int ks, Frags& f, auto frag) __attribute__((always_inline)) {
    constexpr int q = decltype(frag)::value;
    constexpr bool kOfA = q < C::TM, COL = kOfA ? C::A_COL : C::B_COL;
    constexpr int width = kOfA ? C::BM : C::BN;
    const unsigned char* const tile = kOfA ? smem + (c % STAGES_A) * C::A_BYTES
                                           : smem + STAGES_A * C::A_BYTES + (c % STAGES) * C::B_BYTES;
    const int m = kOfA ? wm * C::WM + 32 * q : wn * C::WN + 32 * (q - C::TM);
    auto take = [&](auto& out) __attribute__((always_inline)) {
      constexpr int PLANES = kOfA ? C::A_PLANES : C::B_PLANES;
      unroll<0, PLANES>([&](auto plane) __attribute__((always_inline)) {
        constexpr int p = decltype(plane)::value;
        const unsigned char* const from = tile + p * (kOfA ? C::A_PLANE : C::B_PLANE);
        if constexpr (PLANES == 1) {
          if constexpr (COL) read_col(from, m, ks, width, out);
          else read_row(from, m + frag_row, ks, out);
        } else {
          u32x4 x[1];
          if constexpr (COL) read_col(from, m, ks, width, x);
          else read_row(from, m + frag_row, ks, x);
          out[p] = x[0];
        }
      });
    };
    if constexpr (kOfA) take(f.a[q]);
    else take(f.b[q - C::TM]);
  };
  constexpr int FRAGS = C::TM + C::TN;
  auto read = [&](int c, int ks, Frags& f) __attribute__((always_inline)) {
    unroll<0, FRAGS>([&](auto q) __attribute__((always_inline)) { read_one(c, ks, f, q); });
  };
  // kF32: the least magnitudes of the values this lane has split.
  uint32_t key_a = ~0u, key_b = ~0u;
  auto split = [&](Frags& f) __attribute__((always_inline)) {
    if constexpr (ESZ == 4) {
#pragma unroll
      for (int i = 0; i < C::TM; ++i) {
        const Split3 s = split3(f.a[i][0], f.a[i][1], key_a);
#pragma unroll
        for (int p = 0; p < 3; ++p) f.a[i][p] = s.p[p];
      }
#pragma unroll
      for (int j = 0; j < C::TN; ++j) {
        const Split3 s = split3(f.b[j][0], f.b[j][1], key_b);
#pragma unroll
        for (int p = 0; p < 3; ++p) f.b[j][p] = s.p[p];
      }
    }
  };
  // A step: its products, the fragment reads of the next one (step ks of chunk c) and
  // DMAs from .. to - 1 of a turn. With four MFMAs or more a step, reads and DMAs go one
  // at a time among them, for in bursts they hold the wave, and its MFMAs, until the LDS
  // and the address path, which all waves want at once, have taken them (bf16, 8,192
  // cubed by 256 x 256: 1,005 us, the DMAs spread 979; with A a stage ahead 900, the
  // reads spread too 878. By 64 x 64, one MFMA a step, it loses: 1,024 x 1,024 x 2,048
  // 11.0 us, spread 15.0).
  // The last of split_device.h's products: all of them, (1,0) (0,1) (0,0), the last two or
  // (0,0).
  constexpr int PRODUCTS = C::MODE == kF32 ? kSplitProducts : C::A_PARTS + C::B_PARTS - 1;
  constexpr int ALL = PRODUCTS * C::TM * C::TN;
  constexpr bool kSpread = ESZ == 2 && ALL >= 4;
  auto work = [&](const Frags& cur, Frags& nxt, int c, int ks, int turn, auto from, auto to)
      __attribute__((always_inline)) {
    constexpr int D0 = decltype(from)::value, DMAS = decltype(to)::value - D0;
    if constexpr (!kSpread) {
      read(c, ks, nxt);
      __builtin_amdgcn_sched_barrier(0);
      issue(turn, from, to);
      __builtin_amdgcn_sched_barrier(0);
      split(nxt);
    }
    unroll<0, ALL>([&](auto at) __attribute__((always_inline)) {
      constexpr int e = decltype(at)::value, q = e / (C::TM * C::TN), i = e / C::TN % C::TM,
                    j = e % C::TN;
      constexpr int t = kSplitProducts - PRODUCTS + q, pb = split_b(t), pa = split_a(t);
      f32x16& sum = kApart && q < PRODUCTS - 1 ? small[kApart ? i : 0][j] : acc[i][j];
      sum = product_mfma<C::MODE>(cur.b[j][pb], cur.a[i][pa], sum);
      if constexpr (kSpread) {
        constexpr int r0 = (e * FRAGS + ALL - 1) / ALL, r1 = ((e + 1) * FRAGS + ALL - 1) / ALL;
        constexpr int d0 = e * DMAS / ALL, d1 = (e + 1) * DMAS / ALL;
        __builtin_amdgcn_sched_barrier(0);
        unroll<r0, r1>([&](auto q) __attribute__((always_inline)) { read_one(c, ks, nxt, q); });
        issue(turn, std::integral_constant<int, D0 + d0>{}, std::integral_constant<int, D0 + d1>{});
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    if constexpr (ESZ == 4) {
      // The splitting among the products.
      constexpr int kValu = 56 * FRAGS;
#pragma unroll
      for (int q = 0; q < ALL; ++q) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                        // MFMA
        __builtin_amdgcn_sched_group_barrier(0x002, (kValu + ALL - 1) / ALL, 0);  // VALU
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  // A chunk is waited for (STAGES - 2 younger ones may stay in flight) and the barrier
  // shows everybody's and frees the chunk before, whose stage takes chunk c + STAGES:
  // half of its DMAs go out in the last step of chunk c, whose MFMAs follow that
  // barrier, over the first fragment reads of the next chunk, and half in the next step.
  using None = std::integral_constant<int, 0>;
  using Half = std::integral_constant<int, kSpread ? (DA + DB) / 2 : DA + DB>;
  using Every = std::integral_constant<int, DA + DB>;
  u32x4 held[DA + DB];  // REGS: chunk c + STAGES, until chunk c's stage is free
  if constexpr (C::REGS) {
    u32x4 first[STAGES][DA + DB];
#pragma unroll
    for (int c = 0; c < STAGES; ++c) fetch(c, first[c]);
    fetch(STAGES, held);
#pragma unroll
    for (int c = 0; c < STAGES; ++c) store(c, first[c]);
    ring_barrier();
  } else {
#pragma unroll
    for (int c = -C::AHEAD; c < 0; ++c) issue(c, std::integral_constant<int, DB>{}, Every{});
#pragma unroll
    for (int c = 0; c < STAGES - 1; ++c) issue(c, None{}, Every{});
    ring_wait<C::PENDING>();
    ring_barrier();
    issue(STAGES - 1, None{}, Half{});
  }
  Frags f[2];
  read(0, 0, f[0]);
  split(f[0]);
  auto chunk = [&](int c, auto parity) __attribute__((always_inline)) {
    constexpr int P = decltype(parity)::value;
    unroll<0, C::STEPS - 1>([&](auto step) __attribute__((always_inline)) {
      constexpr int s = decltype(step)::value;
      Frags &cur = f[(P + s) & 1], &nxt = f[(P + s + 1) & 1];
      if constexpr (s == 0 && !C::REGS) work(cur, nxt, c, s + 1, c + STAGES - 1, Half{}, Every{});
      else work(cur, nxt, c, s + 1, 0, None{}, None{});
    });
    if constexpr (!C::REGS) ring_wait<C::PENDING>();
    ring_barrier();
    // Past the last chunk what is read is not used (zeros, with REGS anything).
    Frags &cur = f[(P + C::STEPS - 1) & 1], &nxt = f[(P + C::STEPS) & 1];
    if constexpr (C::REGS) {
      const uint32_t had_a = key_a, had_b = key_b;
      work(cur, nxt, c + 1, 0, 0, None{}, None{});
      if (c + 1 >= nchunks) {
        key_a = had_a;
        key_b = had_b;
      }
      store(c + STAGES, held);
      fetch(c + STAGES + 1, held);
    } else {
      work(cur, nxt, c + 1, 0, c + STAGES, None{}, Half{});
    }
  };
  using Even = std::integral_constant<int, 0>;
  using Odd = std::integral_constant<int, 1>;
  int c = 0;
  if constexpr (C::STEPS % 2) {
#pragma unroll 1
    for (; c + 1 < nchunks; c += 2) {
      chunk(c, Even{});
      chunk(c + 1, Odd{});
    }
    if (c < nchunks) chunk(c, Even{});
  } else {
#pragma unroll 1
    for (; c < nchunks; ++c) chunk(c, Even{});
  }
  if constexpr (!C::REGS) ring_wait<0>();
  bool covered = true;
  if constexpr (kApart)
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j) acc[i][j] += small[i][j];
  if constexpr (C::MODE == kF32) {
    // Infinities, NaN and values or sums that round to an infinity show in the results.
    float probe = 0.0f;
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) probe = fmaf(acc[i][j][e], 0.0f, probe);
    covered = split_covers(wave_min_key(key_a), wave_min_key(key_b)) &&
              __ballot(probe != 0.0f) == 0ull;
    if (lane == 0) reinterpret_cast<uint32_t*>(smem + C::FLAGS)[wave] = !covered;
  }
  __syncthreads();
  if constexpr (C::MODE == kF32) {
    uint32_t again = 0;
#pragma unroll
    for (int w = 0; w < C::NWAVES; ++w) again |= reinterpret_cast<const uint32_t*>(smem + C::FLAGS)[w];
    if (again) {
      // The tile again with fp32 MFMAs (operand q of a step pairs half-wave h with its
      // column 8 h + q), a chunk in flight. Each element then follows from its own row
      // and column alone: split where those are covered and the sum is finite, else fp32,
      // so that it does not depend on the tile it lies in.
      f32x16 full[C::TM][C::TN];
      uint32_t least_a[C::TM], least_b[C::TN];
#pragma unroll
      for (int i = 0; i < C::TM; ++i) least_a[i] = ~0u;
#pragma unroll
      for (int j = 0; j < C::TN; ++j) least_b[j] = ~0u;
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j) clear_block(full[i][j]);
      base_a = first_base_a;
      base_b = first_base_b;
      if constexpr (C::REGS) fetch(0, held);
      else issue(0, None{}, Every{});
#pragma unroll 1
      for (int c = 0; c < nchunks; ++c) {
        if constexpr (C::REGS) {
          store(c, held);
          fetch(c + 1, held);
          ring_barrier();
        } else {
          ring_wait<0>();
          ring_barrier();
          if (c + 1 < nchunks) issue(c + 1, None{}, Every{});
        }
        if (covered) continue;  // the wave only loads
#pragma unroll
        for (int ks = 0; ks < C::STEPS; ++ks) {
          read(c, ks, f[0]);
#pragma unroll
          for (int i = 0; i < C::TM; ++i)
            least_a[i] = least_key(f[0].a[i][0], f[0].a[i][1], least_a[i]);
#pragma unroll
          for (int j = 0; j < C::TN; ++j)
            least_b[j] = least_key(f[0].b[j][0], f[0].b[j][1], least_b[j]);
#pragma unroll
          for (int q = 0; q < 8; ++q)
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
              for (int j = 0; j < C::TN; ++j)
                full[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(
                    __uint_as_float(f[0].b[j][q >> 2][q & 3]),
                    __uint_as_float(f[0].a[i][q >> 2][q & 3]), full[i][j], 0, 0, 0);
        }
      }
      if (!covered) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
          least_a[i] = umin(least_a[i], (uint32_t)__shfl_xor((int)least_a[i], 32));
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
          least_b[j] = umin(least_b[j], (uint32_t)__shfl_xor((int)least_b[j], 32));
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            // A lane's row of block i; its element e's column is this lane's of the fragment.
            const uint32_t kb =
                (uint32_t)__shfl((int)least_b[j], 8 * (e >> 2) + 4 * half + (e & 3));
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
            {
              const float x = acc[i][j][e];
              acc[i][j][e] =
                  split_covers(least_a[i], kb) && fabsf(x) < INFINITY ? x : full[i][j][e];
            }
          }
        }
      }
      __syncthreads();  // the ring is free for the epilogue
    }
  }
}

}  // namespace pinsage
