// Matrix products whose operands lie either way round in memory, on MFMA:
//   C[m, n] = sum over k of A(m, k) B(n, k)
// The passes of a trained layer are all of this form: the outputs take x [R, K] and
// W [N, K], both with the contraction along their rows; the input's gradient takes
// dy [R, N] and W, whose contraction goes down its columns; the weight's gradient takes
// dy and x, where it goes down both.  Nothing is transposed in memory:
//   - A stage of 128 bytes of the contraction (64 bf16, 32 fp32) of both operands moves
//     to LDS by direct loads of 16 bytes a lane, as it lies in memory: rows of 128 bytes
//     along the contraction, or one row of the tile's width for each of its steps.
//   - Operands of the first kind are read back 16 bytes a lane.  Of the second kind bf16
//     goes through the transposing read of gfx950 (ds_read_tr16: 16 lanes read four
//     steps of 16 columns and each gets its column's four), fp32 word by word.
//   - The places of a row's 16 bytes are permuted by the row's number, so that the rows
//     that one read touches lie in different banks.  Direct loads fill LDS in lane
//     order: it is their source that is permuted.
//   - The contraction goes by halves of a stage.  Operands along it lie in a ring of whole
//     stages (their rows are whole cache lines), operands down it in a ring of halves, whose
//     new rows at every half come from other pages and take the longer to arrive: with two
//     whole stages, one under way, 8192 x 4096 x 4096 took 476 us for the weight's gradient
//     and 249 for the input's (209 and 211 now, 1.3 PFLOP/s, the matrix cores 63 % busy).
//   - Each wave has the next half's operands on their way to registers while it multiplies
//     this one's; one barrier for each piece of a ring that is freed and filled again.
// Contractions are cut in parts of whole stages where there are too few tiles to fill the chip:
// each part writes its sums in fp32 to the workspace, and a last launch adds them in order.
#pragma once

#include <algorithm>

#include "act_device.h"
#include "gl_kernels.h"
#include "product_ring.h"
#include "row_device.h"

namespace gl {

enum { kProductStore = 0, kProductPart = 1, kProductGated = 2, kProductGatedPart = 3 };  // what becomes of the sums

struct ProductArgs {
  const void *A, *B;
  long long lda, ldb;  // bytes from row to row, at most 2^22
  int M, N, K;         // K: of the contraction, in elements; whole 16 bytes where it lies along rows
  int cols_a, cols_b;  // 16-byte places of a row, where the contraction goes down the columns
  void* out;           // [M, N], or h [M, N] of the gated layer, whose B has 2 N rows
  float* part;         // [parts, M, N], gated [parts, M, 2 N]
  int parts;           // of the contraction, whole stages each
  const void* bias;    // [2 N] or null (gated)
  void* pre;           // [M, 2 N] or null (gated)
  int act;             // gl_act (gated)
};

// DT 1: bf16, 0: fp32.  KA, KB: the operand's contraction goes down its columns.  Rings: two
// stages where both lie along it; else three, and four halves of the other, or five halves of
// both, within 160 KB for the workgroups of a CU.
template <int DT_, bool KA_, bool KB_, int BM_, int BN_, int WR_, int WC_>
struct ProductCfg {
  static constexpr int DT = DT_, BM = BM_, BN = BN_, WR = WR_, WC = WC_;
  static constexpr bool KA = KA_, KB = KB_;
  static constexpr int ES = DT ? 2 : 4, HALF = 64 / ES;  // contraction of half a stage
  static constexpr int kWaves = WR * WC, kThreads = 64 * kWaves;
  static constexpr int RA = product_ring_depth(KA, KB), RB = product_ring_depth(KB, KA);
  static constexpr int kPieceA = BM * (KA ? 64 : 128), kPieceB = BN * (KB ? 64 : 128);
  static constexpr int kPlaceB = RA * kPieceA;  // of the second operand's ring
  static constexpr int TM = BM / WR / 16, TN = BN / WC / 16;
  static constexpr int WROWS = 16 * TM, WCOLS = 16 * TN;
  static constexpr size_t kSmem = (size_t)RA * kPieceA + RB * kPieceB;
  // rows of the wave's tile that its share of LDS holds in fp32
  static constexpr int kShare = (int)kSmem / kWaves;
  static constexpr int ER = kShare >= WROWS * WCOLS * 4 ? WROWS : kShare >= WROWS * WCOLS * 2 ? WROWS / 2 : WROWS / 4;
  static_assert(kShare >= ER * WCOLS * 4 && ER % 16 == 0 && kSmem <= 163840, "the epilogue's rows fit");
};

// A direct load from a uniform base and 32 bits a lane.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_dma16_at(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// All but the last N of this wave's direct loads have landed and its LDS reads are done; then
// the workgroup's barrier.
template <int N>
__device__ __forceinline__ void dma_wait_barrier() {
  static_assert(N >= 0 && N < 64, "the counter has six bits");
  // vmcnt(N) expcnt(7) lgkmcnt(0) as the instruction's number
  asm volatile("s_waitcnt %0\n\ts_barrier" ::"i"((N & 15) | (N >> 4) << 14 | 7 << 4) : "memory");
}

// One operand's pieces: ROWS rows of outputs by half a stage (KO) or a stage.
// DUAL > 0: of each DUAL rows the second half lies `up` bytes from the first.
template <int DT, bool KO, int ROWS, int WAVES, int DUAL = 0>
struct Staged {
  static constexpr int ES = DT ? 2 : 4, RB = ROWS * ES, BK = (KO ? 64 : 128) / ES, NL = ROWS * BK * ES / 1024 / WAVES;
  static_assert(NL >= 1 && NL * WAVES * 1024 == ROWS * BK * ES && (!KO || 1024 % RB == 0), "whole loads, of whole rows");
  // The permutation of the 16-byte places of contraction row k (KO).  A read of half a wave
  // touches, bf16, 32 bytes of each of rows 8 g + 0 .. 3 for two g, fp32 64 bytes of rows
  // 4 g + j; rows of 128 bytes lie two to a line of all banks.
  __device__ __forceinline__ static int swap(int k) {
    if (!DT) return ((k >> 2) & 3) << 2;
    return RB >= 256 ? ((k & 3) | ((k >> 3) & 1) << 2) << 1 : (((k >> 1) & 1) | ((k >> 3) & 1) << 1) << 1;
  }
  const char* base;   // of the first piece
  uint32_t off[NL];   // the lane's places from it
  long long advance;  // bytes from piece to piece
  long long up = 0;
  int wave;
  int k_of;           // KO: the first load's contraction row; else its place in the 128 bytes

  // row(r): bytes to the operand's row r of the tile (!KO); first, cols: the tile's first
  // 16-byte place and the places there are (KO)
  template <class Row>
  __device__ __forceinline__ void init(const void* p, long long ld, int w, int lane, int first, int cols, Row row) {
    base = static_cast<const char*>(p);
    wave = w;
    advance = KO ? ld * BK : 128;
    k_of = KO ? (w * 1024 + lane * 16) / RB : ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int q = w + WAVES * i;
      if (KO) {
        const int k = (q * 1024 + lane * 16) / RB, slot = (q * 1024 + lane * 16) % RB / 16;
        off[i] = (uint32_t)k * (uint32_t)ld + (uint32_t)min(first + (slot ^ swap(k)), cols - 1) * 16u;
      } else {
        const int r = 8 * q + (lane >> 3);  // r & 7 is lane >> 3
        off[i] = row(r) + k_of;
      }
    }
  }
  // piece s to LDS; what is past the contraction's end is zero
  __device__ __forceinline__ void load(int s, int K, uint32_t lds) const {
    // (whole loads of eight rows lie in either half)
    auto from = [&](int i) {
      return base + s * advance + (DUAL && 8 * (wave + WAVES * i) % (DUAL ? DUAL : 1) >= DUAL / 2 ? up : 0);
    };
    if ((s + 1) * BK <= K) {
#pragma unroll
      for (int i = 0; i < NL; ++i) lds_dma16_at(from(i), off[i], lds + WAVES * i * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const bool in = KO ? s * BK + k_of + WAVES * i * (1024 / RB) < K : s * 128 + k_of < ((K * ES + 15) & ~15);
        lds_dma16(in ? from(i) + off[i] : reinterpret_cast<const char*>(kZero16), lds + WAVES * i * 1024);
      }
    }
  }
};

// A wave's operand registers: tile `blk` of 16 rows of the piece at `st` (!KO: its half kk).
typedef short s16x4 __attribute__((ext_vector_type(4)));
template <int DT, bool KO, int ROWS>
struct Fragment {
  static constexpr int ES = DT ? 2 : 4, RB = ROWS * ES;
  // where the lane reads of block 0 (KO: without the block's permuted place)
  __device__ __forceinline__ static int lane_base(int g, int t) {
    if (!KO) return t * 128;
    return DT ? (8 * g + (t >> 2)) * RB + 8 * (t & 3) : 4 * g * RB + t * 4;
  }
  __device__ __forceinline__ static int lane_swap(int g, int t) {
    if (!KO) return 0;
    if (!DT) return g;
    return RB >= 256 ? (t >> 2) | (g & 1) << 2 : ((t >> 3) & 1) | (g & 1) << 1;
  }
  __device__ __forceinline__ static uint4 read(const char* st, int base, int swap, int blk, int kk, int g, int t) {
    if (!KO) return *reinterpret_cast<const uint4*>(st + base + blk * 2048 + ((kk * 4 + g) ^ (t & 7)) * 16);
    if (DT) {
      using P = __attribute__((address_space(3))) s16x4*;
      const char* p = st + base + ((blk ^ swap) << 5);
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 4 * RB));
      const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
      return make_uint4(x.x, x.y, y.x, y.y);
    }
    const char* p = st + base + ((blk ^ swap) << 6);
    auto word = [&](int j) { return *reinterpret_cast<const uint32_t*>(p + j * RB); };
    return make_uint4(word(0), word(1), word(2), word(3));
  }
};

template <int DT>
__device__ __forceinline__ f32x4 product_mma(const uint4& b, const uint4& a, f32x4 acc) {
  if (DT) return mfma_bf16(b, a, acc);
  acc = mfma_f32(__uint_as_float(b.x), __uint_as_float(a.x), acc);
  acc = mfma_f32(__uint_as_float(b.y), __uint_as_float(a.y), acc);
  acc = mfma_f32(__uint_as_float(b.z), __uint_as_float(a.z), acc);
  return mfma_f32(__uint_as_float(b.w), __uint_as_float(a.w), acc);
}

// Lane (g, t) of MFMA tile (i, j) holds columns 4g .. 4g+3 of row t.  ER rows at a time the
// wave writes its tile to its own part of LDS in fp32 (16-byte places permuted by the row) and
// reads it back in rows, 16 bytes of output a lane.
template <class G, int EPI>
__device__ __forceinline__ void product_epilogue(const ProductArgs& a, char* smem, const f32x4 (&acc)[G::TM][G::TN], int m0,
                                                 int n0, int part) {
  constexpr int DT = G::DT, TN = G::TN;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, t = lane & 15, wm = w / G::WC, wn = w % G::WC;
  using T = Chunk<DT>;
  constexpr bool GATED = EPI == kProductGated || EPI == kProductGatedPart;
  constexpr int E = EPI == kProductPart || EPI == kProductGatedPart ? 4 : T::E;
  constexpr int COLS = GATED ? G::WCOLS / 2 : G::WCOLS;
  constexpr int LPR = COLS / E, RPP = 64 / LPR, ER = G::ER, CSW = G::WCOLS / 4 < 16 ? G::WCOLS / 4 - 1 : 15;
  static_assert(ER % RPP == 0 || RPP % ER == 0, "whole passes, or one");
  const int cq = lane % LPR, rq = lane / LPR;
  const int n = n0 + wn * COLS + cq * E;
  float bias[2][EPI == kProductGated ? E : 1] = {};
  if (EPI == kProductGated && a.bias) {
#pragma unroll
    for (int v = 0; v < E; ++v) {
      bias[0][v] = T::load1(a.bias, min(n + v, a.N - 1));
      bias[1][v] = T::load1(a.bias, a.N + min(n + v, a.N - 1));
    }
  }
  char* st = smem + w * G::kShare;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < G::WROWS / ER; ++e) {
    if (e) __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront"), __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < ER / 16; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        *reinterpret_cast<f32x4*>(st + (i * 16 + t) * (G::WCOLS * 4) + (((j * 4 + g) ^ (t & CSW)) * 16)) =
            acc[e * (ER / 16) + i][j];
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int p = 0; p < (ER + RPP - 1) / RPP; ++p) {
      const int r = p * RPP + (RPP > ER ? rq % ER : rq), row = m0 + wm * G::WROWS + e * ER + r;
      const char* sr = st + r * (G::WCOLS * 4);
      auto from = [&](int col, float* y) {  // E sums from column `col` of the wave's tile
#pragma unroll
        for (int v = 0; v < E; v += 4) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(sr + (((col + v) / 4) ^ (r & CSW)) * 16);
          y[v] = x[0], y[v + 1] = x[1], y[v + 2] = x[2], y[v + 3] = x[3];
        }
      };
      auto put = [&](void* out, size_t at, const float* y) {
        if (n + E <= a.N) {
          T::store(out, at, y);
        } else {
#pragma unroll
          for (int v = 0; v < E; ++v)
            if (n + v < a.N) T::store1(out, at + v, y[v]);
        }
      };
      if (row >= a.M || n >= a.N || (RPP > ER && rq >= ER)) continue;
      float y[E];
      from(cq * E, y);
      if (EPI == kProductStore) {
        put(a.out, (size_t)row * a.N + n, y);
      } else if (EPI == kProductPart || EPI == kProductGatedPart) {
        auto sums = [&](float* o) {
          if (n + E <= a.N) {
            Chunk<0>::store(o, 0, y);
          } else {
#pragma unroll
            for (int v = 0; v < E; ++v)
              if (n + v < a.N) o[v] = y[v];
          }
        };
        float* o = a.part + ((size_t)part * a.M + row) * (GATED ? 2 * (size_t)a.N : a.N) + n;
        sums(o);
        if (GATED) {
          from(COLS + cq * E, y);
          sums(o + a.N);
        }
      } else {
        float u[E];
        from(COLS + cq * E, u);
#pragma unroll
        for (int v = 0; v < E; ++v) y[v] += bias[0][v], u[v] += bias[1][v];
        if (a.pre) {
          put(a.pre, (size_t)row * 2 * a.N + n, y);
          put(a.pre, (size_t)row * 2 * a.N + a.N + n, u);
        }
        gate_acts<DT>(a.act, y);
#pragma unroll
        for (int v = 0; v < E; ++v) y[v] *= u[v];
        put(a.out, (size_t)row * a.N + n, y);
      }
    }
  }
}

// Workgroup `id` of `count` of a product.  EPI: kProductGated or kProductStore, which write
// parts where there are several.
template <class G, int EPI>
__device__ __forceinline__ void product_tile(const ProductArgs& a, char* smem, int id, int count) {
  constexpr int DT = G::DT, ES = G::ES, TM = G::TM, TN = G::TN, BM = G::BM, BN = G::BN;
  constexpr int OUT = EPI == kProductGated ? BN / 2 : BN;  // output columns of a tile
  const int ntm = (a.M + BM - 1) / BM, ntn = (a.N + OUT - 1) / OUT;
  // tiles by bands of eight rows of them, so that what an XCD's workgroups share is in its L2
  int blk = xcd_remap(id, count), part = 0;
  if (a.parts > 1) {
    part = blk / (ntm * ntn);
    blk -= part * ntm * ntn;
  }
  constexpr int BAND = 8;
  const int band = blk / (BAND * ntn), in = blk - band * BAND * ntn, high = min(BAND, ntm - band * BAND);
  const int nt = in / high, mt = band * BAND + in - nt * high;
  const int m0 = mt * BM, n0 = nt * OUT;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, t = lane & 15;
  const int wm = w / G::WC, wn = w % G::WC;

  // halves h0 .. h1 of the contraction, whole stages (the last half may be all zeros)
  const long long stages = (a.K + 2 * G::HALF - 1) / (2 * G::HALF);
  int h0 = 0, h1 = 2 * (int)stages;
  if (a.parts > 1) {
    h0 = 2 * (int)(stages * part / a.parts);
    h1 = 2 * (int)(stages * (part + 1) / a.parts);
  }

  Staged<DT, G::KA, BM, G::kWaves> la;
  Staged<DT, G::KB, BN, G::kWaves, EPI == kProductGated ? G::WCOLS : 0> lb;
  // rows past the last repeat it; what they give is not stored
  la.init(static_cast<const char*>(a.A) + (G::KA ? 0 : (long long)m0 * a.lda), a.lda, w, lane, m0 * ES / 16, a.cols_a,
          [&](int r) { return (uint32_t)min(r, a.M - 1 - m0) * (uint32_t)a.lda; });
  if (EPI == kProductGated) {
    // a wave's columns: as many of the gate, then the same ones of the other product
    constexpr int H = G::WCOLS / 2;
    lb.up = (long long)a.N * a.ldb;
    lb.init(static_cast<const char*>(a.B) + (long long)n0 * a.ldb, a.ldb, w, lane, 0, 0, [&](int r) {
      const int f = r / G::WCOLS * H + r % H;
      return (uint32_t)min(f, a.N - 1 - n0) * (uint32_t)a.ldb;
    });
  } else {
    lb.init(static_cast<const char*>(a.B) + (G::KB ? 0 : (long long)n0 * a.ldb), a.ldb, w, lane, n0 * ES / 16, a.cols_b,
            [&](int r) { return (uint32_t)min(r, a.N - 1 - n0) * (uint32_t)a.ldb; });
  }
  f32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  using FA = Fragment<DT, G::KA, BM>;
  using FB = Fragment<DT, G::KB, BN>;
  const int abase = FA::lane_base(g, t) + (G::KA ? 0 : wm * G::WROWS * 128), aswap = FA::lane_swap(g, t);
  const int bbase = FB::lane_base(g, t) + (G::KB ? 0 : wn * G::WCOLS * 128), bswap = FB::lane_swap(g, t);
  const int ablk = G::KA ? wm * TM : 0, bblk = G::KB ? wn * TN : 0;
  auto multiply = [&](const uint4* af, const uint4* bf) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = product_mma<DT>(bf[j], af[i], acc[i][j]);
  };
  const uint32_t lds0 = lds_offset(smem) + w * 1024;
  auto read = [&](uint32_t qa, uint32_t qb, int kk, uint4* af, uint4* bf) {
#pragma unroll
    for (int j = 0; j < TN; ++j) bf[j] = FB::read(smem + G::kPlaceB + qb, bbase, bswap, bblk + j, kk, g, t);
#pragma unroll
    for (int i = 0; i < TM; ++i) af[i] = FA::read(smem + qa, abase, aswap, ablk + i, kk, g, t);
  };
  // a half's reads among the multiplications before it, not ahead of them all
  auto mix = [&] {
    constexpr int reads = TM * (G::KA ? (DT ? 2 : 4) : 1) + TN * (G::KB ? (DT ? 2 : 4) : 1), mmas = TM * TN * (DT ? 1 : 4);
    constexpr int each = mmas / reads > 0 ? mmas / reads : 1, n = reads < mmas ? reads : mmas;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, each, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, (reads + n - 1) / n, 0);
    }
  };
  uint4 a0[TM], b0[TN], a1[TM], b1[TN];
  using Ring = ProductRing<G::KA, G::KB, decltype(la)::NL, decltype(lb)::NL, G::kPieceA, G::kPieceB>;
  Ring::run(
      h0, h1, [&](int piece, uint32_t at) { la.load(piece, a.K, lds0 + at); },
      [&](int piece, uint32_t at) { lb.load(piece, a.K, lds0 + G::kPlaceB + at); },
      [&](auto n) { dma_wait_barrier<decltype(n)::value>(); }, [&] { dma_wait_barrier(); },
      [&](auto set, uint32_t qa, uint32_t qb) {
        if constexpr (decltype(set)::value) read(qa, qb, 1, a1, b1);
        else read(qa, qb, 0, a0, b0);
      },
      [&](auto set) {
        if constexpr (decltype(set)::value) multiply(a1, b1);
        else multiply(a0, b0);
        mix();
      });

  if (EPI == kProductGated) {
    if (a.parts > 1) product_epilogue<G, kProductGatedPart>(a, smem, acc, m0, n0, part);
    else product_epilogue<G, kProductGated>(a, smem, acc, m0, n0, 0);
  } else if (a.parts > 1)
    product_epilogue<G, kProductPart>(a, smem, acc, m0, n0, part);
  else
    product_epilogue<G, kProductStore>(a, smem, acc, m0, n0, 0);
}

// Two products in one launch, of which either may be missing: x's gradient, whose first
// operand lies along the contraction, and the weight's, whose both lie across it.  They need
// nothing of each other, and fill the chip together where neither does alone.
struct ProductPair {
  ProductArgs dx, dW;
  int dx_count, dW_count;  // workgroups
  int dW_first;            // the one with the longer workgroups goes first
};

template <int DT, int TILE>
struct PairCfg {
  static constexpr int WR = 2, WC = TILE == 256 ? 4 : 2;
  using X = ProductCfg<DT, false, true, TILE, TILE, WR, WC>;
  using W = ProductCfg<DT, true, true, TILE, TILE, WR, WC>;
  static constexpr int kThreads = X::kThreads;
  static_assert(X::kSmem == W::kSmem && kThreads == W::kThreads, "one launch");
};

template <class P>
__global__ __launch_bounds__(P::kThreads) __attribute__((amdgpu_waves_per_eu(2))) void product_pair_kernel(ProductPair p) {
  extern __shared__ __align__(16) char smem[];
  // (the second one's workgroups begin with a whole round of the XCDs)
  const int before = ((p.dW_first ? p.dW_count : p.dx_count) + 7) & ~7, id = blockIdx.x;
  const bool second = id >= before;
  if (second == (p.dW_first != 0)) {
    const int i = second ? id - before : id;
    if (i < p.dx_count) product_tile<typename P::X, kProductStore>(p.dx, smem, i, p.dx_count);
  } else {
    const int i = second ? id - before : id;
    if (i < p.dW_count) product_tile<typename P::W, kProductStore>(p.dW, smem, i, p.dW_count);
  }
}

template <class G>
__global__ __launch_bounds__(G::kThreads) __attribute__((amdgpu_waves_per_eu(2))) void product_gated_kernel(ProductArgs a) {
  extern __shared__ __align__(16) char smem[];
  product_tile<G, kProductGated>(a, smem, blockIdx.x, gridDim.x);
}

// How products are cut: the tile (256, 128, 64 or 32 outputs each way) and the parts of their
// contractions, by an estimate of the time in us.  Workgroups of 128 and 64 lie two and four
// to a CU: a stage takes them a + b n, n of them, and a round of workgroups 1 to 4.5 us more
// (its first stage's trip, its stores); parts cost a launch and their sums' way through
// memory.  Measured, us (tile, parts), bf16:
//                                  256        128        128, parts  64
//   dx 16384 x 2048 x 8192         428        502                    1200
//   dW 16384 x 2048 x 8192         426        565        608, 2      1572
//   dx 12544 x 640 x 5120          118        78.5       102, 2      127
//   dW 12544 x 640 x 5120          99.3, 4    133        97.4, 2     164, 2
//   dx 12544 x 2560 x 640          45.8       50.9                   68.8
//   dW 12544 x 2560 x 640          77.6, 5    68.1, 3    52.3, 5     80.5, 5
//   dx 2000 x 4096 x 1024          33.2       22.0       42.6, 2     31.3
struct ProductTile {
  int size, per_cu;
  double a, b, round;
};
// (the tile of 32 is the gated layer's alone: 777 x 501 x 333 fp32 fills the chip with it.  Its
// activations and its rows of pre and h make a round longer: 12544 x 640 x 2560 117 us with
// 256, 125 with 128, 162 with 64; 100352 x 80 x 320 69, 58, 58; 6272 x 192 x 768 18.8, 18.0, 15.5)
constexpr double kGatedRound[] = {12.5, 6.2, 2.6, 2.4};
constexpr ProductTile kTilesBf16[] = {{256, 1, 0.0, 1.66, 4.5}, {128, 2, 0.5, 0.22, 3.3}, {64, 4, 0.2, 0.15, 1.0}, {32, 8, 0.25, 0.06, 1.0}};
constexpr ProductTile kTilesF32[] = {{128, 2, 0.5, 1.75, 4.0}, {64, 4, 0.4, 0.45, 1.5}, {32, 8, 0.25, 0.15, 1.0}};

struct ProductSize {
  long long M, N, K;
  long long tiles(int size) const { return ((M + size - 1) / size) * ((N + size - 1) / size); }
  long long stages(int dt_bf16) const { return (K + (dt_bf16 ? 63 : 31)) / (dt_bf16 ? 64 : 32); }
};

struct ProductCut {
  int tile, parts;
  double us;
};

// One product alone.
inline ProductCut product_cut(const ProductSize& s, int dt_bf16, bool gated) {
  ProductCut best{64, 1, 1e300};
  const long long stages = s.stages(dt_bf16);
  // (at least four stages a part; the parts' sums stay within 256 MiB)
  const long long most = std::max<long long>(1, std::min<long long>(stages / 4, (64LL << 20) / (s.M * s.N)));
  for (int i = 0; i < (dt_bf16 ? 3 : 2) + (gated ? 1 : 0); ++i) {
    const ProductTile& t = dt_bf16 ? kTilesBf16[i] : kTilesF32[i];
    const long long tiles = s.tiles(t.size), slots = 256LL * t.per_cu;
    if (i && tiles > 1 << 22) break;  // (fewer than 2^31 threads a launch)
    for (const int p : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
      if (p > most || (p > 1 && tiles * p > 3 * slots)) break;
      const long long all = tiles * p, rest = all % slots;
      const double n = (double)((stages + p - 1) / p), round = gated && p == 1 ? kGatedRound[i + !dt_bf16] : t.round;
      double us = (double)(all / slots) * (n * (t.a + t.b * t.per_cu) + round);
      if (rest) us += n * (t.a + t.b * (double)((rest + 255) / 256)) + round;
      if (p > 1) us += 5.0 + (double)(8 * p + 4) * (double)(s.M * s.N) / 5.5e6;
      if (us < best.us) best = ProductCut{t.size, p, us};
    }
  }
  return best;
}

// Two, in one launch with a tile and parts that suit both, or one after the other.  In one
// launch against one after the other, us, bf16: 6272 x 192 x 1536 28 (38), 3008 x 1008 x 336
// 23 (28), 784 x 640 x 5120 29 (41), 12544 x 2560 x 640 103 (110).
struct ProductCuts {
  ProductCut x, W;
  bool together;
};

inline ProductCuts product_cuts(const ProductSize& x, const ProductSize& w, int dt_bf16) {
  ProductCuts best{product_cut(x, dt_bf16, false), product_cut(w, dt_bf16, false), false};
  double least = best.x.us + best.W.us + 8.0;
  const long long sx = x.stages(dt_bf16), sw = w.stages(dt_bf16);
  auto most = [](const ProductSize& s, long long stages) {
    return std::max<long long>(1, std::min<long long>(stages / 4, (64LL << 20) / (s.M * s.N)));
  };
  auto join = [](const ProductSize& s, int p) { return p > 1 ? (double)(8 * p + 4) * (double)(s.M * s.N) / 5.5e6 : 0.0; };
  const long long mx = most(x, sx), mw = most(w, sw);
  for (int i = 0; i < (dt_bf16 ? 3 : 2); ++i) {
    const ProductTile& t = dt_bf16 ? kTilesBf16[i] : kTilesF32[i];
    const long long slots = 256LL * t.per_cu, tx = x.tiles(t.size), tw = w.tiles(t.size);
    if (i && tx + tw > 1 << 22) break;
    const double full = t.a + t.b * t.per_cu;
    for (const int px : {1, 2, 4, 8, 16}) {
      if (px > mx || (px > 1 && tx * px > slots)) break;
      const double nx = (double)((sx + px - 1) / px), x1 = nx * full + t.round, cx = (double)(tx * px);
      for (const int pw : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48}) {
        if (pw > mw || (pw > 1 && tw * pw > 2 * slots)) break;
        const double nw = (double)((sw + pw - 1) / pw), cw = (double)(tw * pw), all = cx + cw;
        double us;
        if (all <= (double)slots) {
          us = std::max(nx, nw) * (t.a + t.b * (double)(((long long)all + 255) / 256)) + t.round;
        } else {
          // the workgroups' time shared out, and half of one at the end; one takes its time at least
          const double w1 = nw * full + t.round;
          us = std::max((cx * x1 + cw * w1) / (double)slots + std::min(x1, w1) / 2, std::max(x1, w1));
        }
        us += join(x, px) + join(w, pw) + (px > 1 || pw > 1 ? 5.0 : 0.0);
        if (us < least) least = us, best = ProductCuts{{t.size, px, us}, {t.size, pw, us}, true};
      }
    }
  }
  return best;
}

}  // namespace gl
