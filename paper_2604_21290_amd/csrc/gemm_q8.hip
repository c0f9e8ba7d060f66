// Fully connected layers on 8-bit rows:
//   out[r, o] = act_out( (sum_k A[r, k] W[o, k]) sa[r] sw[o] + bias[o] ) + residual[r, o]
// The sums are exact (int32, at most 131071 terms); then fp32 and one rounding.  A sum meets
// the row's scale first: the two scales' product alone may overflow (a zero sum would make it
// a NaN) or lose bits below 2^-126 where the result does neither.
//   - Staging: 16 bytes a lane straight into LDS, a row's 16-byte slots permuted by
//     its number so that the rows an operand read touches lie in all banks.
//   - MFMA 16x16x64: a lane's 16 bytes of a row are one operand.  Operands are
//     swapped (W rows first): a lane ends with consecutive output columns of one row.
#include <type_traits>

#include "gl_device.h"
#include "gl_kernels.h"

namespace gl {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4 mfma_i8(const uint4& a, const uint4& b, i32x4 acc) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                               __builtin_bit_cast(i32x4, b), acc, 0, 0, 0);
}

// GELU x Phi(x) = max(x, 0) - |x| Phi(-|x|), where Phi(-a) e^(a^2 / 2) falls like 1 / a for
// large a: with t = 1 / (1 + p a) it is t q(t), q a smooth function on (0, 1].  q is a
// polynomial fitted in float64 to the least largest error relative to Phi(-a), weighted by
// what the output's type shows of it, so that the tail's small results have their bits too:
//   bf16  five terms, within 5.7e-7 e^(1.5 a), never more than 2.8e-3 (2^-8 is its rounding)
//   fp32  eight terms, within 3.8e-8 (1 + a)
// The rest is fp32's own rounding, at most (13 + a + 2 a^2) 2^-24 with the fit (the
// argument's last bit alone moves Phi(-a) by a^2 of its own).  The three terms more cost an
// fp32 layer up to 5 % (100352x80x320 34.2 us for 32.8, 6272x192x768 8.5 for 8.1); in bf16
// they would change one output in a thousand.  Its limits at the infinities.
template <int DT>
__device__ __forceinline__ float gelu_q8(float x) {
  const float a = fabsf(x);
  const float t = __builtin_amdgcn_rcpf(fmaf(DT ? 0.34400001f : 0.3f, a, 1.f));
  float q;
  if (DT) {
    q = fmaf(t, -0.100211024f, 0.2995327891f);
    q = fmaf(t, q, -0.005176517668f);
    q = fmaf(t, q, 0.1722774513f);
    q = fmaf(t, q, 0.1335771899f);
  } else {
    q = fmaf(t, 0.03661797821f, -0.1609455123f);
    q = fmaf(t, q, 0.212445229f);
    q = fmaf(t, q, -0.0589276667f);
    q = fmaf(t, q, 0.1311242333f);
    q = fmaf(t, q, 0.09920725217f);
    q = fmaf(t, q, 0.1208549423f);
    q = fmaf(t, q, 0.1196235572f);
  }
  const float y = x * 0.84932180028801907f;  // sqrt(log2(e) / 2)
  const float e = __builtin_amdgcn_exp2f(-y * y);
  return fmaf(-fminf(a, 3.4e38f), t * q * e, fmaxf(x, 0.f));
}

typedef uint32_t u32x4_w __attribute__((ext_vector_type(4), aligned(4), may_alias));

// 8 consecutive values of a residual at any element's place, as they lie in memory
template <int DT>
struct Raw8 {
  uint4 v[DT ? 1 : 2];
  __device__ __forceinline__ void load(const void* p, size_t i) {
    if (DT) {
      v[0] = load16_any(static_cast<const uint16_t*>(p) + i);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        v[DT ? 0 : h] = __builtin_bit_cast(uint4, reinterpret_cast<const u32x4_w*>(static_cast<const float*>(p) + i)[h]);
    }
  }
  __device__ __forceinline__ void add_to(float* y) const {
    if (DT) {
      float f[8];
      unpack_bf16x8(v[0], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] += f[j];
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4& u = v[DT ? 0 : h];
        y[4 * h] += __uint_as_float(u.x), y[4 * h + 1] += __uint_as_float(u.y);
        y[4 * h + 2] += __uint_as_float(u.z), y[4 * h + 3] += __uint_as_float(u.w);
      }
    }
  }
};
template <int DT>
__device__ __forceinline__ float load1(const void* p, size_t i) {
  return DT ? bf16_bits_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}
template <int DT>
__device__ __forceinline__ void store8(void* p, size_t i, const float* f) {
  if (DT) {
    store16_any(static_cast<uint16_t*>(p) + i, pack_bf16x8(f));
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4_w v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(f[4 * h + j]);
      reinterpret_cast<u32x4_w*>(static_cast<float*>(p) + i)[h] = v;
    }
  }
}
template <int DT>
__device__ __forceinline__ void store1(void* p, size_t i, float f) {
  if (DT) static_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16_bits(f);
  else static_cast<float*>(p)[i] = f;
}

// ---------------------------------------------------------------------------
// Large products: a pipeline that does not drain, neither between stages nor
// between tiles.
//   - A workgroup takes one tile after another, and its stages (128 bytes of K of
//     each row) follow each other across tiles: the first two of the next tile are
//     under way before the last of this one is multiplied.
//   - Operands are double-buffered in registers: while one half stage (64 bytes of
//     K) is multiplied, the next one's are read, a few between every few MFMAs.
//   - The barrier of a stage stands before its last half is multiplied, when that
//     half's operands are in registers: what follows it, the next stage's first
//     reads and the loads into the buffer that is now free, runs under MFMAs.
//   - MFMA tile j of a wave takes W's rows in an order that leaves a lane with eight
//     consecutive columns of a row in tiles 2p and 2p + 1: results go from the
//     accumulators to memory 16 bytes (bf16) a lane, 64 a row, with no trip
//     through LDS.
//   - Small tiles, for few outputs, have KG groups of waves, which take every KG-th stage
//     into buffers of their own and add their sums in LDS.  A stage takes 0.27 us where
//     one wave a SIMD has the tile (64 x 64), 0.2 with two groups (64 x 32), 0.12 with
//     four (32 x 32).
// Tiles are walked so that the 32 that an XCD works on at a time are 8 x 4.
// What bounds it: at 8192 x 8192 x 8192 (420-435 us, 2.6 POP/s; the library's int8
// product 440) the matrix cores are busy 66 % of the cycles, at a clock that falls to
// 1.7-1.8 GHz on random data; with all loads from L2's hottest lines 397 us, so the trip
// to memory costs 8 %.  Its loads alone take 360 us, its products alone 346: each stage's
// loads take about as long as its products, and LDS holds one stage ahead.  Tried and slower there: MFMA 32x32x32 (471 us), stages of 64
// bytes in four buffers (446), 256 x 128 tiles in three buffers (478; also 28.0-30.8 at
// 12544 x 2560 x 640, where 128 x 128 take 26.9-28.1, and no faster at ten sizes more), four
// waves of 128 x 128 (886: operands move between the register files).
// ---------------------------------------------------------------------------
template <int BM_, int BN_, int WR_, int WC_, int NBUF_, int KG_ = 1>
struct PipeCfg {
  static constexpr int BM = BM_, BN = BN_, WR = WR_, WC = WC_, NBUF = NBUF_, KG = KG_, STEP = 128;
  static constexpr int kWaves = WR * WC;  // of one of KG groups, which take every KG-th stage
  static constexpr int kThreads = 64 * kWaves * KG;
  static constexpr int kStage = (BM + BN) * STEP;
  static constexpr int kRPL = 1024 / STEP;  // rows of a wave's load
  static constexpr int kLoadsA = BM / kRPL / kWaves, kLoadsW = BN / kRPL / kWaves;  // per wave and stage
  static constexpr int TM = BM / WR / 16, TN = BN / WC / 16;
  static constexpr int kVec = BM + 2 * BN;  // a tile's scales and bias
  static constexpr int kSums = BM * BN * 4;  // the tile's sums of a group
  static constexpr size_t kBufs = (size_t)KG * NBUF * kStage, kSmem = kBufs + 2 * kVec * 4 + (KG - 1) * kSums;
  static constexpr int kFit = (int)(160 * 1024 / kSmem), kPerCU = kFit * kWaves * KG <= 16 ? kFit : 16 / (kWaves * KG);
  static_assert(BM % (kRPL * kWaves) == 0 && BN % (kRPL * kWaves) == 0, "whole loads per wave");
  static_assert(TN % 2 == 0, "pairs of column tiles");
  static_assert(BM <= kThreads && BN <= kThreads, "a thread loads one of each vector");
};

// 16 bytes a lane from base + off to LDS (lds_dma16 with a uniform base)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void lds_dma16_base(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// v, which the compiler takes for a value of its own each time: what is computed from
// it is not kept in registers across the loop over K.
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// All but this wave's N newest loads have landed and its LDS reads are done; then the
// workgroup's barrier.
template <int N>
__device__ __forceinline__ void dma_wait_barrier_but() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <class G, int DT, int ACT_OUT>
__global__ __launch_bounds__(G::kThreads) __attribute__((amdgpu_waves_per_eu(G::kThreads * G::kPerCU / 256, G::kThreads * G::kPerCU / 256)))
void gemm_q8_pipe_kernel(GemmQ8Args a) {
  extern __shared__ __align__(16) char smem[];
  constexpr int BM = G::BM, BN = G::BN, STEP = G::STEP, TM = G::TM, TN = G::TN, NA = G::kLoadsA, NB = G::kLoadsW;
  constexpr int NL = NA + NB, NBUF = G::NBUF;
  constexpr int WROWS = 16 * TM, WCOLS = 16 * TN;
  const int R = a.R, Cout = a.Cout, rowb = a.Kp;
  const int nstages = (rowb + STEP * G::KG - 1) / (STEP * G::KG);  // of each group
  const int ntm = (R + BM - 1) / BM, ntn = (Cout + BN - 1) / BN, ntiles = ntm * ntn;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = G::KG > 1 ? wv / G::kWaves : 0, w = wv - kg * G::kWaves;
  const int g = lane >> 4, t = lane & 15;
  const int wm = w / G::WC, wn = w % G::WC;

  // place of tile number L of the dispatch order: groups of 8 rows of tiles, walked
  // column by column, a stretch of them for each XCD
  auto place = [&](int L, int& m0, int& n0) {
    const int blk = xcd_remap(L, ntiles);
    const int grp = blk / (8 * ntn), in = blk - grp * 8 * ntn, high = min(8, ntm - grp * 8);
    const int nt = in / high;
    m0 = (grp * 8 + in - nt * high) * BM;
    n0 = nt * BN;
  };

  // staging: load i of wave w fills rows 8 (w + waves i) .. of the stage; lane l's
  // 16 bytes land at place l % 8 of row l / 8 and hold slot place ^ key, where a row
  // of A has key row % 8 and one of W, whose rows are read in fours of every other
  // eight, row % 4 + 4 (row / 8 % 2).  Rows past R or Cout repeat the last one.
  const uint32_t lds0 = lds_offset(smem) + kg * NBUF * G::kStage + w * 1024;
  constexpr int RPL = G::kRPL;
  const int lr = lane >> 3;
  const int slot_a = ((lane & 7) ^ lr) * 16;
  const int slot_w = ((lane & 7) ^ ((lr & 3) | ((w & 1) << 2))) * 16;
  const int lim_a = rowb - 16 - slot_a, lim_w = rowb - 16 - slot_w;  // the row's last slot
  const char *base_a, *base_w;    // of the tile that is being loaded
  uint32_t src_a[NA], src_w[NB];  // at most 256 rows of 2^17 bytes
  int L_load = blockIdx.x, s_load = 0;
  auto aim = [&]() {
    int m0, n0;
    place(L_load, m0, n0);
    base_a = reinterpret_cast<const char*>(a.A) + (size_t)m0 * rowb;
    base_w = reinterpret_cast<const char*>(a.W) + (size_t)n0 * rowb;
    const int r = fresh(RPL * w + lr);
#pragma unroll
    for (int i = 0; i < NA; ++i) src_a[i] = (uint32_t)min(r + RPL * G::kWaves * i, R - 1 - m0) * rowb + slot_a;
#pragma unroll
    for (int i = 0; i < NB; ++i) src_w[i] = (uint32_t)min(r + RPL * G::kWaves * i, Cout - 1 - n0) * rowb + slot_w;
  };
  // past the end of a row, W reads zeros, and A its last slot again
  auto load = [&](int i, int buf) {
    const int off = (s_load * G::KG + kg) * STEP;
    const uint32_t d = lds0 + buf * G::kStage + i * G::kWaves * 1024;
    if (i < NA) {
      lds_dma16_base(base_a, src_a[i < NA ? i : 0] + min(off, lim_a), d);
    } else {
      const char* p = base_w + (src_w[i < NA ? 0 : i - NA] + off);
      lds_dma16(off <= lim_w ? p : reinterpret_cast<const char*>(kZero16), d);
    }
  };
  // after the last stage of the last tile the same stage is loaded again, and not read
  auto next_load = [&]() {
    if (++s_load < nstages) return;
    if (L_load + (int)gridDim.x < ntiles) {
      L_load += gridDim.x;
      s_load = 0;
      aim();
    } else {
      s_load = nstages - 1;
    }
  };

  // operands of half stage kk
  uint4 fa[2][TM], fb[2][TN];
  // (the second half of a stage's row is 64 bytes off: the slot's permutation is an
  // exclusive or)
  const int rd_a = kg * NBUF * G::kStage + (wm * WROWS + t) * STEP + (g ^ (t & 7)) * 16;
  const int rd_b = kg * NBUF * G::kStage + (BM + wn * WCOLS + (t >> 2) * 8 + (t & 3)) * STEP + (g ^ (t & 7)) * 16;
  auto read = [&](int set, int pa, int pb, int i) {  // TM of A, then TN of W
    if (i < TM)
      fa[set][i < TM ? i : 0] = *reinterpret_cast<const uint4*>(smem + pa + i * 16 * STEP);
    else
      fb[set][i < TM ? 0 : i - TM] = *reinterpret_cast<const uint4*>(
          smem + pb + (((i - TM) >> 1) * 32 + ((i - TM) & 1) * 4) * STEP);
  };
  i32x4 acc[TM][TN];
  // multiply half kk (its operands are in set kk) while the next half's are read from
  // `buf` and, in the second half, a stage is loaded into the buffer `lbuf`
  constexpr int kSpread = TM > 2 ? TM / 2 : TM;  // row tiles that the loads are spread over
  auto half = [&](auto KK, int buf, int lbuf) {
    constexpr int kk = decltype(KK)::value;
    constexpr int kPer = TM > 1 ? (TM + TN + TM - 2) / (TM > 1 ? TM - 1 : 1) : TM + TN, kLPer = (NL + kSpread - 1) / kSpread;
    const int pa = buf * G::kStage + (fresh(rd_a) ^ ((kk ^ 1) * 64));
    const int pb = buf * G::kStage + (fresh(rd_b) ^ ((kk ^ 1) * 64));
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = mfma_i8(fb[kk][j], fa[kk][i], acc[i][j]);
      if (kk == 1) {
#pragma unroll
        for (int l = i * kLPer; l < (i + 1) * kLPer && l < NL; ++l) load(l, lbuf);
      }
      // W's first: each of them is needed with every row tile
#pragma unroll
      for (int l = i * kPer; l < (i + 1) * kPer && l < TM + TN; ++l) read(kk ^ 1, pa, pb, l < TN ? TM + l : l - TN);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  aim();
#pragma unroll
  for (int b = 0; b < NBUF; ++b) {
#pragma unroll
    for (int i = 0; i < NL; ++i) load(i, b);
    next_load();
  }
  dma_wait_barrier_but<(NBUF - 1) * NL>();
#pragma unroll
  for (int i = 0; i < TM + TN; ++i) read(0, rd_a, rd_b, i);

  float* const vec0 = reinterpret_cast<float*>(smem + G::kBufs);
  int buf = 0, turn = 0;
  for (int L = blockIdx.x; L < ntiles; L += gridDim.x, turn ^= 1) {
    int m0, n0;
    place(L, m0, n0);
    // the tile's vectors: loaded now, put into LDS before the first barrier
    float* const vec = vec0 + turn * G::kVec;
    float v_sa, v_sw, v_b;
    auto fetch = [&]() {
      const int i = fresh(tid);
      v_sa = i < BM ? a.sa[min(m0 + i, R - 1)] : 0.f;
      v_sw = i < BN ? a.sw[min(n0 + i, Cout - 1)] : 0.f;
      v_b = i < BN && a.bias ? load1<DT>(a.bias, min(n0 + i, Cout - 1)) : 0.f;
    };
    // (tiles whose accumulators leave no room for them load them then)
    constexpr bool kLate = TM * TN >= 32;
    if (!kLate) fetch();
    // The residual's values: for small tiles loaded now, for others before or among the
    // stores, kAhead row tiles ahead.  (Rows past R and columns past Cout are not loaded.)
    constexpr bool kEarly = DT == 1 && TM * TN <= 8;
    constexpr int kAhead = kEarly ? TM : DT == 1 ? 4 : 2;
    Raw8<DT> res[kAhead][TN / 2];
    auto load_res = [&](int i, int lane_e) {
      const int row = m0 + wm * WROWS + i * 16 + (lane_e & 15);
#pragma unroll
      for (int p = 0; p < TN / 2; ++p) {
        const int n = n0 + wn * WCOLS + p * 32 + (lane_e >> 4) * 8;
        if (row < R && n + 8 <= Cout) res[i % kAhead][p].load(a.residual, (size_t)row * Cout + n);
      }
    };
    if (kEarly && a.residual && kg == 0) {
      const int lane_e = fresh(lane);
#pragma unroll
      for (int i = 0; i < TM; ++i) load_res(i, lane_e);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    using std::integral_constant;
    auto fill = [&]() {
      if (kLate) fetch();
      const int i = fresh(tid);
      if (i < BM) vec[i] = v_sa;
      if (i < BN) vec[BM + i] = v_sw, vec[BM + BN + i] = v_b;
    };
    for (int s = 0; s < nstages; ++s) {
      half(integral_constant<int, 0>(), buf, 0);
      if (s == 0) fill();
      // this wave has read all of the stage, and the next one has landed: for all waves
      dma_wait_barrier_but<(NBUF - 2) * NL>();
      const int free = buf;
      buf = buf + 1 == NBUF ? 0 : buf + 1;
      half(integral_constant<int, 1>(), buf, free);
      next_load();
    }

    if (G::KG > 1) {  // the groups' sums meet in LDS; the first group has the rest
      i32x4* const sums = reinterpret_cast<i32x4*>(smem + G::kBufs + 2 * G::kVec * 4) + w * TM * TN * 64 + lane;
      if (kg > 0) {
#pragma unroll
        for (int u = 0; u < TM * TN; ++u) sums[(kg - 1) * (G::kSums / 16) + u * 64] = acc[u / TN][u % TN];
      }
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (kg > 0) continue;
#pragma unroll
      for (int q = 0; q < G::KG - 1; ++q)
#pragma unroll
        for (int u = 0; u < TM * TN; ++u) acc[u / TN][u % TN] += sums[q * (G::kSums / 16) + u * 64];
    }

    // lane (g, t) of MFMA tiles (i, 2p) and (i, 2p + 1): eight columns of row t.  Row
    // tiles outermost: the two halves of a 128-byte line are stored together.
    const int lane_e = fresh(lane), te = lane_e & 15, ge = lane_e >> 4;
    if (!kEarly && a.residual) {
#pragma unroll
      for (int i = 0; i < kAhead - 1; ++i) load_res(i, lane_e);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      // (row tile by row tile, or their addresses and loads would fill the registers)
      if (!kEarly) __builtin_amdgcn_sched_barrier(0);
      if (!kEarly && a.residual && i + kAhead - 1 < TM) load_res(i + kAhead - 1, lane_e);
      const int r = wm * WROWS + i * 16 + te, row = m0 + r;
      const float sar = vec[r];
#pragma unroll
      for (int p = 0; p < TN / 2; ++p) {
        const int c = wn * WCOLS + p * 32 + ge * 8, n = n0 + c;
        float y[8];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          y[v] = fmaf((float)acc[i][2 * p + (v >> 2)][v & 3] * sar, vec[BM + c + v], vec[BM + BN + c + v]);
          if (ACT_OUT) y[v] = gelu_q8<DT>(y[v]);
        }
        if (row >= R || n >= Cout) continue;
        const size_t o = (size_t)row * Cout + n;
        if (n + 8 <= Cout) {
          if (a.residual) res[i % kAhead][p].add_to(y);
          store8<DT>(a.out, o, y);
        } else {
#pragma unroll
          for (int v = 0; v < 8; ++v)
            if (n + v < Cout) {
              if (a.residual) y[v] += load1<DT>(a.residual, o + v);
              store1<DT>(a.out, o + v, y[v]);
            }
        }
      }
    }
    // (the next tile's first operands again: kept across the epilogue they would not leave
    // it enough registers)
    if (kLate) {
#pragma unroll
      for (int i = 0; i < TM + TN; ++i) read(0, buf * G::kStage + rd_a, buf * G::kStage + rd_b, i);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives its workgroup
}

template <class G, int DT>
hipError_t launch_pipe_q8(const GemmQ8Args& a, hipStream_t stream) {
  const void* fn = a.act_out ? (const void*)&gemm_q8_pipe_kernel<G, DT, 1> : (const void*)&gemm_q8_pipe_kernel<G, DT, 0>;
  const long tiles = ((long)(a.R + G::BM - 1) / G::BM) * ((a.Cout + G::BN - 1) / G::BN);
  const dim3 grid((unsigned)std::min(tiles, 256L * G::kPerCU));
  return launch_with_smem(fn, grid, dim3(G::kThreads), G::kSmem, stream, nullptr, nullptr, a);
}

// ---------------------------------------------------------------------------
// Short rows: a workgroup keeps 64 or 96 columns of W, all of K, in LDS, and its four
// waves take strips of 16 rows, each for itself, with no barrier between them.  A strip
// goes straight to registers; each 64 bytes of K of the wave's next strip are requested
// when this one's have been multiplied, and its residual after this one's results.  So
// every wave has a strip on its way from memory (room for 4 to 7 waves a SIMD), where the
// tiles above load W with every tile and meet at a barrier every 128 bytes of K.
//   100352x320x80 with residual 13.7 us (16.3 by tiles), 64 MB of memory traffic, three waves
//   a SIMD of room for four; 6272x192x768 with GELU 7.5 (8.4), of which 3.4 are the GELU's
//   instructions.
// Loading both halves of a 128-byte line together changed nothing; strips of 32 rows
// leave too few waves (6272x192x192 4.0 for 3.6).
// ---------------------------------------------------------------------------
template <int DT_, int KS_, int TN_>
struct StripCfg {  // KS: 64-byte steps of K; TN: 16-column tiles
  static constexpr int DT = DT_, KS = KS_, TN = TN_;
  static constexpr int BM = 16, BN = 16 * TN, NS = (KS + 1) / 2;
  static constexpr int kUnits = NS * BN / 8 / 4;  // 8 rows by 128 bytes of W, per wave
  static constexpr size_t kSmem = (size_t)NS * BN * 128 + 2 * BN * 4;
  // operands of a strip, its sums, a step of W, a residual, addresses and the epilogue
  static constexpr int kRegs = 4 * (KS + 2 * TN) + 2 * TN * (DT ? 1 : 2) + 24;
  static constexpr int kByLds = (int)(160 * 1024 / kSmem), kByRegs = 512 / kRegs;
  static constexpr int kPerCU = kByLds < kByRegs ? kByLds : kByRegs;
  static_assert(TN % 2 == 0 && BN <= 256 && kPerCU >= 1 && kPerCU <= 8, "whole units a wave, a thread a column");
};

template <class G, int ACT_OUT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(G::kPerCU, G::kPerCU)))
void gemm_q8_strip_kernel(GemmQ8Args a) {
  extern __shared__ __align__(16) char smem[];
  constexpr int DT = G::DT, KS = G::KS, TN = G::TN, BM = G::BM, BN = G::BN;
  const int R = a.R, Cout = a.Cout, rowb = a.Kp;
  const int ntm = (R + BM - 1) / BM, ntn = (Cout + BN - 1) / BN, per = (int)gridDim.x / ntn;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, t = lane & 15;
  // workgroups with the same rows follow each other on an XCD
  const int blk = xcd_remap(blockIdx.x, gridDim.x), rb = blk / ntn, n0 = (blk - rb * ntn) * BN;

  // W: unit u is 8 of its rows at 128 bytes of K, its 16-byte slots permuted as in the
  // pipeline; zeros past the rows' end
#pragma unroll
  for (int i = 0; i < G::kUnits; ++i) {
    const int u = w + 4 * i, s = u / (BN / 8), grp = u - s * (BN / 8), lr = lane >> 3;
    const int k = s * 128 + ((lane & 7) ^ ((lr & 3) | ((grp & 1) << 2))) * 16;
    const char* p = reinterpret_cast<const char*>(a.W) + (size_t)min(n0 + 8 * grp + lr, Cout - 1) * rowb + k;
    lds_dma16(k < rowb ? p : reinterpret_cast<const char*>(kZero16), lds_offset(smem) + u * 1024);
  }
  float* const vec = reinterpret_cast<float*>(smem + G::NS * BN * 128);
  if (tid < BN) {
    const int n = min(n0 + tid, Cout - 1);
    vec[tid] = a.sw[n];
    vec[BN + tid] = a.bias ? load1<DT>(a.bias, n) : 0.f;
  }

  uint4 fa[KS];
  float sa;
  Raw8<DT> res[TN / 2];
  // rows past R repeat the last one; past a row's end its last slot, where W is zero
  auto load_step = [&](int k, int m0) {
    const char* base = reinterpret_cast<const char*>(a.A) + (size_t)m0 * rowb;
    const int at = k < KS - 1 ? 64 * k + 16 * g : min(64 * k + 16 * g, rowb - 16);
    fa[k] = *reinterpret_cast<const uint4*>(base + (uint32_t)(min(t, R - 1 - m0) * rowb + at));
  };
  auto load_rest = [&](int m0) {
    const int row = min(m0 + t, R - 1);
    sa = a.sa[row];
    if (!a.residual) return;
#pragma unroll
    for (int p = 0; p < TN / 2; ++p) {
      const int n = n0 + 32 * p + 8 * g;
      if (n + 8 <= Cout) res[p].load(a.residual, (size_t)row * Cout + n);
    }
  };
  const int step = per * 4;
  int mt = rb * 4 + w;
  if (mt < ntm) {
#pragma unroll
    for (int k = 0; k < KS; ++k) load_step(k, mt * BM);
    load_rest(mt * BM);
  }
  dma_wait_barrier();

  const int rd = ((t >> 2) * 8 + (t & 3)) * 128 + (g ^ (t & 7)) * 16;
  auto strip = [&](auto MORE) {
    constexpr bool more = decltype(MORE)::value;
    const int m0 = mt * BM, m1 = m0 + step * BM;
    i32x4 acc[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[j] = i32x4{0, 0, 0, 0};
    const int at = fresh(rd);  // (or all of W would move to registers)
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const char* const pw = smem + (k >> 1) * BN * 128 + (at ^ ((k & 1) * 64));
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[j] = mfma_i8(*reinterpret_cast<const uint4*>(pw + ((j >> 1) * 32 + (j & 1) * 4) * 128), fa[k], acc[j]);
      if (more) load_step(k, m1);
    }
    // lane (g, t) of MFMA tiles 2p and 2p + 1: eight columns of row t
    const int row = m0 + t;
#pragma unroll
    for (int p = 0; p < TN / 2; ++p) {
      const int c = 32 * p + 8 * g, n = n0 + c;
      float y[8];
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        y[v] = fmaf((float)acc[2 * p + (v >> 2)][v & 3] * sa, vec[c + v], vec[BN + c + v]);
        if (ACT_OUT) y[v] = gelu_q8<DT>(y[v]);
      }
      if (row >= R || n >= Cout) continue;
      const size_t o = (size_t)row * Cout + n;
      if (n + 8 <= Cout) {
        if (a.residual) res[p].add_to(y);
        store8<DT>(a.out, o, y);
      } else {
#pragma unroll
        for (int v = 0; v < 8; ++v)
          if (n + v < Cout) {
            if (a.residual) y[v] += load1<DT>(a.residual, o + v);
            store1<DT>(a.out, o + v, y[v]);
          }
      }
    }
    if (more) load_rest(m1);
  };
  for (; mt < ntm - step; mt += step) strip(std::true_type());
  if (mt < ntm) strip(std::false_type());
}

// As many workgroups as the CUs hold together, or fewer with the same number of turns.
template <class G>
hipError_t launch_strip_q8(const GemmQ8Args& a, hipStream_t stream) {
  const void* fn = a.act_out ? (const void*)&gemm_q8_strip_kernel<G, 1> : (const void*)&gemm_q8_strip_kernel<G, 0>;
  const long ntn = (a.Cout + G::BN - 1) / G::BN, fours = ((long)(a.R + G::BM - 1) / G::BM + 3) / 4;
  const long most = std::max(1L, 256L * G::kPerCU / ntn), turns = (fours + most - 1) / most;
  const long per = (fours + turns - 1) / turns;
  return launch_with_smem(fn, dim3((unsigned)(per * ntn)), dim3(256), G::kSmem, stream, nullptr, nullptr, a);
}

template <int DT, int TN>
hipError_t launch_strips_q8(const GemmQ8Args& a, hipStream_t stream) {
  switch ((a.Kp + 63) / 64) {
    case 1: return launch_strip_q8<StripCfg<DT, 1, TN>>(a, stream);
    case 2: return launch_strip_q8<StripCfg<DT, 2, TN>>(a, stream);
    case 3: return launch_strip_q8<StripCfg<DT, 3, TN>>(a, stream);
    case 4: return launch_strip_q8<StripCfg<DT, 4, TN>>(a, stream);
    default: return launch_strip_q8<StripCfg<DT, 5, TN>>(a, stream);
  }
}

// ---------------------------------------------------------------------------
// Few rows: the weights' bytes bound the layer, so every CU has to stream some.  A
// workgroup takes 16 columns and 16 rows; its eight waves split K, 64 bytes of each row
// in turn, and load their operands straight into registers, up to U steps before any is
// used.  The eight partial sums meet in LDS.  (8192 x 8192 weights, one row: 5.2 TB/s.)
// ---------------------------------------------------------------------------
template <int DT, int ACT_OUT>
__global__ __launch_bounds__(512) void gemm_q8_rows_kernel(GemmQ8Args a) {
  constexpr int NW = 8, U = 8;
  __shared__ __align__(16) int part[NW][256];
  const int R = a.R, Cout = a.Cout, rowb = a.Kp;
  // columns first; where there are more rows, an XCD takes a stretch of them with all
  // columns (1885x2699x81 6.8 us for 8.5), and elsewhere most widths give it its own
  // columns with all rows as they are (196x192x768 2.5, 3.1 by stretches)
  const int ntn = (int)gridDim.x, ntm = (int)gridDim.y;
  int nb = blockIdx.x, mb = blockIdx.y;
  if (ntm > ntn) {
    const int blk = xcd_remap(mb * ntn + nb, ntm * ntn);
    mb = blk / ntn;
    nb = blk - mb * ntn;
  }
  const int n0 = nb * 16, m0 = mb * 16;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, t = lane & 15;
  const char* pw = reinterpret_cast<const char*>(a.W) + (size_t)min(n0 + t, Cout - 1) * rowb;
  const char* pa = reinterpret_cast<const char*>(a.A) + (size_t)min(m0 + t, R - 1) * rowb;
  i32x4 acc = {0, 0, 0, 0};
  for (int k0 = w * 64; k0 < rowb; k0 += NW * 64 * U) {
    uint4 fw[U], fa[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int ku = k0 + u * NW * 64, k = ku + g * 16;
      fw[u] = fa[u] = make_uint4(0, 0, 0, 0);
      if (ku < rowb) {  // uniform
        const int at = k < rowb ? k : 0;
        fw[u] = *reinterpret_cast<const uint4*>(pw + at);
        fa[u] = *reinterpret_cast<const uint4*>(pa + at);
        if (k >= rowb) fw[u] = make_uint4(0, 0, 0, 0);  // past the rows' end
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) acc = mfma_i8(fw[u], fa[u], acc);
  }
  *reinterpret_cast<i32x4*>(&part[w][t * 16 + g * 4]) = acc;
  __syncthreads();
  const int row = m0 + (tid >> 4), n = n0 + (tid & 15);
  if (tid >= 256 || row >= R || n >= Cout) return;
  int s = 0;
#pragma unroll
  for (int k = 0; k < NW; ++k) s += part[k][tid];
  float y = fmaf((float)s * a.sa[row], a.sw[n], a.bias ? load1<DT>(a.bias, n) : 0.f);
  if (ACT_OUT) y = gelu_q8<DT>(y);
  const size_t at = (size_t)row * Cout + n;
  if (a.residual) y += load1<DT>(a.residual, at);
  store1<DT>(a.out, at, y);
}

template <int DT>
hipError_t launch_rows_q8(const GemmQ8Args& a, hipStream_t stream) {
  const void* fn = a.act_out ? (const void*)&gemm_q8_rows_kernel<DT, 1> : (const void*)&gemm_q8_rows_kernel<DT, 0>;
  return launch_with_smem(fn, dim3((a.Cout + 15) / 16, (a.R + 15) / 16), dim3(512), 0, stream, nullptr, nullptr, a);
}

// The tile for a layer, by what each takes for one round of all CUs, in us: so much for
// every 128 bytes of K, for the rest of a tile, and for a GELU or a residual in its
// epilogue.  A CU's tiles share it, so part of a round takes its part of the time, but
// no less than the latency of one tile.  Fitted to these (us a call in a row of calls on
// three inputs in turn, bf16, plain / GELU / residual):
//                    256 x 256         128 x 128          64 x 64, 4 a CU    64 x 64, 2 a CU
//   8192x8192x8192   435               549                834                852
//   16384x4096x4096  232               287                423                433
//   12544x640x2560   32.5/45.0/57.5 *  35.0/43.8/49.4 *   43.1/49.5/60.7     48.9/57.0/64.9
//   12544x2560x640   35.9/42.0/40.0    27.2/28.8/28.4 *   38.4/39.4/39.7     38.7/40.0/40.2
//   25088x192x768    21.3/33.3/34.5    15.6/22.1/20.7     17.9/23.6/21.5     20.9/26.6/24.4
//   100352x80x320    29.2/54.2/64.6    20.9/34.0/36.4     21.7/31.0/36.4     27.0/37.6/43.5
//   6272x192x768     11.5/18.0/17.0     8.0/10.1/ 9.8      7.3/ 8.4/ 8.8      8.1/ 9.5/ 9.7
//   1000x8000x1000   85.7              47.1               31.2               18.7 *
// (* the one taken: at 12544x640x2560 the larger tile without GELU or residual; strips
// take three of the others).  The
// kernel for few rows where its 16 x 16 outputs are few or K is short (us, against
// the better 64 x 64 tiles): 1x640x2560 2.5 (4.4), 1x8192x8192 13.0 (16.9), 64x2560x640
// 4.3 (7.4), 128x8192x512 9.6 (16.8), 196x192x768 2.6 (3.5), 1024x2560x64 4.6 (7.4),
// 196x320x1280 3.5 (3.7).  And where its own estimate, by the bytes that its units read (rows
// a multiple of 512 bytes apart meet in the same channels), is below the tiles': 777x1001x333
// 4.9 (5.1).
// Tiles for few outputs, 64 x 32 with K between two groups and 32 x 32 between four (us,
// against 64 x 64, 2 a CU, and 16 x 16):
//   64x4096x4096      8.0   7.5   (10.3, 17.0)      500x3000x500   7.7  6.1  (9.1,  9.6)
//   128x4096x4096     8.2  10.8   (10.7, 30.9)      196x2560x640   5.8  5.2  (7.5,  8.1)
//   871x4336x320     10.6  12.5   (13.2, 16.3)      784x4096x200   7.8  6.8 (10.3, 13.1)
//   531x5531x891     12.1  14.3   (15.6, 29.8)      300x6000x300  12.6  9.4 (16.3, 11.2)
//   256x4096x4096    14.4  17.9   (11.0, 58.9)
//
// Strips where K is short, against the best of the tiles (us, plain / GELU / residual):
//   100352x320x80    11.9/15.9/13.7    14.8/18.0/16.3
//   100352x80x320    17.9/27.6/35.3    20.5/30.6/36.5
//   6272x192x768      6.0/ 7.5/ 7.8     7.3/ 8.4/ 8.8
//   25088x320x320    10.8/12.3/11.0    12.2/13.9/13.7
//   6272x192x192      3.5/ 4.3/ 4.1     4.3/ 4.9/ 4.5
//   1200x320x320      3.5/ 3.9/ 3.6     3.7/ 4.2/ 3.9
// Not taken: K past 320 (6272x384x384 6.1/7.0/7.1 for 5.7/6.4/6.7: each strip reads all of
// W from LDS), rows of 256 bytes (25088x256x512 14.9/17.8/17.5 for 13.6/17.8/15.9), and
// wide or large outputs, which tiles of 128 columns write in longer runs (4096x128x4096
// 12.8/18.6/17.9 for 12.1/17.3/16.6, 100352x80x320 fp32 42/43/67 for 37/42/64).  96
// columns where one such strip is all (100352x320x80 by 64: 12.6/16.8/15.4).
template <int DT>
hipError_t launch_q8(const GemmQ8Args& a, hipStream_t stream) {
  const long units = (long)((a.R + 15) / 16) * ((a.Cout + 15) / 16);
  // (a launch has fewer than 2^32 threads)
  if ((a.R <= 16 && units < 1 << 22) || units <= 256 || (units <= 1280 && units * a.Kp <= 1 << 19))
    return launch_rows_q8<DT>(a, stream);
  const double bytes = (double)a.R * a.Cout * (DT ? 2 : 4);
  if (a.Kp <= 320 && a.Kp != 256 && a.Cout <= 2048 && bytes <= 1 << 26)
    return a.Cout > 64 && a.Cout <= 96 ? launch_strips_q8<DT, 6>(a, stream) : launch_strips_q8<DT, 4>(a, stream);
  const double n = (a.Kp + 127) / 128, gelu = a.act_out ? 1 : 0, res = a.residual ? 1 : 0;
  auto rounds = [&](int bm, int bn) {
    return (double)((((long)(a.R + bm - 1) / bm) * ((a.Cout + bn - 1) / bn) + 255) / 256);
  };
  auto cost = [&](int edge, int per_cu, double round, double tile) {
    return std::max(rounds(edge, edge) / per_cu * round, tile);
  };
  const double c[6] = {cost(256, 1, 1.5 * n + 7.5 + 6 * gelu + 10 * res, 0),
                       cost(128, 2, 1.0 * n + 2.5 + 2.1 * gelu + 3 * res, 0.7 * n + 2),
                       cost(64, 4, 0.78 * n + 1.2 + 1.2 * gelu + 1.7 * res, 0.45 * n + 1.5),
                       cost(64, 2, 0.37 * n + 1.15 + 0.6 * gelu + 0.95 * res, 0.27 * n + 1.5),
                       rounds(64, 32) * (0.2 * n + 1.9), rounds(32, 32) * (0.12 * n + 2.4)};
  const double* best = std::min_element(c, c + 6);
  const double mb = 1e-6 * units * a.Kp * (a.Kp % 512 ? 1 : 1.4);
  if (units <= 4096 && 1.2 + 3.2 * mb < *best) return launch_rows_q8<DT>(a, stream);
  switch (best - c) {
    case 0: return launch_pipe_q8<PipeCfg<256, 256, 2, 4, 2>, DT>(a, stream);
    case 1: return launch_pipe_q8<PipeCfg<128, 128, 2, 4, 2>, DT>(a, stream);
    case 2: return launch_pipe_q8<PipeCfg<64, 64, 2, 2, 2>, DT>(a, stream);
    case 3: return launch_pipe_q8<PipeCfg<64, 64, 2, 2, 4>, DT>(a, stream);
    case 4: return launch_pipe_q8<PipeCfg<64, 32, 4, 1, 4, 2>, DT>(a, stream);
    default: return launch_pipe_q8<PipeCfg<32, 32, 2, 1, 4, 4>, DT>(a, stream);
  }
}

hipError_t launch_gemm_q8(const GemmQ8Args& a, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_q8<1>(a, stream) : launch_q8<0>(a, stream);
}

}  // namespace gl
