// Fully connected layers on 8-bit rows:
//   out[r, o] = act_out( (sum_k A[r, k] W[o, k]) sa[r] sw[o] + bias[o] ) + residual[r, o]
// The sums are exact (int32, at most 131071 terms); then fp32 and one rounding.
//   - Staging as in the bf16 GEMM: 16 bytes a lane straight into LDS, a row's
//     16-byte slots permuted by its number, two buffers and one barrier a stage.
//   - MFMA 16x16x64: a lane's 16 bytes of a row are one operand, so the slots that
//     serve eight bf16 values serve sixteen of these.  Operands are swapped (W rows
//     first): a lane ends with four consecutive output columns of one row.
//   - Epilogue: the tile passes through LDS wave by wave, so that stores and
//     residual loads cover whole rows.
#include "gl_device.h"
#include "gl_kernels.h"

namespace gl {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4 mfma_i8(const uint4& a, const uint4& b, i32x4 acc) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a),
                                               __builtin_bit_cast(i32x4, b), acc, 0, 0, 0);
}

typedef uint32_t u32x4_w __attribute__((ext_vector_type(4), aligned(4), may_alias));

// 8 consecutive values of a bias, a residual or an output at any element's place
template <int DT>
__device__ __forceinline__ void load8(const void* p, size_t i, float* f) {
  if (DT) {
    unpack_bf16x8(load16_any(static_cast<const uint16_t*>(p) + i), f);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4_w v = reinterpret_cast<const u32x4_w*>(static_cast<const float*>(p) + i)[h];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[4 * h + j] = __uint_as_float(v[j]);
    }
  }
}
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

// BM x BN output tile, STEP bytes of K per row and stage, WR x WC waves.
template <int BM_, int BN_, int STEP_, int WR_, int WC_>
struct Q8Cfg {
  static constexpr int BM = BM_, BN = BN_, STEP = STEP_, WR = WR_, WC = WC_;
  static constexpr int kWaves = WR * WC, kThreads = 64 * kWaves;
  static constexpr int kStage = (BM + BN) * STEP;        // bytes of one stage buffer
  static constexpr int kLoads = kStage / 16 / kThreads;  // loads per lane and stage
  static constexpr int TM = BM / WR / 16, TN = BN / WC / 16;
  static constexpr size_t kSmem = (size_t)2 * kStage;
  static_assert((size_t)BM * BN * 4 <= kSmem, "epilogue tile exceeds the stage buffers");
  static_assert(kStage % (1024 * kWaves) == 0 && (STEP == 128 || STEP == 256), "whole loads per wave");
};

template <class G, int DT, int ACT_OUT, bool RES>
__global__ __launch_bounds__(G::kThreads) void gemm_q8_kernel(GemmQ8Args a) {
  extern __shared__ __align__(16) char smem[];
  constexpr int BM = G::BM, BN = G::BN, STEP = G::STEP, TM = G::TM, TN = G::TN, NL = G::kLoads;
  constexpr int SPR = STEP / 16, RPL = 64 / SPR;  // slots per row, rows per wave load
  const int R = a.R, Cout = a.Cout, rowb = a.Kp;
  const int nstages = (rowb + STEP - 1) / STEP;
  const int ntn = (Cout + BN - 1) / BN;
  const int blk = xcd_remap(blockIdx.x, gridDim.x);
  const int mt = blk / ntn, nt = blk - mt * ntn;
  const int m0 = mt * BM, n0 = nt * BN;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, t = lane & 15;
  const int wm = w / G::WC, wn = w % G::WC;

  // staging: rows past R or Cout repeat the last one; slots past Kp read zeros
  const uint32_t lds0 = lds_offset(smem);
  const char* src[NL];
  int slot[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = RPL * (w + G::kWaves * i) + lane / SPR;
    slot[i] = ((lane % SPR) ^ (r & (SPR - 1))) * 16;
    src[i] = (r < BM ? reinterpret_cast<const char*>(a.A) + (size_t)min(m0 + r, R - 1) * rowb
                     : reinterpret_cast<const char*>(a.W) + (size_t)min(n0 + r - BM, Cout - 1) * rowb) +
             slot[i];
  }
  auto stage = [&](int s) {
    const int off = s * STEP;
    const uint32_t d = lds0 + (s & 1) * G::kStage + w * 1024;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const char* p = src[i] + off;
      if (off + STEP > rowb)  // uniform: the last, partial stage
        p = off + slot[i] < rowb ? p : reinterpret_cast<const char*>(kZero16);
      lds_dma16(p, d + G::kWaves * i * 1024);
    }
  };
  stage(0);

  constexpr int WROWS = 16 * TM, WCOLS = 16 * TN;
  constexpr int LPR = WCOLS / 8, RPP = 64 / LPR, NP = WROWS / RPP;  // lanes per row, rows per pass
  constexpr int CSW = WCOLS / 4 < 16 ? WCOLS / 4 - 1 : 15;
  const int cq = lane % LPR, rq = lane / LPR;
  const int n = n0 + wn * WCOLS + cq * 8;
  const int row0 = m0 + wm * WROWS + rq;
  const bool vec = n + 8 <= Cout;
  float bn[8], sw[8];
#pragma unroll
  for (int v = 0; v < 8; ++v) {
    const int c = min(n + v, Cout - 1);
    bn[v] = a.bias ? load1<DT>(a.bias, c) : 0.f;
    sw[v] = a.sw[c];
  }

  i32x4 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  for (int s = 0; s < nstages; ++s) {
    // stage s has landed, and every wave is done reading stage s - 1's buffer
    dma_wait_barrier();
    if (s + 1 < nstages) stage(s + 1);
    const char* sa = smem + (s & 1) * G::kStage + (wm * WROWS + t) * STEP;
    const char* sb = smem + (s & 1) * G::kStage + (BM + wn * WCOLS + t) * STEP;
#pragma unroll
    for (int kk = 0; kk < STEP / 64; ++kk) {
      uint4 af[TM], bf[TN];
      const int co = ((kk * 4 + g) ^ (t & (SPR - 1))) * 16;
#pragma unroll
      for (int i = 0; i < TM; ++i) af[i] = *reinterpret_cast<const uint4*>(sa + i * 16 * STEP + co);
#pragma unroll
      for (int j = 0; j < TN; ++j) bf[j] = *reinterpret_cast<const uint4*>(sb + j * 16 * STEP + co);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma_i8(bf[j], af[i], acc[i][j]);
    }
  }

  // lane (g, t) of MFMA tile (i, j) holds columns 4g .. 4g+3 of row t
  __syncthreads();
  char* st = smem + w * (WROWS * WCOLS * 4);
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
      *reinterpret_cast<i32x4*>(st + (i * 16 + t) * (WCOLS * 4) + (((j * 4 + g) ^ (t & CSW)) * 16)) =
          acc[i][j];
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int r = p * RPP + rq, row = row0 + p * RPP;
    const char* sr = st + r * (WCOLS * 4);
    const i32x4 x0 = *reinterpret_cast<const i32x4*>(sr + ((2 * cq) ^ (r & CSW)) * 16);
    const i32x4 x1 = *reinterpret_cast<const i32x4*>(sr + ((2 * cq + 1) ^ (r & CSW)) * 16);
    if (row >= R || n >= Cout) continue;
    const float sar = a.sa[row];
    float y[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      y[v] = fmaf((float)(v < 4 ? x0[v & 3] : x1[v & 3]), sar * sw[v], bn[v]);
      if (ACT_OUT) y[v] = gelu_f32(y[v]);
    }
    const size_t o = (size_t)row * Cout + n;
    if (vec) {
      if (RES) {
        float f[8];
        load8<DT>(a.residual, o, f);
#pragma unroll
        for (int v = 0; v < 8; ++v) y[v] += f[v];
      }
      store8<DT>(a.out, o, y);
    } else {
#pragma unroll
      for (int v = 0; v < 8; ++v)
        if (n + v < Cout) {
          if (RES) y[v] += load1<DT>(a.residual, o + v);
          store1<DT>(a.out, o + v, y[v]);
        }
    }
  }
}

template <class G, int DT>
hipError_t launch_cfg_q8(const GemmQ8Args& a, hipStream_t stream) {
  const void* fn = a.act_out ? (a.residual ? (const void*)&gemm_q8_kernel<G, DT, 1, true>
                                           : (const void*)&gemm_q8_kernel<G, DT, 1, false>)
                             : (a.residual ? (const void*)&gemm_q8_kernel<G, DT, 0, true>
                                           : (const void*)&gemm_q8_kernel<G, DT, 0, false>);
  const dim3 grid((unsigned)(((long)(a.R + G::BM - 1) / G::BM) * ((a.Cout + G::BN - 1) / G::BN)));
  return launch_with_smem(fn, grid, dim3(G::kThreads), G::kSmem, stream, nullptr, nullptr, a);
}

template <int DT>
hipError_t launch_q8(const GemmQ8Args& a, hipStream_t stream) {
  auto tiles = [&](int bm, int bn) { return (long)((a.R + bm - 1) / bm) * ((a.Cout + bn - 1) / bn); };
  if (tiles(128, 128) >= 384) return launch_cfg_q8<Q8Cfg<128, 128, 128, 4, 2>, DT>(a, stream);
  if (tiles(64, 64) >= 128) return launch_cfg_q8<Q8Cfg<64, 64, 128, 2, 2>, DT>(a, stream);
  return launch_cfg_q8<Q8Cfg<32, 64, 256, 1, 4>, DT>(a, stream);
}

hipError_t launch_gemm_q8(const GemmQ8Args& a, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_q8<1>(a, stream) : launch_q8<0>(a, stream);
}

}  // namespace gl
