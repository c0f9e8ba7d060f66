// Rows of channels: layer norm, and rows brought to 8 bits with a scale each.
//   norm   y = (x - mean) rstd gamma + beta,  rstd = 1 / sqrt(var + eps)
//   8 bits q = rne(127 y / top), scale = top / 127, top = max |y| over the row
// One kernel: a row is read once and stays in registers, in fp32, while its
// statistics are taken (the mean first, then the squares of what is left, which
// loses nothing to cancellation) and its top is found; then it is written once.
// Memory bounds it: us a call in a row of calls on three inputs in turn (and TB/s of what it
// has to read and write; a copy of 1 GiB reaches 5.3) in bf16, norm, 8 bits, norm to 8 bits:
//   32768 x 2560   62.0 (5.4)   47.9 (5.3)   59.1 (4.3)
//   100352 x 320   26.2 (4.9)   17.3 (5.6)   25.3 (3.8)
//   100352 x 80     7.7 (4.2)    6.6 (3.7)    9.4 (2.6)
//   6272 x 192      3.3 (1.5)    2.5 (1.4)    3.5 (1.0)
// Small inputs take a launch and one trip to memory, about 3 us; the norm to 8 bits
// has twice the arithmetic of the norm, which then shows.
#include "gl_kernels.h"
#include "row_device.h"

namespace gl {

enum { kNorm = 0, kNormQ8 = 1, kQ8 = 2 };

// sum / C by 1 / C in two parts, so that the quotient is rounded as if once and a row of
// equal values whose sum is exact has them as its mean (by a rounded 1 / C alone 1000
// channels of 1e5 were 0.008 off it, and the norm 0.93 for 0).  Both parts are positive: an
// infinite sum stays one.
__device__ __forceinline__ float row_mean(float sum, const RowArgs& a) {
  return fmaf(sum, a.mean_hi, sum * a.mean_lo);
}

// 1 / sqrt(var + eps) of the sum of squares.  The hardware's root takes a subnormal for zero:
// where eps leaves room for one (TINY), a small argument is scaled by a power of four first.
// A variant of its own, since the four instructions a row take 3 % of 100352 x 80 (7.70 us
// for 7.50), and a branch on eps in their place as much.
constexpr float kTinyEps = 0x1p-100f;
template <bool TINY>
__device__ __forceinline__ float row_rstd(float sq, const RowArgs& a) {
  const float v = fmaf(sq, a.inv_c, a.eps);
  if (!TINY) return __builtin_amdgcn_rsqf(v);
  const bool tiny = v < kTinyEps;
  return __builtin_amdgcn_rsqf(tiny ? v * 0x1p100f : v) * (tiny ? 0x1p50f : 1.f);
}

// LPR lanes hold a row, VPL chunks each.  A workgroup takes many rows: gamma and beta
// stay in registers, and a row's loads are under way while the one before is worked on.
template <int DT, int MODE, int LPR, int VPL, bool TINY>
__global__ __launch_bounds__(256) void row_kernel(RowArgs a) {
  using T = Chunk<DT>;
  constexpr int E = T::E, GROUPS = 256 / LPR;
  __shared__ uint32_t slots[2][3][4];
  const WaveRows<LPR> rows;
  const int lane = threadIdx.x & (LPR - 1);
  const int C = a.C, n = (C + E - 1) / E;
  const bool ragged = C % E != 0;  // the last chunk repeats values of the one before it

  // lanes past the row's last chunk hold it once more: their values count in no sum, and
  // are not stored
  int at[VPL];  // the chunk's place in its row
#pragma unroll
  for (int v = 0; v < VPL; ++v) at[v] = min(min(lane + v * LPR, n - 1) * E, C - E);
  auto on = [&](int v) { return lane + v * LPR < n; };
  uint4 raw[VPL];
  auto load = [&](long long r0) {
    uint32_t off;
    const char* x = rows.at(a.x, r0 + rows.wave, a.R, a.ldx * (long long)T::kSize, &off);
#pragma unroll
    for (int v = 0; v < VPL; ++v) raw[v] = T::raw_at(x, off + at[v] * (uint32_t)T::kSize);
  };
  const long long step = (long long)gridDim.x * GROUPS;
  long long r0 = (long long)blockIdx.x * GROUPS;
  load(r0);
  uint4 gamma[VPL], beta[VPL];
  if (MODE != kQ8) {
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      gamma[v] = T::ones();
      beta[v] = make_uint4(0, 0, 0, 0);
      if (a.gamma) gamma[v] = T::raw(a.gamma, at[v]);
      if (a.beta) beta[v] = T::raw(a.beta, at[v]);
    }
  }
  int turn = 0;
  // every group of a workgroup makes the same number of turns
  for (; r0 < a.R; r0 += step, turn ^= 1) {
    const long long first = r0 + rows.wave;  // the wave's
    const bool mine = first + rows.lane < a.R;
    float f[VPL][E];
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      T::unpack(raw[v], f[v]);
      if (MODE == kQ8) top = max(top, T::top(raw[v]));
    }
    if (r0 + step < a.R) load(r0 + step);
    if (MODE != kQ8) {
      // sum over the row of what `term` makes of each value
      auto sum = [&](auto term, uint32_t* slot) {
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
          float p = 0.f;
          if (ragged) {
            const int skip = (lane + v * LPR) * E - at[v];
#pragma unroll
            for (int j = 0; j < E; ++j) p = j >= skip ? term(p, f[v][j]) : p;
          } else {
#pragma unroll
            for (int j = 0; j < E; ++j) p = term(p, f[v][j]);
          }
          s += on(v) ? p : 0.f;
        }
        return sum_row<LPR>(s, slot);
      };
      const float mean = row_mean(sum([](float s, float x) { return s + x; }, slots[turn][0]), a);
#pragma unroll
      for (int v = 0; v < VPL; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) f[v][j] -= mean;
      const float rstd = row_rstd<TINY>(sum([](float s, float x) { return fmaf(x, x, s); }, slots[turn][1]), a);
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
        float w[E], b[E];
        if (VPL > 1) keep_packed(gamma[v]), keep_packed(beta[v]);
        T::unpack(gamma[v], w);
        T::unpack(beta[v], b);
#pragma unroll
        for (int j = 0; j < E; ++j) f[v][j] = fmaf(f[v][j] * rstd, w[j], b[j]);
        if (MODE == kNorm && mine && on(v))
          T::store_at(static_cast<char*>(a.out) + first * C * (long long)T::kSize,
                      (rows.lane * (uint32_t)C + at[v]) * (uint32_t)T::kSize, f[v]);
      }
      if (MODE == kNorm && mine && lane == 0) {
        if (a.mean) (a.mean + first)[rows.lane] = mean;
        if (a.rstd) (a.rstd + first)[rows.lane] = rstd;
      }
    }
    if (MODE != kNorm) {
      if (MODE == kNormQ8) {
#pragma unroll
        for (int v = 0; v < VPL; ++v)
#pragma unroll
          for (int j = 0; j < E; ++j) top = max(top, __float_as_uint(f[v][j]) & 0x7fffffffu);
      }
      const RowQ8<DT == 0 && MODE == kQ8> q(max_row<LPR>(top, slots[turn][2]));
      if (mine) {
        int8_t* d = a.q + first * a.Kp;
        const uint32_t off = rows.lane * (uint32_t)a.Kp;
#pragma unroll
        for (int v = 0; v < VPL; ++v)
          if (on(v)) store_q8<E>(d + (off + at[v]), q, f[v]);
        for (int k = lane; k < a.Kp - C; k += LPR) d[off + C + k] = 0;  // fewer than 16
        if (lane == 0) (a.scale + first)[rows.lane] = q.scale;
      }
    }
  }
}

// Rows shorter than a chunk or longer than the largest tile above: a workgroup a
// row, value by value, read once more for each of the steps.
template <int DT, int MODE>
__global__ __launch_bounds__(256) void row_any_kernel(RowArgs a) {
  using T = Chunk<DT>;
  __shared__ uint32_t slots[3][4];
  const int C = a.C;
  for (long long r = blockIdx.x; r < a.R; r += gridDim.x) {
  const size_t row = r;
  const char* x = static_cast<const char*>(a.x) + row * a.ldx * T::kSize;
  float mean = 0.f, rstd = 1.f;
  if (MODE != kQ8) {
    float s = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) s += T::load1(x, c);
    mean = row_mean(sum_row<256>(s, slots[0]), a);
    s = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) {
      const float d = T::load1(x, c) - mean;
      s = fmaf(d, d, s);
    }
    rstd = row_rstd<true>(sum_row<256>(s, slots[1]), a);
  }
  auto value = [&](int c) {
    const float v = T::load1(x, c);
    if (MODE == kQ8) return v;
    return fmaf((v - mean) * rstd, a.gamma ? T::load1(a.gamma, c) : 1.f,
                a.beta ? T::load1(a.beta, c) : 0.f);
  };
  if (MODE == kNorm) {
    for (int c = threadIdx.x; c < C; c += 256) T::store1(a.out, row * C + c, value(c));
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  } else {
    uint32_t top = 0;
    for (int c = threadIdx.x; c < C; c += 256) top = max(top, __float_as_uint(value(c)) & 0x7fffffffu);
    const RowQ8<DT == 0 && MODE == kQ8> q(max_row<256>(top, slots[2]));
    int8_t* d = a.q + row * a.Kp;
    for (int c = threadIdx.x; c < a.Kp; c += 256) d[c] = c < C ? q.one(value(c)) : 0;
    if (threadIdx.x == 0) a.scale[row] = q.scale;
  }
  __syncthreads();  // the words of slots are free again
  }
}

// The lanes and chunks for rows of n chunks: at most three a lane up to 768 chunks, whose
// registers leave four waves a SIMD and more; four up to 1024 (three and more) and eight
// past that (two and more), where a workgroup has no more lanes.  Many short rows lie four
// to a wave, 16 lanes each: their sums take four steps within 16 lanes, and a wave has more
// bytes in flight.  Eight to a wave where that leaves one chunk a lane (100352 x 40 bf16,
// norm 6.0 us for 7.6), and for 8 bits alone, which need no weights, up to three
// (100352 x 192 11.1 for 12.3; the norm would take 17.4 for 15.3).
template <int DT, int MODE, bool TINY>
hipError_t launch_row_tiny(const RowArgs& a, hipStream_t stream) {
  constexpr int E = Chunk<DT>::E;
  const int n = (a.C + E - 1) / E;
  void* argv[] = {const_cast<RowArgs*>(&a)};
  // `rows` a workgroup and turn; at most `per_cu` workgroups a CU, with equal numbers of turns
  auto go = [&](const void* fn, int rows, int per_cu = 16) {
    const long long units = ((long long)a.R + rows - 1) / rows, most = 256LL * per_cu;
    const long long turns = (units + most - 1) / most;
    return hipLaunchKernel(fn, dim3((unsigned)((units + turns - 1) / turns)), dim3(256), argv, 0, stream);
  };
#define GL_ROW(LPR, VPL) go((const void*)&row_kernel<DT, MODE, LPR, VPL, TINY>, 256 / LPR)
  if (a.C < E || n > 2048) return go((const void*)&row_any_kernel<DT, MODE>, 1);
  // the eight rows of a wave lie within 32 bits of the first
  const bool near = a.R == 1 || a.ldx < 1 << 27;
  if (near && a.R >= 16384) {
    if (n <= 8) return GL_ROW(8, 1);
    if constexpr (MODE == kQ8)
      if (n <= 24) return n <= 16 ? GL_ROW(8, 2) : GL_ROW(8, 3);
  }
  if (n <= 16 && near) return GL_ROW(16, 1);
  if (n <= 48 && near && a.R >= 4096) return n <= 32 ? GL_ROW(16, 2) : GL_ROW(16, 3);
  if (n <= 192) return n <= 64 ? GL_ROW(64, 1) : n <= 128 ? GL_ROW(64, 2) : GL_ROW(64, 3);
  if (n <= 384) return n <= 256 ? GL_ROW(128, 2) : GL_ROW(128, 3);
  if (n <= 1024) return n <= 512 ? GL_ROW(256, 2) : n <= 768 ? GL_ROW(256, 3) : GL_ROW(256, 4);
  // two workgroups a CU: more of them would load gamma and beta for a row each (4096 x 8192
  // fp32: 55 us, 91 with 16 a CU)
  return go((const void*)&row_kernel<DT, MODE, 256, 8, TINY>, 1, 2);
#undef GL_ROW
}

template <int DT, int MODE>
hipError_t launch_row_mode(const RowArgs& a, hipStream_t stream) {
  if constexpr (MODE != kQ8)
    if (a.eps < kTinyEps) return launch_row_tiny<DT, MODE, true>(a, stream);
  return launch_row_tiny<DT, MODE, false>(a, stream);
}

hipError_t launch_layer_norm(const RowArgs& a, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_row_mode<1, kNorm>(a, stream) : launch_row_mode<0, kNorm>(a, stream);
}
hipError_t launch_layer_norm_q8(const RowArgs& a, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_row_mode<1, kNormQ8>(a, stream) : launch_row_mode<0, kNormQ8>(a, stream);
}
hipError_t launch_quantize_rows(const RowArgs& a, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_row_mode<1, kQ8>(a, stream) : launch_row_mode<0, kQ8>(a, stream);
}

}  // namespace gl
