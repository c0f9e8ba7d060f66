// Rows of channels: layer norm, and rows brought to 8 bits with a scale each.
//   norm   y = (x - mean) rstd gamma + beta,  rstd = 1 / sqrt(var + eps)
//   8 bits q = rne(127 y / top), scale = top / 127, top = max |y| over the row
// One kernel: a row is read once and stays in registers, in fp32, while its
// statistics are taken (the mean first, then the squares of what is left, which
// loses nothing to cancellation) and its top is found; then it is written once.
#include "gl_kernels.h"
#include "row_device.h"

namespace gl {

enum { kNorm = 0, kNormQ8 = 1, kQ8 = 2 };

// LPR lanes hold a row, VPL chunks each.
template <int DT, int MODE, int LPR, int VPL>
__global__ __launch_bounds__(LPR > 256 ? LPR : 256) void row_kernel(RowArgs a) {
  using T = Chunk<DT>;
  constexpr int E = T::E;
  __shared__ uint32_t slots[3][LPR > 64 ? LPR / 64 : 1];
  const int lane = threadIdx.x & (LPR - 1);
  const long long g = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / LPR;
  const bool mine = g < a.R;
  const size_t row = mine ? g : a.R - 1;
  const int C = a.C, n = (C + E - 1) / E;
  const char* x = static_cast<const char*>(a.x) + row * a.ldx * T::kSize;

  float f[VPL][E];
#pragma unroll
  for (int v = 0; v < VPL; ++v) {
    const int c = lane + v * LPR;
    if (c < n) T::load(x, min(c * E, C - E), f[v]);
  }
  if (MODE != kQ8) {
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR, skip = max(c * E + E - C, 0);
      if (c < n)
#pragma unroll
        for (int j = 0; j < E; ++j) s += j >= skip ? f[v][j] : 0.f;
    }
    const float mean = sum_row<LPR>(s, slots[0]) * a.inv_c;
    s = 0.f;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR, skip = max(c * E + E - C, 0);
      if (c < n)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          f[v][j] -= mean;
          s = fmaf(j >= skip ? f[v][j] : 0.f, f[v][j], s);
        }
    }
    const float rstd = __builtin_amdgcn_rsqf(fmaf(sum_row<LPR>(s, slots[1]), a.inv_c, a.eps));
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR, i = min(c * E, C - E);
      if (c < n) {
        float w[E], b[E];
#pragma unroll
        for (int j = 0; j < E; ++j) w[j] = 1.f, b[j] = 0.f;
        if (a.gamma) T::load(a.gamma, i, w);
        if (a.beta) T::load(a.beta, i, b);
#pragma unroll
        for (int j = 0; j < E; ++j) f[v][j] = fmaf(f[v][j] * rstd, w[j], b[j]);
        if (MODE == kNorm && mine) T::store(a.out, row * C + i, f[v]);
      }
    }
    if (MODE == kNorm && mine && lane == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
  if (MODE != kNorm) {
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < VPL; ++v)
      if (lane + v * LPR < n)
#pragma unroll
        for (int j = 0; j < E; ++j) top = max(top, __float_as_uint(f[v][j]) & 0x7fffffffu);
    const RowQ8 q(max_row<LPR>(top, slots[2]));
    if (mine) {
      int8_t* d = a.q + row * a.Kp;
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
        const int c = lane + v * LPR;
        if (c < n) store_q8<E>(d + min(c * E, C - E), q, f[v]);
      }
      if (lane < a.Kp - C) d[C + lane] = 0;  // fewer than 16
      if (lane == 0) a.scale[row] = q.scale;
    }
  }
}

// Rows shorter than a chunk or longer than the largest tile above: a workgroup a
// row, value by value, read once more for each of the steps.
template <int DT, int MODE>
__global__ __launch_bounds__(256) void row_any_kernel(RowArgs a) {
  using T = Chunk<DT>;
  __shared__ uint32_t slots[3][4];
  const size_t row = blockIdx.x;
  const int C = a.C;
  const char* x = static_cast<const char*>(a.x) + row * a.ldx * T::kSize;
  float mean = 0.f, rstd = 1.f;
  if (MODE != kQ8) {
    float s = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) s += T::load1(x, c);
    mean = sum_row<256>(s, slots[0]) * a.inv_c;
    s = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) {
      const float d = T::load1(x, c) - mean;
      s = fmaf(d, d, s);
    }
    rstd = __builtin_amdgcn_rsqf(fmaf(sum_row<256>(s, slots[1]), a.inv_c, a.eps));
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
    const RowQ8 q(max_row<256>(top, slots[2]));
    int8_t* d = a.q + row * a.Kp;
    for (int c = threadIdx.x; c < a.Kp; c += 256) d[c] = c < C ? (int8_t)(q.bits(value(c)) & 0xff) : 0;
    if (threadIdx.x == 0) a.scale[row] = q.scale;
  }
}

template <int DT, int MODE>
hipError_t launch_row_mode(const RowArgs& a, hipStream_t stream) {
  constexpr int E = Chunk<DT>::E;
  const int n = (a.C + E - 1) / E;
  void* argv[] = {const_cast<RowArgs*>(&a)};
  auto go = [&](const void* fn, int lpr) {
    const int threads = lpr > 256 ? lpr : 256, per = threads / lpr;
    return hipLaunchKernel(fn, dim3((unsigned)((a.R + per - 1) / per)), dim3(threads), argv, 0, stream);
  };
  if (a.C < E || n > 2048) return go((const void*)&row_any_kernel<DT, MODE>, 256);
  if (n <= 16) return go((const void*)&row_kernel<DT, MODE, 16, 1>, 16);
  if (n <= 32) return go((const void*)&row_kernel<DT, MODE, 16, 2>, 16);
  if (n <= 64) return go((const void*)&row_kernel<DT, MODE, 64, 1>, 64);
  if (n <= 128) return go((const void*)&row_kernel<DT, MODE, 64, 2>, 64);
  if (n <= 256) return go((const void*)&row_kernel<DT, MODE, 64, 4>, 64);
  if (n <= 512) return go((const void*)&row_kernel<DT, MODE, 256, 2>, 256);
  if (n <= 1024) return go((const void*)&row_kernel<DT, MODE, 256, 4>, 256);
  return go((const void*)&row_kernel<DT, MODE, 256, 8>, 256);
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
