// The backward pass of layer norm.  With xh = (x - mean) rstd and h = dy gamma,
//   dx     = rstd (h - avg h - xh avg(h xh))      averages over the row's channels
//   dgamma = sum over rows of dy xh,   dbeta = sum over rows of dy
// One kernel reads dy and x once: a row's lanes hold it in registers, take the two
// averages, write dx, and each lane adds its channels' terms of dgamma and dbeta to
// sums of its own over all rows that it meets.  A workgroup then adds its lanes'
// sums and writes them to the workspace, and a second kernel adds the workgroups'.
// Everything is fp32, added in an order that depends on the sizes alone.
#include "gl_kernels.h"
#include "row_device.h"

namespace gl {

// LPR lanes hold a row, VPL chunks each; NT threads a workgroup.
template <int DT, int LPR, int VPL, int NT>
__global__ __launch_bounds__(NT) void norm_grad_kernel(NormGradArgs a) {
  using T = Chunk<DT>;
  constexpr int E = T::E, GROUPS = NT / LPR, NW = NT / 64;
  constexpr int COLS = LPR * VPL * E;  // columns a group covers
  __shared__ uint32_t slots[2][2][LPR > 64 ? LPR / 64 : 1];
  __shared__ float sums[LPR > 64 ? 1 : NW * COLS];
  const int lane = threadIdx.x & (LPR - 1), grp = threadIdx.x / LPR;
  const int C = a.C, n = (C + E - 1) / E;

  float w[VPL][E], dg[VPL][E], db[VPL][E];
#pragma unroll
  for (int v = 0; v < VPL; ++v)
#pragma unroll
    for (int j = 0; j < E; ++j) w[v][j] = 1.f, dg[v][j] = db[v][j] = 0.f;
  if (a.gamma)
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR;
      if (c < n) T::load(a.gamma, min(c * E, C - E), w[v]);
    }
  int turn = 0;
  // every group of a workgroup makes the same number of turns
  for (long long r0 = (long long)blockIdx.x * GROUPS; r0 < a.R; r0 += (long long)gridDim.x * GROUPS) {
    const bool mine = r0 + grp < a.R;
    const size_t row = mine ? r0 + grp : a.R - 1;
    const char* x = static_cast<const char*>(a.x) + row * a.ldx * T::kSize;
    const char* dy = static_cast<const char*>(a.dy) + row * a.lddy * T::kSize;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float f[VPL][E], d[VPL][E];
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR;
      if (c < n) {
        T::load(x, min(c * E, C - E), f[v]);
        T::load(dy, min(c * E, C - E), d[v]);
      }
    }
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR, skip = max(c * E + E - C, 0);
      if (c < n)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          f[v][j] = (f[v][j] - mean) * rstd;
          const float one = mine ? d[v][j] : 0.f;  // rows past the last count for nothing
          dg[v][j] = fmaf(one, f[v][j], dg[v][j]);
          db[v][j] += one;
          d[v][j] *= w[v][j];
          const float h = j >= skip ? d[v][j] : 0.f;
          s0 += h;
          s1 = fmaf(h, f[v][j], s1);
        }
    }
    // two turns' words never meet: a wave is at most one barrier ahead
    s0 = sum_row<LPR>(s0, slots[turn & 1][0]) * a.inv_c;
    s1 = sum_row<LPR>(s1, slots[turn & 1][1]) * a.inv_c;
    ++turn;
    if (a.dx && mine)
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
        const int c = lane + v * LPR;
        if (c < n) {
          float y[E];
#pragma unroll
          for (int j = 0; j < E; ++j) y[j] = (d[v][j] - fmaf(f[v][j], s1, s0)) * rstd;
          T::store(a.dx, row * C + min(c * E, C - E), y);
        }
      }
  }
  if (!a.part) return;

  float* pg = a.part + (size_t)blockIdx.x * 2 * C;
  if (LPR > 64) {  // a lane's columns are its own
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR, i = min(c * E, C - E), skip = max(c * E + E - C, 0);
      if (c < n)
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (j >= skip) {
            pg[i + j] = dg[v][j];
            pg[C + i + j] = db[v][j];
          }
    }
    return;
  }
  const int wave = threadIdx.x >> 6;
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int v = 0; v < VPL; ++v)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        float s = half ? db[v][j] : dg[v][j];
        if (LPR == 16) {  // the wave's four groups
          s += __shfl_xor(s, 16);
          s += __shfl_xor(s, 32);
        }
        if ((threadIdx.x & 63) < LPR) sums[wave * COLS + (lane + v * LPR) * E + j] = s;
      }
    __syncthreads();
    // column c's chunk holds it at its own place, or the last chunk moved back
    for (int c = threadIdx.x; c < C; c += NT) {
      const int last = (n - 1) * E, at = c < last ? c : c + (n * E - C);
      float s = sums[at];
      for (int k = 1; k < NW; ++k) s += sums[k * COLS + at];
      pg[half * C + c] = s;
    }
    __syncthreads();
  }
}

// out[c] = sum over the G rows of part [G, cols]: 64 columns a workgroup, its 16
// waves take every 16th row.
__global__ __launch_bounds__(1024) void norm_grad_sum_kernel(const float* part, int G, int cols,
                                                             float* dgamma, float* dbeta) {
  __shared__ float sums[16][64];
  const int t = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + t;
  float s = 0.f;
  if (c < 2 * cols)
    for (int g = w; g < G; g += 16) s += part[(size_t)g * 2 * cols + c];
  sums[w][t] = s;
  __syncthreads();
  if (w == 0 && c < 2 * cols) {
    for (int k = 1; k < 16; ++k) s += sums[k][t];
    if (c < cols) {
      if (dgamma) dgamma[c] = s;
    } else if (dbeta) dbeta[c - cols] = s;
  }
}

// Rows shorter than a chunk or longer than the largest tile: dx a workgroup a row,
// value by value; the sums over rows by columns, a thread each.
template <int DT>
__global__ __launch_bounds__(256) void norm_grad_any_kernel(NormGradArgs a) {
  using T = Chunk<DT>;
  __shared__ uint32_t slots[2][4];
  const int C = a.C;
  for (long long r = blockIdx.x; r < a.R; r += gridDim.x) {
    const char* x = static_cast<const char*>(a.x) + r * a.ldx * T::kSize;
    const char* dy = static_cast<const char*>(a.dy) + r * a.lddy * T::kSize;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s0 = 0.f, s1 = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) {
      const float h = T::load1(dy, c) * (a.gamma ? T::load1(a.gamma, c) : 1.f);
      s0 += h;
      s1 = fmaf(h, (T::load1(x, c) - mean) * rstd, s1);
    }
    s0 = sum_row<256>(s0, slots[0]) * a.inv_c;
    s1 = sum_row<256>(s1, slots[1]) * a.inv_c;
    for (int c = threadIdx.x; c < C; c += 256) {
      const float h = T::load1(dy, c) * (a.gamma ? T::load1(a.gamma, c) : 1.f);
      T::store1(a.dx, r * C + c, (h - fmaf((T::load1(x, c) - mean) * rstd, s1, s0)) * rstd);
    }
    __syncthreads();  // the words of slots are free again
  }
}

template <int DT>
__global__ __launch_bounds__(256) void norm_grad_any_cols_kernel(NormGradArgs a) {
  using T = Chunk<DT>;
  const int c = blockIdx.x * 256 + threadIdx.x, C = a.C;
  if (c >= C) return;
  float sg = 0.f, sb = 0.f;
  for (long long r = blockIdx.y; r < a.R; r += gridDim.y) {
    const float d = T::load1(static_cast<const char*>(a.dy) + r * a.lddy * T::kSize, c);
    const float f = T::load1(static_cast<const char*>(a.x) + r * a.ldx * T::kSize, c);
    sg = fmaf(d, (f - a.mean[r]) * a.rstd[r], sg);
    sb += d;
  }
  float* p = a.part + (size_t)blockIdx.y * 2 * C;
  p[c] = sg;
  p[C + c] = sb;
}

namespace {

struct Plan {
  const void* fn;  // null: value by value
  int threads, groups, grid;
};

template <int DT>
Plan plan(int R, int C) {
  constexpr int E = Chunk<DT>::E;
  const int n = (C + E - 1) / E;
  auto make = [&](const void* fn, int threads, int lpr, int most) {
    const int groups = threads / lpr;
    return Plan{fn, threads, groups, (int)std::min<long long>(((long long)R + groups - 1) / groups, most)};
  };
  if (C < E || n > 2048) return Plan{nullptr, 256, 1, std::min(R, 256)};
  if (n <= 16) return make((const void*)&norm_grad_kernel<DT, 16, 1, 1024>, 1024, 16, 512);
  if (n <= 32) return make((const void*)&norm_grad_kernel<DT, 16, 2, 512>, 512, 16, 512);
  if (n <= 64) return make((const void*)&norm_grad_kernel<DT, 64, 1, 512>, 512, 64, 512);
  if (n <= 128) return make((const void*)&norm_grad_kernel<DT, 64, 2, 512>, 512, 64, 512);
  if (n <= 256) return make((const void*)&norm_grad_kernel<DT, 64, 4, 256>, 256, 64, 512);
  if (n <= 512) return make((const void*)&norm_grad_kernel<DT, 256, 2, 256>, 256, 256, 512);
  if (n <= 1024) return make((const void*)&norm_grad_kernel<DT, 256, 4, 256>, 256, 256, 512);
  return make((const void*)&norm_grad_kernel<DT, 1024, 2, 1024>, 1024, 1024, 256);
}

template <int DT>
hipError_t launch_grad(NormGradArgs a, hipStream_t stream) {
  const Plan p = plan<DT>(a.R, a.C);
  float* const part = a.part;
  const bool sums = a.dgamma || a.dbeta;
  if (!sums) a.part = nullptr;
  void* argv[] = {&a};
  hipError_t e = hipSuccess;
  if (p.fn) {
    e = hipLaunchKernel(p.fn, dim3(p.grid), dim3(p.threads), argv, 0, stream);
  } else {
    if (a.dx)
      e = hipLaunchKernel((const void*)&norm_grad_any_kernel<DT>, dim3(std::min(a.R, 65536)), dim3(256),
                          argv, 0, stream);
    if (e == hipSuccess && sums)
      e = hipLaunchKernel((const void*)&norm_grad_any_cols_kernel<DT>, dim3((a.C + 255) / 256, p.grid),
                          dim3(256), argv, 0, stream);
  }
  if (e != hipSuccess || !sums) return e;
  norm_grad_sum_kernel<<<(2 * a.C + 63) / 64, 1024, 0, stream>>>(part, p.grid, a.C, a.dgamma, a.dbeta);
  return hipGetLastError();
}

}  // namespace

size_t norm_grad_ws_bytes(int R, int C, int dt_bf16) {
  const int grid = dt_bf16 ? plan<1>(R, C).grid : plan<0>(R, C).grid;
  return (size_t)grid * 2 * C * 4;
}

hipError_t launch_norm_grad(const NormGradArgs& a, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_grad<1>(a, stream) : launch_grad<0>(a, stream);
}

}  // namespace gl
