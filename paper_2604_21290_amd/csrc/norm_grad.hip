// The backward pass of layer norm.  With xh = (x - mean) rstd and h = dy gamma,
//   dx     = rstd (h - avg h - xh avg(h xh))      averages over the row's channels
//   dgamma = sum over rows of dy xh,   dbeta = sum over rows of dy
// One kernel reads dy and x once: a row's lanes hold it in registers, take the two
// averages, write dx, and each lane adds its channels' terms of dgamma and dbeta to
// sums of its own over all rows that it meets.  A workgroup then adds its lanes'
// sums and writes them to the workspace, and a second kernel adds the workgroups'.
// Memory bounds it where rows are many: us (TB/s of dy, x and dx) in bf16, a call in a row of
// calls on three inputs in turn, 32768 x 2560 98 (5.1; 111 in a first run), 100352 x 320
// 43 (4.5), 100352 x 80 14.6 (3.3, of which the second kernel and the gap before it take 4),
// 8193 x 1001 15.3 (3.2).  Few rows take one launch.
// Everything is fp32, added in an order that depends on the sizes alone.
#include "gl_kernels.h"
#include "row_device.h"

namespace gl {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4), may_alias));
__device__ __forceinline__ void store4_any(float* p, const float* f) {
  *reinterpret_cast<f32x4_any*>(p) = f32x4_any{f[0], f[1], f[2], f[3]};
}

// LPR lanes hold a row, VPL chunks each; NT threads a workgroup.  A row's loads are
// under way while the one before it is worked on.
template <int DT, int LPR, int VPL, int NT>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(VPL <= 2 ? 4 : 2)))
void norm_grad_kernel(NormGradArgs a) {
  using T = Chunk<DT>;
  constexpr int E = T::E, GROUPS = NT / LPR, NW = NT / 64;
  constexpr int COLS = LPR * VPL * E;  // columns a group covers
  __shared__ uint32_t slots[2][2][NT / 64];
  __shared__ float sums[LPR > 64 ? 1 : NW * COLS];
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
  uint4 raw_x[VPL], raw_d[VPL];
  float mean, rstd;
  auto load = [&](long long r0) {
    uint32_t off_x, off_d, off;
    const char* x = rows.at(a.x, r0 + rows.wave, a.R, a.ldx * (long long)T::kSize, &off_x);
    const char* dy = rows.at(a.dy, r0 + rows.wave, a.R, a.lddy * (long long)T::kSize, &off_d);
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      raw_x[v] = T::raw_at(x, off_x + at[v] * (uint32_t)T::kSize);
      raw_d[v] = T::raw_at(dy, off_d + at[v] * (uint32_t)T::kSize);
    }
    const char* m = rows.at(a.mean, r0 + rows.wave, a.R, 4, &off);
    mean = *reinterpret_cast<const float*>(m + off);
    const char* s = rows.at(a.rstd, r0 + rows.wave, a.R, 4, &off);
    rstd = *reinterpret_cast<const float*>(s + off);
  };
  const long long step = (long long)gridDim.x * GROUPS;
  long long r0 = (long long)blockIdx.x * GROUPS;
  load(r0);

  float dg[VPL][E], db[VPL][E];
  uint4 raw_w[VPL];
#pragma unroll
  for (int v = 0; v < VPL; ++v) {
#pragma unroll
    for (int j = 0; j < E; ++j) dg[v][j] = db[v][j] = 0.f;
    raw_w[v] = T::ones();
    if (a.gamma) raw_w[v] = T::raw(a.gamma, at[v]);
  }
  int turn = 0;
  // every group of a workgroup makes the same number of turns
  for (; r0 < a.R; r0 += step, turn ^= 1) {
    const long long first = r0 + rows.wave;  // the wave's
    const bool mine = first + rows.lane < a.R;
    float f[VPL][E], d[VPL][E];
    const float mu = mean, rs = rstd;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      T::unpack(raw_x[v], f[v]);
      T::unpack(raw_d[v], d[v]);
    }
    if (r0 + step < a.R) load(r0 + step);
    if (!mine)  // rows past the last count for nothing
#pragma unroll
      for (int v = 0; v < VPL; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) d[v][j] = 0.f;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      float w[E], p0 = 0.f, p1 = 0.f;
      if (VPL > 1) keep_packed(raw_w[v]);
      T::unpack(raw_w[v], w);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        f[v][j] = (f[v][j] - mu) * rs;
        dg[v][j] = fmaf(d[v][j], f[v][j], dg[v][j]);
        db[v][j] += d[v][j];
        d[v][j] *= w[j];
      }
      if (ragged) {
        const int skip = (lane + v * LPR) * E - at[v];
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const float h = j >= skip ? d[v][j] : 0.f;
          p0 += h;
          p1 = fmaf(h, f[v][j], p1);
        }
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) {
          p0 += d[v][j];
          p1 = fmaf(d[v][j], f[v][j], p1);
        }
      }
      s0 += on(v) ? p0 : 0.f;
      s1 += on(v) ? p1 : 0.f;
    }
    // two turns' words never meet: a wave is at most one barrier ahead
    s0 = sum_row<LPR>(s0, slots[turn][0]) * a.inv_c * -rs;
    s1 = sum_row<LPR>(s1, slots[turn][1]) * a.inv_c * -rs;
    if (a.dx && mine)
#pragma unroll
      for (int v = 0; v < VPL; ++v)
        if (on(v)) {
          float y[E];
#pragma unroll
          for (int j = 0; j < E; ++j) y[j] = fmaf(d[v][j], rs, fmaf(f[v][j], s1, s0));
          T::store_at(static_cast<char*>(a.dx) + first * C * (long long)T::kSize,
                      (rows.lane * (uint32_t)C + at[v]) * (uint32_t)T::kSize, y);
        }
  }
  if (!a.part) return;

  float* pg = a.part + (size_t)blockIdx.x * 2 * C;
  if (LPR > 64) {  // a lane's columns are its own
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR, i = min(c * E, C - E), skip = max(c * E + E - C, 0);
      if (c < n && skip == 0) {
#pragma unroll
        for (int j = 0; j < E; j += 4) {
          store4_any(pg + i + j, &dg[v][j]);
          store4_any(pg + C + i + j, &db[v][j]);
        }
      } else if (c < n) {
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (j >= skip) {
            pg[i + j] = dg[v][j];
            pg[C + i + j] = db[v][j];
          }
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
        if (LPR < 64) s = sum_over_groups<LPR>(s);  // the wave's
        if ((threadIdx.x & 63) < LPR) sums[wave * COLS + (lane + v * LPR) * E + j] = s;
      }
    __syncthreads();
    // column c's chunk holds it at its own place, or the last chunk moved back
    for (int c = threadIdx.x; c < C; c += NT) {
      const int last = (n - 1) * E, at = c < last ? c : c + (n * E - C);
      float s = sums[at];
#pragma unroll
      for (int k = 1; k < NW; ++k) s += sums[k * COLS + at];
      pg[half * C + c] = s;
    }
    __syncthreads();
  }
}

// out[c] = sum over the G rows of part [G, 2 cols]: 32 columns a workgroup (whole lines;
// with 8 the second kernel of 8193 x 1001 took 1.7 us more), 32 rows at a time, in the
// same order always.
__global__ __launch_bounds__(1024) void norm_grad_sum_kernel(const float* part, int G, int cols, int first,
                                                             float* dgamma, float* dbeta) {
  constexpr int COLS = 32, ROWS = 1024 / COLS;
  __shared__ float sums[ROWS][COLS + 1];
  const int t = threadIdx.x % COLS, w = threadIdx.x / COLS;
  const int c = first + blockIdx.x * COLS + t;
  float s = 0.f;
  // (eight loads under way at a time, also where there are fewer left)
  for (int g0 = w; g0 < G; g0 += 8 * ROWS) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int g = g0 + u * ROWS;
      v[u] = part[(size_t)min(g, G - 1) * 2 * cols + min(c, 2 * cols - 1)];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) s += g0 + u * ROWS < G ? v[u] : 0.f;
  }
  sums[w][t] = s;
#pragma unroll
  for (int h = ROWS / 2; h >= 1; h /= 2) {
    __syncthreads();
    if (w < h) sums[w][t] += sums[w + h][t];
  }
  if (w == 0 && c < 2 * cols) {
    s = sums[0][t];
    if (c < cols) {
      if (dgamma) dgamma[c] = s;
    } else if (dbeta) dbeta[c - cols] = s;
  }
}

// Few rows, in one launch and without a workspace: the first `row_wgs` workgroups take
// rows, 512 / LPR each, the others 8 chunks of columns each, over all rows: the columns'
// sums need no average of a row, and reading a small input twice is cheap.  What a column
// workgroup takes is trips to memory, of up to 8 x 64 rows each (with 256 threads on 16
// chunks 392 x 2560 bf16 took 7.0 us for 5.5, 784 x 2560 12.6 for 9.3).
template <int DT, int LPR, int VPL>
__global__ __launch_bounds__(512) void norm_grad_few_kernel(NormGradArgs a, int row_wgs) {
  using T = Chunk<DT>;
  constexpr int E = T::E, NT = 512, GROUPS = NT / LPR, CL = 8, RG = NT / CL;
  __shared__ uint32_t slots[2][NT / 64];
  __shared__ float sums[2][NT / 64][CL * E];
  const int C = a.C, n = (C + E - 1) / E;
  if ((int)blockIdx.x < row_wgs) {
    const int lane = threadIdx.x & (LPR - 1);
    const long long r = (long long)blockIdx.x * GROUPS + threadIdx.x / LPR;
    const bool mine = r < a.R;
    const size_t row = mine ? r : a.R - 1;
    const char* x = static_cast<const char*>(a.x) + row * a.ldx * T::kSize;
    const char* dy = static_cast<const char*>(a.dy) + row * a.lddy * T::kSize;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float f[VPL][E], d[VPL][E], s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR, i = min(c * E, C - E);
      if (c >= n) continue;
      T::unpack(T::raw(x, i), f[v]);
      T::unpack(T::raw(dy, i), d[v]);
      if (a.gamma) {
        float w[E];
        T::unpack(T::raw(a.gamma, i), w);
#pragma unroll
        for (int j = 0; j < E; ++j) d[v][j] *= w[j];
      }
    }
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR, skip = max(c * E + E - C, 0);
      if (c >= n) continue;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        f[v][j] = (f[v][j] - mean) * rstd;
        const float h = j >= skip ? d[v][j] : 0.f;
        s0 += h;
        s1 = fmaf(h, f[v][j], s1);
      }
    }
    s0 = sum_row<LPR>(s0, slots[0]) * a.inv_c;
    s1 = sum_row<LPR>(s1, slots[1]) * a.inv_c;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * LPR;
      if (c >= n || !mine) continue;
      float y[E];
#pragma unroll
      for (int j = 0; j < E; ++j) y[j] = (d[v][j] - fmaf(f[v][j], s1, s0)) * rstd;
      T::store(a.dx, row * C + min(c * E, C - E), y);
    }
    return;
  }
  const int lane = threadIdx.x % CL, grp = threadIdx.x / CL;
  const int c = ((int)blockIdx.x - row_wgs) * CL + lane, i = min(c * E, C - E);
  float dg[E] = {}, db[E] = {};
  if (c < n) {
    // (U rows under way at a time, also where there are fewer left)
    constexpr int U = 8;
    for (int first = 0; first < a.R; first += U * RG) {
      uint4 f4[U] = {}, d4[U] = {};
      float mean[U] = {}, rstd[U] = {};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (first + u * RG >= a.R) break;
        const int r = first + u * RG + grp, row = min(r, a.R - 1);
        f4[u] = T::raw(static_cast<const char*>(a.x) + (size_t)row * a.ldx * T::kSize, i);
        d4[u] = T::raw(static_cast<const char*>(a.dy) + (size_t)row * a.lddy * T::kSize, i);
        mean[u] = a.mean[row], rstd[u] = a.rstd[row];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[E], d[E];
        T::unpack(f4[u], f);
        T::unpack(first + u * RG + grp < a.R ? d4[u] : make_uint4(0, 0, 0, 0), d);
#pragma unroll
        for (int j = 0; j < E; ++j) {
          dg[j] = fmaf(d[j], (f[j] - mean[u]) * rstd[u], dg[j]);
          db[j] += d[j];
        }
      }
    }
  }
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const float s0 = sum_over_groups<CL>(dg[j]), s1 = sum_over_groups<CL>(db[j]);  // the wave's
    if ((threadIdx.x & 63) < CL) {
      sums[0][threadIdx.x >> 6][lane * E + j] = s0;
      sums[1][threadIdx.x >> 6][lane * E + j] = s1;
    }
  }
  __syncthreads();
  const int half = threadIdx.x / (CL * E), at = threadIdx.x % (CL * E);
  float* out = half ? a.dbeta : a.dgamma;
  const int ch = ((int)blockIdx.x - row_wgs) * CL + at / E, col = min(ch * E, C - E) + at % E;
  // (the last chunk's first columns are the one before's)
  if (half < 2 && out && ch < n && col >= ch * E) {
    float s = sums[half][0][at];
#pragma unroll
    for (int q = 1; q < NT / 64; ++q) s += sums[half][q][at];
    out[col] = s;
  }
}

// Rows shorter than a chunk or longer than the largest tile: dx a workgroup a row,
// value by value; the sums over rows by columns, a thread each, eight rows under way at a
// time.  A single group of rows has all of them, and writes the sums themselves.
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
  constexpr int U = 8;
  for (long long r0 = blockIdx.y; r0 < a.R; r0 += U * (long long)gridDim.y) {
    float d[U], f[U], mean[U], rstd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long r = min(r0 + u * (long long)gridDim.y, a.R - 1LL);
      d[u] = T::load1(static_cast<const char*>(a.dy) + r * a.lddy * T::kSize, c);
      f[u] = T::load1(static_cast<const char*>(a.x) + r * a.ldx * T::kSize, c);
      mean[u] = a.mean[r], rstd[u] = a.rstd[r];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r0 + u * (long long)gridDim.y < a.R) {
        sg = fmaf(d[u], (f[u] - mean[u]) * rstd[u], sg);
        sb += d[u];
      }
  }
  if (gridDim.y == 1) {
    if (a.dgamma) a.dgamma[c] = sg;
    if (a.dbeta) a.dbeta[c] = sb;
    return;
  }
  float* p = a.part + (size_t)blockIdx.y * 2 * C;
  p[c] = sg;
  p[C + c] = sb;
}

namespace {

struct Plan {
  const void* fn;  // null: value by value
  int threads, groups, grid;  // grid 0: the one launch for few rows; value by value: groups of rows
};

// Up to so many rows take one launch.  Its column workgroups add R / 64 rows a lane, so
// its time grows with R; the two kernels' sums grow with C.  us, one launch (two):
//   bf16 R       C = 80      192          640          2560         1000
//   196          4.2 (5.8)   4.3 (7.0)    4.4          4.6
//   392          4.6         4.6 (7.1)    4.8 (7.1)    5.5 (10.0)
//   640                                                             7.2 (7.4)
//   784          6.2 (6.1)   6.2 (7.4)    6.6 (7.3)    9.3 (12.5)   8.1 (7.6)
//   1200                     7.9 (7.4)                14.4 (14.3)
constexpr int kFewRows = 800, kFewMid = 640, kFewWide = 1024;

template <int DT>
Plan plan(int R, int C) {
  constexpr int E = Chunk<DT>::E;
  const int n = (C + E - 1) / E;
  auto make = [&](const void* fn, int threads, int lpr, int most) {
    const int groups = threads / lpr;
    // (a workgroup that takes few rows costs as much by its sums: 256 of them, or eight rows each)
    const int g = most > 256 ? std::min(std::max(R / 8, 256), most) : most;
    return Plan{fn, threads, groups, (int)std::min<long long>(((long long)R + groups - 1) / groups, g)};
  };
  if (C < E) return Plan{nullptr, 256, 1, std::min(R, 256)};
  // Wide rows fill the GPU by their columns (33 workgroups and more): 32 rows and more a group, so
  // that the groups' sums stay within an eighth of x and dy.  us, this (a group a row, up to
  // 256 of them, which at 256 x 2^20 takes 2 GiB of sums):
  //   256 x 2^20   bf16 4160 (5290)  fp32 4250 (5300)    100 x 40000  bf16 76 (108)  fp32 89 (99)
  //   300 x 20000  bf16 54 (76)      fp32 68 (77)        40 x 8200    bf16 10.8 (10.6)  fp32 17 (20)
  if (n > 2048) return Plan{nullptr, 256, 1, std::min(std::max(R / 32, 1), 256)};
  if (R <= (n > 128 ? kFewWide : n > 96 ? kFewMid : kFewRows) && n <= 1024) {
    if (n <= 16) return Plan{(const void*)&norm_grad_few_kernel<DT, 16, 1>, 512, 32, 0};
    if (n <= 64) return Plan{(const void*)&norm_grad_few_kernel<DT, 64, 1>, 512, 8, 0};
    if (n <= 256) return Plan{(const void*)&norm_grad_few_kernel<DT, 256, 1>, 512, 2, 0};
    return Plan{(const void*)&norm_grad_few_kernel<DT, 256, 4>, 512, 2, 0};
  }
  // (100352 x 40 bf16: 11.4 us, 14.0 with 16 lanes a row)
  if (n <= 8 && R >= 16384) return make((const void*)&norm_grad_kernel<DT, 8, 1, 512>, 512, 8, 512);
  if (n <= 16) return make((const void*)&norm_grad_kernel<DT, 16, 1, 512>, 512, 16, 512);
  if (n <= 32) return make((const void*)&norm_grad_kernel<DT, 16, 2, 512>, 512, 16, 512);
  if (n <= 48) return make((const void*)&norm_grad_kernel<DT, 16, 3, 512>, 512, 16, 256);
  if (n <= 64) return make((const void*)&norm_grad_kernel<DT, 16, 4, 512>, 512, 16, 256);
  if (n <= 128) return make((const void*)&norm_grad_kernel<DT, 64, 2, 512>, 512, 64, 512);
  if (n <= 192) return make((const void*)&norm_grad_kernel<DT, 64, 3, 256>, 256, 64, 512);
  if (n <= 256) return make((const void*)&norm_grad_kernel<DT, 64, 4, 256>, 256, 64, 512);
  // Few turns: a chunk a lane, so that twice as many loads are under way, and half as many
  // sums where those weigh.  us, this (two chunks a lane of 256, 512 workgroups): bf16
  // 1500 x 2560 12.9 (14.2), 2754 x 3000 17.6 (19.7), 5001 x 2201 22.9 (24.2), 10000 x 4096
  // 46.7 (48.2), 32768 x 2560 99.7 (95.7); fp32 20000 x 1500 69.0 (68.2)
  if (n <= 512 && R <= 12288)
    return make((const void*)&norm_grad_kernel<DT, 512, 1, 512>, 512, 512, R < 4096 ? 256 : 512);
  if (n <= 512) return make((const void*)&norm_grad_kernel<DT, 256, 2, 256>, 256, 256, 512);
  if (n <= 768) return make((const void*)&norm_grad_kernel<DT, 256, 3, 256>, 256, 256, 512);
  // (10000 x 8192 bf16: 101 us, 114 with four chunks a lane of 256)
  if (n <= 1024) return make((const void*)&norm_grad_kernel<DT, 1024, 1, 1024>, 1024, 1024, 256);
  return make((const void*)&norm_grad_kernel<DT, 512, 4, 512>, 512, 512, 256);
}

template <int DT>
hipError_t launch_grad(NormGradArgs a, hipStream_t stream) {
  Plan p = plan<DT>(a.R, a.C);
  // the rows of a wave have to lie within 32 bits of the first (any kernel takes any grid)
  const bool near = a.R == 1 || (a.ldx < 1 << 27 && a.lddy < 1 << 27);
  if (!near && p.grid && p.fn && (a.C + Chunk<DT>::E - 1) / Chunk<DT>::E <= 64) {
    p.fn = (const void*)&norm_grad_kernel<DT, 64, 1, 512>;
    p.threads = 512;
  }
  float* const part = a.part;
  const bool sums = a.dgamma || a.dbeta;
  if (!sums) a.part = nullptr;
  void* argv[] = {&a, nullptr};
  hipError_t e = hipSuccess;
  if (!p.grid) {
    int row_wgs = a.dx ? (a.R + p.groups - 1) / p.groups : 0;
    const int n = (a.C + Chunk<DT>::E - 1) / Chunk<DT>::E, col_wgs = sums ? (n + 7) / 8 : 0;
    argv[1] = &row_wgs;
    return hipLaunchKernel(p.fn, dim3(row_wgs + col_wgs), dim3(p.threads), argv, 0, stream);
  }
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
  if (e != hipSuccess || !sums || (!p.fn && p.grid == 1)) return e;
  constexpr int kMost = 1 << 20;  // workgroups a launch: fewer than 2^32 threads
  for (int c = 0; c < 2 * a.C; c += 32 * kMost)
    norm_grad_sum_kernel<<<std::min((2 * a.C - c + 31) / 32, kMost), 1024, 0, stream>>>(part, p.grid, a.C, c,
                                                                                      a.dgamma, a.dbeta);
  return hipGetLastError();
}

}  // namespace

size_t norm_grad_ws_bytes(int R, int C, int dt_bf16) {
  const Plan p = dt_bf16 ? plan<1>(R, C) : plan<0>(R, C);
  return !p.fn && p.grid == 1 ? 0 : (size_t)p.grid * 2 * C * 4;
}

hipError_t launch_norm_grad(const NormGradArgs& a, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_grad<1>(a, stream) : launch_grad<0>(a, stream);
}

}  // namespace gl
