// The end of a block, in one pass over its output b and the features x that went by it:
//   n = (b - mean_b) rstd_b gamma1 + beta1       (post; else n = b)
//   s = x + gate scale n                         a gate for each group of rows, a scale by channel
//   y = (s - mean_s) rstd_s gamma2 + beta2       the norm before the next block
// The norms are over a row's channels, with the mean taken out (layer norm) or not (rms).
// A row's values stay in registers in fp32 from the loads to both stores: y is of the sum
// before its rounding.  Memory bounds it: us a call (TB/s of the four rows; a copy of 1 GiB
// reaches 5.2), with post and a gate for each row, bf16 32768 x 2560 130 (5.2), 8192 x 4096
// 46 (5.8), 100352 x 320 47 (5.5), 100352 x 80 16.1 (4.0; 10 of 16 lanes hold a chunk), 4096 x
// 16384 118 (4.6); fp32 32768 x 2560 229 (5.9).  196 x 192 takes a launch, 3 us.
#include "gl_kernels.h"
#include "row_device.h"

namespace gl {

namespace {

// 1 / sqrt of the mean square plus eps; the hardware's root takes a subnormal for zero, so
// a small argument is scaled by a power of four first
__device__ __forceinline__ float join_rstd(float sq, float inv_c, float eps) {
  const float v = fmaf(sq, inv_c, eps);
  const bool tiny = v < 0x1p-100f;
  return __builtin_amdgcn_rsqf(tiny ? v * 0x1p100f : v) * (tiny ? 0x1p50f : 1.f);
}

// Sum over the lanes of a row: LPR of them (8, 16, 64), or a workgroup's (LPR 0).
template <int LPR>
__device__ __forceinline__ float join_sum(float v, uint32_t* slot) {
  if (LPR) return sum_row<LPR ? LPR : 64>(v, nullptr);
  v = sum_row<64>(v, nullptr);
  const int nw = blockDim.x >> 6;
  if (nw == 1) return v;
  if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = __float_as_uint(v);
  __syncthreads();
  v = __uint_as_float(slot[0]);
  for (int w = 1; w < nw; ++w) v += __uint_as_float(slot[w]);
  return v;
}

// LPR lanes hold a row, VPL chunks each; LPR 0: a workgroup of any number of waves does.
template <int DT, int LPR, int VPL, bool POST>
__global__ __launch_bounds__(LPR ? 256 : 512) void residual_kernel(ResidualArgs a) {
  using T = Chunk<DT>;
  constexpr int E = T::E, GROUPS = LPR ? 256 / (LPR ? LPR : 1) : 1;
  __shared__ uint32_t slots[2][4][16];
  const WaveRows<LPR ? LPR : 1024> rows;
  const int lanes = LPR ? LPR : blockDim.x, lane = LPR ? threadIdx.x & (LPR - 1) : threadIdx.x;
  const int C = a.C, n = (C + E - 1) / E;
  const bool ragged = C % E != 0;  // the last chunk repeats values of the one before it
  int at[VPL];
#pragma unroll
  for (int v = 0; v < VPL; ++v) at[v] = min(min(lane + v * lanes, n - 1) * E, C - E);
  auto on = [&](int v) { return lane + v * lanes < n; };
  uint4 raw_b[VPL], raw_x[VPL];
  auto load = [&](long long r0) {
    uint32_t off_b, off_x;
    const char* b = rows.at(a.b, r0 + rows.wave, a.R, a.ldb * (long long)T::kSize, &off_b);
    const char* x = rows.at(a.x, r0 + rows.wave, a.R, a.ldx * (long long)T::kSize, &off_x);
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      raw_b[v] = T::raw_at(b, off_b + at[v] * (uint32_t)T::kSize);
      raw_x[v] = T::raw_at(x, off_x + at[v] * (uint32_t)T::kSize);
    }
  };
  const long long step = (long long)gridDim.x * GROUPS;
  long long r0 = (long long)blockIdx.x * GROUPS;
  load(r0);
  uint4 g1[VPL], b1[VPL], sc[VPL], g2[VPL], b2[VPL];
#pragma unroll
  for (int v = 0; v < VPL; ++v) {
    g1[v] = sc[v] = g2[v] = T::ones();
    b1[v] = b2[v] = make_uint4(0, 0, 0, 0);
    if (POST && a.gamma1) g1[v] = T::raw(a.gamma1, at[v]);
    if (POST && a.beta1) b1[v] = T::raw(a.beta1, at[v]);
    if (a.scale) sc[v] = T::raw(a.scale, at[v]);
    if (a.gamma2) g2[v] = T::raw(a.gamma2, at[v]);
    if (a.beta2) b2[v] = T::raw(a.beta2, at[v]);
  }
  int turn = 0;
  // every group of a workgroup makes the same number of turns
  for (; r0 < a.R; r0 += step, turn ^= 1) {
    const long long first = r0 + rows.wave;  // the wave's
    const bool mine = first + rows.lane < a.R;
    float f[VPL][E], x[VPL][E];
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      T::unpack(raw_b[v], f[v]);
      T::unpack(raw_x[v], x[v]);
    }
    const float gate = a.gate ? a.gate[(uint32_t)min(first + rows.lane, a.R - 1LL) / (uint32_t)a.per_gate] : 1.f;
    if (r0 + step < a.R) load(r0 + step);
    auto sum = [&](auto term, const float (*p)[E], uint32_t* slot) {
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
        float q = 0.f;
        if (ragged) {
          const int skip = (lane + v * lanes) * E - at[v];
#pragma unroll
          for (int j = 0; j < E; ++j) q = j >= skip ? term(q, p[v][j]) : q;
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j) q = term(q, p[v][j]);
        }
        s += on(v) ? q : 0.f;
      }
      return join_sum<LPR>(s, slot);
    };
    auto add = [](float s, float y) { return s + y; };
    auto square = [](float s, float y) { return fmaf(y, y, s); };
    // takes the mean out of p (layer norm) and returns rstd
    auto norm = [&](float (*p)[E], uint32_t (*slot)[16], float* mean) {
      *mean = 0.f;
      if (!a.rms) {
        const float s = sum(add, p, slot[0]);
        *mean = fmaf(s, a.mean_hi, s * a.mean_lo);
#pragma unroll
        for (int v = 0; v < VPL; ++v)
#pragma unroll
          for (int j = 0; j < E; ++j) p[v][j] -= *mean;
      }
      return join_rstd(sum(square, p, slot[1]), a.inv_c, a.eps);
    };
    auto store = [&](void* out, int v, const float* y) {
      T::store_at(static_cast<char*>(out) + first * C * (long long)T::kSize,
                  (rows.lane * (uint32_t)C + at[v]) * (uint32_t)T::kSize, y);
    };
    auto keep = [&](float* out, float value) {
      if (out && mine && lane == 0) (out + first)[rows.lane] = value;
    };
    float mean, rstd = 1.f;
    if (POST) {
      rstd = norm(f, slots[turn], &mean);
      keep(a.mean_b, mean);
      keep(a.rstd_b, rstd);
    }
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      float w[E], c[E];
      if (VPL > 1) keep_packed(g1[v]), keep_packed(b1[v]), keep_packed(sc[v]);
      if (POST) {
        T::unpack(g1[v], w);
        T::unpack(b1[v], c);
#pragma unroll
        for (int j = 0; j < E; ++j) f[v][j] = fmaf(f[v][j] * rstd, w[j], c[j]);
      }
      T::unpack(sc[v], w);
#pragma unroll
      for (int j = 0; j < E; ++j) f[v][j] = fmaf(f[v][j], gate * w[j], x[v][j]);
      if (mine && on(v)) store(a.s, v, f[v]);
    }
    if (!a.y) continue;
    rstd = norm(f, slots[turn] + 2, &mean);
    keep(a.mean_s, mean);
    keep(a.rstd_s, rstd);
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      float w[E], c[E];
      if (VPL > 1) keep_packed(g2[v]), keep_packed(b2[v]);
      T::unpack(g2[v], w);
      T::unpack(b2[v], c);
#pragma unroll
      for (int j = 0; j < E; ++j) f[v][j] = fmaf(f[v][j] * rstd, w[j], c[j]);
      if (mine && on(v)) store(a.y, v, f[v]);
    }
  }
}

// Rows shorter than a chunk or longer than the largest tile: a workgroup a row, value by
// value, read once more for each of the steps.
template <int DT>
__global__ __launch_bounds__(256) void residual_any_kernel(ResidualArgs a) {
  using T = Chunk<DT>;
  __shared__ uint32_t slots[4][4];
  const int C = a.C;
  for (long long r = blockIdx.x; r < a.R; r += gridDim.x) {
    const char* b = static_cast<const char*>(a.b) + r * a.ldb * T::kSize;
    const char* x = static_cast<const char*>(a.x) + r * a.ldx * T::kSize;
    const float gate = a.gate ? a.gate[r / a.per_gate] : 1.f;
    float mb = 0.f, rb = 1.f, ms = 0.f;
    auto of = [&](const void* w, int c, float otherwise) { return w ? T::load1(w, c) : otherwise; };
    auto value = [&](int c) {
      float n = T::load1(b, c);
      if (a.post) n = fmaf((n - mb) * rb, of(a.gamma1, c, 1.f), of(a.beta1, c, 0.f));
      return fmaf(n, gate * of(a.scale, c, 1.f), T::load1(x, c));
    };
    auto stats = [&](auto at, uint32_t (*slot)[4], float* mean) {
      float s = 0.f;
      if (!a.rms) {
        for (int c = threadIdx.x; c < C; c += 256) s += at(c);
        s = sum_row<256>(s, slot[0]);
        *mean = fmaf(s, a.mean_hi, s * a.mean_lo);
        s = 0.f;
      }
      for (int c = threadIdx.x; c < C; c += 256) {
        const float d = at(c) - *mean;
        s = fmaf(d, d, s);
      }
      return join_rstd(sum_row<256>(s, slot[1]), a.inv_c, a.eps);
    };
    if (a.post) {
      rb = stats([&](int c) { return T::load1(b, c); }, slots, &mb);
      if (threadIdx.x == 0) {
        if (a.mean_b) a.mean_b[r] = mb;
        if (a.rstd_b) a.rstd_b[r] = rb;
      }
    }
    for (int c = threadIdx.x; c < C; c += 256) T::store1(a.s, r * C + c, value(c));
    if (a.y) {
      const float rs = stats(value, slots + 2, &ms);
      for (int c = threadIdx.x; c < C; c += 256)
        T::store1(a.y, r * C + c, fmaf((value(c) - ms) * rs, of(a.gamma2, c, 1.f), of(a.beta2, c, 0.f)));
      if (threadIdx.x == 0) {
        if (a.mean_s) a.mean_s[r] = ms;
        if (a.rstd_s) a.rstd_s[r] = rs;
      }
    }
    __syncthreads();  // the words of slots are free again
  }
}

template <int DT, bool POST>
hipError_t launch_rows(const ResidualArgs& a, hipStream_t stream) {
  constexpr int E = Chunk<DT>::E;
  const int n = (a.C + E - 1) / E;
  void* argv[] = {const_cast<ResidualArgs*>(&a)};
  // `rows` a workgroup and turn; at most `per_cu` workgroups a CU, with equal numbers of turns
  auto go = [&](const void* fn, int rows, int threads, int per_cu) {
    const long long units = ((long long)a.R + rows - 1) / rows, most = 256LL * per_cu;
    const long long turns = (units + most - 1) / most;
    return hipLaunchKernel(fn, dim3((unsigned)((units + turns - 1) / turns)), dim3(threads), argv, 0, stream);
  };
  if (a.C < E || n > 2048) return go((const void*)&residual_any_kernel<DT>, 1, 256, 16);
  // the rows of a wave lie within 32 bits of the first
  const bool near = a.R == 1 || (a.ldx < 1 << 27 && a.ldb < 1 << 27);
  if (near) {
    if (n <= 8 && a.R >= 16384) return go((const void*)&residual_kernel<DT, 8, 1, POST>, 32, 256, 16);
    if (n <= 16) return go((const void*)&residual_kernel<DT, 16, 1, POST>, 16, 256, 16);
    if (n <= 32 && a.R >= 4096) return go((const void*)&residual_kernel<DT, 16, 2, POST>, 16, 256, 16);
  }
  if (n <= 64) return go((const void*)&residual_kernel<DT, 64, 1, POST>, 4, 256, 16);
  if (n > 96 && n <= 128) return go((const void*)&residual_kernel<DT, 64, 2, POST>, 4, 256, 16);
  if (n > 128 && n <= 192) return go((const void*)&residual_kernel<DT, 64, 3, POST>, 4, 256, 3);
  // A row a workgroup: three or two chunks a lane, whichever leaves fewer lanes idle (fewer
  // waves meet for a row's sums: 32768 x 2560 bf16, 3 x 2 waves 134 us, 2 x 3 waves 146, 1 x
  // 5 waves 183 with as many workgroups as fit); as many workgroups as are resident together.
  const int vpl = n <= 96 ? 1 : n > 1024 ? 4 : (n + 191) / 192 * 3 <= (n + 127) / 128 * 2 ? 3 : 2;
  const int waves = (n + 64 * vpl - 1) / (64 * vpl), resident = vpl == 1 ? 24 : vpl == 2 ? (DT ? 16 : 12) : vpl == 3 ? 12 : 8;
  return go(vpl == 1   ? (const void*)&residual_kernel<DT, 0, 1, POST>
            : vpl == 2 ? (const void*)&residual_kernel<DT, 0, 2, POST>
            : vpl == 3 ? (const void*)&residual_kernel<DT, 0, 3, POST>
                       : (const void*)&residual_kernel<DT, 0, 4, POST>,
            1, 64 * waves, std::max(vpl == 2 ? 2 : 1, resident / waves));
}

}  // namespace

hipError_t launch_residual(const ResidualArgs& a, int dt_bf16, hipStream_t stream) {
  if (dt_bf16) return a.post ? launch_rows<1, true>(a, stream) : launch_rows<1, false>(a, stream);
  return a.post ? launch_rows<0, true>(a, stream) : launch_rows<0, false>(a, stream);
}

}  // namespace gl
