// The backward pass of a block's end (residual.hip).  With h = dy gamma2, xs and xb the
// normalised s and b, and k = dv gate scale gamma1,
//   dv = ds + rstd_s (h - avg h - xs avg(h xs))       averages over the row's channels (avg h
//   dx = dv                                           for layer norm alone)
//   db = rstd_b (k - avg k - xb avg(k xb))            (post; else dv gate scale)
// and, over all rows, four sums for each channel,
//   S1 = sum dv gate xb (b without post), S0 = sum dv gate, T1 = sum dy xs, T0 = sum dy,
// make the vectors' gradients:
//   dscale = gamma1 S1 + beta1 S0 (S1), dgamma1 = scale S1, dbeta1 = scale S0,
//   dgamma2 = T1, dbeta2 = T0.  A gate's is the sum of dv scale n over its rows.
// One kernel reads the four rows once, writes dx and db, and each lane adds its channels'
// terms to sums of its own over all rows that it meets; a workgroup adds its lanes' and
// writes them to the workspace, and a second kernel adds the workgroups' and makes the
// vectors.  Memory bounds it where rows are many and wide, us (TB/s of the six rows), with post
// and a gate for each row: bf16 32768 x 2560 259 (3.9; without post 212, 4.7), 8192 x 4096 100
// (4.0), 16384 x 1024 48 (4.2), 8192 x 8192 196 (4.1), fp32 32768 x 2560 374 (5.4).  Four sums a
// channel and four rows under way take the registers of all but two waves a SIMD, and the
// vector units are busy half of the time; 100352 x 80 (28 us without post, 3.5 TB/s) keeps them
// busy 90 %.  Rows wider than the largest tile, 8192 channels of either type, go value by value,
// and eight (bf16) or three times (fp32) slower: bf16 8192 x 8200 1603 us (0.5), 4096 x 16384
// 1416 (0.6), fp32 8192 x 8208 1237 (1.3).
// Everything is fp32, added in an order that depends on the sizes alone.
#include "gl_kernels.h"
#include "row_device.h"

namespace gl {

namespace {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4), may_alias));

// Sums of N values over the lanes of a row, in one trip through LDS where a row has more
// than a wave (LPR 0: the workgroup's).
template <int LPR, int N>
__device__ __forceinline__ void sum_rows(float (&v)[N], float (*slot)[16]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = sum_row<LPR ? LPR : 64>(v[i], nullptr);
  if (LPR) return;
  const int nw = blockDim.x >> 6;
  if (nw == 1) return;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) slot[i][threadIdx.x >> 6] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = slot[i][0];
    for (int w = 1; w < nw; ++w) v[i] += slot[i][w];
  }
}

// LPR lanes hold a row, VPL chunks each; LPR 0: a workgroup of up to NT threads does.  A
// row's loads are under way while the one before it is worked on, but where 1024 threads
// leave 128 registers.
template <int DT, int LPR, int VPL, bool POST, int NT = 512>
__global__ __launch_bounds__(NT) void residual_grad_kernel(ResidualGradArgs a) {
  using T = Chunk<DT>;
  constexpr bool AHEAD = NT <= 512;
  constexpr int E = T::E, GROUPS = LPR ? NT / (LPR ? LPR : 1) : 1, NW = NT / 64;
  constexpr int COLS = LPR * VPL * E;  // columns a group covers
  __shared__ float slots[2][5][16];
  __shared__ float sums[LPR ? NW * COLS : 1];
  const WaveRows<LPR ? LPR : 1024> rows;
  const int lanes = LPR ? LPR : blockDim.x, lane = LPR ? threadIdx.x & (LPR - 1) : threadIdx.x;
  const int C = a.C, n = (C + E - 1) / E;
  const bool ragged = C % E != 0;  // the last chunk repeats values of the one before it
  int at[VPL];
#pragma unroll
  for (int v = 0; v < VPL; ++v) at[v] = min(min(lane + v * lanes, n - 1) * E, C - E);
  auto on = [&](int v) { return lane + v * lanes < n; };
  // adds up what `term` makes of the chunk's values that count: not those that the chunk
  // before it has too, and none of a lane past the row's end
  auto add_up = [&](int v, float& sum, auto term) {
    float q = 0.f;
    if (ragged) {
      const int skip = (lane + v * lanes) * E - at[v];
#pragma unroll
      for (int j = 0; j < E; ++j) q = j >= skip ? term(q, j) : q;
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) q = term(q, j);
    }
    sum += on(v) ? q : 0.f;
  };
  uint4 raw_d[VPL], raw_y[VPL], raw_b[VPL], raw_s[VPL];
  float mb = 0.f, rb = 1.f, ms = 0.f, rs = 0.f, gate = 1.f;
  auto load = [&](long long r0) {
    auto from = [&](const void* p, long long ld, uint4* raw) {
      uint32_t off;
      const char* q = rows.at(p, r0 + rows.wave, a.R, ld * (long long)T::kSize, &off);
#pragma unroll
      for (int v = 0; v < VPL; ++v) raw[v] = T::raw_at(q, off + at[v] * (uint32_t)T::kSize);
    };
    const long long r = min(r0 + rows.wave + rows.lane, a.R - 1LL);
    if (a.ds) from(a.ds, a.ldds, raw_d);
    from(a.b, a.ldb, raw_b);
    if (a.dy) {
      from(a.dy, a.lddy, raw_y);
      from(a.s, a.lds, raw_s);
      rs = a.rstd_s[r];
      if (!a.rms) ms = a.mean_s[r];
    }
    if (POST) {
      rb = a.rstd_b[r];
      if (!a.rms) mb = a.mean_b[r];
    }
    if (a.gate) gate = a.gate[(uint32_t)r / (uint32_t)a.per_gate];
  };
#pragma unroll
  for (int v = 0; v < VPL; ++v) raw_d[v] = raw_y[v] = raw_s[v] = make_uint4(0, 0, 0, 0);
  const long long step = (long long)gridDim.x * GROUPS;
  long long r0 = (long long)blockIdx.x * GROUPS;
  if (AHEAD) load(r0);
  uint4 g1[VPL], b1[VPL], sc[VPL], g2[VPL];
  float S1[VPL][E] = {}, S0[VPL][E] = {}, T1[VPL][E] = {}, T0[VPL][E] = {};
#pragma unroll
  for (int v = 0; v < VPL; ++v) {
    g1[v] = sc[v] = g2[v] = T::ones();
    b1[v] = make_uint4(0, 0, 0, 0);
    if (POST && a.gamma1) g1[v] = T::raw(a.gamma1, at[v]);
    if (POST && a.beta1) b1[v] = T::raw(a.beta1, at[v]);
    if (a.scale) sc[v] = T::raw(a.scale, at[v]);
    if (a.gamma2) g2[v] = T::raw(a.gamma2, at[v]);
  }
  int turn = 0;
  // every group of a workgroup makes the same number of turns
  for (; r0 < a.R; r0 += step, turn ^= 1) {
    const long long first = r0 + rows.wave;  // the wave's
    // a row past the last repeats it: nothing of it is stored, and the sums over rows leave it
    // out, where 0 times its values would not be 0 for an infinity
    const bool mine = !LPR || first + rows.lane < a.R;
    float d[VPL][E], h[VPL][E], f[VPL][E], x[VPL][E];
    if (!AHEAD) load(r0);
    const float mbr = mb, rbr = rb, msr = ms, rsr = rs, gr = gate;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      T::unpack(raw_d[v], d[v]);
      T::unpack(raw_y[v], h[v]);
      T::unpack(raw_s[v], x[v]);
      T::unpack(raw_b[v], f[v]);
    }
    if (AHEAD && r0 + step < a.R) load(r0 + step);
    auto store = [&](void* out, int v, const float* y) {
      T::store_at(static_cast<char*>(out) + first * C * (long long)T::kSize,
                  (rows.lane * (uint32_t)C + at[v]) * (uint32_t)T::kSize, y);
    };
    if (a.dy) {
      float p[2] = {0.f, 0.f};
#pragma unroll
      for (int v = 0; v < VPL; ++v) {
        float w[E];
        if (VPL > 1) keep_packed(g2[v]);
        T::unpack(g2[v], w);
#pragma unroll
        for (int j = 0; j < E; ++j) x[v][j] = (x[v][j] - msr) * rsr;
        if (mine)
#pragma unroll
          for (int j = 0; j < E; ++j) {
            T1[v][j] = fmaf(h[v][j], x[v][j], T1[v][j]);
            T0[v][j] += h[v][j];
          }
#pragma unroll
        for (int j = 0; j < E; ++j) h[v][j] *= w[j];
        if (!a.rms) add_up(v, p[0], [&](float q, int j) { return q + h[v][j]; });
        add_up(v, p[1], [&](float q, int j) { return fmaf(h[v][j], x[v][j], q); });
      }
      sum_rows<LPR>(p, slots[turn]);
      const float s0 = a.rms ? 0.f : p[0] * a.inv_c * -rsr, s1 = p[1] * a.inv_c * -rsr;
#pragma unroll
      for (int v = 0; v < VPL; ++v)
#pragma unroll
        for (int j = 0; j < E; ++j) d[v][j] += fmaf(h[v][j], rsr, fmaf(x[v][j], s1, s0));
    }
    // h: k from here on; p: the sums of k, of k xb and of dv scale n
    float p[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      if (a.dx && mine && on(v)) store(a.dx, v, d[v]);
      float w[E], sv[E], c[E];
      if (VPL > 1) keep_packed(g1[v]), keep_packed(b1[v]), keep_packed(sc[v]);
      T::unpack(sc[v], sv);
      if (POST) {
        T::unpack(g1[v], w);
        T::unpack(b1[v], c);
      }
      if (POST)
#pragma unroll
        for (int j = 0; j < E; ++j) f[v][j] = (f[v][j] - mbr) * rbr;
      if (mine)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const float dg = d[v][j] * gr;
          S1[v][j] = fmaf(dg, f[v][j], S1[v][j]);
          if (POST) S0[v][j] += dg;
        }
#pragma unroll
      for (int j = 0; j < E; ++j) {
        d[v][j] *= sv[j];
        h[v][j] = POST ? d[v][j] * gr * w[j] : d[v][j] * gr;
      }
      if (POST) {
        if (!a.rms) add_up(v, p[0], [&](float q, int j) { return q + h[v][j]; });
        add_up(v, p[1], [&](float q, int j) { return fmaf(h[v][j], f[v][j], q); });
      }
      if (a.dots) add_up(v, p[2], [&](float q, int j) { return fmaf(d[v][j], POST ? fmaf(f[v][j], w[j], c[j]) : f[v][j], q); });
    }
    if (POST || a.dots) sum_rows<LPR>(p, slots[turn] + 2);
    if (a.dots && mine && lane == 0) (a.dots + first)[rows.lane] = p[2];
    const float s0 = a.rms ? 0.f : p[0] * a.inv_c * -rbr, s1 = p[1] * a.inv_c * -rbr;
    if (a.db && mine)
#pragma unroll
      for (int v = 0; v < VPL; ++v)
        if (on(v)) {
          float y[E];
#pragma unroll
          for (int j = 0; j < E; ++j) y[j] = POST ? fmaf(h[v][j], rbr, fmaf(f[v][j], s1, s0)) : h[v][j];
          store(a.db, v, y);
        }
  }
  if (!a.part) return;

  float* part = a.part + (size_t)blockIdx.x * 4 * C;
  if (!LPR) {  // a lane's columns are its own
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
      const int c = lane + v * lanes, i = min(c * E, C - E), skip = max(c * E + E - C, 0);
      if (c >= n) continue;
      auto put = [&](int q, const float* s) {
        float* o = part + (size_t)q * C + i;
        if (skip == 0) {
#pragma unroll
          for (int j = 0; j < E; j += 4) *reinterpret_cast<f32x4_any*>(o + j) = f32x4_any{s[j], s[j + 1], s[j + 2], s[j + 3]};
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j)
            if (j >= skip) o[j] = s[j];
        }
      };
      put(0, S1[v]);
      put(1, S0[v]);
      put(2, T1[v]);
      put(3, T0[v]);
    }
    return;
  }
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
#pragma unroll
    for (int v = 0; v < VPL; ++v)
#pragma unroll
      for (int j = 0; j < E; ++j) {
        float s = q == 0 ? S1[v][j] : q == 1 ? S0[v][j] : q == 2 ? T1[v][j] : T0[v][j];
        if (LPR < 64) s = sum_over_groups<LPR ? LPR : 8>(s);  // the wave's
        if ((threadIdx.x & 63) < LPR) sums[wave * COLS + (lane + v * LPR) * E + j] = s;
      }
    __syncthreads();
    // column c's chunk holds it at its own place, or the last chunk moved back
    for (int c = threadIdx.x; c < C; c += NT) {
      const int last = (n - 1) * E, i = c < last ? c : c + (n * E - C);
      float s = sums[i];
#pragma unroll
      for (int k = 1; k < NW; ++k) s += sums[k * COLS + i];
      part[(size_t)q * C + c] = s;
    }
    __syncthreads();
  }
}

// The groups' sums and the vectors' gradients from them: 32 columns a workgroup, 32 groups
// at a time and eight of those under way, in the same order always.  Workgroups past
// `vectors` sum the gates' rows, a wave or (many rows) a workgroup each.
constexpr int kGateWave = 512;
template <int DT>
__global__ __launch_bounds__(1024) void residual_vectors_kernel(ResidualGradArgs a, int G, int vectors) {
  using T = Chunk<DT>;
  constexpr int COLS = 32, ROWS = 1024 / COLS, U = 8;
  __shared__ float sums[4][ROWS][COLS + 1];
  if ((int)blockIdx.x >= vectors) {
    const long long gates = ((long long)a.R + a.per_gate - 1) / a.per_gate;
    const bool wide = a.per_gate > kGateWave;
    const int id = blockIdx.x - vectors, lanes = wide ? 1024 : 64, lane = threadIdx.x & (lanes - 1);
    const long long step = ((long long)gridDim.x - vectors) * (1024 / lanes);
    for (long long gate = (long long)id * (1024 / lanes) + threadIdx.x / lanes; gate < gates; gate += step) {
      const long long first = gate * a.per_gate, end = min(first + a.per_gate, (long long)a.R);
      float s = 0.f;
      for (long long r = first + lane; r < end; r += lanes) s += a.dots[r];
      s = wide ? sum_row<1024>(s, reinterpret_cast<uint32_t*>(sums)) : sum_row<64>(s, nullptr);
      if (lane == 0) a.dgate[gate] = s;
      if (wide) __syncthreads();  // the words of sums are free again
    }
    return;
  }
  const int t = threadIdx.x % COLS, w = threadIdx.x / COLS, C = a.C;
  for (int c0 = blockIdx.x * COLS; c0 < C; c0 += vectors * COLS) {
    const int c = c0 + t, col = min(c, C - 1);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int g0 = w; g0 < G; g0 += U * ROWS) {
      float v[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[u][q] = a.part[((size_t)min(g0 + u * ROWS, G - 1) * 4 + q) * C + col];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) s[q] += g0 + u * ROWS < G ? v[u][q] : 0.f;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[q][w][t] = s[q];
#pragma unroll
    for (int h = ROWS / 2; h >= 1; h /= 2) {
      __syncthreads();
      if (w < h)
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[q][w][t] += sums[q][w + h][t];
    }
    if (!w && c < C) {
      const float S1 = sums[0][0][t], S0 = sums[1][0][t];
      const float sc = a.scale ? T::load1(a.scale, c) : 1.f;
      if (a.dscale)
        a.dscale[c] = a.post ? fmaf(a.gamma1 ? T::load1(a.gamma1, c) : 1.f, S1, a.beta1 ? T::load1(a.beta1, c) * S0 : 0.f) : S1;
      if (a.dgamma1) a.dgamma1[c] = sc * S1;
      if (a.dbeta1) a.dbeta1[c] = sc * S0;
      if (a.dgamma2) a.dgamma2[c] = sums[2][0][t];
      if (a.dbeta2) a.dbeta2[c] = sums[3][0][t];
    }
    __syncthreads();  // sums is free again
  }
}

// Rows shorter than a chunk or longer than the largest tile: dx and db a workgroup a row,
// value by value; the row's averages of h and h xs are kept for the sums over rows, which
// go by columns, a thread each, and a group of rows a workgroup.
template <int DT>
struct AnyRow {
  using T = Chunk<DT>;
  const ResidualGradArgs& a;
  const char *ds, *dy, *b, *s;
  float mb = 0.f, rb = 1.f, ms = 0.f, rs = 0.f, gate, s0 = 0.f, s1 = 0.f;
  __device__ __forceinline__ AnyRow(const ResidualGradArgs& a, long long r) : a(a) {
    auto at = [&](const void* p, long long ld) { return static_cast<const char*>(p) + r * ld * (long long)T::kSize; };
    ds = at(a.ds, a.ldds), dy = at(a.dy, a.lddy), b = at(a.b, a.ldb), s = at(a.s, a.lds);
    if (a.dy) rs = a.rstd_s[r], ms = a.rms ? 0.f : a.mean_s[r];
    if (a.post) rb = a.rstd_b[r], mb = a.rms ? 0.f : a.mean_b[r];
    gate = a.gate ? a.gate[r / a.per_gate] : 1.f;
  }
  __device__ __forceinline__ static float of(const void* w, int c, float otherwise) { return w ? T::load1(w, c) : otherwise; }
  __device__ __forceinline__ float xs(int c) const { return (T::load1(s, c) - ms) * rs; }
  __device__ __forceinline__ float xb(int c) const { return (T::load1(b, c) - mb) * rb; }
  __device__ __forceinline__ float h(int c) const { return T::load1(dy, c) * of(a.gamma2, c, 1.f); }
  __device__ __forceinline__ float dv(int c) const {
    const float d = a.ds ? T::load1(ds, c) : 0.f;
    return a.dy ? d + fmaf(h(c), rs, fmaf(xs(c), s1, s0)) : d;
  }
};

template <int DT>
__global__ __launch_bounds__(256) void residual_grad_any_kernel(ResidualGradArgs a) {
  using T = Chunk<DT>;
  __shared__ uint32_t slots[5][4];
  const int C = a.C;
  for (long long r = blockIdx.x; r < a.R; r += gridDim.x) {
    AnyRow<DT> row(a, r);
    if (a.dy) {
      float p0 = 0.f, p1 = 0.f;
      for (int c = threadIdx.x; c < C; c += 256) {
        const float h = row.h(c);
        p0 += h;
        p1 = fmaf(h, row.xs(c), p1);
      }
      p0 = sum_row<256>(p0, slots[0]);
      p1 = sum_row<256>(p1, slots[1]);
      row.s0 = a.rms ? 0.f : p0 * a.inv_c * -row.rs;
      row.s1 = p1 * a.inv_c * -row.rs;
      if (a.rows && threadIdx.x == 0) a.rows[2 * r] = row.s0, a.rows[2 * r + 1] = row.s1;
    }
    auto factor = [&](int c) { return row.gate * row.of(a.scale, c, 1.f); };
    float p0 = 0.f, p1 = 0.f, p2 = 0.f;
    for (int c = threadIdx.x; c < C; c += 256) {
      const float dv = row.dv(c), w = row.of(a.gamma1, c, 1.f), f = a.post ? row.xb(c) : T::load1(row.b, c);
      if (a.dx) T::store1(a.dx, r * C + c, dv);
      const float k = dv * factor(c) * w;
      p0 += k;
      p1 = fmaf(k, f, p1);
      p2 = fmaf(dv * row.of(a.scale, c, 1.f), a.post ? fmaf(f, w, row.of(a.beta1, c, 0.f)) : f, p2);
    }
    p0 = sum_row<256>(p0, slots[2]);
    p1 = sum_row<256>(p1, slots[3]);
    p2 = sum_row<256>(p2, slots[4]);
    if (a.dots && threadIdx.x == 0) a.dots[r] = p2;
    const float s0 = a.rms ? 0.f : p0 * a.inv_c * -row.rb, s1 = p1 * a.inv_c * -row.rb;
    if (a.db)
      for (int c = threadIdx.x; c < C; c += 256) {
        const float k = row.dv(c) * factor(c);
        T::store1(a.db, r * C + c, a.post ? fmaf(k * row.of(a.gamma1, c, 1.f), row.rb, fmaf(row.xb(c), s1, s0)) : k);
      }
    __syncthreads();  // the words of slots are free again
  }
}

template <int DT>
__global__ __launch_bounds__(256) void residual_grad_any_cols_kernel(ResidualGradArgs a) {
  using T = Chunk<DT>;
  const int c = blockIdx.x * 256 + threadIdx.x, C = a.C;
  if (c >= C) return;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  for (long long r = blockIdx.y; r < a.R; r += gridDim.y) {
    AnyRow<DT> row(a, r);
    if (a.dy) {
      row.s0 = a.rows[2 * r], row.s1 = a.rows[2 * r + 1];
      const float d = T::load1(row.dy, c);
      s[2] = fmaf(d, row.xs(c), s[2]);
      s[3] += d;
    }
    const float dg = row.dv(c) * row.gate;
    s[0] = fmaf(dg, a.post ? row.xb(c) : T::load1(row.b, c), s[0]);
    s[1] += dg;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) a.part[((size_t)blockIdx.y * 4 + q) * C + c] = s[q];
}

struct Plan {
  int lpr, vpl;  // lpr -1: value by value
  int threads, grid;
};

template <int DT>
Plan plan(int R, int C, bool near) {
  constexpr int E = Chunk<DT>::E;
  const int n = (C + E - 1) / E;
  auto make = [&](int lpr, int vpl, int threads, int most) {
    const int groups = lpr ? threads / lpr : 1;
    // (a workgroup that takes few rows costs as much by its sums)
    const int g = most > 256 ? std::min(std::max(R / 8, 256), most) : most;
    return Plan{lpr, vpl, threads, (int)std::min<long long>(((long long)R + groups - 1) / groups, g)};
  };
  if (C < E || n > (DT ? 1024 : 2048)) return Plan{-1, 0, 256, std::min(std::max(R / 32, 1), C < E ? 256 : 64)};
  if (near) {
    if (n <= 8 && R >= 16384) return make(8, 1, 512, 512);
    if (n <= 16) return make(16, 1, 512, 512);
    if (n <= 32) return make(16, 2, 512, 256);
  }
  if (n <= 64) return make(64, 1, 512, 512);
  if (n <= 128) return make(64, 2, 512, 256);
  // A row a workgroup, as many of them as are resident together.  us, chunks a lane x waves:
  //   bf16 32768 x 2560  2 x 3 266, 1 x 5 342      8192 x 4096  2 x 4 98, 1 x 8 120
  //        20000 x 1536  1 x 3 88, 2 x 2 99
  //   fp32 32768 x 2560  3 x 4 381, 2 x 5 439      8192 x 4096  3 x 6 168, 2 x 8 164
  //        20000 x 1536  1 x 6 140, 3 x 2 145
  const int vpl = n <= (DT ? 256 : 512) ? 1 : DT || n > 1536 ? 2 : 3, waves = (n + 64 * vpl - 1) / (64 * vpl);
  return make(0, vpl, 64 * waves, 256 * std::max(1, (vpl == 1 ? 12 : 8) / waves));
}


template <int DT, bool POST>
hipError_t launch_rows(ResidualGradArgs a, void* ws, hipStream_t stream) {
  const bool near = a.R == 1 || (std::max(std::max(a.ldds, a.lddy), std::max(a.ldb, a.lds)) < 1 << 27);
  const Plan p = plan<DT>(a.R, a.C, near);
  char* w = static_cast<char*>(ws);
  const bool sums = a.dscale || a.dgamma1 || a.dbeta1 || a.dgamma2 || a.dbeta2;
  a.dots = !a.dgate ? nullptr : a.per_gate == 1 ? a.dgate : reinterpret_cast<float*>(w);
  w += whole256((size_t)a.R * 4);
  a.rows = reinterpret_cast<float*>(w);
  if (p.lpr < 0) w += whole256((size_t)a.R * 8);
  a.part = sums ? reinterpret_cast<float*>(w) : nullptr;
  void* argv[] = {&a};
  hipError_t e = hipSuccess;
  auto go = [&](const void* fn) { return hipLaunchKernel(fn, dim3(p.grid), dim3(p.threads), argv, 0, stream); };
  if (p.lpr < 0) {
    if (!sums) a.rows = nullptr;
    if (a.dx || a.db || a.dots || a.rows)
      e = hipLaunchKernel((const void*)&residual_grad_any_kernel<DT>, dim3(std::min(a.R, 65536)), dim3(256), argv, 0, stream);
    if (e == hipSuccess && sums)
      e = hipLaunchKernel((const void*)&residual_grad_any_cols_kernel<DT>, dim3((a.C + 255) / 256, p.grid), dim3(256), argv, 0,
                          stream);
  } else if (p.lpr == 8) {
    e = go((const void*)&residual_grad_kernel<DT, 8, 1, POST>);
  } else if (p.lpr == 16) {
    e = go(p.vpl == 1 ? (const void*)&residual_grad_kernel<DT, 16, 1, POST> : (const void*)&residual_grad_kernel<DT, 16, 2, POST>);
  } else if (p.lpr == 64) {
    e = go(p.vpl == 1 ? (const void*)&residual_grad_kernel<DT, 64, 1, POST> : (const void*)&residual_grad_kernel<DT, 64, 2, POST>);
  } else {
    e = go(p.vpl == 1                 ? (const void*)&residual_grad_kernel<DT, 0, 1, POST>
           : p.vpl == 3               ? (const void*)&residual_grad_kernel<DT, 0, DT ? 2 : 3, POST>
           : DT || p.threads <= 512 ? (const void*)&residual_grad_kernel<DT, 0, 2, POST>
                                    : (const void*)&residual_grad_kernel<DT, 0, 2, POST, DT ? 512 : 1024>);
  }
  const int vectors = sums ? std::min((a.C + 31) / 32, 1 << 16) : 0;
  long long gates = a.dgate && a.per_gate > 1 ? ((long long)a.R + a.per_gate - 1) / a.per_gate : 0;
  gates = std::min<long long>(a.per_gate > kGateWave ? gates : (gates + 15) / 16, 1 << 16);
  if (e == hipSuccess && vectors + gates) {
    residual_vectors_kernel<DT><<<(unsigned)(vectors + gates), 1024, 0, stream>>>(a, p.grid, vectors);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

// The same for rows near and far: the larger of the two plans'.
size_t residual_grad_ws_bytes(int R, int C, int dt_bf16) {
  size_t most = 0;
  for (const bool near : {false, true}) {
    const Plan p = dt_bf16 ? plan<1>(R, C, near) : plan<0>(R, C, near);
    most = std::max(most, (p.lpr < 0 ? whole256((size_t)R * 8) : 0) + (size_t)p.grid * 4 * C * 4);
  }
  return whole256((size_t)R * 4) + most;
}

hipError_t launch_residual_grad(const ResidualGradArgs& a, void* ws, int dt_bf16, hipStream_t stream) {
  if (dt_bf16) return a.post ? launch_rows<1, true>(a, ws, stream) : launch_rows<1, false>(a, ws, stream);
  return a.post ? launch_rows<0, true>(a, ws, stream) : launch_rows<0, false>(a, ws, stream);
}

}  // namespace gl
