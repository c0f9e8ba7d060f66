// The backward passes of the fully connected layers, plain and gated.
//   dx = dy W,  dW = dy^T x,  db = sum over rows of dy
// are two products of product.h and a sum over rows.  The gated layer's dy is
//   dpre = [dh u act'(g) | dh act(g)],  pre = [g | u]
// which one pass over dh and pre writes to the workspace, rounded to the operands' type (a
// product's operands are 16 bits; the sum db is of the values before that rounding).
#include "product.h"

namespace gl {

namespace {

constexpr int kSumGroups = 256;  // most groups of rows whose sums are kept apart

size_t packed_row(int C, int dt_bf16) { return ((size_t)C * (dt_bf16 ? 2 : 4) + 15) & ~(size_t)15; }
size_t whole256(size_t n) { return (n + 255) & ~(size_t)255; }

// rows [R, C] to rows of `row` bytes, whole 16-byte vectors with zeros at their ends: 64
// vectors of four rows a workgroup and turn
template <int DT>
__global__ __launch_bounds__(256) void pack_rows_kernel(const void* src, int R, int C, char* dst, int row) {
  using T = Chunk<DT>;
  constexpr int ES = DT ? 2 : 4, E = T::E;
  const int v = blockIdx.x * 64 + (threadIdx.x & 63), c = v * E;
  if (v * 16 >= row) return;
  for (long long r = blockIdx.y * 4 + (threadIdx.x >> 6); r < R; r += 4LL * gridDim.y) {
    const char* p = static_cast<const char*>(src) + r * C * ES;
    uint4 q;
    if (c + E <= C) {
      q = T::raw(p, c);
    } else {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (c + j < C) {
          if (DT) w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[c + j] << (j % 2 * 16);
          else w[j] = reinterpret_cast<const uint32_t*>(p)[c + j];
        }
      q = make_uint4(w[0], w[1], w[2], w[3]);
    }
    *reinterpret_cast<uint4*>(dst + r * row + v * 16) = q;
  }
}

struct GateGradArgs {
  const void *dh, *pre;  // [R, F], [R, 2 F]
  char* dpre;            // rows of `row` bytes: dpre, then zeros
  float* part;           // [gridDim.y, 2 F]: the groups' sums of dpre, or null
  int R, F, row, act;
};

// 32 lanes take 32 chunks of columns, eight rows a turn.
// dpre and its groups' sums (GATED), or the sums of rows dh alone.
template <int DT, bool GATED>
__global__ __launch_bounds__(256) void gate_grad_kernel(GateGradArgs a) {
  using T = Chunk<DT>;
  constexpr int E = T::E, ES = DT ? 2 : 4, CL = 32, RL = 256 / CL, NS = GATED ? 2 : 1;
  __shared__ float sums[RL][CL * E + 4];
  const int lane = threadIdx.x % CL, rl = threadIdx.x / CL;
  const int F = a.F, c = (blockIdx.x * CL + lane) * E;
  const bool on = c < F, whole = c + E <= F;
  auto load = [&](const void* p, size_t at, float* f) {
    if (whole) {
      T::unpack(T::raw(p, at), f);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) f[j] = c + j < F ? T::load1(p, at + j) : 0.f;
    }
  };
  auto put = [&](char* p, size_t at, const float* f) {
    if (whole) {
      T::store(p, at, f);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (c + j < F) T::store1(p, at + j, f[j]);
    }
  };
  float s[NS][E] = {};
  const long long step = (long long)RL * gridDim.y;
  if (on)
    for (long long r = (long long)blockIdx.y * RL + rl; r < a.R; r += step) {
      float d[E];
      load(a.dh, (size_t)r * F + c, d);
      if (!GATED) {
#pragma unroll
        for (int j = 0; j < E; ++j) s[0][j] += d[j];
        continue;
      }
      float p[E], u[E];
      load(a.pre, (size_t)r * 2 * F + c, p);
      load(a.pre, (size_t)r * 2 * F + F + c, u);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        float da;
        const float act = gate_act_grad(a.act, p[j], &da);
        p[j] = d[j] * u[j] * da;
        u[j] = d[j] * act;
        s[0][j] += p[j];
        s[NS - 1][j] += u[j];
      }
      char* o = a.dpre + (size_t)r * a.row;
      put(o, c, p);
      put(o, F + c, u);
      if (!whole || c + E == F)  // the row's last chunk
        for (int k = 2 * F; k < a.row / ES; ++k) T::store1(o, k, 0.f);
    }
  if (!a.part) return;
#pragma unroll
  for (int h = 0; h < NS; ++h) {
    if (h) __syncthreads();
#pragma unroll
    for (int j = 0; j < E; ++j) sums[rl][lane * E + j] = s[h][j];
    __syncthreads();
    for (int i = threadIdx.x; i < CL * E; i += 256) {
      const int col = blockIdx.x * CL * E + i;
      float v = sums[0][i];
#pragma unroll
      for (int q = 1; q < RL; ++q) v += sums[q][i];
      if (col < F) a.part[(size_t)blockIdx.y * NS * F + h * F + col] = v;
    }
  }
}

// out[i] = sum over p of part[p, i], i < n, in the order of the parts
template <int DT>
__global__ __launch_bounds__(256) void product_join_kernel(const float* part, int parts, long long n, void* out) {
  for (long long i = (blockIdx.x * 256LL + threadIdx.x) * 4; i < n; i += 1024LL * gridDim.x) {
    const int m = (int)min(4LL, n - i);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (m == 4) {
      for (int p = 0; p < parts; ++p) {
        float f[4];
        Chunk<0>::unpack(Chunk<0>::raw_at(reinterpret_cast<const char*>(part + p * n + i), 0), f);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] += f[j];
      }
      if (DT) store8_any(static_cast<uint16_t*>(out) + i,
                         make_uint2(f32x2_to_bf16x2_bits(s[0], s[1]), f32x2_to_bf16x2_bits(s[2], s[3])));
      else Chunk<0>::store(out, i, s);
    } else {
      for (int j = 0; j < m; ++j) {
        for (int p = 0; p < parts; ++p) s[0] += part[p * n + i + j];
        Chunk<DT>::store1(out, i + j, s[0]);
        s[0] = 0.f;
      }
    }
  }
}

// out[c] = sum over the G rows of part [G, cols]: 32 columns a workgroup, 32 rows at a time,
// in the same order always (a thread a column took 62 us for 256 x 1536).
__global__ __launch_bounds__(1024) void sum_groups_kernel(const float* part, int G, int cols, float* out) {
  constexpr int COLS = 32, ROWS = 1024 / COLS;
  __shared__ float sums[ROWS][COLS + 1];
  const int t = threadIdx.x % COLS, w = threadIdx.x / COLS, c = blockIdx.x * COLS + t;
  float s = 0.f;
  for (int g0 = w; g0 < G; g0 += 8 * ROWS) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = part[(size_t)min(g0 + u * ROWS, G - 1) * cols + min(c, cols - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += g0 + u * ROWS < G ? v[u] : 0.f;
  }
  sums[w][t] = s;
#pragma unroll
  for (int h = ROWS / 2; h >= 1; h /= 2) {
    __syncthreads();
    if (w < h) sums[w][t] += sums[w + h][t];
  }
  if (w == 0 && c < cols) out[c] = sums[0][t];
}

size_t part_bytes(const ProductCut& c, long long M, long long N) { return c.parts > 1 ? (size_t)c.parts * M * N * 4 : 0; }

template <int DT, bool KA, bool KB, int EPI>
hipError_t launch_cut(const ProductArgs& a, int tile, hipStream_t stream) {
  if constexpr (DT == 1)
    if (tile == 256) return launch_product<ProductCfg<1, KA, KB, 256, 256, 2, 4>, EPI>(a, stream);
  if (tile == 128) return launch_product<ProductCfg<DT, KA, KB, 128, 128, 2, 2>, EPI>(a, stream);
  return launch_product<ProductCfg<DT, KA, KB, 64, 64, 2, 2>, EPI>(a, stream);
}

template <int DT, bool KA, bool KB>
hipError_t product(ProductArgs a, float* part, hipStream_t stream) {
  const ProductCut c = product_cut(a.M, a.N, a.K, DT, true);
  if (c.parts == 1) return launch_cut<DT, KA, KB, kProductStore>(a, c.tile, stream);
  a.parts = c.parts;
  a.part = part;
  hipError_t e = launch_cut<DT, KA, KB, kProductPart>(a, c.tile, stream);
  if (e != hipSuccess) return e;
  const long long n = (long long)a.M * a.N;
  product_join_kernel<DT><<<(unsigned)std::min<long long>((n + 1023) / 1024, 4096), 256, 0, stream>>>(part, c.parts, n, a.out);
  return hipGetLastError();
}

// Groups of rows of the sums over rows.
int sum_groups(int R, int F, int dt_bf16) {
  const long long cols = ((long long)F + (dt_bf16 ? 255 : 127)) / (dt_bf16 ? 256 : 128);
  const long long rows = ((long long)R + 7) / 8;
  return (int)std::max<long long>(1, std::min<long long>({rows, (2048 + cols - 1) / cols, kSumGroups}));
}

// The workspace of a backward pass, its pieces 256 bytes apart.
struct GradPlan {
  size_t x = 0, dy = 0, W = 0, sums = 0, part = 0, bytes = 0;  // offsets; W, x, dy: packed rows
  bool pack_x, pack_dy;
  int groups;
};

GradPlan plan(int R, int K, int N, int dt_bf16, bool gated) {
  GradPlan p;
  const int e = dt_bf16 ? 8 : 4;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += whole256(n);
    return o;
  };
  p.pack_x = K % e != 0;
  p.pack_dy = gated || N % e != 0;
  if (p.pack_x) {
    p.x = take(R * packed_row(K, dt_bf16));
    p.W = take(N * packed_row(K, dt_bf16));
  }
  if (p.pack_dy) p.dy = take(R * packed_row(N, dt_bf16));
  p.groups = sum_groups(R, gated ? N / 2 : N, dt_bf16);
  p.sums = take(p.groups > 1 ? (size_t)p.groups * N * 4 : 0);
  p.part = take(std::max(part_bytes(product_cut(R, K, N, dt_bf16, true), R, K),
                         part_bytes(product_cut(N, K, R, dt_bf16, true), N, K)));
  p.bytes = at;
  return p;
}

template <int DT>
hipError_t launch_grad(const LinearGradArgs& g, hipStream_t stream) {
  constexpr int es = DT ? 2 : 4, E = 16 / es;
  const bool gated = g.pre != nullptr;
  const GradPlan p = plan(g.R, g.K, g.N, DT, gated);
  char* ws = static_cast<char*>(g.ws);
  const void *x = g.x, *W = g.W, *dy = g.dy;
  const int F = gated ? g.N / 2 : g.N;
  hipError_t e = hipSuccess;
  if (p.pack_x) {
    if (g.dW) e = launch_pack_rows(g.x, g.R, g.K, ws + p.x, DT, stream);
    if (e == hipSuccess && g.dx) e = launch_pack_rows(g.W, g.N, g.K, ws + p.W, DT, stream);
    x = ws + p.x;
    W = ws + p.W;
  }
  if (e != hipSuccess) return e;
  GateGradArgs s{};
  s.dh = g.dy;
  s.pre = g.pre;
  s.R = g.R;
  s.F = F;
  s.act = g.act;
  s.row = (int)packed_row(g.N, DT);
  s.dpre = ws + p.dy;
  s.part = !g.db ? nullptr : p.groups > 1 ? reinterpret_cast<float*>(ws + p.sums) : g.db;
  const dim3 grid((F + 32 * E - 1) / (32 * E), p.groups);
  if (gated) gate_grad_kernel<DT, true><<<grid, 256, 0, stream>>>(s);
  else if (g.db) gate_grad_kernel<DT, false><<<grid, 256, 0, stream>>>(s);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (g.db && p.groups > 1) {
    sum_groups_kernel<<<(g.N + 31) / 32, 1024, 0, stream>>>(reinterpret_cast<float*>(ws + p.sums), p.groups, g.N, g.db);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (!gated && p.pack_dy && (g.dx || g.dW)) e = launch_pack_rows(g.dy, g.R, g.N, ws + p.dy, DT, stream);
  if (p.pack_dy) dy = ws + p.dy;
  if (e != hipSuccess) return e;
  ProductArgs a{};
  const long long krow = (long long)packed_row(g.K, DT), nrow = (long long)packed_row(g.N, DT);
  float* part = reinterpret_cast<float*>(ws + p.part);
  a.A = dy;
  a.lda = nrow;
  a.ldb = krow;
  a.N = g.K;
  a.cols_a = (int)(nrow / 16);
  a.cols_b = (int)(krow / 16);
  if (g.dx) {
    a.B = W;
    a.M = g.R;
    a.K = g.N;
    a.out = g.dx;
    if ((e = product<DT, false, true>(a, part, stream)) != hipSuccess) return e;
  }
  if (g.dW) {
    a.B = x;
    a.M = g.N;
    a.K = g.R;
    a.out = g.dW;
    e = product<DT, true, true>(a, part, stream);
  }
  return e;
}

}  // namespace

hipError_t launch_pack_rows(const void* src, int R, int C, void* dst, int dt_bf16, hipStream_t stream) {
  const int row = (int)packed_row(C, dt_bf16);
  const dim3 grid((row / 16 + 63) / 64, std::min((R + 3) / 4, 4096));
  if (dt_bf16) pack_rows_kernel<1><<<grid, 256, 0, stream>>>(src, R, C, static_cast<char*>(dst), row);
  else pack_rows_kernel<0><<<grid, 256, 0, stream>>>(src, R, C, static_cast<char*>(dst), row);
  return hipGetLastError();
}

size_t linear_grad_ws_bytes(int R, int K, int N, int dt_bf16, bool gated) { return plan(R, K, N, dt_bf16, gated).bytes; }

hipError_t launch_linear_grad(const LinearGradArgs& g, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_grad<1>(g, stream) : launch_grad<0>(g, stream);
}

}  // namespace gl
