// The backward passes of the fully connected layers, plain and gated.
//   dx = dy W,  dW = dy^T x,  db = sum over rows of dy
// are two products of product.h and a sum over rows.  The gated layer's dy is
//   dpre = [dh u act'(g) | dh act(g)],  pre = [g | u]
// which one pass over dh and pre writes to the workspace, rounded to the operands' type (a
// product's operands are 16 bits; the sum db is of the values before that rounding).  Three
// launches: before, both products, after.  us, bf16: gated 16384 x 2048 x 4096 976 (113 at
// 5.9 TB/s, then 860: 1.28 PFLOP/s), 6272 x 192 x 768 36 (12.5, 21, 5); plain 12544 x 2560 x 640
// 112 (5, 100, 7).
#include "product.h"

namespace gl {

namespace {

constexpr int kSumGroups = 512;  // most groups of rows whose sums are kept apart

// rows [R, C] to rows of whole 16-byte vectors with zeros at their ends: 64 vectors of four
// rows a workgroup and turn, workgroup `id` of `count`
template <int DT>
__device__ __forceinline__ void pack_rows(const PackRows& a, int id, int count) {
  using T = Chunk<DT>;
  constexpr int ES = DT ? 2 : 4, E = T::E;
  const int C = a.C, row = (C * ES + 15) & ~15, across = (row / 16 + 63) / 64;
  const int y = id / across, v = (id - y * across) * 64 + (threadIdx.x & 63), c = v * E;
  if (v * 16 >= row) return;
  const long long step = 4LL * (count / across);
  constexpr int U = 4;  // rows under way
  for (long long r = y * 4 + (threadIdx.x >> 6); r < a.R; r += U * step) {
    uint4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const char* p = static_cast<const char*>(a.src) + min(r + u * step, a.R - 1LL) * C * ES;
      if (c + E <= C) {
        q[u] = T::raw(p, c);
      } else {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < E; ++j)
          if (c + j < C) {
            if (DT) w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[c + j] << (j % 2 * 16);
            else w[j] = reinterpret_cast<const uint32_t*>(p)[c + j];
          }
        q[u] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (r + u * step < a.R) *reinterpret_cast<uint4*>(static_cast<char*>(a.dst) + (r + u * step) * row + v * 16) = q[u];
  }
}
// workgroups for it, whole rows of them
int pack_count(const PackRows& a, int dt_bf16) {
  if (!a.src) return 0;
  const int across = (int)((packed_row(a.C, dt_bf16) / 16 + 63) / 64);
  return across * std::min((a.R + 15) / 16, std::max(1, 4096 / across));
}

template <int DT>
__global__ __launch_bounds__(256) void pack_rows_kernel(PackPair p, int first) {
  if ((int)blockIdx.x < first) pack_rows<DT>(p.t[0], blockIdx.x, first);
  else pack_rows<DT>(p.t[1], blockIdx.x - first, gridDim.x - first);
}

// What comes before the products, in one launch: dpre and its sums over groups of rows
// (GATED), or the sums of dy and, where its rows are no whole vectors, their copy; and the
// copies of x and W.
struct PrepareArgs {
  const void *dy, *pre;  // [R, F] (GATED: dh), [R, 2 F]
  char* out;             // rows of `row` bytes: dpre or dy, then zeros; null: not wanted
  float* part;           // [groups, 2 F or F]: the groups' sums, or null
  int R, F, row, act;
  int across, groups;    // workgroups: by columns, by groups of rows
  PackPair pack;
  int pack_first;        // workgroups of the first copy
};

// CL lanes take as many chunks of columns, 256 / CL rows a turn and two turns' loads under way.
template <int DT, bool GATED, int CL>
__global__ __launch_bounds__(256) void prepare_kernel(PrepareArgs a) {
  using T = Chunk<DT>;
  constexpr int E = T::E, ES = DT ? 2 : 4, RL = 256 / CL, NS = GATED ? 2 : 1, U = 2;
  __shared__ float sums[RL][CL * E + 4];
  int id = blockIdx.x;
  if (id >= a.across * a.groups) {
    id -= a.across * a.groups;
    if (id < a.pack_first) pack_rows<DT>(a.pack.t[0], id, a.pack_first);
    else pack_rows<DT>(a.pack.t[1], id - a.pack_first, gridDim.x - a.across * a.groups - a.pack_first);
    return;
  }
  const int group = id / a.across, block = id - group * a.across;
  const int lane = threadIdx.x % CL, rl = threadIdx.x / CL;
  const int F = a.F, c = (block * CL + lane) * E;
  const bool on = c < F, whole = c + E <= F;
  // the lane's columns of the row that begins `row` elements from p
  auto load = [&](const void* p, size_t row) {
    const char* q = static_cast<const char*>(p) + row * ES;
    if (whole) return T::raw(q, c);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (c + j < F) {
        if (DT) w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(q)[c + j] << (j % 2 * 16);
        else w[j] = reinterpret_cast<const uint32_t*>(q)[c + j];
      }
    return make_uint4(w[0], w[1], w[2], w[3]);
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
  const long long step = (long long)RL * a.groups;
  if (on)
    for (long long r0 = (long long)group * RL + rl; r0 < a.R; r0 += U * step) {
      uint4 rd[U], rp[U], ru[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const long long r = min(r0 + k * step, a.R - 1LL);
        rd[k] = load(a.dy, (size_t)r * F);
        if (GATED) {
          rp[k] = load(a.pre, (size_t)r * 2 * F);
          ru[k] = load(a.pre, (size_t)r * 2 * F + F);
        }
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const long long r = r0 + k * step;
        if (r >= a.R) break;
        float d[E];
        T::unpack(rd[k], d);
        char* o = a.out + (size_t)r * a.row;
        if (GATED) {
          float act[E], p[E], u[E];
          T::unpack(rp[k], act);
          T::unpack(ru[k], u);
          gate_act_grads(a.act, act, p);
#pragma unroll
          for (int j = 0; j < E; ++j) {
            p[j] *= d[j] * u[j];
            u[j] = d[j] * act[j];
            s[0][j] += p[j];
            s[NS - 1][j] += u[j];
          }
          if (a.out) {
            put(o, c, p);
            put(o, F + c, u);
          }
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j) s[0][j] += d[j];
          if (a.out) put(o, c, d);
        }
        if (a.out && c + E >= F)  // the row's last chunk
          for (int q = NS * F; q < a.row / ES; ++q) T::store1(o, q, 0.f);
      }
    }
  if (!a.part) return;
#pragma unroll
  for (int h = 0; h < NS; ++h) {
    if (h) __syncthreads();
#pragma unroll
    for (int j = 0; j < E; ++j) sums[rl][lane * E + j] = s[h][j];
    __syncthreads();
    for (int i = threadIdx.x; i < CL * E; i += 256) {
      const int col = block * CL * E + i;
      float v = sums[0][i];
#pragma unroll
      for (int q = 1; q < RL; ++q) v += sums[q][i];
      if (col < F) a.part[(size_t)group * NS * F + h * F + col] = v;
    }
  }
}

// What comes after the products, in one launch: the parts of dx and of dW added in order, and
// the groups' sums of db.
struct FinishArgs {
  const float* part[2];
  void* out[2];
  long long n[2];
  int parts[2], count[2];  // workgroups; 0: not parted
  const float* sums;       // [groups, cols], or null
  float* db;
  int groups, cols;
};

template <int DT>
__global__ __launch_bounds__(256) void finish_kernel(FinishArgs a) {
  int id = blockIdx.x;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (id < a.count[k]) {
      const float* part = a.part[k];
      const long long n = a.n[k];
      for (long long i = (id * 256LL + threadIdx.x) * 4; i < n; i += 1024LL * a.count[k]) {
        const int m = (int)min(4LL, n - i);
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        if (m == 4) {
          // (eight loads under way at a time)
          for (int p0 = 0; p0 < a.parts[k]; p0 += 8) {
            uint4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
              v[u] = Chunk<0>::raw_at(reinterpret_cast<const char*>(part + min(p0 + u, a.parts[k] - 1) * n + i), 0);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              float f[4];
              Chunk<0>::unpack(v[u], f);
#pragma unroll
              for (int j = 0; j < 4; ++j) s[j] += p0 + u < a.parts[k] ? f[j] : 0.f;
            }
          }
          if (DT) store8_any(static_cast<uint16_t*>(a.out[k]) + i,
                             make_uint2(f32x2_to_bf16x2_bits(s[0], s[1]), f32x2_to_bf16x2_bits(s[2], s[3])));
          else Chunk<0>::store(a.out[k], i, s);
        } else {
          for (int j = 0; j < m; ++j) {
            float v = 0.f;
            for (int p = 0; p < a.parts[k]; ++p) v += part[p * n + i + j];
            Chunk<DT>::store1(a.out[k], i + j, v);
          }
        }
      }
      return;
    }
    id -= a.count[k];
  }
  // 32 columns a workgroup, eight groups at a time and eight of those under way
  constexpr int COLS = 32, ROWS = 256 / COLS;
  __shared__ float sums[ROWS][COLS + 1];
  const int t = threadIdx.x % COLS, w = threadIdx.x / COLS, c = id * COLS + t;
  float s = 0.f;
  for (int g0 = w; g0 < a.groups; g0 += 8 * ROWS) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = a.sums[(size_t)min(g0 + u * ROWS, a.groups - 1) * a.cols + min(c, a.cols - 1)];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += g0 + u * ROWS < a.groups ? v[u] : 0.f;
  }
  sums[w][t] = s;
#pragma unroll
  for (int h = ROWS / 2; h >= 1; h /= 2) {
    __syncthreads();
    if (w < h) sums[w][t] += sums[w + h][t];
  }
  if (w == 0 && c < a.cols) a.db[c] = sums[0][t];
}

size_t part_bytes(int parts, const ProductSize& s) { return parts > 1 ? whole256((size_t)parts * s.M * s.N * 4) : 0; }

template <int DT, int TILE>
hipError_t launch_pair(ProductPair p, hipStream_t stream) {
  using G = typename PairCfg<DT, TILE>::X;
  auto count = [](const ProductArgs& a) {
    return a.out ? ((long long)(a.M + TILE - 1) / TILE) * ((a.N + TILE - 1) / TILE) * a.parts : 0;
  };
  const long long x = count(p.dx), w = count(p.dW);
  if (x + w + 8 > INT32_MAX / G::kThreads) return hipErrorInvalidConfiguration;
  p.dx_count = (int)x;
  p.dW_count = (int)w;
  p.dW_first = (long long)p.dW.K / std::max(1, p.dW.parts) > (long long)p.dx.K / std::max(1, p.dx.parts);
  const long long all = (((p.dW_first ? w : x) + 7) & ~7LL) + (p.dW_first ? x : w);
  return launch_with_smem((const void*)&product_pair_kernel<PairCfg<DT, TILE>>, dim3((unsigned)all), dim3(G::kThreads), G::kSmem, stream,
                          nullptr, nullptr, p);
}

template <int DT>
hipError_t launch_tile(const ProductPair& p, int tile, hipStream_t stream) {
  if constexpr (DT == 1)
    if (tile == 256) return launch_pair<DT, 256>(p, stream);
  return tile == 128 ? launch_pair<DT, 128>(p, stream) : launch_pair<DT, 64>(p, stream);
}

// Lanes to a row of F columns (narrow rows would leave most of 32 idle), and groups of rows of
// the sums over rows.
int row_lanes(int F, int dt_bf16) { return F <= (dt_bf16 ? 64 : 32) ? 8 : 32; }
int sum_groups(int R, int F, int dt_bf16) {
  const int lanes = row_lanes(F, dt_bf16), e = dt_bf16 ? 8 : 4;
  const long long cols = ((long long)F + lanes * e - 1) / (lanes * e), rows = ((long long)R + 256 / lanes - 1) / (256 / lanes);
  return (int)std::max<long long>(1, std::min<long long>({(rows + 1) / 2, (2048 + cols - 1) / cols, kSumGroups}));
}

// The workspace of a backward pass, its pieces 256 bytes apart.
struct GradPlan {
  size_t x = 0, dy = 0, W = 0, sums = 0, part_x = 0, part_W = 0, bytes = 0;  // offsets; W, x, dy: packed rows
  bool pack_x, pack_dy;
  int groups;
  ProductCuts cuts;
};

GradPlan make_plan(int R, int K, int N, int dt_bf16, bool gated) {
  GradPlan p{};
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
  const ProductSize x{R, K, N}, W{N, K, R};
  p.cuts = product_cuts(x, W, dt_bf16);
  p.part_x = take(part_bytes(p.cuts.x.parts, x));
  p.part_W = take(part_bytes(p.cuts.W.parts, W));
  p.bytes = at;
  return p;
}

// A call asks three times: for the workspace's size, its check and the launch.
const GradPlan& plan(int R, int K, int N, int dt_bf16, bool gated) {
  thread_local int key[5] = {};
  thread_local GradPlan last;
  const int now[5] = {R, K, N, dt_bf16, gated};
  if (!std::equal(key, key + 5, now)) {
    last = make_plan(R, K, N, dt_bf16, gated);
    std::copy(now, now + 5, key);
  }
  return last;
}

template <int DT>
hipError_t launch_grad(const LinearGradArgs& g, hipStream_t stream) {
  constexpr int es = DT ? 2 : 4, E = 16 / es;
  const bool gated = g.pre != nullptr, products = g.dx || g.dW;
  const GradPlan p = plan(g.R, g.K, g.N, DT, gated);
  char* ws = static_cast<char*>(g.ws);
  const int F = gated ? g.N / 2 : g.N;
  hipError_t e = hipSuccess;

  PrepareArgs s{};
  s.dy = g.dy;
  s.pre = g.pre;
  s.R = g.R;
  s.F = F;
  s.act = g.act;
  s.row = (int)packed_row(g.N, DT);
  s.out = products && p.pack_dy ? ws + p.dy : nullptr;
  s.part = !g.db ? nullptr : p.groups > 1 ? reinterpret_cast<float*>(ws + p.sums) : g.db;
  const int lanes = row_lanes(F, DT);
  s.across = (F + lanes * E - 1) / (lanes * E);
  s.groups = s.out || s.part ? p.groups : 0;
  if (p.pack_x && g.dW) s.pack.t[0] = {g.x, ws + p.x, g.R, g.K};
  if (p.pack_x && g.dx) s.pack.t[1] = {g.W, ws + p.W, g.N, g.K};
  s.pack_first = pack_count(s.pack.t[0], DT);
  const int before = s.across * s.groups + s.pack_first + pack_count(s.pack.t[1], DT);
  if (before) {
    void* argv[] = {&s};
    const void* fn = gated ? (lanes == 8 ? (const void*)&prepare_kernel<DT, true, 8> : (const void*)&prepare_kernel<DT, true, 32>)
                           : (lanes == 8 ? (const void*)&prepare_kernel<DT, false, 8> : (const void*)&prepare_kernel<DT, false, 32>);
    if ((e = hipLaunchKernel(fn, dim3(before), dim3(256), argv, 0, stream)) != hipSuccess) return e;
  }

  ProductPair q{};
  ProductArgs a{};
  const long long krow = (long long)packed_row(g.K, DT), nrow = (long long)packed_row(g.N, DT);
  a.A = p.pack_dy ? ws + p.dy : g.dy;
  a.lda = nrow;
  a.ldb = krow;
  a.N = g.K;
  a.cols_a = (int)(nrow / 16);
  a.cols_b = (int)(krow / 16);
  q.dx = q.dW = a;
  q.dx.B = p.pack_x ? ws + p.W : g.W;
  q.dx.M = g.R;
  q.dx.K = g.N;
  q.dx.out = g.dx;
  q.dx.parts = p.cuts.x.parts;
  q.dx.part = reinterpret_cast<float*>(ws + p.part_x);
  q.dW.B = p.pack_x ? ws + p.x : g.x;
  q.dW.M = g.N;
  q.dW.K = g.R;
  q.dW.out = g.dW;
  q.dW.parts = p.cuts.W.parts;
  q.dW.part = reinterpret_cast<float*>(ws + p.part_W);
  if (products && p.cuts.together) {
    e = launch_tile<DT>(q, p.cuts.x.tile, stream);
  } else {
    ProductPair x = q, W = q;
    x.dW.out = W.dx.out = nullptr;
    if (g.dx) e = launch_tile<DT>(x, p.cuts.x.tile, stream);
    if (g.dW && e == hipSuccess) e = launch_tile<DT>(W, p.cuts.W.tile, stream);
  }
  if (e != hipSuccess) return e;

  FinishArgs f{};
  const ProductArgs* both[2] = {&q.dx, &q.dW};
  for (int k = 0; k < 2; ++k) {
    f.part[k] = both[k]->part;
    f.out[k] = both[k]->out;
    f.n[k] = (long long)both[k]->M * both[k]->N;
    f.parts[k] = both[k]->parts;
    f.count[k] = both[k]->out && both[k]->parts > 1 ? (int)std::min<long long>((f.n[k] + 1023) / 1024, 4096) : 0;
  }
  const bool sums = g.db && p.groups > 1;
  f.sums = reinterpret_cast<const float*>(ws + p.sums);
  f.db = g.db;
  f.groups = p.groups;
  f.cols = g.N;
  const int after = f.count[0] + f.count[1] + (sums ? (g.N + 31) / 32 : 0);
  if (after) finish_kernel<DT><<<after, 256, 0, stream>>>(f);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_pack_rows(const PackPair& p, int dt_bf16, hipStream_t stream) {
  const int first = pack_count(p.t[0], dt_bf16), all = first + pack_count(p.t[1], dt_bf16);
  if (dt_bf16) pack_rows_kernel<1><<<all, 256, 0, stream>>>(p, first);
  else pack_rows_kernel<0><<<all, 256, 0, stream>>>(p, first);
  return hipGetLastError();
}

size_t linear_grad_ws_bytes(int R, int K, int N, int dt_bf16, bool gated) { return plan(R, K, N, dt_bf16, gated).bytes; }

hipError_t launch_linear_grad(const LinearGradArgs& g, int dt_bf16, hipStream_t stream) {
  return dt_bf16 ? launch_grad<1>(g, stream) : launch_grad<0>(g, stream);
}

}  // namespace gl
