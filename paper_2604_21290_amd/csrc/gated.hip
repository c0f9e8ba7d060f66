// The gated fully connected layer
//   pre = x W^T + b,  W [2 F, K];  h = act(pre[:, :F]) * pre[:, F:]
// in one pass: a wave's tile holds as many columns of the gate as of the other product, the
// same ones, so that both of an output's products end in the same lane's registers and only
// h (and, for a backward pass, pre) is written.  Many rows: product.h; us, GELU, with pre:
// bf16 16384 x 2048 x 4096 494 (1.11 PFLOP/s), 12544 x 640 x 2560 117 (0.70: ten stages, then
// the activations, for which the matrix cores wait), 6272 x 192 x 768 15.
// Few rows (serving): the kernel below, which reads W once straight into registers; one row of
// 640 x 2560 bf16 3.9 us (W's 6.6 MB from the last level of cache and a launch).
#include <type_traits>

#include "product.h"

namespace gl {

namespace {

// Up to 16 RT rows.  A workgroup takes 16 columns of the gate and the same of the other
// product; its eight waves share the contraction, 128 bytes of every row at a time: a lane
// has 32 consecutive bytes of one row of W, and of one row of x, whose place in the
// instruction's contraction both agree on.  Rows of x are few and stay in the caches;
// W's bytes bound it.
template <int DT, int RT>
__global__ __launch_bounds__(512) void gated_few_kernel(ProductArgs a) {
  using T = Chunk<DT>;
  constexpr int E = T::E, ES = DT ? 2 : 4, BK = 128 / ES, NW = 8;
  __shared__ float sums[NW][2][RT * 16][17];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, t = lane & 15;
  const int n0 = blockIdx.x * 16, K = a.K;
  const char* wg = static_cast<const char*>(a.B) + (size_t)min(n0 + t, a.N - 1) * K * ES;
  const char* wu = wg + (size_t)a.N * K * ES;
  const char* x[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) x[r] = static_cast<const char*>(a.A) + (size_t)min(r * 16 + t, a.M - 1) * K * ES;
  f32x4 acc[2][RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) acc[0][r] = acc[1][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  // E values from k on, zeros past the row's end
  auto load = [&](const char* p, int k) {
    if (k + E <= K) return T::raw(p, k);
    uint32_t v[4] = {0, 0, 0, 0};
    for (int j = 0; k + j < K && j < E; ++j) {
      if (DT) v[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[k + j] << (j % 2 * 16);
      else v[j] = reinterpret_cast<const uint32_t*>(p)[k + j];
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
  };
  // N steps from k0 on; whole: within the rows, so that no load is behind a branch and those of
  // a later step may be under way (5 x 3936 x 8 fp32, one workgroup: 13.7 us for 15)
  auto steps = [&](int k0, auto n, auto whole) {
    constexpr int N = decltype(n)::value;
    uint4 wf[N][2][2], xf[N][RT][2];
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = k0 + s * NW * BK + g * 2 * E + h * E;
        auto at = [&](const char* p) { return decltype(whole)::value ? T::raw(p, k) : load(p, k); };
        wf[s][0][h] = at(wg);
        wf[s][1][h] = at(wu);
#pragma unroll
        for (int r = 0; r < RT; ++r) xf[s][r][h] = at(x[r]);
      }
#pragma unroll
    for (int s = 0; s < N; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          acc[0][r] = product_mma<DT>(wf[s][0][h], xf[s][r][h], acc[0][r]);
          acc[1][r] = product_mma<DT>(wf[s][1][h], xf[s][r][h], acc[1][r]);
        }
  };
  constexpr int U = RT == 1 ? 4 : 2;
  using std::integral_constant;
  int k0 = w * BK;
  for (; k0 + (U - 1) * NW * BK + BK <= K; k0 += U * NW * BK) steps(k0, integral_constant<int, U>{}, std::true_type{});
  for (; k0 + BK <= K; k0 += NW * BK) steps(k0, integral_constant<int, 1>{}, std::true_type{});
  if (k0 < K) steps(k0, integral_constant<int, 1>{}, std::false_type{});
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int v = 0; v < 4; ++v) sums[w][h][r * 16 + t][4 * g + v] = acc[h][r][v];
  __syncthreads();
  for (int i = threadIdx.x; i < RT * 256; i += 512) {
    const int r = i >> 4, c = i & 15, n = n0 + c;
    if (r >= a.M || n >= a.N) continue;
    float y = 0.f, u = 0.f;
#pragma unroll
    for (int q = 0; q < NW; ++q) y += sums[q][0][r][c], u += sums[q][1][r][c];
    if (a.bias) y += T::load1(a.bias, n), u += T::load1(a.bias, (size_t)a.N + n);
    if (a.pre) {
      T::store1(a.pre, (size_t)r * 2 * a.N + n, y);
      T::store1(a.pre, (size_t)r * 2 * a.N + a.N + n, u);
    }
    float g[1] = {y};
    gate_acts<DT>(a.act, g);
    T::store1(a.out, (size_t)r * a.N + n, g[0] * u);
  }
}

// (32 x 640 x 2560 bf16 5.3 us, by tiles 5.5; 64 x 512 x 2048 fp32 would take 10.6 for 8.0)
constexpr int kFewRows = 32;

// Where the contraction is parted: the parts' sums added in order, four columns of the gate and
// of the other product a thread, then the layer's end.
template <int DT>
__global__ __launch_bounds__(256) void gated_join_kernel(ProductArgs a) {
  using T = Chunk<DT>;
  const int N = a.N, across = (N + 3) / 4;
  const long long n = (long long)a.M * across;
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += 256LL * gridDim.x) {
    const long long row = i / across;
    const int c = (int)(i - row * across) * 4, m = min(4, N - c);
    const float* p = a.part + row * 2 * N + c;
    const size_t step = (size_t)a.M * 2 * N;
    float g[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
    if (m == 4) {
#pragma unroll 4
      for (int q = 0; q < a.parts; ++q) {
        float f[4];
        Chunk<0>::unpack(Chunk<0>::raw_at(reinterpret_cast<const char*>(p + q * step), 0), f);
#pragma unroll
        for (int j = 0; j < 4; ++j) g[j] += f[j];
        Chunk<0>::unpack(Chunk<0>::raw_at(reinterpret_cast<const char*>(p + q * step + N), 0), f);
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] += f[j];
      }
    } else {
      for (int q = 0; q < a.parts; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < m) g[j] += p[q * step + j], u[j] += p[q * step + N + j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j >= m) break;
      if (a.bias) g[j] += T::load1(a.bias, c + j), u[j] += T::load1(a.bias, (size_t)N + c + j);
      if (a.pre) {
        T::store1(a.pre, row * 2 * N + c + j, g[j]);
        T::store1(a.pre, row * 2 * N + N + c + j, u[j]);
      }
    }
    gate_acts<DT>(a.act, g);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < m) T::store1(a.out, row * N + c + j, g[j] * u[j]);
  }
}

template <int DT>
hipError_t launch_few(const ProductArgs& a, hipStream_t stream) {
  const void* fn = a.M <= 16 ? (const void*)&gated_few_kernel<DT, 1> : (const void*)&gated_few_kernel<DT, 2>;
  void* argv[] = {const_cast<ProductArgs*>(&a)};
  return hipLaunchKernel(fn, dim3((a.N + 15) / 16), dim3(512), argv, 0, stream);
}

template <class G>
hipError_t launch_tile(const ProductArgs& a, hipStream_t stream) {
  const long long tiles = ((long long)(a.M + G::BM - 1) / G::BM) * ((a.N + G::BN / 2 - 1) / (G::BN / 2)) * a.parts;
  if (tiles > INT32_MAX / G::kThreads) return hipErrorInvalidConfiguration;
  return launch_with_smem((const void*)&product_gated_kernel<G>, dim3((unsigned)tiles), dim3(G::kThreads), G::kSmem, stream,
                          nullptr, nullptr, a);
}

template <int DT>
hipError_t launch_tiles(const ProductArgs& a, int tile, hipStream_t stream) {
  if constexpr (DT == 1)
    if (tile == 256) return launch_tile<ProductCfg<1, false, false, 256, 256, 2, 4>>(a, stream);
  if (tile == 128) return launch_tile<ProductCfg<DT, false, false, 128, 128, 2, 2>>(a, stream);
  if (tile == 64) return launch_tile<ProductCfg<DT, false, false, 64, 64, 2, 2>>(a, stream);
  return launch_tile<ProductCfg<DT, false, false, 32, 32, 2, 2>>(a, stream);
}

// The workspace: rows of x and W brought to whole vectors, the parts' sums.
struct GatedPlan {
  size_t W = 0, part = 0, bytes = 0;  // offsets
  bool pack;
  ProductCut cut;
};

GatedPlan make_plan(int R, int K, int F, int dt_bf16) {
  GatedPlan p{};
  if (R <= kFewRows) return p;
  p.pack = K % (dt_bf16 ? 8 : 4) != 0;
  if (p.pack) {
    p.W = whole256(R * packed_row(K, dt_bf16));
    p.part = p.W + whole256(2 * (size_t)F * packed_row(K, dt_bf16));
  }
  p.cut = product_cut({R, 2LL * F, K}, dt_bf16, true);
  p.bytes = p.part + (p.cut.parts > 1 ? (size_t)p.cut.parts * R * 2 * F * 4 : 0);
  return p;
}

// A call asks three times: for the workspace's size, its check and the launch.
const GatedPlan& plan(int R, int K, int F, int dt_bf16) {
  thread_local int key[4] = {};
  thread_local GatedPlan last;
  const int now[4] = {R, K, F, dt_bf16};
  if (!std::equal(key, key + 4, now)) {
    last = make_plan(R, K, F, dt_bf16);
    std::copy(now, now + 4, key);
  }
  return last;
}

}  // namespace

size_t gated_ws_bytes(int R, int K, int F, int dt_bf16) { return plan(R, K, F, dt_bf16).bytes; }

hipError_t launch_gated(const GatedArgs& g, int dt_bf16, hipStream_t stream) {
  ProductArgs a{};
  a.A = g.x;
  a.B = g.W;
  a.lda = a.ldb = (long long)g.K * (dt_bf16 ? 2 : 4);
  a.M = g.R;
  a.N = g.F;
  a.K = g.K;
  a.out = g.h;
  a.bias = g.bias;
  a.pre = g.pre;
  a.act = g.act;
  if (g.R <= kFewRows) return dt_bf16 ? launch_few<1>(a, stream) : launch_few<0>(a, stream);
  const GatedPlan& p = plan(g.R, g.K, g.F, dt_bf16);
  char* ws = static_cast<char*>(g.ws);
  if (p.pack) {
    hipError_t e = launch_pack_rows(PackPair{{{g.x, ws, g.R, g.K}, {g.W, ws + p.W, 2 * g.F, g.K}}}, dt_bf16, stream);
    if (e != hipSuccess) return e;
    a.A = ws;
    a.B = ws + p.W;
    a.lda = a.ldb = (long long)packed_row(g.K, dt_bf16);
  }
  a.parts = p.cut.parts;
  a.part = reinterpret_cast<float*>(ws + p.part);
  hipError_t e = dt_bf16 ? launch_tiles<1>(a, p.cut.tile, stream) : launch_tiles<0>(a, p.cut.tile, stream);
  if (e != hipSuccess || a.parts == 1) return e;
  const unsigned grid = (unsigned)std::min<long long>(((long long)g.R * ((g.F + 3) / 4) + 255) / 256, 8192);
  if (dt_bf16) gated_join_kernel<1><<<grid, 256, 0, stream>>>(a);
  else gated_join_kernel<0><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace gl
