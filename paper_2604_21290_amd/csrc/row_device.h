// Device helpers of the kernels that work on whole rows of channels (layer norm,
// its gradient, the 8-bit rows): a row in chunks of 16 bytes, sums and maxima over
// the lanes that share a row, and the rounding to 8 bits.
#pragma once

#include "gl_device.h"

namespace gl {

// ---------------------------------------------------------------------------
// chunks: 8 bf16 or 4 fp32 values, 16 bytes at any element's place.  A row of C
// channels is covered by ceil(C / E) of them; where C is not a whole number of
// chunks the last one is moved back to end with the row, and its first `skip`
// values, which the chunk before it has too, are left out of sums.  So every
// access lies inside the row and no width or alignment needs a loop over single
// values (rows shorter than one chunk aside).
// ---------------------------------------------------------------------------
template <int DT>
struct Chunk;  // DT 1: bf16, 0: fp32

typedef uint32_t u32x4_any4 __attribute__((ext_vector_type(4), aligned(4), may_alias));

template <>
struct Chunk<1> {
  static constexpr int E = 8;
  static constexpr size_t kSize = 2;
  __device__ __forceinline__ static uint4 raw(const void* p, size_t i) {
    return load16_any(static_cast<const uint16_t*>(p) + i);
  }
  __device__ __forceinline__ static uint4 raw_at(const char* p, uint32_t byte) { return load16_any(p + byte); }
  __device__ __forceinline__ static void store_at(char* p, uint32_t byte, const float* f) {
    store16_any(p + byte, pack_bf16x8(f));
  }
  __device__ __forceinline__ static uint4 ones() {
    return make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
  }
  __device__ __forceinline__ static void unpack(const uint4& v, float* f) { unpack_bf16x8(v, f); }
  // the largest magnitude's bits as fp32, two values at a time
  __device__ __forceinline__ static uint32_t top(const uint4& v) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    auto mag = [](uint32_t w) { return __builtin_bit_cast(u16x2, w & 0x7fff7fffu); };
    const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(mag(v.x), mag(v.y)),
                                              __builtin_elementwise_max(mag(v.z), mag(v.w)));
    return (uint32_t)max(m[0], m[1]) << 16;
  }
  __device__ __forceinline__ static void store(void* p, size_t i, const float* f) {
    store16_any(static_cast<uint16_t*>(p) + i, pack_bf16x8(f));
  }
  __device__ __forceinline__ static float load1(const void* p, size_t i) {
    return bf16_bits_to_f32(static_cast<const uint16_t*>(p)[i]);
  }
  __device__ __forceinline__ static void store1(void* p, size_t i, float f) {
    static_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16_bits(f);
  }
};

template <>
struct Chunk<0> {
  static constexpr int E = 4;
  static constexpr size_t kSize = 4;
  __device__ __forceinline__ static uint4 raw(const void* p, size_t i) {
    return raw_at(static_cast<const char*>(p), (uint32_t)i * 4);
  }
  __device__ __forceinline__ static uint4 raw_at(const char* p, uint32_t byte) {
    return __builtin_bit_cast(uint4, *reinterpret_cast<const u32x4_any4*>(p + byte));
  }
  __device__ __forceinline__ static void store_at(char* p, uint32_t byte, const float* f) {
    store(p + byte, 0, f);
  }
  __device__ __forceinline__ static uint4 ones() {
    return make_uint4(0x3f800000u, 0x3f800000u, 0x3f800000u, 0x3f800000u);
  }
  __device__ __forceinline__ static void unpack(const uint4& v, float* f) {
    f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
  }
  __device__ __forceinline__ static uint32_t top(const uint4& v) {
    return max(max(v.x & 0x7fffffffu, v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu));
  }
  __device__ __forceinline__ static void store(void* p, size_t i, const float* f) {
    u32x4_any4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(f[j]);
    *reinterpret_cast<u32x4_any4*>(static_cast<float*>(p) + i) = v;
  }
  __device__ __forceinline__ static float load1(const void* p, size_t i) {
    return static_cast<const float*>(p)[i];
  }
  __device__ __forceinline__ static void store1(void* p, size_t i, float f) {
    static_cast<float*>(p)[i] = f;
  }
};

// Where the rows of a workgroup lie, LPR lanes to each: a wave's first row is uniform, so
// that rows are addressed by a uniform base and 32 bits a lane (LPR < 64: the caller's
// strides leave the wave's other rows within them).
template <int LPR>
struct WaveRows {
  static constexpr int kRows = LPR < 64 ? 64 / LPR : 1;  // rows of a wave
  int wave, lane;  // the wave's first row in the workgroup, the lane's row in the wave
  __device__ __forceinline__ WaveRows()
      : wave(__builtin_amdgcn_readfirstlane(LPR < 64 ? (threadIdx.x >> 6) * kRows : threadIdx.x / LPR)),
        lane(LPR < 64 ? (threadIdx.x & 63) / LPR : 0) {}
  // rows of `bytes` from row `first` of R on: the base, and where the lane's row lies from
  // it; rows past the last repeat it
  __device__ __forceinline__ const char* at(const void* p, long long first, long long R, long long bytes,
                                            uint32_t* off) const {
    const long long f = min(first, R - 1);
    int l = lane;
    if (LPR < 64 && f + kRows > R) l = min(l, (int)(R - 1 - f));
    *off = LPR < 64 ? (uint32_t)l * (uint32_t)bytes : 0u;
    return static_cast<const char*>(p) + f * bytes;
  }
};

// A packed vector that a loop keeps: hides from the compiler that it does not change, or
// it would keep the unpacked values, twice the registers, instead.
__device__ __forceinline__ void keep_packed(uint4& v) {
  asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w));
}

// ---------------------------------------------------------------------------
// sums and maxima over the LPR lanes (8, 16, 64, or a workgroup's LPR / 64 waves) of
// one row; every lane of the group gets the result, in the same order always.
// `slot`: a word of LDS for each wave, for this reduction alone (LPR > 64).
// ---------------------------------------------------------------------------
struct AddF {
  __device__ __forceinline__ static uint32_t of(uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }
};
struct MaxU {
  __device__ __forceinline__ static uint32_t of(uint32_t a, uint32_t b) { return max(a, b); }
};

template <class Op>
__device__ __forceinline__ uint32_t reduce8(uint32_t v) {
  v = Op::of(v, dpp_mov<0xB1>(v));      // quad_perm [1,0,3,2]
  v = Op::of(v, dpp_mov<0x4E>(v));      // quad_perm [2,3,0,1]
  return Op::of(v, dpp_mov<0x141>(v));  // half-row mirror: the other quad of eight
}
template <class Op>
__device__ __forceinline__ uint32_t reduce16(uint32_t v) {
  v = reduce8<Op>(v);
  return Op::of(v, dpp_mov<0x140>(v));  // row mirror: the other eight
}

// Sum over the groups of 8 or 16 lanes of a wave, lane by lane (gfx950 swaps rows of two
// registers: with both the same, each ends with one of each pair's rows twice).
template <int LPR>
__device__ __forceinline__ float sum_over_groups(float v) {
  if (LPR == 8) v += __uint_as_float(dpp_mov<0x128>(__float_as_uint(v)));  // row rotate by 8
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t w = __float_as_uint(v);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <class Op, int LPR>
__device__ __forceinline__ uint32_t reduce_row(uint32_t v, uint32_t* slot) {
  if (LPR == 8) return reduce8<Op>(v);
  v = reduce16<Op>(v);
  if (LPR == 16) return v;
  const uint32_t a = Op::of(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16));
  const uint32_t b = Op::of(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48));
  v = Op::of(a, b);
  if (LPR == 64) return v;
  constexpr int NW = LPR / 64;
  slot += threadIdx.x / LPR * NW;
  if ((threadIdx.x & 63) == 0) slot[(threadIdx.x >> 6) % NW] = v;
  __syncthreads();
  v = slot[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v = Op::of(v, slot[w]);
  return v;
}

template <int LPR>
__device__ __forceinline__ float sum_row(float v, uint32_t* slot) {
  return __uint_as_float(reduce_row<AddF, LPR>(__float_as_uint(v), slot));
}
// of the bits of magnitudes: an infinity ranks above every number, a NaN above it
template <int LPR>
__device__ __forceinline__ uint32_t max_row(uint32_t v, uint32_t* slot) {
  return reduce_row<MaxU, LPR>(v, slot);
}

// ---------------------------------------------------------------------------
// 8-bit rows: q = rne(127 x / top), scale = top / 127, top the row's largest
// magnitude.  The quotient is the correctly rounded one, so that it ties exactly where
// 127 x / top does: 127 / top is held in two parts, hi + lo, and fma(x, hi, x lo) rounds
// their sum once (for bf16 the quotient is never nearer to a tie than 2^-17 of itself
// without being one).  Stored fp32 (F32) takes the quotient of the rounded 127 x, which is
// the definition computed in fp32; 2^-e, e top's exponent, keeps it in range.  Adding 1.5 2^23
// rounds to the nearest even whole number and leaves it in the low byte.
// ---------------------------------------------------------------------------
constexpr uint32_t kTopMin = 0x04800000u;  // 2^-118: a row below it counts as zero

template <bool F32>
struct RowQ8 {
  float c, hi, lo, scale;
  uint32_t keep;  // 0: the row is not finite, and all its values are 0
  __device__ __forceinline__ explicit RowQ8(uint32_t top) {
    const bool zero = top < kTopMin, bad = top >= 0x7f800000u;  // an infinity or a NaN in the row
    const uint32_t t = zero || bad ? 0x3f800000u : top;
    const float f = __uint_as_float(t);
    const float a = __uint_as_float((t & 0x7fffffu) | 0x3f800000u);  // f 2^-e, in [1, 2)
    const float r = __builtin_amdgcn_rcpf(a);
    const float inv = fmaf(fmaf(-a, r, 1.f), r, r);
    // 127 2^-e; 0 brings every value to 0
    c = zero || bad ? 0.f : __uint_as_float(((133u + 127u - (t >> 23)) << 23) | 0x7e0000u);
    if (F32) {  // the reciprocal of a in two parts
      hi = inv;
      lo = fmaf(-inv, a, 1.f) * inv;
    } else {
      hi = c * inv;
      lo = zero || bad ? 0.f : fmaf(-hi, f, 127.f) * inv * (c * (1.f / 127.f));
    }
    const float s = f * (1.f / 127.f);
    scale = zero ? 0.f : bad ? __uint_as_float(0x7fc00000u)
                             : fmaf(fmaf(-127.f, s, f), 1.f / 127.f, s);
    keep = bad ? 0 : ~0u;
  }
  // the quotient's whole number in the low byte
  __device__ __forceinline__ uint32_t bits(float x) const {
    const float t = F32 ? x * c : x;
    return __float_as_uint(fmaf(t, hi, t * lo) + 12582912.f);
  }
  __device__ __forceinline__ int8_t one(float x) const { return (int8_t)(bits(x) & keep); }
  __device__ __forceinline__ uint32_t pack4(const float* f) const {
    const uint32_t lo4 = __builtin_amdgcn_perm(bits(f[1]), bits(f[0]), 0x0c0c0400u);
    const uint32_t hi4 = __builtin_amdgcn_perm(bits(f[3]), bits(f[2]), 0x04000c0cu);
    return (lo4 | hi4) & keep;
  }
};

typedef uint32_t u32_any __attribute__((aligned(1), may_alias));
typedef uint32_t u32x2_any1 __attribute__((ext_vector_type(2), aligned(1), may_alias));

// E values of a chunk to 8 bits at any place
template <int E, class Q>
__device__ __forceinline__ void store_q8(int8_t* p, const Q& q, const float* f) {
  if (E == 8) *reinterpret_cast<u32x2_any1*>(p) = u32x2_any1{q.pack4(f), q.pack4(f + 4)};
  else *reinterpret_cast<u32_any*>(p) = q.pack4(f);
}

}  // namespace gl
