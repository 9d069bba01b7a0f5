// Device code that the operators' kernels share: bf16, 16-byte vectors of a type at
// an element's alignment, reductions over a wave.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace un {

typedef uint16_t bf16_t;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// vectors at an element's alignment (rows of any stride): gfx950 takes such
// global accesses as they are
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef u32x2 u32x2_a1 __attribute__((aligned(1)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
typedef uint32_t u32_a1 __attribute__((aligned(1)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));

namespace {

__device__ __forceinline__ float bf2f(uint32_t h) { return __uint_as_float(h << 16); }
__device__ __forceinline__ uint32_t f2bf(float f) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t f2bf2(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}

// A 16-byte vector of T as floats and back.
template <typename T> struct V16;
template <> struct V16<float> {
  static constexpr int N = 4;
  __device__ static void unpack(u32x4 v, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = __uint_as_float(v[e]);
  }
  __device__ static u32x4 pack(const float* f) {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(f[e]);
    return v;
  }
  __device__ static float load1(const float* p) { return *p; }
  __device__ static void store1(float* p, float f) { *p = f; }
};
template <> struct V16<bf16_t> {
  static constexpr int N = 8;
  __device__ static void unpack(u32x4 v, float* f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(v[e] << 16);
      f[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
    }
  }
  __device__ static u32x4 pack(const float* f) {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = f2bf2(f[2 * e], f[2 * e + 1]);
    return v;
  }
  __device__ static float load1(const bf16_t* p) { return bf2f(*p); }
  __device__ static void store1(bf16_t* p, float f) { *p = (bf16_t)f2bf(f); }
};

// n (0 .. N) values to p
template <typename T> __device__ __forceinline__ void store_vec(T* p, int n, const float* f) {
  constexpr int N = V16<T>::N;
  if (n == N) {
    *(u32x4_a2*)p = V16<T>::pack(f);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) V16<T>::store1(p + e, f[e]);
  }
}
// n (0 .. N) values at p; the rest are zeros
template <int N> __device__ __forceinline__ void load_f32(const float* p, int n, float* f) {
  if (n == N) {
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      const f32x4 v = ((const f32x4_a4*)p)[q];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[4 * q + e] = v[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = e < n ? p[e] : 0.f;
  }
}

// Reductions over the 16 lanes of a DPP row (quad swaps, then the halves of a
// row mirrored), whose result every lane of the row has, and over a wave (the
// four rows' values read to scalars, in order). No LDS traffic.
template <typename F> __device__ __forceinline__ float row16(float v, F&& op) {
  auto dpp = [](float x, auto ctrl) {
    const int i = __float_as_int(x);
    return __int_as_float(__builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, 0xf, 0xf, false));
  };
  v = op(v, dpp(v, std::integral_constant<int, 0xB1>{}));   // quad_perm [1, 0, 3, 2]
  v = op(v, dpp(v, std::integral_constant<int, 0x4E>{}));   // quad_perm [2, 3, 0, 1]
  v = op(v, dpp(v, std::integral_constant<int, 0x141>{}));  // row_half_mirror
  v = op(v, dpp(v, std::integral_constant<int, 0x140>{}));  // row_mirror
  return v;
}
template <typename F> __device__ __forceinline__ float wave64(float v, F&& op) {
  v = row16(v, op);
  auto lane = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return op(op(lane(0), lane(16)), op(lane(32), lane(48)));
}
struct Add {
  __device__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
  __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
__device__ __forceinline__ float wave_max(float v) { return wave64(v, Max{}); }

template <int N> using Int = std::integral_constant<int, N>;
constexpr int64_t LAST_LEVEL = (int64_t)256 << 20;  // bytes of the cache that all XCDs share

}  // namespace
}  // namespace un
