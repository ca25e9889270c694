// Values of fp32 or bf16 rows in registers, 4 or 8 at a time by 16-byte accesses,
// and sums over the lanes of a wave. Device code.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace mt::vio {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float low_bf16(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float high_bf16(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
// two values rounded to nearest even
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  bf16x2 t;
  t[0] = (__bf16)a;
  t[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, t);
}

// Wide accesses at any element's address: the hardware takes them, so that odd
// widths and pitches run by the same kernels as aligned ones.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// The VEC (4 or 8) values from element i on.
template <bool BF, int VEC>
__device__ __forceinline__ void load(const void* p, int64_t i, float (&v)[VEC]) {
  if constexpr (BF && VEC == 4) {
    const u32x2 u = *(const u32x2_any*)((const unsigned short*)p + i);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      v[2 * e] = low_bf16(u[e]);
      v[2 * e + 1] = high_bf16(u[e]);
    }
  } else if constexpr (BF) {
    static_assert(VEC == 8);
    const u32x4 u = *(const u32x4_any*)((const unsigned short*)p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = low_bf16(u[e]);
      v[2 * e + 1] = high_bf16(u[e]);
    }
  } else {
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q) {
      const f32x4 t = *(const f32x4_any*)((const float*)p + i + 4 * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = t[e];
    }
  }
}
template <bool BF, int VEC>
__device__ __forceinline__ void store(void* p, int64_t i, const float (&v)[VEC]) {
  if constexpr (BF && VEC == 4) {
    *(u32x2_any*)((unsigned short*)p + i) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
  } else if constexpr (BF) {
    static_assert(VEC == 8);
    *(u32x4_any*)((unsigned short*)p + i) = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
  } else {
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q)
      *(f32x4_any*)((float*)p + i + 4 * q) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
  }
}

template <bool BF>
__device__ __forceinline__ float load_one(const void* p, int64_t i) {
  if constexpr (BF) return __uint_as_float((uint32_t)((const unsigned short*)p)[i] << 16);
  else return ((const float*)p)[i];
}
template <bool BF>
__device__ __forceinline__ void store_one(void* p, int64_t i, float v) {
  if constexpr (BF) ((__bf16*)p)[i] = (__bf16)v;
  else ((float*)p)[i] = v;
}

// The same where only the first n values exist (a row's end); n <= 0: none.
// Values that do not exist are `fill`.
template <bool BF, int VEC>
__device__ __forceinline__ void load_some(const void* p, int64_t i, int n, float fill, float (&v)[VEC]) {
  if (n >= VEC) {
    load<BF, VEC>(p, i, v);
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = e < n ? load_one<BF>(p, i + e) : fill;
  }
}
template <bool BF, int VEC>
__device__ __forceinline__ void store_some(void* p, int64_t i, int n, const float (&v)[VEC]) {
  if (n >= VEC) {
    store<BF, VEC>(p, i, v);
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (e < n) store_one<BF>(p, i + e, v[e]);
  }
}

// The value of a lane's partner, by the vector instructions' own lane paths
// (__shfl goes through LDS): lanes 1 and 2 apart, then the mirrored one of 8 and of
// 16, which holds the same as the one 4 and 8 apart once the smaller groups agree.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Every lane of L (a power of two up to 64) consecutive ones gets their reduction.
template <typename Op>
__device__ __forceinline__ float lanes_reduce(float v, int L, Op op) {
  if (L > 1) v = op(v, dpp<0xb1>(v));   // quad_perm 1 0 3 2
  if (L > 2) v = op(v, dpp<0x4e>(v));   // quad_perm 2 3 0 1
  if (L > 4) v = op(v, dpp<0x141>(v));  // row_half_mirror
  if (L > 8) v = op(v, dpp<0x140>(v));  // row_mirror
  if (L > 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  if (L > 32) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  return v;
}
__device__ __forceinline__ float lanes_sum(float v, int L) {
  return lanes_reduce(v, L, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float lanes_max(float v, int L) {
  return lanes_reduce(v, L, [](float a, float b) { return fmaxf(a, b); });
}

// A view of int32 values (tokens, classes), row-major index m of [m / inner, m % inner].
struct Index {
  const int32_t* p;
  int64_t inner, s0, s1;  // inner 0: one after another
  __device__ __forceinline__ int32_t operator[](int64_t m) const {
    if (inner == 0) return p[m];
    const uint32_t r = (uint32_t)m / (uint32_t)inner;
    return p[r * s0 + ((uint32_t)m - r * (uint32_t)inner) * s1];
  }
};

}  // namespace mt::vio
