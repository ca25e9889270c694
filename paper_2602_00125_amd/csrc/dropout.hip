// Dropout with the residual sum, and its gradient, gfx950:
//
//   y = residual + x keep / (1 - p)        dx = dy keep / (1 - p)
//
// The mask is never stored: whether an element stays is a function of (seed,
// offset, its row-major index), computed again by the backward. The generator
// is Philox4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel
// random numbers: as easy as 1, 2, 3", SC 2011), key = seed, counter = offset
// + index / 8; element i takes the 16 bits i % 8 of the four words (low half
// first) and is dropped where they are below round(65536 p). One counter
// serves eight elements: two multiplications of a round are the cost (a 64-bit
// product each), and 32 bits an element would make the kernel bound by them
// rather than by HBM. The scale is one over the probability in use, so that
// the mean is kept whatever p rounds to.
//
// Bound: HBM (8192 x 8192 fp32 with a residual, 0.81 GB: 134 us = 6.0 TB/s, where a
// large copy reaches 4.8). A thread takes eight consecutive elements, so a tensor
// without gaps is one flat array whatever its width; rows with a pitch go by
// vectors where the width is a multiple of eight, by element elsewhere. Small
// tensors cost the launch (509 x 383 bf16: 2.5 us of kernel, 5 a call).
#include <hip/hip_runtime.h>

#include "kernels.hpp"

namespace mt {
namespace dropout {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The four words of counter c under key k.
__device__ __forceinline__ u32x4 philox(uint64_t c, uint64_t k) {
  uint32_t x0 = (uint32_t)c, x1 = (uint32_t)(c >> 32), x2 = 0, x3 = 0;
  uint32_t k0 = (uint32_t)k, k1 = (uint32_t)(k >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
    x0 = (uint32_t)(b >> 32) ^ x1 ^ k0;
    x1 = (uint32_t)b;
    x2 = (uint32_t)(a >> 32) ^ x3 ^ k1;
    x3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return u32x4{x0, x1, x2, x3};
}
// the 16 bits of element e of eight
__device__ __forceinline__ uint32_t draw_of(const u32x4& w, int e) { return e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu; }

template <bool BF>
__device__ __forceinline__ void load8(const void* p, int64_t i, float (&v)[8]) {
  if constexpr (BF) {
    const u32x4 u = *(const u32x4*)((const unsigned short*)p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(u[e] << 16);
      v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
  } else {
    const f32x4 a = *(const f32x4*)((const float*)p + i), b = *(const f32x4*)((const float*)p + i + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = a[e];
      v[4 + e] = b[e];
    }
  }
}
template <bool BF>
__device__ __forceinline__ void store8(void* p, int64_t i, const float (&v)[8]) {
  if constexpr (BF) {
    u32x4 u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bf16x2 t;
      t[0] = (__bf16)v[2 * e];
      t[1] = (__bf16)v[2 * e + 1];
      u[e] = __builtin_bit_cast(uint32_t, t);
    }
    *(u32x4*)((unsigned short*)p + i) = u;
  } else {
    *(f32x4*)((float*)p + i) = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)((float*)p + i + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
}
template <bool BF>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
  if constexpr (BF) return __uint_as_float((unsigned)((const unsigned short*)p)[i] << 16);
  else return ((const float*)p)[i];
}
template <bool BF>
__device__ __forceinline__ void store1(void* p, int64_t i, float v) {
  if constexpr (BF) ((__bf16*)p)[i] = (__bf16)v;
  else ((float*)p)[i] = v;
}

// A dropped element is x's zero whatever x holds (an infinity or NaN too).
__device__ __forceinline__ float one(float x, uint32_t draw, const DropoutParams& p) {
  return draw >= p.drop ? x * p.scale : 0.f;
}

// vec: N is a multiple of 8 and every pitch and base allows 16-byte accesses
// (or the tensors are flat: M = 1, any N, the last few elements one by one).
template <bool XB, bool YB, bool RES, bool VEC>
__global__ __launch_bounds__(256) void kernel(const DropoutParams p) {
  const int64_t total = p.M * p.N, groups = (total + 7) >> 3;
  for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < groups; g += (int64_t)gridDim.x * 256) {
    int64_t m = 0, n = 8 * g;
    if (p.M > 1) {
      m = n / p.N;
      n -= m * p.N;
    }
    const u32x4 w = philox(p.offset + (uint64_t)g, p.seed);
    if (VEC && n + 8 <= p.N) {
      float x[8], r[8];
      load8<XB>(p.x, m * p.ldx + n, x);
      if constexpr (RES) load8<YB>(p.res, m * p.ldr + n, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = one(x[e], draw_of(w, e), p);
        if constexpr (RES) x[e] += r[e];
      }
      store8<YB>(p.y, m * p.ldy + n, x);
    } else {
      const int left = total - 8 * g < 8 ? (int)(total - 8 * g) : 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e >= left) break;
        float v = one(load1<XB>(p.x, m * p.ldx + n), draw_of(w, e), p);
        if constexpr (RES) v += load1<YB>(p.res, m * p.ldr + n);
        store1<YB>(p.y, m * p.ldy + n, v);
        if (++n == p.N) {
          n = 0;
          ++m;
        }
      }
    }
  }
}

template <bool XB, bool YB, bool RES>
hipError_t launch(const DropoutParams& p, bool vec, hipStream_t stream) {
  const int64_t groups = (p.M * p.N + 7) / 8, blocks = (groups + 255) / 256;
  const dim3 grid((unsigned)(blocks < (1 << 23) ? blocks : 1 << 23));  // a launch has fewer than 2^32 threads
  if (vec) kernel<XB, YB, RES, true><<<grid, 256, 0, stream>>>(p);
  else kernel<XB, YB, RES, false><<<grid, 256, 0, stream>>>(p);
  return hipGetLastError();
}
template <bool XB, bool YB>
hipError_t launch(const DropoutParams& p, bool vec, hipStream_t stream) {
  return p.res ? launch<XB, YB, true>(p, vec, stream) : launch<XB, YB, false>(p, vec, stream);
}

}  // namespace dropout

hipError_t dropout_run(const DropoutParams& p, bool x_bf16, bool y_bf16, bool vec, hipStream_t stream) {
  if (x_bf16) return y_bf16 ? dropout::launch<true, true>(p, vec, stream) : dropout::launch<true, false>(p, vec, stream);
  return y_bf16 ? dropout::launch<false, true>(p, vec, stream) : dropout::launch<false, false>(p, vec, stream);
}

}  // namespace mt
