// The cross-entropy of logits and classes with its gradient (MiniTensor Sec. 3.3
// Eq. (8)), gfx950. For a row z of V logits and its class t:
//
//   lse = log sum_v exp z_v,   loss = mean over the counted rows of lse - z_t,
//   dz_v = (exp(z_v - lse) - [v = t]) / n        n: how many rows count
//
// A row whose class is not one of 0 .. V-1 does not count: its loss and gradient
// are 0, and it is not read.
//
// Bound: HBM. A row is read once, held in registers by a block (or, where it is
// short, by some lanes of a wave) through its maximum, its sum and the gradient;
// exponentials stay in the logits' registers. Rows longer than a block's registers
// are read twice.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "language.hpp"

namespace mt {
namespace xent {

using namespace vio;

constexpr float kLog2E = 1.4426950408889634f, kLog2ELow = 1.9259629911266175e-8f, kLn2 = 0.6931471805599453f;

// e^d for d <= 0: d log2(e) in two parts, so that its rounding does not grow with |d|.
__device__ __forceinline__ float exp_of(float d) {
  const float t = d * kLog2E;
  const float e = __builtin_amdgcn_exp2f(t);
  const float low = fmaf(d, kLog2ELow, fmaf(d, kLog2E, -t));
  return d < -126.f ? e : fmaf(e, low * kLn2, e);  // past it e is 0 or tiny, and -inf - -inf none
}

// The maximum and the sum of a block's values, the same in every thread; two
// buffers, so that the barrier of one covers the other's next use.
__device__ __forceinline__ float block_max(float v, float* red) {
  v = lanes_max(v, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = red[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) m = fmaxf(m, red[w]);
  return m;
}
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = lanes_sum(v, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += red[w];
  return s;
}

template <bool BF>
__device__ __forceinline__ const char* row_at(const void* p, int64_t m, int64_t ld) {
  return (const char*)p + m * ld * (BF ? 2 : 4);
}

// The gradient of a row that does not count.
template <bool YB, int VEC>
__device__ __forceinline__ void clear(void* dr, int step, int V) {
  const float zero[VEC] = {};
  if (dr)
    for (int e0 = (int)threadIdx.x * VEC; e0 < V; e0 += step) store_some<YB, VEC>(dr, e0, V - e0, zero);
}

// A block a row, NV groups of VEC values a thread.
template <bool XB, bool YB, int VEC, int NV>
__global__ __launch_bounds__(1024) void row_kernel(const CrossEntropyParams p) {
  __shared__ float red[2][16];
  const int step = (int)blockDim.x * VEC;
  for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x) {
    const int32_t t = p.targets[m];
    const char* zr = row_at<XB>(p.z, m, p.ldz);
    char* dr = p.dz ? (char*)row_at<YB>(p.dz, m, p.ldd) : nullptr;
    if ((uint32_t)t >= (uint32_t)p.V) {
      if (threadIdx.x == 0) p.row_loss[m] = 0.f;
      clear<YB, VEC>(dr, step, p.V);
      continue;
    }
    float z[NV][VEC], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e0 = k * step + (int)threadIdx.x * VEC;
      load_some<XB, VEC>(zr, e0, p.V - e0, -INFINITY, z[k]);
    }
    const float zt = load_one<XB>(zr, t);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) top = fmaxf(top, z[k][e]);
    top = block_max(top, red[0]);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        z[k][e] = exp_of(z[k][e] - top);
        sum += z[k][e];
      }
    sum = block_sum(sum, red[1]);
    if (threadIdx.x == 0) p.row_loss[m] = (top - zt) + logf(sum);
    if (!dr) continue;
    const float inv_n = 1.f / (float)*p.counted, c = inv_n / sum;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int e0 = k * step + (int)threadIdx.x * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[k][e] = e0 + e == t ? fmaf(z[k][e], c, -inv_n) : z[k][e] * c;
      store_some<YB, VEC>(dr, e0, p.V - e0, z[k]);
    }
  }
}

// A block a row of any length, read twice: the maximum and the sum together,
// raised where a thread meets a larger value.
template <bool XB, bool YB, int VEC>
__global__ __launch_bounds__(1024) void long_kernel(const CrossEntropyParams p) {
  __shared__ float red[2][16];
  const int step = (int)blockDim.x * VEC;
  for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x) {
    const int32_t t = p.targets[m];
    const char* zr = row_at<XB>(p.z, m, p.ldz);
    char* dr = p.dz ? (char*)row_at<YB>(p.dz, m, p.ldd) : nullptr;
    if ((uint32_t)t >= (uint32_t)p.V) {
      if (threadIdx.x == 0) p.row_loss[m] = 0.f;
      clear<YB, VEC>(dr, step, p.V);
      continue;
    }
    float top = -INFINITY, sum = 0.f;
    const float zt = load_one<XB>(zr, t);
    for (int e0 = (int)threadIdx.x * VEC; e0 < p.V; e0 += step) {
      float z[VEC];
      load_some<XB, VEC>(zr, e0, p.V - e0, -INFINITY, z);
      float most = top;
#pragma unroll
      for (int e = 0; e < VEC; ++e) most = fmaxf(most, z[e]);
      if (most > top) {
        sum *= exp_of(top - most);
        top = most;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum += z[e] == -INFINITY ? 0.f : exp_of(z[e] - top);
    }
    const float mine = top;
    top = block_max(top, red[0]);
    // a thread that met nothing but -inf adds nothing, unless it met a NaN or all did
    if (mine > -INFINITY || top == -INFINITY) sum *= exp_of(mine - top);
    sum = block_sum(sum, red[1]);
    if (threadIdx.x == 0) p.row_loss[m] = (top - zt) + logf(sum);
    if (!dr) continue;
    const float inv_n = 1.f / (float)*p.counted, c = inv_n / sum;
    for (int e0 = (int)threadIdx.x * VEC; e0 < p.V; e0 += step) {
      float z[VEC];
      load_some<XB, VEC>(zr, e0, p.V - e0, -INFINITY, z);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        z[e] = exp_of(z[e] - top);
        z[e] = e0 + e == t ? fmaf(z[e], c, -inv_n) : z[e] * c;
      }
      store_some<YB, VEC>(dr, e0, p.V - e0, z);
    }
  }
}

// L lanes a row, NV values a lane, one after another: short rows.
template <bool XB, bool YB, int NV>
__global__ __launch_bounds__(256) void lanes_kernel(const CrossEntropyParams p, int L, int L_shift) {
  const int l = threadIdx.x & (L - 1);
  const int64_t rows = 256 >> L_shift;
  // a row's lanes stay together
  for (int64_t m = (int64_t)blockIdx.x * rows + (threadIdx.x >> L_shift); m < p.M; m += gridDim.x * rows) {
    const int32_t t = p.targets[m];
    const bool counts = (uint32_t)t < (uint32_t)p.V;
    const char* zr = row_at<XB>(p.z, m, p.ldz);
    float z[NV], top = -INFINITY, sum = 0.f, zt = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = l + (k << L_shift);
      z[k] = counts && v < p.V ? load_one<XB>(zr, v) : -INFINITY;
    }
    if (counts) zt = load_one<XB>(zr, t);
#pragma unroll
    for (int k = 0; k < NV; ++k) top = fmaxf(top, z[k]);
    top = lanes_max(top, L);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      z[k] = exp_of(z[k] - top);
      sum += z[k];
    }
    sum = lanes_sum(sum, L);
    if (l == 0) p.row_loss[m] = counts ? (top - zt) + logf(sum) : 0.f;
    if (!p.dz) continue;
    const float inv_n = counts ? 1.f / (float)*p.counted : 0.f, c = inv_n / sum;
    char* dr = (char*)row_at<YB>(p.dz, m, p.ldd);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = l + (k << L_shift);
      if (v < p.V) store_one<YB>(dr, v, !counts ? 0.f : v == t ? fmaf(z[k], c, -inv_n) : z[k] * c);
    }
  }
}

__global__ __launch_bounds__(1024) void count_kernel(const Index targets, int64_t M, int64_t V, int32_t* counted) {
  __shared__ int32_t red[16];
  int n = 0;
#pragma unroll 8
  for (int64_t m = threadIdx.x; m < M; m += 1024) n += (uint32_t)targets[m] < (uint64_t)V;
  for (int o = 32; o; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x) return;
  n = 0;
  for (int w = 0; w < 16; ++w) n += red[w];
  *counted = n;
}

// loss = sum of the rows' in a fixed order / n; 0 where no row counts
__global__ __launch_bounds__(1024) void mean_kernel(const float* row_loss, int64_t M, const int32_t* counted, float* loss) {
  __shared__ float red[16];
  float s = 0.f;
#pragma unroll 8
  for (int64_t m = threadIdx.x; m < M; m += 1024) s += row_loss[m];
  s = block_sum(s, red);
  const int n = *counted;
  if (threadIdx.x == 0) *loss = n > 0 ? s / (float)n : 0.f;
}

constexpr int64_t kMostBlocks = 1 << 20;  // a launch has fewer than 2^32 threads

template <bool XB, bool YB>
hipError_t rows(const CrossEntropyParams& p, const CrossEntropyForm& f, hipStream_t stream) {
  constexpr int VEC = XB ? 8 : 4;  // of the logits alone: a row's loss does not depend on what else is asked for
  if (f.L) {
    const int64_t per = 256 >> f.L_shift;
    lanes_kernel<XB, YB, 8><<<dim3((unsigned)std::min((p.M + per - 1) / per, kMostBlocks)), 256, 0, stream>>>(p, f.L, f.L_shift);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)std::min(p.M, kMostBlocks));
  if (f.values == 0) long_kernel<XB, YB, VEC><<<grid, f.threads, 0, stream>>>(p);
  else if (f.values <= 16) row_kernel<XB, YB, VEC, 16 / VEC><<<grid, f.threads, 0, stream>>>(p);
  else if (f.values <= 32) row_kernel<XB, YB, VEC, 32 / VEC><<<grid, f.threads, 0, stream>>>(p);
  else row_kernel<XB, YB, VEC, 64 / VEC><<<grid, f.threads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace xent

hipError_t cross_entropy_count(const vio::Index& targets, int64_t M, int64_t V, int32_t* counted, hipStream_t stream) {
  xent::count_kernel<<<1, 1024, 0, stream>>>(targets, M, V, counted);
  return hipGetLastError();
}

hipError_t cross_entropy_rows(const CrossEntropyParams& p, const CrossEntropyForm& f, bool z_bf16, bool d_bf16,
                              hipStream_t stream) {
  if (z_bf16) return d_bf16 ? xent::rows<true, true>(p, f, stream) : xent::rows<true, false>(p, f, stream);
  return d_bf16 ? xent::rows<false, true>(p, f, stream) : xent::rows<false, false>(p, f, stream);
}

hipError_t cross_entropy_mean(const float* row_loss, int64_t M, const int32_t* counted, float* loss, hipStream_t stream) {
  xent::mean_kernel<<<1, 1024, 0, stream>>>(row_loss, M, counted, loss);
  return hipGetLastError();
}

}  // namespace mt
