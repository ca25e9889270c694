// The cross-entropy of logits and classes with its gradient (MiniTensor Sec. 3.3
// Eq. (8)), gfx950. For a row z of V logits and its class t:
//
//   lse = log sum_v exp z_v,   loss = mean over the counted rows of lse - z_t,
//   dz_v = (exp(z_v - lse) - [v = t]) / n        n: how many rows count
//
// A row whose class is not one of 0 .. V-1 does not count: its loss and gradient
// are 0, and it is not read.
//
// Bound: HBM. Rows of up to 1024 logits are held by up to 64 lanes, several rows a
// wave (134217 x 1000 fp32 228 us, 4.7 TB/s; by blocks of 256 threads 437). Longer
// ones have a block each, whose threads hold 16 or 32 values through the row's
// maximum, its sum and the gradient, exponentials in the logits' registers. Of rows
// longer than that a thread keeps a running maximum and sum and reads them again,
// from the caches: 8192 x 50001 fp32 to bf16, a fifth of it padding, 460 us, 4.64
// TB/s of what has to move. Holding nothing took 500 us, 16 values 488, 64 (too many
// registers for two blocks a CU) 563, and rows held whole by 1024 threads 811: one
// block a CU, whose loads, arithmetic and stores took turns.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "language.hpp"

namespace mt {
namespace xent {

using namespace vio;

constexpr float kLog2E = 1.4426950408889634f, kLog2ELow = 1.9259629911266175e-8f, kLn2 = 0.6931471805599453f;

// e^d for d <= 0, the difference of two logits. fp32 logits' are rounded by up to
// 2^-24 |d|, which the product with log2(e) would double: its rest is added back.
// bf16 logits' are exact, or nearly so, and the product's rounding may stay.
template <bool XB>
__device__ __forceinline__ float exp_of(float d) {
  const float t = d * kLog2E;
  const float e = __builtin_amdgcn_exp2f(t);
  if constexpr (XB) return e;
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
// of the rows' losses, in 64 bits: one number that a program follows for long
__device__ __forceinline__ double block_sum64(double v, double* red) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += red[w];
  return s;
}

__device__ __forceinline__ int block_count(int n, int* red) {
  for (int o = 32; o; o >>= 1) n += __shfl_xor(n, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) n += red[w];
  return n;
}

// How many rows count: a launch of its own has written it, or, of few rows, every
// block counts them (128 x 2624 9.8 -> 7.5 us, 1000 x 500 9.3 -> 8.1; of 2000 x
// 1100 bf16 it costs more than the launch, 11 -> 14).
__device__ __forceinline__ int counted(const CrossEntropyParams& p, int* red) {
  if (p.counted) return *p.counted;
  int n = 0;
  for (int m = threadIdx.x; m < (int)p.M; m += blockDim.x) n += (uint32_t)p.targets[m] < (uint32_t)p.V;
  return block_count(n, red);
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

// dz = e c, and one less 1 / n at the class (of n values from e0 on).
template <bool YB, int VEC>
__device__ __forceinline__ void put(void* dr, int e0, int n, int32_t t, float c, float inv_n, float (&e)[VEC]) {
  if ((uint32_t)(t - e0) < (uint32_t)VEC) {  // one group of the row
#pragma unroll
    for (int i = 0; i < VEC; ++i) e[i] = e0 + i == t ? fmaf(e[i], c, -inv_n) : e[i] * c;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) e[i] *= c;
  }
  store_some<YB, VEC>(dr, e0, n, e);
}

// A block a row. A thread holds the first NV groups of VEC values it meets; of
// the rest (REST: the held part is whole) it keeps the maximum and the sum so
// far, raised together, and reads them again for the gradient, 16 values at a
// time, from the caches. Sixteens are added in 64 bits: a thread meets 16384 values
// of a row of 2^24, and a sum in fp32 was off by 2e-4 of like ones.
template <bool XB, bool YB, int VEC, int NV, bool REST>
__global__ __launch_bounds__(REST ? 1024 : 512, REST ? 4 : 6) void row_kernel(const CrossEntropyParams p) {
  __shared__ float red[2][16];
  __shared__ int counts[16];
  const int step = (int)blockDim.x * VEC, first = (int)threadIdx.x * VEC;
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
    for (int k = 0; k < NV; ++k)
      load_some<XB, VEC>(zr, first + k * step, REST ? VEC : p.V - first - k * step, -INFINITY, z[k]);
    const float zt = load_one<XB>(zr, t);
    const int n = dr ? counted(p, counts) : 1;
    constexpr int U = 16 / VEC;  // groups of the rest in flight
    double sum_rest = 0.0;
    if constexpr (REST) {
      for (int e0 = first + NV * step; e0 < p.V; e0 += U * step) {
        float v[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) load_some<XB, VEC>(zr, e0 + u * step, p.V - e0 - u * step, -INFINITY, v[u]);
        float most = top;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < VEC; ++e) most = fmaxf(most, v[u][e]);
        if (most > top) {
          sum_rest *= exp_of<XB>(top - most);
          top = most;
        }
        const float from = top == -INFINITY ? 0.f : top;  // nothing but -inf so far adds nothing
        float some = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < VEC; ++e) some += exp_of<XB>(v[u][e] - from);
        sum_rest += some;
      }
    }
    const float rest = top;  // of the rest
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) top = fmaxf(top, z[k][e]);
    top = block_max(top, red[0]);
    // a rest of nothing but -inf adds nothing, unless there was a NaN
    if constexpr (REST) sum = (float)(rest > -INFINITY ? sum_rest * exp_of<XB>(rest - top) : sum_rest);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        z[k][e] = exp_of<XB>(z[k][e] - top);
        sum += z[k][e];
      }
    sum = block_sum(sum, red[1]);
    if (threadIdx.x == 0) p.row_loss[m] = (top - zt) + logf(sum);
    if (!dr) continue;
    const float inv_n = 1.f / (float)n, c = inv_n / sum;
#pragma unroll
    for (int k = 0; k < NV; ++k) put<YB, VEC>(dr, first + k * step, REST ? VEC : p.V - first - k * step, t, c, inv_n, z[k]);
    if constexpr (REST) {
      for (int e0 = first + NV * step; e0 < p.V; e0 += U * step) {
        float v[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) load_some<XB, VEC>(zr, e0 + u * step, p.V - e0 - u * step, -INFINITY, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[u][e] = exp_of<XB>(v[u][e] - top);
          put<YB, VEC>(dr, e0 + u * step, p.V - e0 - u * step, t, c, inv_n, v[u]);
        }
      }
    }
  }
}

// A row by L lanes of a wave, l each one's place: up to 16 values a lane. The
// row's loss, in every lane.
template <bool XB, bool YB, int VEC>
__device__ __forceinline__ float lanes_row(const CrossEntropyParams& p, int64_t m, int l, int L, int n) {
  constexpr int NV = 16 / VEC;
  const int32_t t = p.targets[m];
  const bool counts = (uint32_t)t < (uint32_t)p.V;
  const char* zr = row_at<XB>(p.z, m, p.ldz);
  float z[NV][VEC], top = -INFINITY, sum = 0.f, zt = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int e0 = (l + k * L) * VEC;
    load_some<XB, VEC>(zr, e0, counts ? p.V - e0 : 0, -INFINITY, z[k]);
  }
  if (counts) zt = load_one<XB>(zr, t);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) top = fmaxf(top, z[k][e]);
  top = lanes_max(top, L);
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      z[k][e] = exp_of<XB>(z[k][e] - top);
      sum += z[k][e];
    }
  sum = lanes_sum(sum, L);
  const float loss = counts ? (top - zt) + logf(sum) : 0.f;
  if (l == 0) p.row_loss[m] = loss;
  if (!p.dz) return loss;
  char* dr = (char*)row_at<YB>(p.dz, m, p.ldd);
  const float inv_n = 1.f / (float)n, c = inv_n / sum;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int e0 = (l + k * L) * VEC;
    if (!counts)
#pragma unroll
      for (int e = 0; e < VEC; ++e) z[k][e] = 0.f;
    put<YB, VEC>(dr, e0, p.V - e0, counts ? t : -1, counts ? c : 0.f, inv_n, z[k]);
  }
  return loss;
}

// Short rows: 256 / L a block.
template <bool XB, bool YB, int VEC>
__global__ __launch_bounds__(256) void lanes_kernel(const CrossEntropyParams p, int L, int L_shift) {
  __shared__ int counts[16];
  const int64_t rows = 256 >> L_shift;
  const int n = p.dz ? counted(p, counts) : 1;
  // a row's lanes stay together
  for (int64_t m = (int64_t)blockIdx.x * rows + (threadIdx.x >> L_shift); m < p.M; m += gridDim.x * rows)
    lanes_row<XB, YB, VEC>(p, m, threadIdx.x & (L - 1), L, n);
}

// A few short rows: the count, the rows and the mean by one block, one launch.
template <bool XB, bool YB, int VEC>
__global__ __launch_bounds__(1024) void few_kernel(const CrossEntropyParams p, int L, int L_shift, float* loss) {
  __shared__ double red[16];
  __shared__ int counts[16];
  const int n = counted(p, counts);
  double sum = 0.0;
  for (int64_t m = threadIdx.x >> L_shift; m < p.M; m += 1024 >> L_shift) {
    const float one = lanes_row<XB, YB, VEC>(p, m, threadIdx.x & (L - 1), L, n);
    if ((threadIdx.x & (L - 1)) == 0) sum += one;
  }
  sum = block_sum64(sum, red);
  if (loss && threadIdx.x == 0) *loss = n > 0 ? (float)(sum / n) : 0.f;
}

// How many rows count; the mean of their losses, 0 where none does. Blocks take
// shares of the rows, and one adds their results in order.
__global__ __launch_bounds__(1024) void count_kernel(const Index targets, int64_t M, int64_t V, int32_t* out) {
  __shared__ int red[16];
  const int64_t share = (M + gridDim.x - 1) / gridDim.x, m0 = blockIdx.x * share, m1 = min(m0 + share, M);
  int n = 0;
#pragma unroll 8
  for (int64_t m = m0 + threadIdx.x; m < m1; m += 1024) n += (uint32_t)targets[m] < (uint64_t)V;
  n = block_count(n, red);
  if (threadIdx.x == 0) out[blockIdx.x] = n;
}
__global__ __launch_bounds__(kCrossEntropyParts) void add_counts_kernel(const int32_t* part, int parts, int32_t* counted) {
  __shared__ int red[16];
  const int n = block_count((int)threadIdx.x < parts ? part[threadIdx.x] : 0, red);
  if (threadIdx.x == 0) *counted = n;
}
// from: fp32 losses or 64-bit partial sums; to: those, or the mean
template <typename From, typename To>
__global__ __launch_bounds__(1024) void mean_kernel(const CrossEntropyParams p, const From* from, int64_t M, To* out) {
  __shared__ double red[16];
  __shared__ int counts[16];
  const int64_t share = (M + gridDim.x - 1) / gridDim.x, m0 = blockIdx.x * share, m1 = min(m0 + share, M);
  double s = 0.0;
#pragma unroll 8
  for (int64_t m = m0 + threadIdx.x; m < m1; m += 1024) s += from[m];
  s = block_sum64(s, red);
  if constexpr (sizeof(To) == 8) {
    if (threadIdx.x == 0) out[blockIdx.x] = s;
  } else {
    const int n = counted(p, counts);
    if (threadIdx.x == 0) *out = n > 0 ? (float)(s / n) : 0.f;
  }
}

constexpr int64_t kMostBlocks = 1 << 20;  // a launch has fewer than 2^32 threads

template <bool XB, bool YB>
hipError_t rows(const CrossEntropyParams& p, const CrossEntropyForm& f, float* loss, hipStream_t stream) {
  constexpr int VEC = XB ? 8 : 4;  // of the logits alone: a row's loss does not depend on what else is asked for
  if (f.few) {
    few_kernel<XB, YB, VEC><<<1, 1024, 0, stream>>>(p, f.L, f.L_shift, loss);
    return hipGetLastError();
  }
  if (f.L) {
    const int64_t per = 256 >> f.L_shift;
    lanes_kernel<XB, YB, VEC><<<dim3((unsigned)std::min((p.M + per - 1) / per, kMostBlocks)), 256, 0, stream>>>(p, f.L, f.L_shift);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)std::min(p.M, kMostBlocks));
  if (f.values <= 16) row_kernel<XB, YB, VEC, 16 / VEC, false><<<grid, f.threads, 0, stream>>>(p);
  else if (f.values <= 32) row_kernel<XB, YB, VEC, 32 / VEC, false><<<grid, f.threads, 0, stream>>>(p);
  else row_kernel<XB, YB, VEC, 32 / VEC, true><<<grid, f.threads, 0, stream>>>(p);
  return hipGetLastError();
}

int parts_of(int64_t M) { return (int)std::min<int64_t>(kCrossEntropyParts, (M + kCrossEntropyPartRows - 1) / kCrossEntropyPartRows); }

}  // namespace xent

hipError_t cross_entropy_count(const vio::Index& targets, int64_t M, int64_t V, int32_t* part, int32_t* counted,
                               hipStream_t stream) {
  const int parts = xent::parts_of(M);
  xent::count_kernel<<<dim3(parts > 1 ? parts : 1), 1024, 0, stream>>>(targets, M, V, parts > 1 ? part : counted);
  if (parts > 1) xent::add_counts_kernel<<<1, kCrossEntropyParts, 0, stream>>>(part, parts, counted);
  return hipGetLastError();
}

hipError_t cross_entropy_rows(const CrossEntropyParams& p, const CrossEntropyForm& f, bool z_bf16, bool d_bf16, float* loss,
                              hipStream_t stream) {
  if (z_bf16) return d_bf16 ? xent::rows<true, true>(p, f, loss, stream) : xent::rows<true, false>(p, f, loss, stream);
  return d_bf16 ? xent::rows<false, true>(p, f, loss, stream) : xent::rows<false, false>(p, f, loss, stream);
}

hipError_t cross_entropy_mean(const CrossEntropyParams& p, double* part, float* loss, hipStream_t stream) {
  const int parts = xent::parts_of(p.M);
  if (parts > 1) {
    xent::mean_kernel<<<dim3(parts), 1024, 0, stream>>>(p, (const float*)p.row_loss, p.M, part);
    xent::mean_kernel<<<1, 1024, 0, stream>>>(p, (const double*)part, (int64_t)parts, loss);
  } else {
    xent::mean_kernel<<<1, 1024, 0, stream>>>(p, (const float*)p.row_loss, p.M, loss);
  }
  return hipGetLastError();
}

}  // namespace mt
