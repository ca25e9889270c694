// The norm over the gradients of all parameters and their clipping, gfx950:
//
//   N = (sum over tensors of g^2)^(1/2),   out = g min(1, max_norm / N)
//
// Squares are formed and added in 64 bits: no finite gradient overflows or
// vanishes in them, and the sum of hundreds of millions of values keeps its
// digits. So is the factor, and a result is rounded once, to bf16 too. Bound: HBM
// (vector instructions 11% busy).
//
// Two launches for each 188 tensors, or 313 in place. norm_kernel: blocks take the
// chunks of the tensors in turn and write a partial sum each. scale_kernel: every
// block adds all partial sums in one order, so that all find the same factor, and
// takes the chunks again, the last first: those are in the caches. In place and
// with nothing to clip it ends there. 134 million fp32 values into others: 308 us
// (118 and 189), 5.2 TB/s of two readings and a writing; stores that pass the
// caches by took 302 there, but 477 for 466 at 201 million values.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "language.hpp"

namespace mt {
namespace clip {

using namespace vio;

// The tensor that chunk c belongs to; the same in every lane.
__device__ __forceinline__ int tensor_of(const ClipBatch& b, int c) {
  const int lane = threadIdx.x & 63;
  const uint32_t* starts = b.starts();
  int n = 0;
  for (int i = 0; i < b.n; i += 64) n += __popcll(__ballot(i + lane < b.n && starts[min(i + lane, b.n - 1)] <= (uint32_t)c));
  return __builtin_amdgcn_readfirstlane(n - 1);
}
typedef __attribute__((address_space(1))) void Global;  // an address that is not of LDS
__device__ __forceinline__ void* address(uint64_t w) { return (void*)(Global*)(w & 0xffffffffffffull); }
// Where it is, its kind, the chunk's first value and how many it has.
struct Chunk {
  void* src;
  int kind, n;
  int64_t first;
};
__device__ __forceinline__ Chunk chunk_of(const ClipBatch& b, int t, int c) {
  const uint64_t s = b.w[t];
  const uint32_t* starts = b.starts();
  const uint32_t next = t + 1 < b.n ? starts[t + 1] : (uint32_t)b.chunks;
  return Chunk{address(s), (int)(s >> 48) & 15, (uint32_t)c + 1 < next ? kClipChunk : (int)(s >> 52) + 1,
               (int64_t)((uint32_t)c - starts[t]) * kClipChunk};
}

// The 256 threads' values added by a fixed tree.
__device__ __forceinline__ double block_sum(double v, double* red) {
  red[threadIdx.x] = v;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
    __syncthreads();
  }
  return red[0];
}

// v cut off to fp32, the last bit set where that is not v: what is rounded to bf16
// from there is v itself (by way of the nearest fp32 value it would be rounded twice).
__device__ __forceinline__ float cut_odd(double v) {
  const float f = (float)v;
  const uint32_t u = __float_as_uint(f) - (fabs((double)f) > fabs(v));
  return __uint_as_float((double)f != v ? u | 1u : u);
}

constexpr int kPer = kClipChunk / 256;  // values a thread of a chunk

// f(i, n, values): the thread's values of a chunk by eights, the first n of which
// exist.
template <bool BF, typename F>
__device__ __forceinline__ void values(const Chunk& k, F f) {
  float v[kPer / 8][8];
  const int at = (int)threadIdx.x * 8;
#pragma unroll
  for (int j = 0; j < kPer / 8; ++j) load_some<BF, 8>(k.src, k.first + at + j * 2048, k.n - at - j * 2048, 0.f, v[j]);
#pragma unroll
  for (int j = 0; j < kPer / 8; ++j) f(k.first + at + j * 2048, k.n - at - j * 2048, v[j]);
}

__global__ __launch_bounds__(256) void norm_kernel(const ClipBatch b, double* part) {
  __shared__ double red[256];
  double sum = 0.0;
  auto add = [&](int64_t, int, const float (&v)[8]) {
    for (float x : v) sum = fma((double)x, (double)x, sum);
  };
  for (int c = blockIdx.x; c < b.chunks; c += gridDim.x) {
    const Chunk k = chunk_of(b, tensor_of(b, c), c);
    if (k.kind & kClipSourceBf16) values<true>(k, add);
    else values<false>(k, add);
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(256) void scale_kernel(const ClipBatch b, const double* part, int parts, double max_norm, float* out_norm) {
  __shared__ double red[256];
  double sum = 0.0;
  for (int i = threadIdx.x; i < parts; i += 256) sum += part[i];
  const double norm = sqrt(block_sum(sum, red));
  if (out_norm && blockIdx.x == 0 && threadIdx.x == 0) *out_norm = (float)norm;
  // a norm that is not finite, as the caller reads it, clips nothing
  const bool clips = norm > max_norm && (float)norm < INFINITY;
  if (!clips && b.in_place) return;
  const double f = clips ? max_norm / norm : 1.0;
  for (int c = b.chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const int t = tensor_of(b, c);
    const Chunk k = chunk_of(b, t, c);
    void* dst = b.in_place ? k.src : address(b.w[b.n + t]);
    auto put = [&](int64_t i, int n, float (&v)[8]) {
      if (k.kind & kClipDestBf16) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = cut_odd(v[e] * f);
        store_some<true, 8>(dst, i, n, v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)(v[e] * f);
        store_some<false, 8>(dst, i, n, v);
      }
    };
    if (k.kind & kClipSourceBf16) values<true>(k, put);
    else values<false>(k, put);
  }
}

}  // namespace clip

int clip_blocks(int64_t chunks) { return (int)std::min<int64_t>(chunks, 2048); }

hipError_t clip_norm(const ClipBatch& b, double* part, int blocks, hipStream_t stream) {
  clip::norm_kernel<<<dim3((unsigned)blocks), 256, 0, stream>>>(b, part);
  return hipGetLastError();
}

hipError_t clip_scale(const ClipBatch& b, const double* part, int parts, double max_norm, float* norm, int blocks,
                      hipStream_t stream) {
  clip::scale_kernel<<<dim3((unsigned)blocks), 256, 0, stream>>>(b, part, parts, max_norm, norm);
  return hipGetLastError();
}

}  // namespace mt
