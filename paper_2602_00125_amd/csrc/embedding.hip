// Embedding lookup with scaling, and its gradient, gfx950:
//
//   y[m] = s E[id_m]            dE[v] = s sum of dy[m] over the m with id_m = v
//
// A token whose id is not a row of E (padding) gets zeros and gives nothing.
//
// The lookup is bound by HBM: a group of lanes copies a token's row.
//
// The gradient groups the tokens by id, without atomics in memory and with the
// tokens of an id in ascending order, so that its sums have one order:
//
// 1. group_kernel. The low bits of an id name its bucket, a block each. A block
//    reads all ids: it counts those of lower buckets (where its own begin) and
//    its own, by wave and id, in LDS; a scan turns the counts into places; a
//    second reading hands the places out, 64 tokens at a time, tokens of one id
//    by their order among the lanes. Integers throughout. Blocks past the
//    buckets clear dE meanwhile.
// 2. sum_kernel. Chunks of the grouped tokens, a group of lanes each: a run
//    (the tokens of an id) inside a chunk goes to dE, what belongs to a run that
//    the chunk cuts goes to the workspace. Work is even whatever the ids are.
// 3. join_kernel. Where a run goes on past its first chunk, its pieces are added
//    in order.
#include <hip/hip_runtime.h>

#include "language.hpp"

namespace mt {
namespace embedding {

using namespace vio;

// VEC values a lane, G lanes a row (or a tile of it: blockIdx.y), 256 / G rows a block.
template <bool TB, bool YB, int VEC>
__global__ __launch_bounds__(256) void fwd_kernel(const EmbeddingParams p, int G_shift) {
  const int G = 1 << G_shift;
  const int64_t d = ((int64_t)blockIdx.y * G + (threadIdx.x & (G - 1))) * VEC;
  if (d >= p.D) return;
  const int64_t step = (int64_t)gridDim.x * (256 >> G_shift);
  for (int64_t m = (int64_t)blockIdx.x * (256 >> G_shift) + (threadIdx.x >> G_shift); m < p.M; m += step) {
    const int32_t id = p.ids[m];
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = 0.f;
    if ((uint32_t)id < (uint64_t)p.V) {
      load_some<TB, VEC>(p.table, id * p.ldt + d, (int)(p.D - d), 0.f, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] *= p.scale;
    }
    store_some<YB, VEC>(p.y, m * p.ldy + d, (int)(p.D - d), v);
  }
}

constexpr int kGroupWaves = 16, kGroupThreads = 64 * kGroupWaves;
constexpr int kAhead = 8;  // loads of ids in flight a lane

// Clears the rows of dE, by blocks of kGroupThreads.
__device__ __forceinline__ void clear(const EmbeddingGradParams& p, int64_t block, int64_t blocks) {
  const int64_t total = p.V * p.D, first = block * kGroupThreads + threadIdx.x, step = blocks * kGroupThreads;
  if (p.ldt == p.D) {
    // up to three values before the first 16-byte boundary and after the last
    const int64_t head = min((int64_t)((16 - ((uintptr_t)p.dtable & 15)) & 15) / 4, total), quads = (total - head) / 4;
    f32x4* q = (f32x4*)(p.dtable + head);
    for (int64_t i = first; i < quads; i += step) q[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (first < head) p.dtable[first] = 0.f;
    if (head + 4 * quads + first < total) p.dtable[head + 4 * quads + first] = 0.f;
  } else {
    for (int64_t i = first; i < total; i += step) {
      const int64_t v = i / p.D;
      p.dtable[v * p.ldt + (i - v * p.D)] = 0.f;
    }
  }
}

// counts: [kGroupWaves][locals], of the bucket's ids local 2^shift + bucket.
__global__ __launch_bounds__(kGroupThreads) void group_kernel(const EmbeddingGradParams p, int locals) {
  __shared__ int32_t counts[kGroupWaves * kEmbedBucketIds];
  __shared__ int32_t wave_lower[kGroupWaves], wave_sum[kGroupWaves];
  const int buckets = 1 << p.bucket_shift, bucket = blockIdx.x;
  if (bucket >= buckets) {
    clear(p, bucket - buckets, gridDim.x - buckets);
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < kGroupWaves * locals; i += kGroupThreads) counts[i] = 0;
  __syncthreads();
  int32_t* mine = counts + wave * locals;
  // a wave's share of the tokens: whole batches of 64
  const int64_t share = ((p.M + kGroupThreads - 1) / kGroupThreads) * 64;
  const int64_t m0 = wave * share, m1 = min(m0 + share, p.M);
  int lower = 0;  // of the wave, the same in every lane
  for (int64_t m = m0; m < m1; m += 64 * kAhead) {
    int32_t id[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int64_t i = m + 64 * j + lane;
      id[j] = i < m1 ? p.ids[i] : -1;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const bool ok = (uint32_t)id[j] < (uint64_t)p.V;
      const int b = id[j] & (buckets - 1);
      lower += __popcll(__ballot(ok && b < bucket));
      if (ok && b == bucket) atomicAdd(&mine[id[j] >> p.bucket_shift], 1);
    }
  }
  if (lane == 0) wave_lower[wave] = lower;
  __syncthreads();
  // places: ids in order, an id's waves in order
  const int per = (locals + kGroupThreads - 1) / kGroupThreads, l0 = threadIdx.x * per, l1 = min(l0 + per, locals);
  int sum = 0;
  for (int l = l0; l < l1; ++l)
    for (int w = 0; w < kGroupWaves; ++w) sum += counts[w * locals + l];
  int scan = sum;  // inclusive over the wave
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(scan, o, 64);
    if (lane >= o) scan += t;
  }
  if (lane == 63) wave_sum[wave] = scan;
  __syncthreads();
  int at = scan - sum, own = 0;
  for (int w = 0; w < kGroupWaves; ++w) {
    at += wave_lower[w] + (w < wave ? wave_sum[w] : 0);
    own += wave_lower[w] + wave_sum[w];
  }
  if (bucket == buckets - 1 && threadIdx.x == 0) *p.total = own;  // of all buckets
  for (int l = l0; l < l1; ++l)
    for (int w = 0; w < kGroupWaves; ++w) {
      const int n = counts[w * locals + l];
      counts[w * locals + l] = at;
      at += n;
    }
  __syncthreads();
  for (int64_t m = m0; m < m1; m += 64 * kAhead) {
    int32_t id[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int64_t i = m + 64 * j + lane;
      id[j] = i < m1 ? p.ids[i] : -1;
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      uint64_t left = __ballot((uint32_t)id[j] < (uint64_t)p.V && (id[j] & (buckets - 1)) == bucket);
      while (left) {  // an id at a time; the same in every lane
        const int leader = __ffsll((unsigned long long)left) - 1;
        const int32_t v = __shfl(id[j], leader, 64);
        const uint64_t same = __ballot(id[j] == v);
        int place = 0;
        if (lane == leader) place = atomicAdd(&mine[v >> p.bucket_shift], (int)__popcll(same));
        place = __shfl(place, leader, 64);
        if (id[j] == v) {
          const int k = place + (int)__popcll(same & ((1ull << lane) - 1));
          p.id[k] = v;
          p.pos[k] = (int32_t)(m + 64 * j + lane);
        }
        left &= ~same;
      }
    }
  }
}

// dE's values from column d on (+)= s sum
template <int VEC>
__device__ __forceinline__ void put(const EmbeddingGradParams& p, int32_t id, int64_t d, const float (&sum)[VEC]) {
  float* row = p.dtable + id * p.ldt;
  float v[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) v[e] = p.scale * sum[e];
  if (p.accumulate) {
    float old[VEC];
    load_some<false, VEC>(row, d, (int)(p.D - d), 0.f, old);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] += old[e];
  }
  store_some<false, VEC>(row, d, (int)(p.D - d), v);
}

template <bool BF, int VEC>
__global__ __launch_bounds__(256) void sum_kernel(const EmbeddingGradParams p, int G_shift) {
  constexpr int U = 4;  // rows in flight
  const int G = 1 << G_shift;
  const int64_t c = (int64_t)blockIdx.x * (256 >> G_shift) + (threadIdx.x >> G_shift);
  const int64_t d = ((int64_t)blockIdx.y * G + (threadIdx.x & (G - 1))) * VEC;
  const int64_t total = *p.total, i0 = c * p.chunk, i1 = min(i0 + p.chunk, total);
  if (i0 >= i1 || d >= p.D) return;
  const int32_t before = i0 > 0 ? p.id[i0 - 1] : -1, after = i1 < total ? p.id[i1] : -1;
  int32_t cur = p.id[i0];
  bool cut = cur == before;  // the run began in an earlier chunk
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  for (int64_t i = i0; i < i1; i += U) {
    int32_t id[U];
    float v[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      id[u] = -1;
      if (i + u < i1) {
        id[u] = p.id[i + u];
        load_some<BF, VEC>(p.dy, p.pos[i + u] * p.ldy + d, (int)(p.D - d), 0.f, v[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (id[u] < 0) break;
      if (id[u] != cur) {
        if (cut) store_some<false, VEC>(p.head + c * p.D, d, (int)(p.D - d), acc);
        else put<VEC>(p, cur, d, acc);
        cur = id[u];
        cut = false;
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += v[u][e];
    }
  }
  if (cut) store_some<false, VEC>(p.head + c * p.D, d, (int)(p.D - d), acc);
  else if (cur == after) store_some<false, VEC>(p.tail + c * p.D, d, (int)(p.D - d), acc);
  else put<VEC>(p, cur, d, acc);
}

// A block for each chunk whose last run began in it and goes on. Its 256 / G
// groups of lanes take the later pieces in turn; their sums meet in LDS.
template <int VEC>
__global__ __launch_bounds__(256) void join_kernel(const EmbeddingGradParams p, int G_shift) {
  __shared__ float sums[256 * VEC];
  const int G = 1 << G_shift, groups = 256 >> G_shift, grp = threadIdx.x >> G_shift, lane = threadIdx.x & 63;
  const int64_t c = blockIdx.x, total = *p.total, i0 = c * p.chunk, i1 = i0 + p.chunk;
  if (i1 >= total) return;  // nothing after it
  const int32_t id = p.id[i1];
  if (p.id[i1 - 1] != id || (p.id[i0] == id && i0 > 0 && p.id[i0 - 1] == id)) return;
  // how many chunks begin with the run
  int64_t pieces = 1;
  for (;;) {
    const int64_t i = (c + 1 + pieces + lane) * p.chunk;
    const uint64_t in = __ballot(i < total && p.id[i < total ? i : 0] == id);
    const int n = in == ~0ull ? 64 : __ffsll((unsigned long long)~in) - 1;
    pieces += n;
    if (n < 64) break;
  }
  const int64_t d = ((int64_t)blockIdx.y * G + (threadIdx.x & (G - 1))) * VEC;
  float acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  if (d < p.D) {
    // a group takes a share of the pieces, one after another
    const int64_t share = (pieces + groups - 1) / groups, j0 = grp * share, j1 = min(j0 + share, pieces);
    if (grp == 0) load_some<false, VEC>(p.tail + c * p.D, d, (int)(p.D - d), 0.f, acc);
#pragma unroll 4
    for (int64_t j = j0; j < j1; ++j) {
      float v[VEC];
      load_some<false, VEC>(p.head + (c + 1 + j) * p.D, d, (int)(p.D - d), 0.f, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[threadIdx.x * VEC + e] = acc[e];
  __syncthreads();
  if (grp || d >= p.D) return;
  for (int g = 1; g < groups; ++g)
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] += sums[(g * G + threadIdx.x) * VEC + e];
  put<VEC>(p, id, d, acc);
}

// Lanes of a row: a power of two, 256 at most.
int lanes_shift(int64_t D, int vec) {
  int s = 0;
  while (s < 8 && (int64_t)vec << s < D) ++s;
  return s;
}

}  // namespace embedding

hipError_t embedding_fwd(const EmbeddingParams& p, bool t_bf16, bool y_bf16, hipStream_t stream) {
  using namespace embedding;
  const int vec = t_bf16 || y_bf16 ? 8 : 4, s = lanes_shift(p.D, vec);
  const int64_t rows = 256 >> s, tile = (int64_t)vec << s;
  const int64_t blocks = (p.M + rows - 1) / rows;
  const dim3 grid((unsigned)(blocks < (1 << 22) ? blocks : 1 << 22), (unsigned)((p.D + tile - 1) / tile));
  if (t_bf16) {
    if (y_bf16) fwd_kernel<true, true, 8><<<grid, 256, 0, stream>>>(p, s);
    else fwd_kernel<true, false, 8><<<grid, 256, 0, stream>>>(p, s);
  } else {
    if (y_bf16) fwd_kernel<false, true, 8><<<grid, 256, 0, stream>>>(p, s);
    else fwd_kernel<false, false, 4><<<grid, 256, 0, stream>>>(p, s);
  }
  return hipGetLastError();
}

hipError_t embedding_bwd(const EmbeddingGradParams& p, bool bf16, hipStream_t stream) {
  using namespace embedding;
  const int buckets = 1 << p.bucket_shift, locals = (int)((p.V + buckets - 1) >> p.bucket_shift);
  // blocks that clear: 16 KB each at a time, two a CU at most
  int64_t clear = p.accumulate ? 0 : (p.V * p.D + 4095) / 4096;
  if (clear > 512) clear = 512;
  group_kernel<<<dim3((unsigned)(buckets + clear)), kGroupThreads, 0, stream>>>(p, locals);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.M == 0) return e;
  const int vec = bf16 ? 8 : 4, s = lanes_shift(p.D, vec);
  const int64_t rows = 256 >> s, tile = (int64_t)vec << s;
  const dim3 sums((unsigned)((p.chunks + rows - 1) / rows), (unsigned)((p.D + tile - 1) / tile));
  if (bf16) sum_kernel<true, 8><<<sums, 256, 0, stream>>>(p, s);
  else sum_kernel<false, 4><<<sums, 256, 0, stream>>>(p, s);
  if ((e = hipGetLastError()) != hipSuccess || p.chunks < 2) return e;
  const dim3 joins((unsigned)p.chunks, sums.y);
  if (bf16) join_kernel<8><<<joins, 256, 0, stream>>>(p, s);
  else join_kernel<4><<<joins, 256, 0, stream>>>(p, s);
  return hipGetLastError();
}

}  // namespace mt
