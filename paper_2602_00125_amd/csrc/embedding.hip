// Embedding lookup with scaling, and its gradient, gfx950:
//
//   y[m] = s E[id_m]            dE[v] = s sum of dy[m] over the m with id_m = v
//
// A token whose id is not a row of E (padding) gets zeros and gives nothing.
//
// The lookup is bound by HBM: a group of lanes copies a token's row, four at a time
// where there are many (16384 x 1024 fp32 22.8 -> 20.6 us: 4.4 TB/s).
//
// The gradient groups the tokens by id, without atomics in memory and with the
// tokens of an id in ascending order, so that its sums have one order:
//
// 1. group_kernel. The low bits of an id name its bucket, a block each. A block
//    reads all ids: it counts those of lower buckets (where its own begin) and
//    its own, by wave and id, in LDS; a scan turns the counts into places; the
//    ids, still in registers or read again, are handed the places, 64 tokens at a
//    time, tokens of one id by their order among the lanes. Integers throughout.
// 2. sum_kernel. Chunks of the grouped tokens, a wave or less each and tile of
//    columns: a run (the tokens of an id) inside a chunk goes to dE, what belongs
//    to a run that the chunk cuts goes to the workspace. Work is even whatever the
//    ids are. Beside it, blocks clear the rows without a token.
// 3. join_kernel. Where a run goes on past its first chunk, its pieces are added
//    in order, in 64 bits.
//
// 16384 tokens of 1024 fp32 values into 50001 rows: 74 us for 272 MB, of which the
// first launch takes 9 (it waits for loads, LDS and its own order), the second 55
// (276 MB moved, 5.0 TB/s), the third 8 (a chain of loads). Clearing part of the
// rows in the first and the last launch too moved their time, and saved none.
// A few tokens take one launch instead (few_kernel).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "language.hpp"

namespace mt {
namespace embedding {

using namespace vio;

// VEC values a lane, G lanes a row (or a tile of it: blockIdx.y), U rows at a time.
template <bool TB, bool YB, int VEC, int U>
__global__ __launch_bounds__(256) void fwd_kernel(const EmbeddingParams p, int G_shift) {
  const int G = 1 << G_shift, rows = 256 >> G_shift;
  const int d = ((int)blockIdx.y * G + (threadIdx.x & (G - 1))) * VEC, n = (int)p.D - d;
  if (n <= 0) return;
  for (int64_t m0 = (int64_t)blockIdx.x * rows * U + (threadIdx.x >> G_shift); m0 < p.M; m0 += (int64_t)gridDim.x * rows * U) {
    int32_t id[U];
    float v[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) id[u] = m0 + u * rows < p.M ? p.ids[m0 + u * rows] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u)
      load_some<TB, VEC>(p.table, id[u] * p.ldt + d, (uint32_t)id[u] < (uint64_t)p.V ? n : 0, 0.f, v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[u][e] = (uint32_t)id[u] < (uint64_t)p.V ? v[u][e] * p.scale : 0.f;
      store_some<YB, VEC>(p.y, (m0 + u * rows) * p.ldy + d, m0 + u * rows < p.M ? n : 0, v[u]);
    }
  }
}

constexpr int64_t kManyBlocks = 4096;  // a lookup of so many keeps four rows in flight a lane
constexpr int kGroupWaves = 16, kGroupThreads = 64 * kGroupWaves;
constexpr int kAhead = 16;  // ids in flight a lane

// counts: [kGroupWaves][locals], of the bucket's ids local 2^shift + bucket.
__global__ __launch_bounds__(kGroupThreads) void group_kernel(const EmbeddingGradParams p, int locals) {
  __shared__ int32_t counts[kGroupWaves * kEmbedBucketIds];
  __shared__ int32_t wave_lower[kGroupWaves], wave_sum[kGroupWaves];
  const int buckets = 1 << p.bucket_shift, bucket = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int i = threadIdx.x; i < kGroupWaves * locals; i += kGroupThreads) counts[i] = 0;
  __syncthreads();
  int32_t* mine = counts + wave * locals;
  // a wave's share of the tokens: whole batches of 64
  const int64_t share = ((p.M + kGroupThreads - 1) / kGroupThreads) * 64;
  const int64_t m0 = wave * share, m1 = min(m0 + share, p.M);
  int lower = 0;  // of the wave, the same in every lane
  int32_t id[kAhead];
  auto read = [&](int64_t m) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int64_t i = m + 64 * j + lane;
      id[j] = i < m1 ? p.ids[i] : -1;
    }
  };
  for (int64_t m = m0; m < m1; m += 64 * kAhead) {
    read(m);
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
#pragma unroll
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
  if (bucket == buckets - 1)  // its end is that of all: no id after it
    for (int64_t i = own + threadIdx.x; i < p.M; i += kGroupThreads) p.id[i] = -1;
  for (int l = l0; l < l1; ++l) {
    const int from = at;
    int n[kGroupWaves];
#pragma unroll
    for (int w = 0; w < kGroupWaves; ++w) n[w] = counts[w * locals + l];
#pragma unroll
    for (int w = 0; w < kGroupWaves; ++w) {
      counts[w * locals + l] = at;
      at += n[w];
    }
    const int64_t v = ((int64_t)l << p.bucket_shift) + bucket;
    if (v < p.V) p.seen[v] = at > from;
  }
  __syncthreads();
  for (int64_t m = m0; m < m1; m += 64 * kAhead) {
    if (share > 64 * kAhead) read(m);  // else it still holds them
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      uint64_t left = __ballot((uint32_t)id[j] < (uint64_t)p.V && (id[j] & (buckets - 1)) == bucket);
      while (left) {  // an id at a time; the same in every lane
        const int leader = __ffsll((unsigned long long)left) - 1;
        const int32_t v = __builtin_amdgcn_readlane(id[j], leader);
        const uint64_t same = __ballot(id[j] == v);
        int place = 0;
        if (lane == leader) place = atomicAdd(&mine[v >> p.bucket_shift], (int)__popcll(same));
        place = __builtin_amdgcn_readlane(place, leader);
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

// dE[id] = s sum (+ old), n values from column d on.
template <int VEC>
__device__ __forceinline__ void put(const EmbeddingGradParams& p, int32_t id, int d, int n, const float (&sum)[VEC], const float (&old)[VEC]) {
  float v[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) v[e] = p.scale * sum[e];
  if (p.accumulate)
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] += old[e];
  store_some<false, VEC>(p.dtable, id * p.ldt + d, n, v);
}
template <int VEC>
__device__ __forceinline__ void load_old(const EmbeddingGradParams& p, int32_t id, int d, int n, float (&old)[VEC]) {
  load_some<false, VEC>(p.dtable, id * p.ldt + d, p.accumulate ? n : 0, 0.f, old);
}

// Rows without a token become 0, by blocks past those of the sums.
__device__ __forceinline__ void clear(const EmbeddingGradParams& p, int block, int blocks, int G_shift) {
  const int G = 1 << G_shift, rows = 256 >> G_shift;
  const float zero[4] = {};
  for (int64_t v = (int64_t)block * rows + (threadIdx.x >> G_shift); v < p.V; v += (int64_t)blocks * rows) {
    if (p.seen[v]) continue;
    for (int d = (threadIdx.x & (G - 1)) * 4; d < p.D; d += G * 4) store_some<false, 4>(p.dtable, v * p.ldt + d, (int)p.D - d, zero);
  }
}

// Sum: what a run's rows are added in, fp32 where a chunk has up to kEmbedChunk of
// them (64 bits take registers: three waves a SIMD, not four).
template <bool BF, typename Sum>
__global__ __launch_bounds__(256) void sum_kernel(const EmbeddingGradParams p, int G_shift, int tiles, int sum_blocks) {
  if ((int)blockIdx.x >= sum_blocks) {
    clear(p, blockIdx.x - sum_blocks, gridDim.x - sum_blocks, G_shift);
    return;
  }
  constexpr int VEC = 4, U = 8;  // rows in flight
  const int G = 1 << G_shift, tile = blockIdx.x % tiles;
  const int64_t c = (int64_t)(blockIdx.x / tiles) * (256 >> G_shift) + (threadIdx.x >> G_shift);
  const int d = (tile * G + (threadIdx.x & (G - 1))) * VEC, n = (int)p.D - d;
  const int64_t i0 = c * p.chunk, i1 = min(i0 + p.chunk, p.M);
  if (i0 >= i1 || n <= 0) return;
  const int32_t before = i0 > 0 ? p.id[i0 - 1] : -1;
  bool cut = before == p.id[i0];  // the run began in an earlier chunk
  Sum acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0;
  for (int64_t i = i0; i < i1; i += U) {  // a chunk is whole but for the last one's end, past which ids are -1
    int32_t id[U + 1], pos[U];
    float v[U][VEC], old[U][VEC];
#pragma unroll
    for (int u = 0; u <= U; ++u) id[u] = i + u < p.M ? p.id[i + u] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) pos[u] = i + u < i1 ? p.pos[i + u] : 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      load_some<BF, VEC>(p.dy, pos[u] * p.ldy + d, id[u] >= 0 ? n : 0, 0.f, v[u]);
      load_old(p, id[u], d, id[u] >= 0 && id[u] != id[u + 1] ? n : 0, old[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (id[u] < 0) return;
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += v[u][e];
      const bool ends = id[u] != id[u + 1];
      if (!ends && i + u < i1 - 1) continue;
      float sum[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) sum[e] = (float)acc[e];
      if (cut) store_some<false, VEC>(p.head, c * p.D + d, n, sum);
      else if (ends) put(p, id[u], d, n, sum, old[u]);
      else store_some<false, VEC>(p.tail, c * p.D + d, n, sum);
      cut = false;
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] = 0;
    }
  }
}

// A block for each chunk whose last run began in it and goes on. Its 256 / G
// groups of lanes take equal shares of the later pieces; their sums meet in LDS. In
// 64 bits: a frequent id has a piece in every chunk, and added in fp32 the like
// rows of 2^24 tokens were off by 6e-4 of their sum.
__global__ __launch_bounds__(256) void join_kernel(const EmbeddingGradParams p, int G_shift, int tiles) {
  constexpr int VEC = 4, U = 8;
  __shared__ double sums[256 * VEC];
  const int G = 1 << G_shift, groups = 256 >> G_shift, grp = threadIdx.x >> G_shift, lane = threadIdx.x & 63;
  const int tile = blockIdx.x % tiles;
  const int64_t c = blockIdx.x / tiles, i0 = c * p.chunk, i1 = i0 + p.chunk;
  // together: the chunk's first id and the one before it, its last and the one after it
  const int32_t id = i1 < p.M ? p.id[i1] : -1, last = p.id[min(i1, p.M) - 1], first = p.id[i0], before = i0 > 0 ? p.id[i0 - 1] : -1;
  if (id < 0 || last != id || (first == id && before == id)) return;
  // how many chunks begin with the run
  int64_t pieces = 1;
  for (;;) {
    const int64_t i = (c + 1 + pieces + lane) * p.chunk;
    const uint64_t in = __ballot(i < p.M && p.id[i < p.M ? i : 0] == id);
    const int n = in == ~0ull ? 64 : __ffsll((unsigned long long)~in) - 1;
    pieces += n;
    if (n < 64) break;
  }
  const int d = (tile * G + (threadIdx.x & (G - 1))) * VEC, n = (int)p.D - d;
  float first_piece[VEC], old[VEC];
  // a group takes a share of the pieces, one after another
  const int64_t share = (pieces + groups - 1) / groups, j1 = min((grp + 1) * share, pieces);
  load_some<false, VEC>(p.tail, c * p.D + d, grp == 0 ? n : 0, 0.f, first_piece);
  double acc[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = first_piece[e];
  load_old(p, id, d, grp == 0 ? n : 0, old);
  for (int64_t j = grp * share; j < j1; j += U) {
    float v[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) load_some<false, VEC>(p.head, (c + 1 + j + u) * p.D + d, j + u < j1 ? n : 0, 0.f, v[u]);
    // all loads first: else a value is widened behind its own load, which waits for it (65536 tokens of 64 columns, 16
    // ids 68 -> 97 us)
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e) __asm__ __volatile__("" : "+v"(v[u][e]));
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += v[u][e];
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[threadIdx.x * VEC + e] = acc[e];
  __syncthreads();
  if (grp || n <= 0) return;
  for (int g = 1; g < groups; ++g)
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] += sums[(g * G + threadIdx.x) * VEC + e];
  float sum[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = (float)acc[e];
  put(p, id, d, n, sum, old);
}

constexpr int kFewThreads = 512;
// A few tokens: one launch, no lists. A block takes a token and a tile of
// columns; where no earlier token has its id it finds those that have, in order,
// and its groups of G lanes add equal shares of their rows, which meet in
// LDS. Blocks past these clear ranges of rows, which they look up in all tokens.
template <bool BF>
__global__ __launch_bounds__(kFewThreads) void few_kernel(const EmbeddingGradParams p, int G_shift, int tiles, int sum_blocks, int clear_rows) {
  constexpr int VEC = 4, U = 8, PER = kEmbedFewTokens / kFewThreads;
  __shared__ float sums[kFewThreads * VEC];
  __shared__ uint16_t list[kEmbedFewTokens];
  __shared__ int wave_count[kFewThreads / 64];
  __shared__ uint8_t seen[kEmbedFewClear];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, M = (int)p.M;
  const int G = 1 << G_shift, groups = kFewThreads >> G_shift, grp = threadIdx.x >> G_shift, D = (int)p.D;
  int32_t id[PER];  // of the wave's share of the tokens, 64 at a time
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int m = wave * (64 * PER) + 64 * j + lane;
    id[j] = m < M ? p.ids[m] : -1;
  }
  if ((int)blockIdx.x >= sum_blocks) {
    const int64_t v0 = (int64_t)(blockIdx.x - sum_blocks) * clear_rows;
    for (int i = threadIdx.x; i < clear_rows; i += kFewThreads) seen[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PER; ++j)
      if (id[j] >= v0 && id[j] < v0 + clear_rows) seen[id[j] - v0] = 1;
    __syncthreads();
    const float zero[4] = {};
    for (int i = grp; i < clear_rows && v0 + i < p.V; i += groups) {
      if (seen[i]) continue;
      for (int d = (threadIdx.x & (G - 1)) * 4; d < D; d += G * 4) store_some<false, 4>(p.dtable, (v0 + i) * p.ldt + d, D - d, zero);
    }
    return;
  }
  const int m = blockIdx.x / tiles, tile = blockIdx.x % tiles;
  const int32_t v = p.ids[m];
  if ((uint32_t)v >= (uint64_t)p.V) return;
  uint64_t same[PER];
  int mine = 0, earlier = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    same[j] = __ballot(id[j] == v);
    mine += __popcll(same[j]);
    earlier += __popcll(__ballot(id[j] == v && wave * (64 * PER) + 64 * j + lane < m));
  }
  if (__syncthreads_or(earlier)) return;
  if (lane == 0) wave_count[wave] = mine;
  __syncthreads();
  int at = 0, n = 0;
  for (int w = 0; w < kFewThreads / 64; ++w) {
    at += w < wave ? wave_count[w] : 0;
    n += wave_count[w];
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (id[j] == v) list[at + __popcll(same[j] & ((1ull << lane) - 1))] = (uint16_t)(wave * (64 * PER) + 64 * j + lane);
    at += __popcll(same[j]);
  }
  __syncthreads();
  const int d = (tile * G + (threadIdx.x & (G - 1))) * VEC, left = D - d;
  float acc[VEC], old[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
  load_some<false, VEC>(p.dtable, v * p.ldt + d, p.accumulate && grp == 0 ? left : 0, 0.f, old);
  const int share = (n + groups - 1) / groups, i1 = min((grp + 1) * share, n);
  for (int i = grp * share; i < i1; i += U) {
    float x[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u)
      load_some<BF, VEC>(p.dy, (i + u < i1 ? list[i + u] : 0) * p.ldy + d, i + u < i1 ? left : 0, 0.f, x[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e) acc[e] += x[u][e];
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[threadIdx.x * VEC + e] = acc[e];
  __syncthreads();
  if (grp || left <= 0) return;
  for (int g = 1; g < groups && g * share < n; ++g)
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] += sums[(g * G + threadIdx.x) * VEC + e];
  put(p, v, d, left, acc, old);
}

// Lanes of a row: a power of two, 2^most at most.
int lanes_shift(int64_t D, int vec, int most) {
  int s = 0;
  while (s < most && (int64_t)vec << s < D) ++s;
  return s;
}

template <bool TB, bool YB, int VEC>
hipError_t lookup(const EmbeddingParams& p, hipStream_t stream) {
  const int s = lanes_shift(p.D, VEC, 8);
  const int64_t rows = 256 >> s, tile = (int64_t)VEC << s, tiles = (p.D + tile - 1) / tile;
  auto grid = [&](int U) { return dim3((unsigned)std::min<int64_t>((p.M + rows * U - 1) / (rows * U), 1 << 22), (unsigned)tiles); };
  if (p.M / rows * tiles >= kManyBlocks) fwd_kernel<TB, YB, VEC, 4><<<grid(4), 256, 0, stream>>>(p, s);
  else fwd_kernel<TB, YB, VEC, 1><<<grid(1), 256, 0, stream>>>(p, s);
  return hipGetLastError();
}

}  // namespace embedding

hipError_t embedding_fwd(const EmbeddingParams& p, bool t_bf16, bool y_bf16, hipStream_t stream) {
  using namespace embedding;
  if (t_bf16) return y_bf16 ? lookup<true, true, 8>(p, stream) : lookup<true, false, 8>(p, stream);
  return y_bf16 ? lookup<false, true, 8>(p, stream) : lookup<false, false, 4>(p, stream);
}

EmbeddingGradForm embedding_grad_form(int64_t M, int64_t D) {
  EmbeddingGradForm f;
  f.shift = embedding::lanes_shift(D, 4, 6);
  f.tiles = (int32_t)((D + (4 << f.shift) - 1) >> (f.shift + 2));
  // 4096 waves, then chunks of up to kEmbedChunk tokens; longer ones for what a launch holds
  auto items = [&] { return (M + f.chunk - 1) / f.chunk * f.tiles; };
  for (f.chunk = 8; items() > (int64_t)4096 * (64 >> f.shift) && (f.chunk < kEmbedChunk || items() > 1 << 22);) f.chunk *= 2;
  f.chunks = (int32_t)((M + f.chunk - 1) / f.chunk);
  return f;
}

hipError_t embedding_bwd(const EmbeddingGradParams& p, const EmbeddingGradForm& f, bool bf16, hipStream_t stream) {
  using namespace embedding;
  // One launch for few tokens: 64 of 64 columns into 50001 rows 16.1 -> 5.7 us, 2000 of 256 added to 20000 rows
  // 16.2 -> 8.1, 1000 of 1024 bf16 17.7 -> 15.5; past 4096 tiles each block's search costs more than the other two
  // launches (1000 of 2048: 19 -> 27). A batch of one token alone may lose (2000 of 256: 22 -> 36).
  if (p.M > 0 && p.M <= kEmbedFewTokens && p.M * f.tiles <= 4096) {
    const int sums = (int)p.M * f.tiles;
    const int clear_rows = (int)std::max<int64_t>((p.V + 1023) / 1024, std::max<int64_t>(1, std::min<int64_t>(1024, 4096 / p.D)));
    const int clears = p.accumulate ? 0 : (int)((p.V + clear_rows - 1) / clear_rows);
    const dim3 grid((unsigned)(sums + clears));
    if (bf16) few_kernel<true><<<grid, kFewThreads, 0, stream>>>(p, f.shift, f.tiles, sums, clear_rows);
    else few_kernel<false><<<grid, kFewThreads, 0, stream>>>(p, f.shift, f.tiles, sums, clear_rows);
    return hipGetLastError();
  }
  const int buckets = 1 << p.bucket_shift, locals = (int)((p.V + buckets - 1) >> p.bucket_shift);
  group_kernel<<<dim3((unsigned)buckets), kGroupThreads, 0, stream>>>(p, locals);
  const int rows = 256 >> f.shift;
  const int sums = (int)((f.chunks + rows - 1) / rows) * f.tiles;
  // 16 KB each at a time, eight a CU at most
  const int clears = p.accumulate ? 0 : (int)std::min<int64_t>((p.V * p.D + 4095) / 4096, 2048);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sums + clears == 0) return e;
  const dim3 grid((unsigned)(sums + clears));
  auto sum = [&](auto kernel) { kernel<<<grid, 256, 0, stream>>>(p, f.shift, f.tiles, sums); };
  if (f.chunk <= kEmbedChunk) bf16 ? sum(sum_kernel<true, float>) : sum(sum_kernel<false, float>);
  else bf16 ? sum(sum_kernel<true, double>) : sum(sum_kernel<false, double>);
  if ((e = hipGetLastError()) != hipSuccess || f.chunks < 2) return e;
  join_kernel<<<dim3((unsigned)(f.chunks * f.tiles)), 256, 0, stream>>>(p, f.shift, f.tiles);
  return hipGetLastError();
}

}  // namespace mt
