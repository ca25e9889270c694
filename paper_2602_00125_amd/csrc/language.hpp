// Kernels of the embedding, the layer norm, the cross-entropy loss and the
// clipping of gradients (embedding.hip, layer_norm.hip, cross_entropy.hip,
// grad_clip.hip), as their host code (language_host.cpp) launches them.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "vector_io.hpp"

namespace mt {

// y[m] = scale table[ids[m]], rows of zeros for ids outside 0 .. V-1.
struct EmbeddingParams {
  vio::Index ids;
  const void* table;
  void* y;
  int64_t M, V, D, ldt, ldy;
  float scale;
};
hipError_t embedding_fwd(const EmbeddingParams& p, bool t_bf16, bool y_bf16, hipStream_t stream);

// Its gradient. ws holds the tokens grouped by id and the sums of runs that
// chunks cut.
struct EmbeddingGradParams {
  vio::Index ids;
  const void* dy;
  float* dtable;
  int64_t M, V, D, ldy, ldt;
  float scale;
  int accumulate;
  int32_t chunk;               // tokens of a chunk
  int32_t bucket_shift;        // 2^bucket_shift buckets: the low bits of an id
  int32_t *id, *pos;           // [M]: ids grouped (-1 after the last), and the tokens they come from
  uint8_t* seen;               // [V]: whether a row has a token
  float *head, *tail;          // [chunks][D]: a run that began before the chunk; one that ends after it
};
constexpr int kEmbedBucketIds = 1024;  // ids of a bucket, at most
constexpr int kEmbedChunk = 64;        // rows of an id that are added in fp32, at most
constexpr int kEmbedFewTokens = 2048, kEmbedFewClear = 16384;  // tokens of a single launch, rows that a block of it clears, at most
// How the sums are shared out: 2^shift lanes a row or tile of it, chunks of tokens.
struct EmbeddingGradForm {
  int32_t shift, tiles, chunk, chunks;
};
EmbeddingGradForm embedding_grad_form(int64_t M, int64_t D);
hipError_t embedding_bwd(const EmbeddingGradParams& p, const EmbeddingGradForm& f, bool bf16, hipStream_t stream);

constexpr int kLayerNormMaxC = 16384;
constexpr int kLayerNormLaneRows = 128;  // rows whose dy and dy n a lane adds in fp32, at most
struct LayerNormParams {
  const void *x, *dy;
  const float *w, *b;
  void* out;  // y, or dx (NULL: none)
  float* part;  // backward: [blocks][2][C] sums of dw and db, or NULL
  int64_t M, ldx, ldd, ldo;
  int32_t C, L;  // L lanes a row: a power of two up to a wave, or whole waves
  int32_t accumulate;
  float eps, C_f, inv_C;  // C as a float and 1 / C: a quotient where the mean of like values must be exact
};
// nv: groups of values (8 where a side is bf16, else 4) a lane holds, 16 values
// at most; threads of a block, blocks.
hipError_t layer_norm_fwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, int nv, int threads, int blocks,
                          hipStream_t stream);
hipError_t layer_norm_bwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, int nv, int threads, int blocks,
                          hipStream_t stream);
// dw, db (+)= the sum of the parts and, where not NULL, of from; to: receives it instead ([2][C]).
hipError_t layer_norm_finish(const float* part, int parts, int C, const double* from, double* to, float* dw, float* db, bool add,
                             hipStream_t stream);

// Cross-entropy: row_loss[m] = lse_m - z[m][t], dz = (softmax - onehot) / n.
struct CrossEntropyParams {
  const void* z;
  void* dz;  // or NULL
  vio::Index targets;
  float* row_loss;
  const int32_t* counted;  // n, or NULL where blocks count the rows themselves
  int64_t M, ldz, ldd;
  int32_t V;
};
// How a row is held (cross_entropy.hip).
struct CrossEntropyForm {
  int32_t threads, values;  // a block a row: values a thread meets
  int32_t L, L_shift;       // lanes a row where a wave holds several, else 0
  bool few;                 // one launch of one block for everything
};
// The passes over the rows' classes and losses: shares of kCrossEntropyPartRows
// rows, up to kCrossEntropyParts of them.
constexpr int kCrossEntropyParts = 256, kCrossEntropyPartRows = 16384;
hipError_t cross_entropy_count(const vio::Index& targets, int64_t M, int64_t V, int32_t* part, int32_t* counted,
                               hipStream_t stream);
// loss: written where f.few
hipError_t cross_entropy_rows(const CrossEntropyParams& p, const CrossEntropyForm& f, bool z_bf16, bool d_bf16, float* loss,
                              hipStream_t stream);
hipError_t cross_entropy_mean(const CrossEntropyParams& p, double* part, float* loss, hipStream_t stream);

// The tensors of a launch, cut into chunks of kClipChunk values, 20 bytes a tensor
// in a launch's arguments (12 where they are scaled in place):
//   w[0 .. n)       sources: 48 bits of address, kind, values of the last chunk - 1
//   w[n .. 2 n)     destinations (not in place)
//   then n 32-bit   chunks before each tensor
constexpr int kClipChunk = 4096;
constexpr int kClipWords = 470;
constexpr int kClipSourceBf16 = 1, kClipDestBf16 = 2;  // kinds
struct ClipBatch {
  uint64_t w[kClipWords];
  int32_t n, in_place, chunks;
  static int most(bool in_place) { return kClipWords * 8 / (in_place ? 12 : 20); }
  static uint64_t source(const void* p, int kind, int64_t numel) {
    return ((uint64_t)(uintptr_t)p & 0xffffffffffffull) | (uint64_t)kind << 48 | (uint64_t)((numel - 1) % kClipChunk) << 52;
  }
#if defined(__HIPCC__)
  __host__ __device__
#endif
  const uint32_t* starts() const { return (const uint32_t*)(w + (in_place ? n : 2 * n)); }
};
// part[block] = the block's sum of squares; blocks <= clip_blocks(chunks).
int clip_blocks(int64_t chunks);
hipError_t clip_norm(const ClipBatch& b, double* part, int blocks, hipStream_t stream);
// norm = sqrt of the parts' sum (where not NULL); dst = src min(1, max_norm / norm).
hipError_t clip_scale(const ClipBatch& b, const double* part, int parts, double max_norm, float* norm, int blocks,
                      hipStream_t stream);

}  // namespace mt
