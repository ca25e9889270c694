// Launch descriptions of the attention kernels (attention.hip), filled by
// attention_host.cpp.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "kernels.hpp"

namespace mt {

struct AttnParams {
  HeadView q, k, v, o, dout, dq, dk, dv;
  float* lse;           // [B, HQ, TQ]: written by the forward (NULL: skipped), read by the backward
  float* delta;         // [2][B, HQ, TQ]: -lse / scale and -sum_d do o, from the dq pass to the dk / dv pass
  const int32_t* kv_len;   // [B] or NULL: keys of each batch element
  const int32_t* q_start;  // [B] or NULL: key position of query 0 (causal)
  int32_t B, TQ, TK, HQ, HK, G, D;
  int32_t causal, accumulate, with_dq, paired;
  float scale, scale_log2;  // scale and scale * log2(e)
  // keys shared out over splits (forward) / query tiles over splits (dk, dv)
  int32_t splits;
  float* part;  // the splits' partial results
};

// D <= 128. bf16 inputs, or fp32. vec: every base and stride allows 16-byte
// accesses and D is a multiple of a 16-byte chunk; else element accesses.
hipError_t attn_fwd(const AttnParams& p, bool bf16, bool vec, hipStream_t stream);
// The same with 32 queries (of all heads of a key head) and a share of the
// keys a block: p.splits shares, whose results (D + 2 floats for each query and
// head) meet in p.part unless there is one.
hipError_t attn_fwd_split(const AttnParams& p, bool bf16, bool vec, hipStream_t stream);
// The dq pass (which also writes p.delta; with_dq = 0: nothing else) and the
// dk / dv pass: p.splits shares of the query tiles a block of keys, which meet in
// p.part (2 B HK TK D floats each) unless there is one.
hipError_t attn_bwd_dq(const AttnParams& p, bool bf16, bool vec, hipStream_t stream);
hipError_t attn_bwd_dkv(const AttnParams& p, bool bf16, bool vec, hipStream_t stream);

constexpr int kAttnRows = 128;  // queries (forward, dq) or keys (dk, dv) a block holds
constexpr int kAttnMaxD = 128;

// Keys a block of the dk / dv pass holds: in bf16 half as many where there
// would be fewer blocks than CUs.
inline int attn_kv_block(const AttnParams& p, bool bf16) {
  return bf16 && (int64_t)p.B * p.HK * ((p.TK + 127) / 128) < 256 ? 64 : 128;
}

}  // namespace mt
