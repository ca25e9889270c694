// Host-side pieces shared by the C-ABI translation units (capi.cpp and
// conv_host.cpp): error recording, tensor checks, the product planner and
// launcher, and the test / tuning knobs. Internal: not part of the ABI.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>
#include <string>

#include "../../include/minitensor_hip.h"
#include "gemm_params.hpp"

namespace mt::host {

// knobs set by mt_debug_set (-1 / 0 = automatic); atomics, read once per use
extern std::atomic<int> g_force_cfg, g_force_vec1, g_force_splits, g_force_parts, g_krot;
extern std::atomic<int> g_conv_gather, g_stream_k, g_sk_blocks, g_phase_grid, g_persist, g_attn_splits;

// records the message for mt_last_error() and returns s
mt_status fail(mt_status s, const std::string& msg);
mt_status hip_status(hipError_t e);
mt_status check_tensor(const mt_tensor* t, const char* name, int min_nd, int max_nd);
mt_status check_vector(const mt_tensor* t, const char* name, int64_t n);
bool overlaps(const mt_tensor* a, const mt_tensor* b);
int64_t numel(const mt_tensor* t);
size_t elem_size(int32_t dt);
bool is_row_major(const mt_tensor* t);
bool vec_ok_operand(const void* base, int64_t rows_other, int64_t contig_extent, int64_t ld,
                    const int64_t* bstrides, int nb, int per);

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// One matrix product as the planner sees it: launch description, operand
// layouts, vector width, tile configuration (-1 = choose), gathered operand.
struct GemmCall {
  mt::GemmParams p;
  bool a_kc, b_kc;
  bool vec;   // 16-byte operand loads and output stores
  bool bf16;  // bf16 operands (else fp32)
  int cfg;
  int conv;   // 1 / 2 / 3: the convolution product gathering an operand (p.cg), else 0
  int sk;     // stream-K blocks (conv 1 and 3 on the 256x256 tile), else 0
  int runs;   // most split-K runs (0: as many as the kind of product takes)
};


void init_params(mt::GemmParams* p);
// resolves tile, vector width, split-K / stream-K; returns the workspace the
// split needs (0 = none)
size_t plan_gemm(GemmCall& g, bool may_split);
// plans and launches (split partials in ws if it is large enough), then the
// split's finish
mt_status launch_gemm(GemmCall& g, hipStream_t stream, void* ws, size_t ws_bytes);

// the convolution entry points' bodies (conv_host.cpp); ws_query non-null:
// validate and report the workspace size only
mt_status conv_fwd_impl(const mt_tensor* x, const mt_tensor* w, const mt_tensor* b,
                        const mt_tensor* y, int32_t sh, int32_t sw, int32_t ph, int32_t pw,
                        void* ws, size_t ws_bytes, hipStream_t stream, size_t* ws_query);
mt_status conv_bwd_impl(const mt_tensor* x, const mt_tensor* w, const mt_tensor* dy,
                        const mt_tensor* dx, const mt_tensor* dw, const mt_tensor* db, int32_t sh,
                        int32_t sw, int32_t ph, int32_t pw, uint32_t flags, void* ws,
                        size_t ws_bytes, hipStream_t stream, size_t* ws_query);

// the bodies of attention, the head norms with rotation and dropout
// (attention_host.cpp); ws_query as above
mt_status attention_fwd_impl(const mt_tensor* q, const mt_tensor* k, const mt_tensor* v, const mt_tensor* kv_len,
                             const mt_tensor* q_start, const mt_tensor* o, const mt_tensor* lse, float scale,
                             uint32_t flags, void* ws, size_t ws_bytes, hipStream_t stream, size_t* ws_query);
mt_status attention_bwd_impl(const mt_tensor* q, const mt_tensor* k, const mt_tensor* v, const mt_tensor* kv_len,
                             const mt_tensor* q_start, const mt_tensor* o, const mt_tensor* lse, const mt_tensor* dout,
                             const mt_tensor* dq, const mt_tensor* dk, const mt_tensor* dv, float scale, uint32_t flags,
                             void* ws, size_t ws_bytes, hipStream_t stream, size_t* ws_query);
mt_status qk_norm_rope_fwd_impl(const mt_tensor* q, const mt_tensor* k, const mt_tensor* wq, const mt_tensor* wk,
                                const mt_tensor* cos, const mt_tensor* sin, const mt_tensor* yq, const mt_tensor* yk,
                                float eps, uint32_t flags, hipStream_t stream);
mt_status qk_norm_rope_bwd_impl(const mt_tensor* q, const mt_tensor* k, const mt_tensor* wq, const mt_tensor* wk,
                                const mt_tensor* cos, const mt_tensor* sin, const mt_tensor* dyq, const mt_tensor* dyk,
                                const mt_tensor* dq, const mt_tensor* dk, const mt_tensor* dwq, const mt_tensor* dwk,
                                float eps, uint32_t flags, void* ws, size_t ws_bytes, hipStream_t stream,
                                size_t* ws_query);
mt_status dropout_impl(const mt_tensor* x, const mt_tensor* residual, float p, uint64_t seed, uint64_t offset,
                       const mt_tensor* y, uint32_t flags, bool backward, hipStream_t stream);

}  // namespace mt::host
