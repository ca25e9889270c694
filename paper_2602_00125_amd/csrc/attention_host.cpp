// Argument validation and dispatch of attention, the head norms with rotation
// and dropout. Contracts: include/minitensor_hip.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "attention.hpp"
#include "host.hpp"
#include "kernels.hpp"

namespace mt::host {
namespace {

// [B, T, H, D] with contiguous vectors.
mt_status check_heads(const mt_tensor* t, const char* name) {
  mt_status s = check_tensor(t, name, 4, 4);
  if (s) return s;
  if (t->shape[3] > 1 && t->stride[3] != 1)
    return fail(MT_ERR_LAYOUT, std::string(name) + ": a head's vector must be contiguous");
  for (int i = 0; i < 4; ++i)
    if (t->shape[i] > INT32_MAX / 2) return fail(MT_ERR_SHAPE, std::string(name) + ": size beyond 2^30");
  return MT_OK;
}

mt_status same_heads(const mt_tensor* t, const char* name, const mt_tensor* like, const char* like_name) {
  for (int i = 0; i < 4; ++i)
    if (t->shape[i] != like->shape[i])
      return fail(MT_ERR_SHAPE, std::string(name) + " must have the shape of " + like_name);
  return MT_OK;
}

// An output addresses every element once: by ascending stride, each dim steps
// past what the smaller ones span.
mt_status check_out_heads(const mt_tensor* t, const char* name) {
  int dims[3] = {0, 1, 2};
  std::sort(dims, dims + 3, [&](int a, int b) { return t->stride[a] < t->stride[b]; });
  int64_t span = t->shape[3];
  if (numel(t) == 0) return MT_OK;
  for (int d : dims) {
    if (t->shape[d] <= 1) continue;
    if (t->stride[d] < span) return fail(MT_ERR_LAYOUT, std::string(name) + ": elements overlap");
    span += t->stride[d] * (t->shape[d] - 1);
  }
  return MT_OK;
}

// Whether two [B, T, H, D] views may share an element. Views of one packed
// buffer have overlapping ranges but no common element. Over the first `dims`
// dims, with equal sizes and pitches, the larger pitches multiples of the
// smallest, only the places within that one count: 2 dims for queries, keys and
// values side by side in each token's row, 3 for those of each head.
bool apart_within_pitch(const mt_tensor* a, const mt_tensor* b, int dims) {
  auto inner_bytes = [&](const mt_tensor* t) {  // what the other dims span
    return ((dims < 3 ? (t->shape[2] - 1) * t->stride[2] : 0) + t->shape[3]) * (int64_t)elem_size(t->dtype);
  };
  auto pitch = [](const mt_tensor* t, int d) { return t->stride[d] * (int64_t)elem_size(t->dtype); };
  int64_t p = 0;
  for (int d = 0; d < dims; ++d) {
    if (a->shape[d] != b->shape[d]) return false;
    if (a->shape[d] > 1 && (p == 0 || pitch(a, d) < p)) p = pitch(a, d);
  }
  if (p == 0) return false;
  for (int d = 0; d < dims; ++d)
    if (a->shape[d] > 1 && (pitch(a, d) != pitch(b, d) || pitch(a, d) % p)) return false;
  int64_t at = ((int64_t)((uintptr_t)b->data - (uintptr_t)a->data)) % p;  // b's place within a's pitch
  if (at < 0) at += p;
  return inner_bytes(a) <= at && at + inner_bytes(b) <= p;
}
bool heads_overlap(const mt_tensor* a, const mt_tensor* b) {
  return overlaps(a, b) && !apart_within_pitch(a, b, 2) && !apart_within_pitch(a, b, 3);
}

// The outputs against the inputs and one another (nulls are skipped).
mt_status check_apart(const mt_tensor* const* outs, const char* const* names, int n, const mt_tensor* const* ins, int m,
                      bool (*over)(const mt_tensor*, const mt_tensor*)) {
  for (int i = 0; i < n; ++i) {
    if (!outs[i]) continue;
    bool bad = false;
    for (int j = 0; j < m && !bad; ++j) bad = ins[j] && over(outs[i], ins[j]);
    for (int j = 0; j < i && !bad; ++j) bad = outs[j] && over(outs[i], outs[j]);
    if (bad) return fail(MT_ERR_ALIAS, std::string(names[i]) + " overlaps an input or another output");
  }
  return MT_OK;
}
// heads_overlap where both are [B, T, H, D], byte ranges elsewhere
bool any_overlap(const mt_tensor* a, const mt_tensor* b) {
  return a->ndim == 4 && b->ndim == 4 ? heads_overlap(a, b) : overlaps(a, b);
}

mt_status check_index(const mt_tensor* t, const char* name, int64_t n) {
  if (t->ndim != 1) return fail(MT_ERR_NDIM, std::string(name) + ": must have rank 1");
  if (t->dtype != MT_I32) return fail(MT_ERR_DTYPE, std::string(name) + ": must be i32");
  if (t->shape[0] != n) return fail(MT_ERR_SHAPE, std::string(name) + ": one value a batch element");
  if (n > 1 && t->stride[0] != 1) return fail(MT_ERR_LAYOUT, std::string(name) + ": must be contiguous");
  if (n > 0 && !t->data) return fail(MT_ERR_NULL, std::string(name) + ": null data pointer");
  return MT_OK;
}

// Byte range of an index tensor (check_tensor's dtypes do not hold it).
bool index_overlaps(const mt_tensor* out, const mt_tensor* idx) {
  if (!out || !idx) return false;
  mt_tensor t = *idx;
  t.dtype = MT_F32;  // the same four bytes an element
  return overlaps(out, &t);
}

HeadView view(const mt_tensor* t) {
  return t ? HeadView{t->data, t->stride[0], t->stride[1], t->stride[2]} : HeadView{nullptr, 0, 0, 0};
}

// Whether a view allows accesses of `bytes` at a time (a power of two, at most 16).
bool vector_ok(const mt_tensor* t, int bytes) {
  if (!t) return true;
  const int64_t es = (int64_t)elem_size(t->dtype);
  if ((uintptr_t)t->data & (bytes - 1) || t->shape[t->ndim - 1] * es % bytes) return false;
  for (int i = 0; i + 1 < t->ndim; ++i)
    if (t->shape[i] > 1 && t->stride[i] * es % bytes) return false;
  return true;
}

// ---------------------------------------------------------------- attention
// A launch has fewer than 2^32 threads, blocks up to 512.
constexpr int64_t kMostBlocks = (1 << 23) - 8;

struct AttnArgs {
  const mt_tensor *q, *k, *v, *kv_len, *q_start, *o, *lse;
};

mt_status check_attention(const AttnArgs& a, float scale, mt::AttnParams* p) {
  mt_status s;
  if ((s = check_heads(a.q, "q")) || (s = check_heads(a.k, "k")) || (s = check_heads(a.v, "v"))) return s;
  if (a.k->dtype != a.q->dtype || a.v->dtype != a.q->dtype) return fail(MT_ERR_DTYPE, "q, k and v must share a dtype");
  const int64_t B = a.q->shape[0], TQ = a.q->shape[1], HQ = a.q->shape[2], D = a.q->shape[3];
  const int64_t TK = a.k->shape[1], HK = a.k->shape[2];
  if (a.k->shape[0] != B || a.k->shape[3] != D) return fail(MT_ERR_SHAPE, "k must be [B, TK, HK, D] with q [B, TQ, HQ, D]");
  if ((s = same_heads(a.v, "v", a.k, "k"))) return s;
  if (D < 1 || D > mt::kAttnMaxD) return fail(MT_ERR_SHAPE, "the head width must be 1 to 128");
  if (HK > 0 ? HQ % HK != 0 : HQ != 0) return fail(MT_ERR_SHAPE, "the query heads must be a multiple of the key heads");
  // Past these lse / scale (what the dk / dv pass starts its sums from; lse is 22
  // at most more than the largest score) or scale log2(e) might not be finite
  if (!(scale >= 0x1p-100f && scale <= 0x1p100f)) return fail(MT_ERR_INVALID, "scale must lie in 2^-100 .. 2^100");
  if (a.kv_len && (s = check_index(a.kv_len, "kv_len", B))) return s;
  if (a.q_start && (s = check_index(a.q_start, "q_start", B))) return s;
  if (B * HQ > kMostBlocks || B * HK > kMostBlocks || B * HQ * cdiv(TQ, mt::kAttnRows) > kMostBlocks ||
      B * HK * cdiv(TK, mt::kAttnRows) > kMostBlocks)
    return fail(MT_ERR_SHAPE, "too many blocks of tokens and heads");
  *p = mt::AttnParams{};
  p->q = view(a.q);
  p->k = view(a.k);
  p->v = view(a.v);
  p->o = view(a.o);
  p->lse = a.lse ? (float*)a.lse->data : nullptr;
  p->kv_len = a.kv_len ? (const int32_t*)a.kv_len->data : nullptr;
  p->q_start = a.q_start ? (const int32_t*)a.q_start->data : nullptr;
  p->B = (int32_t)B;
  p->TQ = (int32_t)TQ;
  p->TK = (int32_t)TK;
  p->HQ = (int32_t)HQ;
  p->HK = (int32_t)HK;
  p->G = HK > 0 ? (int32_t)(HQ / HK) : 1;
  p->D = (int32_t)D;
  p->scale = scale;
  p->scale_log2 = scale * 1.4426950408889634f;
  p->splits = 1;
  return MT_OK;
}

mt_status check_lse(const mt_tensor* lse, const mt_tensor* q) {
  mt_status s = check_tensor(lse, "lse", 3, 3);
  if (s) return s;
  if (lse->dtype != MT_F32) return fail(MT_ERR_DTYPE, "lse must be f32");
  if (lse->shape[0] != q->shape[0] || lse->shape[1] != q->shape[2] || lse->shape[2] != q->shape[1])
    return fail(MT_ERR_SHAPE, "lse must be [B, HQ, TQ]");
  if (numel(lse) > 0 && !is_row_major(lse)) return fail(MT_ERR_LAYOUT, "lse must be contiguous");
  return MT_OK;
}

// 16-byte accesses, and token pitches that 32-bit offsets within a tile reach.
bool attn_vector_ok(const mt_tensor* const* ts, int n) {
  if (g_force_vec1) return false;
  for (int i = 0; i < n; ++i)
    if (ts[i] && (!vector_ok(ts[i], 16) || (ts[i]->shape[1] > 1 && ts[i]->stride[1] > (1 << 21)))) return false;
  return true;
}

// The most shares of the keys that the split forward can launch (0: not even
// one): its blocks hold 32 queries, and more than one meet in a join of a block
// of 256 threads a query and head.
int most_attn_splits(const mt::AttnParams& p) {
  const int64_t blocks = (int64_t)p.B * p.HK * cdiv((int64_t)p.G * p.TQ, 32);
  if (blocks > kMostBlocks) return 0;
  return (int64_t)p.B * p.HQ * p.TQ < 1 << 24 ? (int)std::min<int64_t>(64, kMostBlocks / blocks) : 1;
}

// Shares of the keys for the split forward, 0 for the forward by blocks of 128
// queries: whichever is estimated shorter, in us a key from what was measured
// (bf16 / fp32, heads of up to 64 / 128; one block a CU, then two):
//   by blocks of 128: 8 x 500 queries, 16 heads, 2000 keys, bf16: 81 us against
//   217 split; 2 x 400, 12 heads of 96: 11.4 against 14.4;
//   split: 1 query, 32 heads, 16384 keys, bf16: 21 us (32 shares) against 358;
//   16 x 1 query, 32 over 8 heads, 4096 keys, fp32: 110 us (2 shares) against
//   757; 1 x 2000, 8 heads, fp32: 131 (1 share) against 163.
int choose_attn_splits(const mt::AttnParams& p, bool bf16) {
  const int most = most_attn_splits(p);
  if (const int fs = g_attn_splits; fs >= 0) return std::min(fs, most);
  const int64_t whole = (int64_t)p.B * p.HQ * cdiv(p.TQ, mt::kAttnRows);
  if (whole > 512 && p.TQ > 32) return 0;
  const int64_t blocks = (int64_t)p.B * p.HK * cdiv((int64_t)p.G * p.TQ, 32);
  const bool wide = p.D > 64;
  const double one = bf16 ? (wide ? 0.0165 : 0.012) : (wide ? 0.08 : 0.0445);
  const double round = bf16 ? (wide ? 0.0106 : 0.0117) : (wide ? 0.043 : 0.0245);
  const int64_t slots = bf16 && !wide ? 512 : 256;  // blocks at a time, by their LDS
  // Causal blocks of unequal length fill rounds after the first better: 1 x 626,
  // 16 heads of 128, fp32: 42 us against 56 without this factor; 3 x 410, 12 over
  // 4: 47 against 38; over 40 drawn sizes that it decides, 1.03 times. (Lengths
  // in kv_len, which may all be full, count for nothing: a factor of 0.88 for
  // them made 100 drawn sizes that it decided 1.12 times as long where they were
  // full and 1.08 where they were a quarter to all of the keys.)
  const double later = p.causal ? 1.0 - 0.25 * std::min(1.0, (double)p.TQ / std::max(p.TK, 1)) : 1.0;
  double best = 4.0 + p.TK * one *
                          (whole <= 256 ? 1.0 : later * (!bf16 && wide ? cdiv(whole, 256) : 1.7 * cdiv(whole, 512)));
  int splits = 0;
  // what the shares of every row write and the join reads, at 4 TB/s
  const double bytes = 8.0 * p.B * p.HQ * p.TQ * (p.D + 2) / 4e6;
  // a share holds a tile of 32 keys a wave
  for (int s = 1; s <= most && (s == 1 || s * 128 <= p.TK); ++s) {
    const double join = s > 1 ? 3.0 + (0.12 + bytes) * s : 0.0;
    const int64_t rounds = cdiv(blocks * s, slots);
    const double t = rounds * (5.0 + p.TK * round / s) * (rounds > 1 ? later : 1.0) + join;
    if (t < best) {
      best = t;
      splits = s;
    }
  }
  return splits;
}

// Shares of the query tiles (of all heads of a key head) for the dk / dv pass,
// where its blocks are fewer than the CUs: whatever is estimated shortest, in us
// a tile and for the join. Gradients with one share and with those chosen:
//   1 x 2048, 8 heads over 1 of 128, bf16: 251 us against 86 (8 shares), fp32: 2327
//   against 365 (16); 1 x 512, 16 over 4 of 64, fp32: 158 against 62 (16); 1 x 71,
//   8 over 1 of 96, fp32: 98 against 33 (24); 4 x 512, 12 over 4 of 96, bf16: 42.5
//   against 43.1 (2), where the estimates meet.
int choose_dkv_splits(const mt::AttnParams& p, bool bf16) {
  const int keys = mt::attn_kv_block(p, bf16);
  const int64_t items = (int64_t)p.B * p.HK * cdiv(p.TK, keys);
  const int64_t tiles = p.G * cdiv(p.TQ, bf16 ? (keys == 64 ? 128 : 64) : p.D > 64 ? 32 : 64);
  const double tile = bf16 ? 1.8 : 3.5;
  // what a share of every key writes and the join reads, at 4 TB/s
  const double bytes = 16.0 * p.B * p.HK * p.TK * p.D / 4e6;
  double best = tiles * tile;
  int splits = 1;
  for (int64_t s = 2; s <= tiles && s * items <= 256; ++s) {
    const double t = cdiv(tiles, s) * tile + 4.0 + (0.1 + bytes) * s;
    if (t < best) {
      best = t;
      splits = (int)s;
    }
  }
  return splits;
}

}  // namespace

mt_status attention_fwd_impl(const mt_tensor* q, const mt_tensor* k, const mt_tensor* v, const mt_tensor* kv_len,
                             const mt_tensor* q_start, const mt_tensor* o, const mt_tensor* lse, float scale,
                             uint32_t flags, void* ws, size_t ws_bytes, hipStream_t stream, size_t* ws_query) {
  if (flags & ~MT_CAUSAL) return fail(MT_ERR_INVALID, "mt_attention_fwd: unknown flags");
  mt::AttnParams p;
  mt_status s = check_attention({q, k, v, kv_len, q_start, o, lse}, scale, &p);
  if (s) return s;
  if ((s = check_heads(o, "o")) || (s = same_heads(o, "o", q, "q")) || (s = check_out_heads(o, "o"))) return s;
  if (o->dtype != q->dtype) return fail(MT_ERR_DTYPE, "o must have q's dtype");
  if (lse && (s = check_lse(lse, q))) return s;
  const mt_tensor *outs[] = {o, lse}, *ins[] = {q, k, v};
  const char* names[] = {"o", "lse"};
  if ((s = check_apart(outs, names, 2, ins, 3, any_overlap))) return s;
  for (int i = 0; i < 2; ++i)
    if (index_overlaps(outs[i], kv_len) || index_overlaps(outs[i], q_start))
      return fail(MT_ERR_ALIAS, std::string(names[i]) + " overlaps kv_len or q_start");
  p.causal = (flags & MT_CAUSAL) != 0;
  const bool empty = p.B == 0 || p.TQ == 0 || p.HQ == 0;
  const int splits = empty ? 0 : choose_attn_splits(p, q->dtype == MT_BF16);
  const size_t need = splits > 1 ? (size_t)splits * p.B * p.HQ * p.TQ * (p.D + 2) * sizeof(float) : 0;
  if (ws_query) {
    *ws_query = need;
    return MT_OK;
  }
  if (ws && ((uintptr_t)ws & 255)) return fail(MT_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (empty) return MT_OK;
  p.splits = ws && ws_bytes >= need ? splits : std::min(splits, 1);
  p.part = (float*)ws;
  const mt_tensor* all[] = {q, k, v, o};
  const bool bf = q->dtype == MT_BF16, vec = attn_vector_ok(all, 4);
  (void)hipGetLastError();
  return hip_status(splits ? mt::attn_fwd_split(p, bf, vec, stream) : mt::attn_fwd(p, bf, vec, stream));
}

mt_status attention_bwd_impl(const mt_tensor* q, const mt_tensor* k, const mt_tensor* v, const mt_tensor* kv_len,
                             const mt_tensor* q_start, const mt_tensor* o, const mt_tensor* lse, const mt_tensor* dout,
                             const mt_tensor* dq, const mt_tensor* dk, const mt_tensor* dv, float scale, uint32_t flags,
                             void* ws, size_t ws_bytes, hipStream_t stream, size_t* ws_query) {
  if (flags & ~(MT_CAUSAL | MT_ACCUMULATE)) return fail(MT_ERR_INVALID, "mt_attention_bwd: unknown flags");
  mt::AttnParams p;
  mt_status s = check_attention({q, k, v, kv_len, q_start, o, lse}, scale, &p);
  if (s) return s;
  if ((s = check_heads(o, "o")) || (s = same_heads(o, "o", q, "q")) || (s = check_heads(dout, "dout")) ||
      (s = same_heads(dout, "dout", q, "q")) || (s = check_lse(lse, q)))
    return s;
  if (o->dtype != q->dtype || dout->dtype != q->dtype) return fail(MT_ERR_DTYPE, "o and dout must have q's dtype");
  const mt_tensor *outs[] = {dq, dk, dv}, *like[] = {q, k, k}, *ins[] = {q, k, v, o, lse, dout};
  const char *names[] = {"dq", "dk", "dv"}, *like_names[] = {"q", "k", "k"};
  if (!dq && !dk && !dv) return fail(MT_ERR_NULL, "no output requested");
  for (int i = 0; i < 3; ++i) {
    if (!outs[i]) continue;
    if ((s = check_heads(outs[i], names[i])) || (s = same_heads(outs[i], names[i], like[i], like_names[i])) ||
        (s = check_out_heads(outs[i], names[i])))
      return s;
    if (outs[i]->dtype != q->dtype) return fail(MT_ERR_DTYPE, std::string(names[i]) + " must have q's dtype");
    if (index_overlaps(outs[i], kv_len) || index_overlaps(outs[i], q_start))
      return fail(MT_ERR_ALIAS, std::string(names[i]) + " overlaps kv_len or q_start");
  }
  if ((s = check_apart(outs, names, 3, ins, 6, any_overlap))) return s;
  const size_t stats = (2 * (size_t)p.B * p.HQ * p.TQ * sizeof(float) + 255) / 256 * 256;
  const int splits = (dk || dv) && p.TK > 0 && stats > 0 ? choose_dkv_splits(p, q->dtype == MT_BF16) : 1;
  const size_t need = stats + (splits > 1 ? 2 * (size_t)splits * p.B * p.HK * p.TK * p.D * sizeof(float) : 0);
  if (ws_query) {
    *ws_query = need;
    return MT_OK;
  }
  if (ws && ((uintptr_t)ws & 255)) return fail(MT_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(MT_ERR_WORKSPACE, "mt_attention_bwd needs the workspace that mt_attention_bwd_workspace reports");
  if (p.B == 0) return MT_OK;
  p.dout = view(dout);
  p.dq = view(dq);
  p.dk = view(dk);
  p.dv = view(dv);
  p.delta = (float*)ws;
  p.causal = (flags & MT_CAUSAL) != 0;
  p.accumulate = (flags & MT_ACCUMULATE) != 0;
  p.with_dq = dq != nullptr;
  const mt_tensor* all[] = {q, k, v, o, dout, dq, dk, dv};
  const bool bf = q->dtype == MT_BF16, vec = attn_vector_ok(all, 8);
  (void)hipGetLastError();
  if (p.TQ > 0 && p.HQ > 0 && (s = hip_status(mt::attn_bwd_dq(p, bf, vec, stream)))) return s;
  p.splits = splits;
  p.part = (float*)((char*)ws + stats);
  // without queries too: dk and dv are empty sums then
  if ((dk || dv) && p.TK > 0 && p.HK > 0) return hip_status(mt::attn_bwd_dkv(p, bf, vec, stream));
  return MT_OK;
}

// ----------------------------------------------- head norms with rotation
namespace {

struct NormArgs {
  const mt_tensor *q, *k, *wq, *wk, *cos, *sin, *yq, *yk;  // y: the forward's y or the backward's dy
  const char *yq_name, *yk_name;
};

mt_status check_table(const mt_tensor* t, const char* name, int64_t B, int64_t T) {
  mt_status s = check_tensor(t, name, 3, 3);
  if (s) return s;
  if (t->dtype != MT_F32) return fail(MT_ERR_DTYPE, std::string(name) + ": must be f32");
  if (t->shape[0] != B || t->shape[1] != T)
    return fail(MT_ERR_SHAPE, std::string(name) + ": must be [B, T, R / 2] (a stride may be 0)");
  if (t->shape[2] > 1 && t->stride[2] != 1) return fail(MT_ERR_LAYOUT, std::string(name) + ": rows must be contiguous");
  return MT_OK;
}

mt_status check_norm(const NormArgs& a, float eps, uint32_t flags, mt::HeadNormParams* p) {
  mt_status s;
  if ((s = check_heads(a.q, "q")) || (s = check_heads(a.yq, a.yq_name)) || (s = same_heads(a.yq, a.yq_name, a.q, "q")))
    return s;
  if (!a.k != !a.yk) return fail(MT_ERR_NULL, std::string("k and ") + a.yk_name + " go together");
  if (!a.k && a.wk) return fail(MT_ERR_NULL, "wk is given without k");
  const int64_t B = a.q->shape[0], T = a.q->shape[1], D = a.q->shape[3];
  if (a.k) {
    if ((s = check_heads(a.k, "k")) || (s = check_heads(a.yk, a.yk_name)) ||
        (s = same_heads(a.yk, a.yk_name, a.k, "k")))
      return s;
    if (a.k->shape[0] != B || a.k->shape[1] != T || a.k->shape[3] != D)
      return fail(MT_ERR_SHAPE, "k must be [B, T, HK, D] with q [B, T, HQ, D]");
    if (a.k->dtype != a.q->dtype) return fail(MT_ERR_DTYPE, "q and k must share a dtype");
    if (a.yk->dtype != a.yq->dtype)
      return fail(MT_ERR_DTYPE, std::string(a.yq_name) + " and " + a.yk_name + " must share a dtype");
  }
  if (D < 1 || D > mt::kHeadNormMaxD) return fail(MT_ERR_SHAPE, "the head width must be 1 to 1024");
  if (a.wq && (s = check_vector(a.wq, "wq", D))) return s;
  if (a.wk && (s = check_vector(a.wk, "wk", D))) return s;
  if (!a.cos != !a.sin) return fail(MT_ERR_NULL, "cos and sin go together");
  int64_t R = 0;
  if (a.cos) {
    if ((s = check_table(a.cos, "cos", B, T)) || (s = check_table(a.sin, "sin", B, T))) return s;
    R = 2 * a.cos->shape[2];
    if (a.sin->shape[2] != a.cos->shape[2]) return fail(MT_ERR_SHAPE, "cos and sin must share a shape");
    if (R > D) return fail(MT_ERR_SHAPE, "the tables hold more pairs than a head has");
  }
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MT_ERR_INVALID, "eps must be finite and not negative");
  *p = mt::HeadNormParams{};
  p->q = view(a.q);
  p->k = view(a.k);
  p->wq = a.wq ? (const float*)a.wq->data : nullptr;
  p->wk = a.wk ? (const float*)a.wk->data : nullptr;
  if (a.cos) {
    p->cos = (const float*)a.cos->data;
    p->sin = (const float*)a.sin->data;
    p->cos_sb = a.cos->stride[0];
    p->cos_st = a.cos->stride[1];
    p->sin_sb = a.sin->stride[0];
    p->sin_st = a.sin->stride[1];
  }
  p->B = (int32_t)B;
  p->T = (int32_t)T;
  p->HQ = (int32_t)a.q->shape[2];
  p->HK = a.k ? (int32_t)a.k->shape[2] : 0;
  p->D = (int32_t)D;
  p->R = (int32_t)R;
  p->interleaved = (flags & MT_ROPE_INTERLEAVED) != 0;
  p->eps = eps;
  p->inv_D = 1.f / (float)D;
  if ((int64_t)p->HQ + p->HK > INT32_MAX / 2 || B * T > INT32_MAX / 2 || B * T * (p->HQ + p->HK) > INT32_MAX / 2)
    return fail(MT_ERR_SHAPE, "too many rows");
  return MT_OK;
}

// Values a lane: 8 where a bf16 row allows it (16 bytes), else 4, else by
// element. A lane's values lie in one half of the rotated pairs.
int norm_vector(mt::HeadNormParams* p, const mt_tensor* const* ts, int n) {
  bool bf = false;
  for (int i = 0; i < n; ++i) bf = bf || (ts[i] && ts[i]->dtype == MT_BF16);
  for (int vec = bf ? 8 : 4; vec >= 4 && !g_force_vec1; vec -= 4) {
    bool ok = p->D % vec == 0 && p->D <= 64 * vec && (p->interleaved || (p->R / 2) % vec == 0) &&
              aligned16(p->wq) && aligned16(p->wk);
    for (int i = 0; i < n && ok; ++i)
      ok = !ts[i] || vector_ok(ts[i], std::min<int>(16, vec * (int)elem_size(ts[i]->dtype)));
    if (!ok) continue;
    for (p->L = 1, p->L_shift = 0; p->L * vec < p->D; p->L *= 2) ++p->L_shift;
    return vec;
  }
  return 0;
}

// Blocks of the backward: at most four a CU; each holds partial sums of dw.
constexpr int kNormBlocks = 1024;

}  // namespace

mt_status qk_norm_rope_fwd_impl(const mt_tensor* q, const mt_tensor* k, const mt_tensor* wq, const mt_tensor* wk,
                                const mt_tensor* cos, const mt_tensor* sin, const mt_tensor* yq, const mt_tensor* yk,
                                float eps, uint32_t flags, hipStream_t stream) {
  if (flags & ~MT_ROPE_INTERLEAVED) return fail(MT_ERR_INVALID, "mt_qk_norm_rope_fwd: unknown flags");
  mt::HeadNormParams p;
  mt_status s = check_norm({q, k, wq, wk, cos, sin, yq, yk, "yq", "yk"}, eps, flags, &p);
  if (s) return s;
  if ((s = check_out_heads(yq, "yq")) || (yk && (s = check_out_heads(yk, "yk")))) return s;
  const mt_tensor *outs[] = {yq, yk}, *ins[] = {q, k, wq, wk, cos, sin};
  const char* names[] = {"yq", "yk"};
  if ((s = check_apart(outs, names, 2, ins, 6, any_overlap))) return s;
  const int64_t rows = (int64_t)p.B * p.T * (p.HQ + p.HK);
  if (rows == 0) return MT_OK;
  p.yq = view(yq);
  p.yk = view(yk);
  const mt_tensor* all[] = {q, k, yq, yk};
  const int vec = norm_vector(&p, all, 4);
  // Four heads a group of lanes share the tables' row and keep four loads in
  // flight, where that still leaves each CU two blocks
  const int hpg = vec && rows / 4 >= 512 * (256 >> p.L_shift) ? 4 : 1;
  (void)hipGetLastError();
  return hip_status(mt::head_norm_fwd(p, q->dtype == MT_BF16, yq->dtype == MT_BF16, vec, hpg, stream));
}

mt_status qk_norm_rope_bwd_impl(const mt_tensor* q, const mt_tensor* k, const mt_tensor* wq, const mt_tensor* wk,
                                const mt_tensor* cos, const mt_tensor* sin, const mt_tensor* dyq, const mt_tensor* dyk,
                                const mt_tensor* dq, const mt_tensor* dk, const mt_tensor* dwq, const mt_tensor* dwk,
                                float eps, uint32_t flags, void* ws, size_t ws_bytes, hipStream_t stream,
                                size_t* ws_query) {
  if (flags & ~(MT_ROPE_INTERLEAVED | MT_ACCUMULATE)) return fail(MT_ERR_INVALID, "mt_qk_norm_rope_bwd: unknown flags");
  mt::HeadNormParams p;
  mt_status s = check_norm({q, k, wq, wk, cos, sin, dyq, dyk, "dyq", "dyk"}, eps, flags, &p);
  if (s) return s;
  if (!dq && !dk && !dwq && !dwk) return fail(MT_ERR_NULL, "no output requested");
  if (!k && (dk || dwk)) return fail(MT_ERR_NULL, "dk or dwk is given without k");
  if (k && !dq != !dk) return fail(MT_ERR_NULL, "dq and dk go together");
  const mt_tensor *outs[] = {dq, dk, dwq, dwk}, *like[] = {q, k}, *ins[] = {q, k, wq, wk, cos, sin, dyq, dyk};
  const char *names[] = {"dq", "dk", "dwq", "dwk"}, *like_names[] = {"q", "k"};
  for (int i = 0; i < 2; ++i) {
    if (!outs[i]) continue;
    if ((s = check_heads(outs[i], names[i])) || (s = same_heads(outs[i], names[i], like[i], like_names[i])) ||
        (s = check_out_heads(outs[i], names[i])))
      return s;
    if (outs[i]->dtype != dyq->dtype) return fail(MT_ERR_DTYPE, std::string(names[i]) + " must have dyq's dtype");
  }
  for (int i = 2; i < 4; ++i)
    if (outs[i] && (s = check_vector(outs[i], names[i], p.D))) return s;
  if ((s = check_apart(outs, names, 4, ins, 8, any_overlap))) return s;
  const mt_tensor* all[] = {q, k, dyq, dyk, dq, dk};
  const int vec = norm_vector(&p, all, 6);
  const int64_t rows = (int64_t)p.B * p.T * (p.HQ + p.HK);
  const int64_t per = vec ? 2 * (256 >> p.L_shift) : 4;  // rows a block takes at a time
  const int blocks = (int)std::min<int64_t>(kNormBlocks, std::max<int64_t>(1, cdiv(rows, per)));
  const bool weights = dwq || dwk;
  const size_t one = 2 * (size_t)p.D * sizeof(float), need = weights ? blocks * one : 0;
  if (ws_query) {
    *ws_query = need;
    return MT_OK;
  }
  if (ws && ((uintptr_t)ws & 255)) return fail(MT_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (weights && (!ws || ws_bytes < need))
    return fail(MT_ERR_WORKSPACE, "dwq and dwk need the workspace that mt_qk_norm_rope_bwd_workspace reports");
  p.dyq = view(dyq);
  p.dyk = view(dyk);
  p.yq = view(dq);
  p.yk = view(dk);
  p.with_dx = dq != nullptr;
  p.accumulate = (flags & MT_ACCUMULATE) != 0;
  p.part = weights ? (float*)ws : nullptr;
  (void)hipGetLastError();
  if ((rows > 0 || weights) &&
      (s = hip_status(mt::head_norm_bwd(p, q->dtype == MT_BF16, dyq->dtype == MT_BF16, vec, blocks, stream))))
    return s;
  if (!weights) return MT_OK;
  return hip_status(mt::head_norm_finish(p.part, blocks, p.D, dwq ? (float*)dwq->data : nullptr,
                                         dwk ? (float*)dwk->data : nullptr, p.accumulate, stream));
}

// ------------------------------------------------------------------ dropout
mt_status dropout_impl(const mt_tensor* x, const mt_tensor* residual, float p, uint64_t seed, uint64_t offset,
                       const mt_tensor* y, uint32_t flags, bool backward, hipStream_t stream) {
  const char *xn = backward ? "dy" : "x", *yn = backward ? "dx" : "y";
  if (flags & ~(backward ? MT_ACCUMULATE : 0u)) return fail(MT_ERR_INVALID, "mt_dropout: unknown flags");
  mt_status s;
  auto matrix = [&](const mt_tensor* t, const char* name) {
    if ((s = check_tensor(t, name, 2, 2))) return s;
    if (t->shape[1] > 1 && t->stride[1] != 1)
      return fail(MT_ERR_LAYOUT, std::string(name) + ": inner dimension must be contiguous");
    if (x && (t->shape[0] != x->shape[0] || t->shape[1] != x->shape[1]))
      return fail(MT_ERR_SHAPE, std::string(name) + " must have the shape of " + xn);
    return MT_OK;
  };
  if ((s = matrix(x, xn)) || (s = matrix(y, yn)) || (residual && (s = matrix(residual, "residual")))) return s;
  if (residual && residual->dtype != y->dtype) return fail(MT_ERR_DTYPE, "residual must have y's dtype");
  if (y->shape[0] > 1 && y->stride[0] < y->shape[1])
    return fail(MT_ERR_LAYOUT, std::string(yn) + ": rows overlap (row pitch < columns)");
  if (!(p >= 0.f && p <= 1.f)) return fail(MT_ERR_INVALID, "p must lie in 0 .. 1");
  if (overlaps(y, x) || overlaps(y, residual))
    return fail(MT_ERR_ALIAS, std::string(yn) + " overlaps an input");
  const int64_t M = x->shape[0], N = x->shape[1];
  if (M == 0 || N == 0) return MT_OK;
  mt::DropoutParams d{};
  const mt_tensor* res = flags & MT_ACCUMULATE ? y : residual;  // dx += : the sum's other term is dx itself
  auto pitch = [&](const mt_tensor* t) { return M > 1 ? t->stride[0] : N; };
  d.x = x->data;
  d.y = y->data;
  d.res = res ? res->data : nullptr;
  d.M = M;
  d.N = N;
  d.ldx = pitch(x);
  d.ldy = pitch(y);
  d.ldr = res ? pitch(res) : N;
  bool vec = aligned16(d.x) && aligned16(d.y) && (!d.res || aligned16(d.res)) && !g_force_vec1;
  if (d.ldx == N && d.ldy == N && d.ldr == N) {  // no gaps: one flat row
    d.M = 1;
    d.N = M * N;
  } else {
    vec = vec && N % 8 == 0 && d.ldx % 8 == 0 && d.ldy % 8 == 0 && d.ldr % 8 == 0;
  }
  d.seed = seed;
  d.offset = offset;
  d.drop = (uint32_t)std::lround(p * 65536.f);
  d.scale = d.drop < 65536 ? (float)(65536.0 / (65536 - d.drop)) : 0.f;
  (void)hipGetLastError();
  return hip_status(mt::dropout_run(d, x->dtype == MT_BF16, y->dtype == MT_BF16, vec, stream));
}

}  // namespace mt::host
