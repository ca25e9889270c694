// Argument validation and dispatch of the embedding, the layer norm, the
// cross-entropy loss and the clipping of gradients. Contracts:
// include/minitensor_hip.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "host.hpp"
#include "language.hpp"

namespace mt::host {
namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;

// Rank 1 or 2, any strides: tokens or classes.
mt_status check_ids(const mt_tensor* t, const char* name, mt::vio::Index* out, int64_t* count) {
  if (!t) return fail(MT_ERR_NULL, std::string(name) + ": null tensor descriptor");
  if (t->ndim < 1 || t->ndim > 2) return fail(MT_ERR_NDIM, std::string(name) + ": must have rank 1 or 2");
  if (t->dtype != MT_I32) return fail(MT_ERR_DTYPE, std::string(name) + ": must be i32");
  for (int i = 0; i < t->ndim; ++i) {
    if (t->shape[i] < 0) return fail(MT_ERR_SHAPE, std::string(name) + ": negative size");
    if (t->shape[i] > kMostRows) return fail(MT_ERR_SHAPE, std::string(name) + ": size beyond 2^30");
    if (t->stride[i] < 0) return fail(MT_ERR_LAYOUT, std::string(name) + ": negative stride");
  }
  const int64_t n = numel(t);
  if (n > kMostRows) return fail(MT_ERR_SHAPE, std::string(name) + ": more than 2^30 values");
  if (n > 0 && !t->data) return fail(MT_ERR_NULL, std::string(name) + ": null data pointer");
  *count = n;
  const int64_t inner = t->shape[t->ndim - 1], s1 = t->stride[t->ndim - 1], s0 = t->ndim > 1 ? t->stride[0] : 0;
  const bool rows = t->ndim > 1 && t->shape[0] > 1, flat = (inner <= 1 || s1 == 1) && (!rows || s0 == inner);
  *out = mt::vio::Index{(const int32_t*)t->data, flat ? 0 : inner, s0, s1};
  return MT_OK;
}

// [rows, columns], the columns contiguous; `out`: rows apart.
mt_status check_rows(const mt_tensor* t, const char* name, bool out) {
  mt_status s = check_tensor(t, name, 2, 2);
  if (s) return s;
  if (t->shape[1] > 1 && t->stride[1] != 1)
    return fail(MT_ERR_LAYOUT, std::string(name) + ": inner dimension must be contiguous");
  if (t->shape[0] > kMostRows) return fail(MT_ERR_SHAPE, std::string(name) + ": more than 2^30 rows");
  if (out && t->shape[0] > 1 && t->stride[0] < t->shape[1])
    return fail(MT_ERR_LAYOUT, std::string(name) + ": rows overlap (row pitch < columns)");
  return MT_OK;
}
int64_t row_pitch(const mt_tensor* t) { return t->shape[0] > 1 ? t->stride[0] : t->shape[1]; }

// Byte ranges; tokens and classes have four bytes an element too.
bool apart(const mt_tensor* a, const mt_tensor* b) {
  if (!a || !b) return true;
  mt_tensor x = *a, y = *b;
  if (x.dtype == MT_I32) x.dtype = MT_F32;
  if (y.dtype == MT_I32) y.dtype = MT_F32;
  return !overlaps(&x, &y);
}
mt_status check_apart(std::initializer_list<const mt_tensor*> outs, std::initializer_list<const mt_tensor*> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (const mt_tensor* i : ins)
      if (!apart(*o, i)) return fail(MT_ERR_ALIAS, "an output overlaps an input");
    for (auto q = outs.begin(); q != o; ++q)
      if (!apart(*o, *q)) return fail(MT_ERR_ALIAS, "two outputs overlap");
  }
  return MT_OK;
}

mt_status check_workspace(const void* ws, size_t ws_bytes, size_t need, const char* who) {
  if (ws && ((uintptr_t)ws & 255)) return fail(MT_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (need > 0 && (!ws || ws_bytes < need))
    return fail(MT_ERR_WORKSPACE, std::string(who) + " needs the workspace that its _workspace call reports");
  return MT_OK;
}

// Values of a lane's group: 16 bytes of the narrower type.
int vector_of(std::initializer_list<const mt_tensor*> ts) {
  for (const mt_tensor* t : ts)
    if (t && t->dtype == MT_BF16) return 8;
  return 4;
}

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

// ---------------------------------------------------------------- embedding
mt_status embedding_fwd_impl(const mt_tensor* ids, const mt_tensor* table, float scale, const mt_tensor* y,
                             hipStream_t stream) {
  mt::EmbeddingParams p{};
  mt_status s;
  if ((s = check_ids(ids, "ids", &p.ids, &p.M)) || (s = check_rows(table, "table", false)) ||
      (s = check_rows(y, "y", true)))
    return s;
  p.V = table->shape[0];
  p.D = table->shape[1];
  if (y->shape[0] != p.M || y->shape[1] != p.D) return fail(MT_ERR_SHAPE, "y must be [tokens, D] with table [V, D]");
  if (p.D > (1 << 20)) return fail(MT_ERR_SHAPE, "rows of more than 2^20 values");
  if (!std::isfinite(scale)) return fail(MT_ERR_INVALID, "scale must be finite");
  if ((s = check_apart({y}, {ids, table}))) return s;
  if (p.M == 0 || p.D == 0) return MT_OK;
  p.table = table->data;
  p.y = y->data;
  p.ldt = row_pitch(table);
  p.ldy = row_pitch(y);
  p.scale = scale;
  (void)hipGetLastError();
  return hip_status(mt::embedding_fwd(p, table->dtype == MT_BF16, y->dtype == MT_BF16, stream));
}

mt_status embedding_bwd_impl(const mt_tensor* ids, const mt_tensor* dy, float scale, const mt_tensor* dtable,
                             uint32_t flags, void* ws, size_t ws_bytes, hipStream_t stream, size_t* ws_query) {
  if (flags & ~MT_ACCUMULATE) return fail(MT_ERR_INVALID, "mt_embedding_bwd: unknown flags");
  mt::EmbeddingGradParams p{};
  mt_status s;
  if ((s = check_ids(ids, "ids", &p.ids, &p.M)) || (s = check_rows(dy, "dy", false)) ||
      (s = check_rows(dtable, "dtable", true)))
    return s;
  if (dtable->dtype != MT_F32) return fail(MT_ERR_DTYPE, "dtable must be f32");
  p.V = dtable->shape[0];
  p.D = dtable->shape[1];
  if (dy->shape[0] != p.M || dy->shape[1] != p.D)
    return fail(MT_ERR_SHAPE, "dy must be [tokens, D] with dtable [V, D]");
  if (p.D > (1 << 20)) return fail(MT_ERR_SHAPE, "rows of more than 2^20 values");
  if (p.V > (1 << 24)) return fail(MT_ERR_SHAPE, "more than 2^24 rows of dtable");
  if (p.M > (1 << 26)) return fail(MT_ERR_SHAPE, "more than 2^26 tokens");
  if (!std::isfinite(scale)) return fail(MT_ERR_INVALID, "scale must be finite");
  if ((s = check_apart({dtable}, {ids, dy}))) return s;
  const mt::EmbeddingGradForm f = mt::embedding_grad_form(p.M, p.D);
  p.chunk = f.chunk;
  const size_t list = round256(p.M * sizeof(int32_t)), sums = round256((size_t)f.chunks * p.D * sizeof(float));
  const size_t need = p.V && p.D ? 2 * list + 2 * sums + round256(p.V) : 0;
  if (ws_query) {
    *ws_query = need;
    return MT_OK;
  }
  if ((s = check_workspace(ws, ws_bytes, need, "mt_embedding_bwd"))) return s;
  if (p.V == 0 || p.D == 0) return MT_OK;
  char* at = (char*)ws;
  p.id = (int32_t*)at;
  p.pos = (int32_t*)(at += list);
  p.head = (float*)(at += list);
  p.tail = (float*)(at += sums);
  p.seen = (uint8_t*)(at += sums);
  p.dy = dy->data;
  p.dtable = (float*)dtable->data;
  p.ldy = row_pitch(dy);
  p.ldt = row_pitch(dtable);
  p.scale = scale;
  p.accumulate = (flags & MT_ACCUMULATE) != 0;
  // buckets of 256 blocks, or as many as leave a bucket no more ids than it has counters for
  while (p.bucket_shift < 8 && (int64_t)1 << p.bucket_shift < p.V) ++p.bucket_shift;
  while (p.V > (int64_t)mt::kEmbedBucketIds << p.bucket_shift) ++p.bucket_shift;
  (void)hipGetLastError();
  return hip_status(mt::embedding_bwd(p, f, dy->dtype == MT_BF16, stream));
}

// --------------------------------------------------------------- layer norm
namespace {

mt_status check_norm(const mt_tensor* x, const mt_tensor* w, float eps, mt::LayerNormParams* p) {
  mt_status s = check_rows(x, "x", false);
  if (s) return s;
  const int64_t C = x->shape[1];
  if (C < 1 || C > mt::kLayerNormMaxC) return fail(MT_ERR_SHAPE, "a row must have 1 to 16384 values");
  if (w && (s = check_vector(w, "w", C))) return s;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MT_ERR_INVALID, "eps must be finite and not negative");
  *p = mt::LayerNormParams{};
  p->x = x->data;
  p->w = w ? (const float*)w->data : nullptr;
  p->M = x->shape[0];
  p->C = (int32_t)C;
  p->ldx = row_pitch(x);
  p->eps = eps;
  p->C_f = (float)C;
  p->inv_C = 1.f / (float)C;
  return MT_OK;
}

mt_status like(const mt_tensor* t, const char* name, const mt_tensor* x, bool out) {
  mt_status s = check_rows(t, name, out);
  if (s) return s;
  if (t->shape[0] != x->shape[0] || t->shape[1] != x->shape[1])
    return fail(MT_ERR_SHAPE, std::string(name) + " must have the shape of x");
  return MT_OK;
}

// How a row is held: L lanes with nv groups of vec values, blocks of `threads`.
struct NormForm {
  int nv, threads, blocks;
};
NormForm norm_form(mt::LayerNormParams* p, int vec, int values, int threads, int most_blocks) {
  NormForm f{1, threads, 1};
  const int most = values / vec;  // groups a lane
  for (p->L = 1; p->L < 64 && p->L * vec * most < p->C;) p->L *= 2;
  if (p->L * vec * most < p->C) {
    // as few whole waves as hold a row (13107 x 2560 bf16 40 us by four, 29 by three; 2730 x 12288 46 by 16, 36 by
    // 12), but eight rather than six or seven (5461 x 6144 34 us by eight, 35 by six)
    int waves = (int)cdiv(p->C, (int64_t)64 * vec * most);
    if (waves == 6 || waves == 7) waves = 8;
    p->L = 64 * waves;
  }
  f.nv = (int)cdiv(p->C, (int64_t)p->L * vec);
  const int rows = std::max(1, threads / p->L);
  f.threads = rows * p->L;
  f.blocks = (int)std::min<int64_t>(most_blocks, std::max<int64_t>(1, cdiv(p->M, rows)));
  return f;
}

}  // namespace

mt_status layer_norm_fwd_impl(const mt_tensor* x, const mt_tensor* w, const mt_tensor* b, float eps,
                              const mt_tensor* y, hipStream_t stream) {
  mt::LayerNormParams p;
  mt_status s;
  if ((s = check_norm(x, w, eps, &p)) || (b && (s = check_vector(b, "b", p.C))) || (s = like(y, "y", x, true)) ||
      (s = check_apart({y}, {x, w, b})))
    return s;
  if (p.M == 0) return MT_OK;
  p.b = b ? (const float*)b->data : nullptr;
  p.out = y->data;
  p.ldo = row_pitch(y);
  // 16 values a lane, or 8 where that takes a part of a wave, three, four or eight waves (524288 x 64 bf16 37 -> 28
  // us, 21845 x 1536 37 -> 31, 8192 x 4096 33 -> 29; by five waves 13107 x 2560 29 -> 32)
  const int waves = (int)cdiv(p.C, 512);
  const int values = p.C <= 512 || waves == 3 || waves == 4 || waves == 8 ? 8 : 16;
  // eight blocks a CU, or seven of the forms of 512 to 1024 columns, whose registers have room for no more: of eight the
  // last would run alone (32768 x 1024 bf16 31 -> 26 us, 32768 x 1023 33 -> 30)
  const int blocks = p.C > 512 && p.C <= 1024 ? 7 * 256 : 8 * 256;
  const NormForm f = norm_form(&p, vector_of({x, y}), values, 256, blocks);
  (void)hipGetLastError();
  return hip_status(mt::layer_norm_fwd(p, x->dtype == MT_BF16, y->dtype == MT_BF16, f.nv, f.threads, f.blocks, stream));
}

mt_status layer_norm_bwd_impl(const mt_tensor* x, const mt_tensor* w, const mt_tensor* dy, float eps,
                              const mt_tensor* dx, const mt_tensor* dw, const mt_tensor* db, uint32_t flags, void* ws,
                              size_t ws_bytes, hipStream_t stream, size_t* ws_query) {
  if (flags & ~MT_ACCUMULATE) return fail(MT_ERR_INVALID, "mt_layer_norm_bwd: unknown flags");
  mt::LayerNormParams p;
  mt_status s;
  if ((s = check_norm(x, w, eps, &p)) || (s = like(dy, "dy", x, false))) return s;
  if (!dx && !dw && !db) return fail(MT_ERR_NULL, "no output requested");
  if (dx) {
    if ((s = like(dx, "dx", x, true))) return s;
    if (dx->dtype != dy->dtype) return fail(MT_ERR_DTYPE, "dx must have dy's dtype");
  }
  if ((dw && (s = check_vector(dw, "dw", p.C))) || (db && (s = check_vector(db, "db", p.C))) ||
      (s = check_apart({dx, dw, db}, {x, w, dy})))
    return s;
  // two blocks a CU up to 4096 columns (524288 x 64 bf16 51 -> 48 us, 16384 x 2048 bf16 65 -> 57); of longer rows
  // one, whose sums of dw and db are half as many (2048 x 16384 bf16 73 us, two blocks 88; 512 x 6075 fp32 23, 29; bf16
  // rows of 6144 and 8192 alone take two the better, 4096 x 8192 70 us, 63)
  // 8 values a lane for short rows (524288 x 64 bf16 53 -> 48), 16 for others (32768 x 1024 bf16 49, 8 values 61)
  const NormForm f = norm_form(&p, vector_of({x, dy}), p.C <= 512 ? 8 : 16, p.C <= 4096 ? 512 : 1024,
                               p.C <= 4096 ? 512 : 256);
  const bool weights = dw || db;
  // dw and db: launches whose lanes meet up to kLayerNormLaneRows rows each; the parts of up to 64 are added at a time
  // (524288 x 8192 bf16 by eight launches 6.24 ms, by one 6.12)
  const int64_t rows = f.threads / p.L, most = f.blocks * rows * mt::kLayerNormLaneRows, M = p.M;
  const int64_t launches = weights ? std::max<int64_t>(1, cdiv(M, most)) : 1, each = cdiv(M, launches);
  const int64_t group = std::min<int64_t>(launches, 64), part = f.blocks * 2 * p.C;
  const size_t parts = group * part * sizeof(float);
  const size_t need = weights ? parts + (launches > group ? 2 * p.C * sizeof(double) : 0) : 0;
  if (ws_query) {
    *ws_query = need;
    return MT_OK;
  }
  if ((s = check_workspace(ws, ws_bytes, need, "mt_layer_norm_bwd"))) return s;
  p.dy = dy->data;
  p.ldd = row_pitch(dy);
  p.out = dx ? dx->data : nullptr;
  p.ldo = dx ? row_pitch(dx) : 0;
  p.accumulate = (flags & MT_ACCUMULATE) != 0;
  (void)hipGetLastError();
  // without rows too: dw and db are empty sums then
  double* carry = launches > group ? (double*)((char*)ws + parts) : nullptr;
  for (int64_t i = 0; i < launches && (M > 0 || weights); ++i) {
    const int64_t m0 = i * each;
    mt::LayerNormParams q = p;
    q.M = std::max<int64_t>(0, std::min(each, M - m0));
    q.x = (const char*)p.x + m0 * p.ldx * elem_size(x->dtype);
    q.dy = (const char*)p.dy + m0 * p.ldd * elem_size(dy->dtype);
    if (dx) q.out = (char*)p.out + m0 * p.ldo * elem_size(dx->dtype);
    q.part = weights ? (float*)ws + i % group * part : nullptr;
    if ((s = hip_status(mt::layer_norm_bwd(q, x->dtype == MT_BF16, dy->dtype == MT_BF16, f.nv, f.threads, f.blocks, stream))))
      return s;
    const bool last = i + 1 == launches;
    if (!weights || !(last || (i + 1) % group == 0)) continue;
    if ((s = hip_status(mt::layer_norm_finish((const float*)ws, (int)((i % group + 1) * f.blocks), p.C,
                                              i < group ? nullptr : carry, last ? nullptr : carry,
                                              dw ? (float*)dw->data : nullptr, db ? (float*)db->data : nullptr,
                                              p.accumulate, stream))))
      return s;
  }
  return MT_OK;
}

// ------------------------------------------------------------ cross-entropy
mt_status cross_entropy_impl(const mt_tensor* logits, const mt_tensor* targets, const mt_tensor* loss,
                             const mt_tensor* losses, const mt_tensor* dlogits, void* ws, size_t ws_bytes,
                             hipStream_t stream, size_t* ws_query) {
  mt::CrossEntropyParams p{};
  mt_status s;
  int64_t n = 0;
  if ((s = check_rows(logits, "logits", false)) || (s = check_ids(targets, "targets", &p.targets, &n))) return s;
  p.M = logits->shape[0];
  const int64_t V = logits->shape[1];
  if (n != p.M) return fail(MT_ERR_SHAPE, "targets must hold one class for each row of logits");
  if (V < 1 || V > (1 << 24)) return fail(MT_ERR_SHAPE, "a row must have 1 to 2^24 logits");
  const size_t need = 256 + kCrossEntropyParts * sizeof(double) + round256(p.M * sizeof(float));
  if (ws_query) {
    *ws_query = need;
    return MT_OK;
  }
  if (!loss && !losses && !dlogits) return fail(MT_ERR_NULL, "mt_cross_entropy: no output requested");
  if (loss) {
    if ((s = check_tensor(loss, "loss", 0, MT_MAX_DIMS))) return s;
    if (loss->dtype != MT_F32) return fail(MT_ERR_DTYPE, "loss must be f32");
    if (numel(loss) != 1) return fail(MT_ERR_SHAPE, "loss must hold exactly one element");
  }
  if (losses && (s = check_vector(losses, "losses", p.M))) return s;
  if (dlogits) {
    if ((s = check_rows(dlogits, "dlogits", true))) return s;
    if (dlogits->shape[0] != p.M || dlogits->shape[1] != V)
      return fail(MT_ERR_SHAPE, "dlogits must have the shape of logits");
  }
  if ((s = check_apart({loss, losses, dlogits}, {logits, targets})) ||
      (s = check_workspace(ws, ws_bytes, need, "mt_cross_entropy")))
    return s;
  void* part = (char*)ws + 256;
  p.V = (int32_t)V;
  p.row_loss = losses && p.M ? (float*)losses->data : (float*)((char*)part + kCrossEntropyParts * sizeof(double));
  p.z = logits->data;
  p.ldz = row_pitch(logits);
  const bool zb = logits->dtype == MT_BF16, db = dlogits ? dlogits->dtype == MT_BF16 : zb;
  if (dlogits) {
    p.dz = dlogits->data;
    p.ldd = row_pitch(dlogits);
  }
  mt::CrossEntropyForm f{64, 0, 0, 0, false};
  if (V <= 1024) {
    for (f.L = 1; f.L < 64 && f.L * 16 < V; f.L *= 2) ++f.L_shift;
    f.few = p.M * f.L <= 4096;
  } else {
    // 16 values a thread, of bf16 32 (8192 x 16384 fp32 189 us against 200 the other way, bf16 128 against
    // 131). 1024 threads, one block a CU, where the rows of two would not stay in the caches (2048 x 131072
    // fp32 565 -> 493, 4096 x 65537 485 -> 460; 5336 x 50001 fp32 to bf16 355 -> 368, so not below 65536) or
    // where all rows have a CU (64 x 50001 20.5 -> 17.4); only past 32 values a thread: shorter rows' kernels
    // take 512 threads at most
    while (f.threads < 512 && f.threads * (zb ? 32 : 16) < V) f.threads *= 2;
    if (V > 65536 || (V > 32768 && p.M <= 256)) f.threads = 1024;
    f.values = (int32_t)cdiv(V, f.threads);
  }
  float* to = loss ? (float*)loss->data : nullptr;
  (void)hipGetLastError();
  // every block counts the rows itself where they read 2^18 classes in all
  const int64_t blocks = f.L ? cdiv(p.M * f.L, 256) : p.M;
  if (!f.few && blocks * p.M > (1 << 18)) p.counted = (int32_t*)ws;
  if (p.counted && (loss || dlogits) &&
      (s = hip_status(mt::cross_entropy_count(p.targets, p.M, V, (int32_t*)part, (int32_t*)ws, stream))))
    return s;
  if ((p.M > 0 || f.few) && (s = hip_status(mt::cross_entropy_rows(p, f, zb, db, to, stream)))) return s;
  if (f.few || !loss) return MT_OK;
  return hip_status(mt::cross_entropy_mean(p, (double*)part, to, stream));
}

// ----------------------------------------------------------------- clipping
namespace {

// How many values a tensor that clipping takes has, -1 where something about it
// is wrong; what, the checks of check_clip say.
int64_t dense_numel(const mt_tensor* t) {
  if (t->ndim < 0 || t->ndim > MT_MAX_DIMS || (t->dtype != MT_F32 && t->dtype != MT_BF16)) return -1;
  bool none = false;
  for (int i = 0; i < t->ndim; ++i) {
    if (t->shape[i] < 0 || t->stride[i] < 0) return -1;
    none = none || t->shape[i] == 0;
  }
  if (none) return 0;
  int64_t n = 1;
  for (int i = t->ndim - 1; i >= 0; --i) {
    const int64_t size = t->shape[i];
    if (size != 1 && t->stride[i] != n) return -1;
    if (size > ((int64_t)1 << 40) / n) return -1;
    n *= size;
  }
  return t->data ? n : -1;
}
mt_status check_clip(const mt_tensor* t, bool out, int32_t i) {
  const std::string name = (out ? "out " : "grad ") + std::to_string(i);
  mt_status s = check_tensor(t, name.c_str(), 0, MT_MAX_DIMS);
  if (s) return s;
  if (!is_row_major(t)) return fail(MT_ERR_LAYOUT, name + ": must be contiguous");
  return fail(MT_ERR_SHAPE, name + ": more than 2^40 values");
}

// A gradient that is not empty.
struct ClipItem {
  const mt_tensor* grad;
  const mt_tensor* out;
  int64_t numel;
  int64_t chunks() const { return cdiv(numel, mt::kClipChunk); }
};
// What one launch takes of the items from `first` on: up to which, and its chunks.
size_t clip_batch(const std::vector<ClipItem>& items, size_t first, bool in_place, int64_t* chunks) {
  const size_t end = std::min(items.size(), first + (size_t)mt::ClipBatch::most(in_place));
  *chunks = 0;
  size_t i = first;
  for (; i < end && *chunks + items[i].chunks() <= (1 << 30); ++i) *chunks += items[i].chunks();
  return i;
}
size_t clip_parts(const std::vector<ClipItem>& items, bool in_place) {
  size_t parts = 0;
  int64_t chunks;
  for (size_t i = 0; i < items.size(); parts += mt::clip_blocks(chunks)) i = clip_batch(items, i, in_place, &chunks);
  return parts;
}
void clip_pack(const std::vector<ClipItem>& items, size_t first, size_t end, int64_t chunks, bool in_place, mt::ClipBatch* b) {
  b->n = (int32_t)(end - first);
  b->in_place = in_place;
  b->chunks = (int32_t)chunks;
  uint32_t* starts = (uint32_t*)b->starts();
  uint32_t at = 0;
  for (size_t i = first; i < end; ++i) {
    const ClipItem& t = items[i];
    const int kind = (t.grad->dtype == MT_BF16 ? mt::kClipSourceBf16 : 0) | (t.out->dtype == MT_BF16 ? mt::kClipDestBf16 : 0);
    b->w[i - first] = mt::ClipBatch::source(t.grad->data, kind, t.numel);
    if (!in_place) b->w[end - first + (i - first)] = (uint64_t)(uintptr_t)t.out->data;
    starts[i - first] = at;
    at += (uint32_t)t.chunks();
  }
}

struct Range {
  uintptr_t lo, hi;
  bool written;
};
// Whether what is written overlaps anything else. Tensors cut from one buffer
// mostly come by ascending address.
bool any_written_overlaps(std::vector<Range>& r) {
  auto before = [](const Range& a, const Range& b) { return a.lo < b.lo; };
  if (!std::is_sorted(r.begin(), r.end(), before)) std::sort(r.begin(), r.end(), before);
  uintptr_t far = 0, far_written = 0;  // ends of what came before: of all, of what is written
  for (const Range& x : r) {
    if (x.lo < far_written || (x.written && x.lo < far)) return true;
    far = std::max(far, x.hi);
    if (x.written) far_written = std::max(far_written, x.hi);
  }
  return false;
}

}  // namespace

mt_status clip_grad_norm_impl(int32_t n, const mt_tensor* grads, double max_norm, const mt_tensor* out,
                              const mt_tensor* norm, void* ws, size_t ws_bytes, hipStream_t stream, size_t* ws_query) {
  if (n < 0) return fail(MT_ERR_INVALID, "mt_clip_grad_norm: negative tensor count");
  if (n > 0 && !grads) return fail(MT_ERR_NULL, "mt_clip_grad_norm: null array");
  mt_status s;
  std::vector<ClipItem> items;
  std::vector<Range> ranges;
  items.reserve(n);
  ranges.reserve((size_t)n * (out ? 2 : 1) + 1);
  auto take = [&](const mt_tensor* t, int64_t count, bool written) {
    const uintptr_t lo = (uintptr_t)t->data;
    ranges.push_back({lo, lo + (uintptr_t)count * elem_size(t->dtype), written});
  };
  for (int32_t i = 0; i < n; ++i) {
    const int64_t count = dense_numel(&grads[i]);
    if (count < 0) return check_clip(&grads[i], false, i);
    if (out) {
      if (dense_numel(&out[i]) < 0) return check_clip(&out[i], true, i);
      if (out[i].ndim != grads[i].ndim || !std::equal(out[i].shape, out[i].shape + out[i].ndim, grads[i].shape))
        return fail(MT_ERR_SHAPE, "out " + std::to_string(i) + " must have the shape of its gradient");
    }
    if (count == 0) continue;
    items.push_back({&grads[i], out ? &out[i] : &grads[i], count});
    take(&grads[i], count, !out);
  }
  // a workspace serves both forms: the query does not know of out
  const size_t parts = clip_parts(items, !out);
  const size_t need = round256(std::max({(size_t)1, parts, clip_parts(items, out != nullptr)}) * sizeof(double));
  if (ws_query) {
    *ws_query = need;
    return MT_OK;
  }
  if (!(max_norm >= 0.0)) return fail(MT_ERR_INVALID, "mt_clip_grad_norm: max_norm must not be negative");
  if (norm) {
    if ((s = check_tensor(norm, "norm", 0, MT_MAX_DIMS))) return s;
    if (norm->dtype != MT_F32) return fail(MT_ERR_DTYPE, "norm must be f32");
    if (numel(norm) != 1) return fail(MT_ERR_SHAPE, "norm must hold exactly one element");
    take(norm, 1, true);
  }
  if (out)
    for (const ClipItem& t : items) take(t.out, t.numel, true);
  if (any_written_overlaps(ranges)) return fail(MT_ERR_ALIAS, "mt_clip_grad_norm: a tensor that is written overlaps another");
  if ((s = check_workspace(ws, ws_bytes, need, "mt_clip_grad_norm"))) return s;
  mt::ClipBatch b;
  double* part = (double*)ws;
  float* to = norm ? (float*)norm->data : nullptr;
  (void)hipGetLastError();
  if (items.empty()) {
    if (!to) return MT_OK;
    b.n = b.chunks = 0;
    b.in_place = 1;
    return hip_status(mt::clip_scale(b, part, 0, max_norm, to, 1, stream));
  }
  int64_t chunks;
  size_t at = 0, end = 0;
  for (size_t first = 0; first < items.size(); first = end) {
    end = clip_batch(items, first, !out, &chunks);
    clip_pack(items, first, end, chunks, !out, &b);
    const int blocks = mt::clip_blocks(chunks);
    if ((s = hip_status(mt::clip_norm(b, part + at, blocks, stream)))) return s;
    at += blocks;
  }
  for (size_t first = 0; first < items.size(); first = end) {
    end = clip_batch(items, first, !out, &chunks);
    if (end - first < items.size()) clip_pack(items, first, end, chunks, !out, &b);  // else it still holds them
    if ((s = hip_status(mt::clip_scale(b, part, (int)parts, max_norm, to, mt::clip_blocks(chunks), stream)))) return s;
    to = nullptr;
  }
  return MT_OK;
}

}  // namespace mt::host
