// Entry points of the decoder operators (declared and documented in ios.h):
// every size, pointer and alignment that the host can see is checked here,
// before anything is launched.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "decoder.h"

using namespace ios;

namespace {

template <class F>
int guarded(F &&f) {
  try {
    f();
    return IOS_OK;
  } catch (const Error &e) {
    set_last_error_text(e.msg.c_str());
    return e.code;
  } catch (const std::bad_alloc &) {
    set_last_error_text("host allocation failed");
    return IOS_E_OOM;
  } catch (const std::exception &e) {
    set_last_error_text(e.what());
    return IOS_E_ARG;
  }
}

void need(bool ok, int code, const char *msg) {
  if (!ok) fail(code, msg);
}
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int type_size(int dtype) { return dtype == IOS_F32 ? 4 : 2; }

// Tokens of a call are bounded so that offsets and grids stay in 32 bits (the
// elements' own offsets are 64-bit everywhere).
constexpr int64_t kMaxTokens = (int64_t)1 << 28;
constexpr int32_t kMaxSeqs = 1 << 21, kMaxAttnSeqs = 65535;
constexpr int32_t kMaxHeads = 1 << 14;
// a tile of 64 rows is addressed with 32-bit byte offsets from its first
constexpr int64_t kMaxStride = (int64_t)1 << 22;

void check_tokens(const ios_tokens *t, int dtype, const char *what) {
  need(t != nullptr, IOS_E_ARG, "null tensor");
  const int64_t unit = 16 / type_size(dtype);
  const std::string w(what);
  if (t->tokens < 0 || t->tokens > kMaxTokens) fail(IOS_E_ARG, w + ": tokens out of range");
  if (t->tokens > 0 && !t->data) fail(IOS_E_ARG, w + ": null data");
  if (!aligned16(t->data) || t->token_stride % unit || t->head_stride % unit)
    fail(IOS_E_ARG, w + ": data and strides must be multiples of 16 bytes");
  if (t->token_stride < 0 || t->token_stride > kMaxStride || t->head_stride < 0 || t->head_stride > ((int64_t)1 << 40))
    fail(IOS_E_ARG, w + ": stride out of range");
}

// A tensor that the call writes: no two rows share an element.
void check_out(const ios_tokens *t, int dtype, int heads, const char *what) {
  check_tokens(t, dtype, what);
  if ((t->tokens > 1 && t->token_stride == 0) || (heads > 1 && t->head_stride == 0))
    fail(IOS_E_ARG, std::string(what) + ": an output's strides must not be 0");
}

void check_type(int dtype) { need(dtype >= IOS_F32 && dtype <= IOS_BF16, IOS_E_ARG, "unknown element type"); }

void check_desc(const ios_attn_desc *d) {
  need(d != nullptr, IOS_E_ARG, "null attention descriptor");
  check_type(d->dtype);
  need(d->heads >= 1 && d->kv_heads >= 1 && d->heads <= kMaxHeads, IOS_E_ARG, "head count out of range");
  need(d->heads % d->kv_heads == 0, IOS_E_SHAPE, "heads must be a multiple of kv_heads");
  need(d->head_dim >= 1, IOS_E_ARG, "head_dim out of range");
  need(d->head_dim % 8 == 0 && d->head_dim <= 128, IOS_E_UNSUPPORTED,
       "head_dim must be a multiple of 8 up to 128");
  need(d->seqs >= 1 && d->seqs <= kMaxAttnSeqs, IOS_E_ARG, "seqs out of range");
  need(d->causal == 0 || d->causal == 1, IOS_E_ARG, "causal must be 0 or 1");
  need(d->max_keys >= 0, IOS_E_ARG, "negative max_keys");
  need(std::isfinite(d->scale), IOS_E_ARG, "scale must be finite");
}

// The cache's sizes; `state`: its pointers too.
void check_cache(const ios_cache *c, bool state) {
  need(c != nullptr, IOS_E_ARG, "null cache");
  need(c->layers >= 1 && c->kv_heads >= 1 && c->kv_heads <= kMaxHeads && c->pages >= 1 && c->slots >= 1 &&
           c->row >= 1 && c->head_dim >= 1 && c->page_tokens >= 1,
       IOS_E_ARG, "cache sizes must be positive");
  need(c->head_dim % kGroup == 0 && c->head_dim <= 4 * kGroup, IOS_E_UNSUPPORTED,
       "a cache's head_dim must be 32, 64, 96 or 128");
  need(c->page_tokens == 32 || c->page_tokens == 64 || c->page_tokens == 128 || c->page_tokens == 256,
       IOS_E_UNSUPPORTED, "page_tokens must be 32, 64, 128 or 256");
  need((int64_t)c->slots * c->row <= INT32_MAX && (int64_t)c->row * c->page_tokens <= kMaxTokens &&
           c->pages <= INT32_MAX / 2 && c->slots <= kMaxSeqs,
       IOS_E_UNSUPPORTED, "cache tables too large");
  if (!state) return;
  need(c->pool && c->refs && c->table && c->lens && c->work, IOS_E_ARG, "null pointer in the cache");
  need(aligned16(c->pool) && aligned16(c->work), IOS_E_ARG, "pool and work must be 16-byte aligned");
}

int64_t page_bytes(const ios_cache &c) {
  return (int64_t)c.kv_heads * (c.page_tokens / kTileKeys) * tile_bytes(c.head_dim / kGroup);
}

CacheView view(const ios_cache &c, int layer) {
  need(layer >= 0 && layer < c.layers, IOS_E_ARG, "layer out of range");
  CacheView v{};
  v.page_bytes = page_bytes(c);
  v.pool = (unsigned char *)c.pool + (int64_t)layer * c.pages * v.page_bytes;
  v.table = c.table;
  v.lens = c.lens;
  v.head_bytes = c.page_tokens / kTileKeys * tile_bytes(c.head_dim / kGroup);
  v.pages = c.pages;
  v.slots = c.slots;
  v.row = c.row;
  v.heads = c.kv_heads;
  while ((1 << v.page_lg) < c.page_tokens) ++v.page_lg;
  return v;
}

void launched(hipError_t e, const char *what) { hip_check(e, what); }

void check_list(const ios_cache *c, int32_t n, const void *a, const void *b) {
  check_cache(c, true);
  need(n >= 0 && n <= c->slots, IOS_E_ARG, "list longer than the cache has slots");
  need(n == 0 || (a && b), IOS_E_ARG, "null list");
}

int64_t split_bytes(int64_t rows, int heads, int dim, int splits) {
  return splits > 1 ? rows * heads * splits * (int64_t)(dim + 2) * (int64_t)sizeof(float) : 0;
}

// Splits that a call with this workspace takes.
int usable(int splits, int64_t rows, const ios_attn_desc &d, const void *work, int64_t work_bytes) {
  if (!work || splits <= 1) return 1;
  need(aligned16(work) && work_bytes >= split_bytes(rows, d.heads, d.head_dim, splits), IOS_E_ARG,
       "workspace below ios_attn_work_bytes or misaligned");
  return splits;
}

// A rotation of heads of this size.
void check_rotary(const ios_rotary *r, int head_dim) {
  need(r != nullptr, IOS_E_ARG, "null rotation");
  need(r->dim >= 2 && r->dim % 2 == 0 && r->dim <= head_dim, IOS_E_ARG, "a rotation's dim must be even, from 2 to head_dim");
  need(r->interleaved == 0 || r->interleaved == 1, IOS_E_ARG, "interleaved must be 0 or 1");
  need(r->reserved == 0, IOS_E_ARG, "reserved must be 0");
  need(std::isfinite(r->amplitude), IOS_E_ARG, "amplitude must be finite");
  for (int i = 0; i < r->dim / 2; ++i)
    need(std::fabs(r->freq[i]) <= 1024.0, IOS_E_ARG, "a frequency must be within 1024");   // not a NaN's either
}

// An output that is its input or lies apart.
void check_turned(const ios_tokens *in, const ios_tokens *out, int dtype, int heads, const char *what) {
  check_tokens(in, dtype, what);
  check_out(out, dtype, heads, what);
  const std::string w(what);
  if (heads < 1 || heads > kMaxHeads) fail(IOS_E_ARG, w + ": head count out of range");
  if (in->tokens != out->tokens) fail(IOS_E_SHAPE, w + ": input and output have different lengths");
  if (in->data == out->data && in->data && (in->token_stride != out->token_stride || in->head_stride != out->head_stride))
    fail(IOS_E_ARG, w + ": in place, the strides must be the same");
}

// A cache, a type and the tensors that go into one of its layers.
void check_append(const ios_cache *c, int32_t dtype, const ios_tokens *k, const ios_tokens *v) {
  check_type(dtype);
  check_tokens(k, dtype, "k");
  check_tokens(v, dtype, "v");
  need(k->tokens == v->tokens, IOS_E_SHAPE, "k and v have different lengths");
}

void check_drafts(int32_t most) {
  need(most >= 1 && most <= kMaxDrafts, IOS_E_ARG, "drafts of a sequence must be 1 to 64");
}

// Rows of all heads, as many as fit a grid of a wave each (fewer than 2^32 threads), and of one sequence.
void check_tree(const ios_attn_desc &d, int64_t q_tokens, int32_t most) {
  need(q_tokens * d.heads <= INT32_MAX / 64 && (int64_t)most * d.heads <= 65535, IOS_E_UNSUPPORTED, "too many rows and heads");
}

void check_rows(const ios_rows *t, const ios_verify_desc *d, const char *what) {
  const std::string w(what);
  if (!t) fail(IOS_E_ARG, w + ": null matrix");
  if (t->rows < 0 || t->rows > kMaxTokens) fail(IOS_E_ARG, w + ": rows out of range");
  if (t->rows > 0 && !t->data) fail(IOS_E_ARG, w + ": null data");
  if (reinterpret_cast<uintptr_t>(t->data) % type_size(d->dtype)) fail(IOS_E_ARG, w + ": misaligned data");
  if (t->row_stride < 0 || t->row_stride > ((int64_t)1 << 32)) fail(IOS_E_ARG, w + ": stride out of range");
}

void check_verify(const ios_verify_desc *d) {
  need(d != nullptr, IOS_E_ARG, "null descriptor");
  check_type(d->dtype);
  need(d->seqs >= 1 && d->seqs <= kMaxAttnSeqs, IOS_E_ARG, "seqs out of range");
  need(d->vocab >= 1, IOS_E_ARG, "vocab out of range");
  check_drafts(d->max_drafts);
}

int move_tokens(bool read, const ios_cache *c, int32_t layer, int32_t dtype, const ios_tokens *k, const ios_tokens *v,
                int32_t n, const int32_t *seqs, const int32_t *cu, void *hip_stream) {
  return guarded([&] {
    check_list(c, n, seqs, cu);
    check_type(dtype);
    if (read) {
      check_out(k, dtype, c->kv_heads, "k");
      check_out(v, dtype, c->kv_heads, "v");
    } else {
      check_tokens(k, dtype, "k");
      check_tokens(v, dtype, "v");
    }
    need(k->tokens == v->tokens, IOS_E_SHAPE, "k and v have different lengths");
    const CacheView cv = view(*c, layer);
    if (n == 0 || k->tokens == 0) return;
    launched((read ? launch_read : launch_append)(cv, c->head_dim / kGroup, dtype, *k, *v, n, seqs, cu,
                                                  (hipStream_t)hip_stream),
             read ? "ios_cache_read" : "ios_cache_append");
  });
}

}  // namespace

extern "C" int ios_attn_work_bytes(const ios_attn_desc *d, int64_t q_tokens, int64_t *bytes) {
  return guarded([&] {
    check_desc(d);
    need(bytes != nullptr, IOS_E_ARG, "null bytes");
    need(q_tokens >= 0 && q_tokens <= kMaxTokens, IOS_E_ARG, "q_tokens out of range");
    const int64_t single = q_tokens == d->seqs ? split_bytes(q_tokens, d->heads, d->head_dim, cache_splits(*d)) : 0;
    *bytes = std::max(single, split_bytes(q_tokens, d->heads, d->head_dim, prompt_splits(*d, q_tokens)));
  });
}

extern "C" int ios_attn_prompt(const ios_attn_desc *d, const ios_tokens *q, const ios_tokens *k, const ios_tokens *v,
                               const ios_tokens *out, float *lse, const int32_t *cu_q, const int32_t *cu_k,
                               void *work, int64_t work_bytes, void *hip_stream) {
  return guarded([&] {
    check_desc(d);
    check_tokens(q, d->dtype, "q");
    check_tokens(k, d->dtype, "k");
    check_tokens(v, d->dtype, "v");
    check_out(out, d->dtype, d->heads, "out");
    need(k->tokens == v->tokens, IOS_E_SHAPE, "k and v have different lengths");
    need(q->tokens == out->tokens, IOS_E_SHAPE, "q and out have different lengths");
    need(cu_q && cu_k, IOS_E_ARG, "null offsets");
    if (q->tokens == 0) return;
    need((q->tokens / 64 + d->seqs) * d->heads < ((int64_t)1 << 32) / 512, IOS_E_UNSUPPORTED, "too many queries and heads");
    const int splits = usable(prompt_splits(*d, q->tokens), q->tokens, *d, work, work_bytes);
    launched(launch_attn_prompt(*d, *q, *k, *v, *out, lse, cu_q, cu_k, work, splits, (hipStream_t)hip_stream),
             "ios_attn_prompt");
  });
}

extern "C" int ios_attn_cache(const ios_cache *c, int32_t layer, const ios_attn_desc *d, const ios_tokens *q,
                              const ios_tokens *out, float *lse, const int32_t *seqs, void *work,
                              int64_t work_bytes, void *hip_stream) {
  return guarded([&] {
    check_cache(c, true);
    check_desc(d);
    check_tokens(q, d->dtype, "q");
    check_out(out, d->dtype, d->heads, "out");
    need(d->kv_heads == c->kv_heads && d->head_dim == c->head_dim, IOS_E_SHAPE, "the cache has other heads");
    need(q->tokens == d->seqs && out->tokens == d->seqs, IOS_E_SHAPE, "q and out must have one row per sequence");
    need(seqs != nullptr, IOS_E_ARG, "null sequence list");
    const CacheView cv = view(*c, layer);
    const int splits = usable(cache_splits(*d), d->seqs, *d, work, work_bytes);
    launched(launch_attn_cache(cv, *d, *q, *out, lse, seqs, work, splits, (hipStream_t)hip_stream),
             "ios_attn_cache");
  });
}

extern "C" int ios_cache_page_bytes(const ios_cache *c, int64_t *bytes) {
  return guarded([&] {
    check_cache(c, false);
    need(bytes != nullptr, IOS_E_ARG, "null bytes");
    *bytes = page_bytes(*c);
  });
}

extern "C" int ios_cache_work_bytes(const ios_cache *c, int64_t *bytes) {
  return guarded([&] {
    check_cache(c, false);
    need(bytes != nullptr, IOS_E_ARG, "null bytes");
    *bytes = cache_work_words(c->pages, c->slots) * (int64_t)sizeof(int32_t);
  });
}

extern "C" int ios_cache_reserve(const ios_cache *c, int32_t n, const int32_t *seqs, const int32_t *add,
                                 void *hip_stream) {
  return guarded([&] {
    check_list(c, n, seqs, add);
    if (n) launched(launch_reserve(*c, page_bytes(*c), n, seqs, add, (hipStream_t)hip_stream), "ios_cache_reserve");
  });
}

extern "C" int ios_cache_append(const ios_cache *c, int32_t layer, int32_t dtype, const ios_tokens *k,
                                const ios_tokens *v, int32_t n, const int32_t *seqs, const int32_t *cu,
                                void *hip_stream) {
  return move_tokens(false, c, layer, dtype, k, v, n, seqs, cu, hip_stream);
}

extern "C" int ios_cache_read(const ios_cache *c, int32_t layer, int32_t dtype, const ios_tokens *k,
                              const ios_tokens *v, int32_t n, const int32_t *seqs, const int32_t *cu,
                              void *hip_stream) {
  return move_tokens(true, c, layer, dtype, k, v, n, seqs, cu, hip_stream);
}

extern "C" int ios_rotary_freqs(ios_rotary *r, double base, double factor, double original, double low, double high) {
  return guarded([&] {
    need(r != nullptr, IOS_E_ARG, "null rotation");
    need(r->dim >= 2 && r->dim % 2 == 0 && r->dim <= 128, IOS_E_ARG, "a rotation's dim must be even, from 2 to 128");
    need(base > 1.0 && std::isfinite(base), IOS_E_ARG, "base must be above 1");
    need(factor > 0.0 && std::isfinite(factor), IOS_E_ARG, "factor must be above 0");
    need(original >= 0.0 && std::isfinite(original), IOS_E_ARG, "original must not be negative");
    need(original == 0.0 || (low < high && std::isfinite(low) && std::isfinite(high)), IOS_E_ARG, "low must be below high");
    double f[64];
    for (int i = 0; i < r->dim / 2; ++i) {
      f[i] = std::pow(base, -2.0 * i / r->dim);
      double keep = 0.0;
      if (original > 0.0) keep = std::min(std::max((original * f[i] / (2 * M_PI) - low) / (high - low), 0.0), 1.0);
      f[i] = original > 0.0 ? f[i] * (keep + (1.0 - keep) / factor) : f[i] / factor;
      need(f[i] <= 1024.0, IOS_E_ARG, "factor makes a frequency above 1024");
    }
    std::copy(f, f + r->dim / 2, r->freq);
  });
}

extern "C" int ios_rotate(const ios_rotary *r, int32_t dtype, int32_t head_dim, const ios_tokens *q,
                          const ios_tokens *q_out, int32_t heads, const ios_tokens *k, const ios_tokens *k_out,
                          int32_t kv_heads, const int32_t *pos, void *hip_stream) {
  return guarded([&] {
    check_type(dtype);
    need(head_dim >= 1, IOS_E_ARG, "head_dim out of range");
    need(head_dim % 8 == 0 && head_dim <= 128, IOS_E_UNSUPPORTED, "head_dim must be a multiple of 8 up to 128");
    check_rotary(r, head_dim);
    check_turned(q, q_out, dtype, heads, "q");
    const ios_tokens none{};
    need(!k == !k_out, IOS_E_ARG, "k and k_out must be given together");
    if (k) {
      check_turned(k, k_out, dtype, kv_heads, "k");
      need(k->tokens == q->tokens, IOS_E_SHAPE, "q and k have different lengths");
    }
    if (q->tokens == 0) return;
    need(pos != nullptr, IOS_E_ARG, "null positions");
    launched(launch_rotate(*r, dtype, head_dim, *q, *q_out, heads, k ? *k : none, k ? *k_out : none, k ? kv_heads : 0, pos,
                           (hipStream_t)hip_stream),
             "ios_rotate");
  });
}

extern "C" int ios_cache_append_rotary(const ios_cache *c, int32_t layer, int32_t dtype, const ios_rotary *r,
                                       const ios_tokens *q, const ios_tokens *q_out, int32_t heads, const ios_tokens *k,
                                       const ios_tokens *v, int32_t n, const int32_t *seqs, const int32_t *cu,
                                       void *hip_stream) {
  return guarded([&] {
    check_list(c, n, seqs, cu);
    check_append(c, dtype, k, v);
    check_rotary(r, c->head_dim);
    need(!q == !q_out, IOS_E_ARG, "q and q_out must be given together");
    if (q) {
      check_turned(q, q_out, dtype, heads, "q");
      need(q->tokens == k->tokens, IOS_E_SHAPE, "q and k have different lengths");
    }
    const CacheView cv = view(*c, layer);
    if (n == 0 || k->tokens == 0) return;
    launched(launch_append_rotary(cv, c->head_dim / kGroup, dtype, *r, q, q_out, heads, *k, *v, n, seqs, cu,
                                  (hipStream_t)hip_stream),
             "ios_cache_append_rotary");
  });
}

extern "C" int ios_cache_keep(const ios_cache *c, int32_t layer, int32_t dtype, const ios_tokens *k, const ios_tokens *v,
                              int32_t n, const int32_t *seqs, const int32_t *path, int32_t max_path,
                              const int32_t *count, void *hip_stream) {
  return guarded([&] {
    check_list(c, n, seqs, path);
    check_append(c, dtype, k, v);
    check_drafts(max_path);
    need(n == 0 || count != nullptr, IOS_E_ARG, "null list");
    const CacheView cv = view(*c, layer);
    if (n == 0) return;
    launched(launch_keep(cv, c->head_dim / kGroup, dtype, *k, *v, n, seqs, path, max_path, count, (hipStream_t)hip_stream),
             "ios_cache_keep");
  });
}

extern "C" int ios_attn_tree_work_bytes(const ios_attn_desc *d, int64_t q_tokens, int32_t max_drafts, int64_t *bytes) {
  return guarded([&] {
    check_desc(d);
    check_drafts(max_drafts);
    need(bytes != nullptr, IOS_E_ARG, "null bytes");
    need(q_tokens >= 0 && q_tokens <= kMaxTokens, IOS_E_ARG, "q_tokens out of range");
    check_tree(*d, q_tokens, max_drafts);
    *bytes = tree_bytes(*d, q_tokens, max_drafts);
  });
}

extern "C" int ios_attn_tree(const ios_cache *c, int32_t layer, const ios_attn_desc *d, const ios_tokens *q,
                             const ios_tokens *k, const ios_tokens *v, const ios_tokens *out, float *lse,
                             const int32_t *seqs, const int32_t *cu, const int32_t *parent, int32_t max_drafts, void *work,
                             int64_t work_bytes, void *hip_stream) {
  return guarded([&] {
    check_cache(c, true);
    check_desc(d);
    check_drafts(max_drafts);
    check_tokens(q, d->dtype, "q");
    check_tokens(k, d->dtype, "k");
    check_tokens(v, d->dtype, "v");
    check_out(out, d->dtype, d->heads, "out");
    need(d->kv_heads == c->kv_heads && d->head_dim == c->head_dim, IOS_E_SHAPE, "the cache has other heads");
    need(k->tokens == q->tokens && v->tokens == q->tokens && out->tokens == q->tokens, IOS_E_SHAPE,
         "q, k, v and out must have the same rows");
    need(seqs && cu && parent, IOS_E_ARG, "null list");
    const CacheView cv = view(*c, layer);
    if (q->tokens == 0) return;
    check_tree(*d, q->tokens, max_drafts);
    need(!work || (aligned16(work) && work_bytes >= tree_bytes(*d, q->tokens, max_drafts)), IOS_E_ARG,
         "workspace below ios_attn_tree_work_bytes or misaligned");
    launched(launch_attn_tree(cv, *d, *q, *k, *v, *out, lse, seqs, cu, parent, max_drafts, work, (hipStream_t)hip_stream),
             "ios_attn_tree");
  });
}

extern "C" int ios_verify_work_bytes(const ios_verify_desc *d, int64_t *bytes) {
  return guarded([&] {
    check_verify(d);
    need(bytes != nullptr, IOS_E_ARG, "null bytes");
    *bytes = verify_bytes(*d);
  });
}

extern "C" int ios_verify(const ios_verify_desc *d, const ios_rows *p, const ios_rows *q, const int32_t *tokens,
                          const int32_t *parent, const int32_t *cu, const float *accept, const float *sample,
                          int32_t *path, int32_t *count, int32_t *next, void *work, int64_t work_bytes,
                          void *hip_stream) {
  return guarded([&] {
    check_verify(d);
    check_rows(p, d, "p");
    if (q) {
      check_rows(q, d, "q");
      need(q->rows == p->rows, IOS_E_SHAPE, "p and q have different lengths");
    }
    need(cu && path && count && next && sample, IOS_E_ARG, "null list");
    need(p->rows == 0 || (tokens && parent && accept), IOS_E_ARG, "null list");
    const int64_t size = verify_bytes(*d);
    need(size == 0 || (work && aligned16(work) && work_bytes >= size), IOS_E_ARG,
         "workspace below ios_verify_work_bytes or misaligned");
    launched(launch_verify(*d, *p, q, tokens, parent, cu, accept, sample, path, count, next, work, (hipStream_t)hip_stream),
             "ios_verify");
  });
}

extern "C" int ios_cache_fork(const ios_cache *c, int32_t n, const int32_t *parents, const int32_t *children,
                              void *hip_stream) {
  return guarded([&] {
    check_list(c, n, parents, children);
    if (n) launched(launch_fork(*c, n, parents, children, (hipStream_t)hip_stream), "ios_cache_fork");
  });
}

extern "C" int ios_cache_free(const ios_cache *c, int32_t n, const int32_t *seqs, void *hip_stream) {
  return guarded([&] {
    check_list(c, n, seqs, seqs);
    if (n) launched(launch_free(*c, n, seqs, (hipStream_t)hip_stream), "ios_cache_free");
  });
}

extern "C" int ios_cache_compact(const ios_cache *c, int32_t *live, void *hip_stream) {
  return guarded([&] {
    check_cache(c, true);
    launched(launch_compact(*c, page_bytes(*c), live, (hipStream_t)hip_stream), "ios_cache_compact");
  });
}

extern "C" int ios_cache_copy(const ios_cache *c, int32_t n, const int32_t *src, const int32_t *dst,
                              void *hip_stream) {
  return guarded([&] {
    check_cache(c, true);
    need(n >= 0 && n <= c->pages, IOS_E_ARG, "more pairs than pages");
    need(n == 0 || (src && dst), IOS_E_ARG, "null list");
    if (n) launched(launch_copy(*c, page_bytes(*c), n, src, dst, (hipStream_t)hip_stream), "ios_cache_copy");
  });
}

extern "C" int ios_cache_status(const ios_cache *c, void *hip_stream, int32_t *flags) {
  return guarded([&] {
    check_cache(c, true);
    need(flags != nullptr, IOS_E_ARG, "null flags");
    hipStream_t s = (hipStream_t)hip_stream;
    int32_t f = 0;
    int32_t *word = (int32_t *)c->work + CW_FLAGS;
    hip_check(hipMemcpyAsync(&f, word, sizeof(f), hipMemcpyDeviceToHost, s), "hipMemcpyAsync");
    hip_check(hipStreamSynchronize(s), "hipStreamSynchronize");
    if (f) {                                                 // on the caller's stream: before whatever is called next
      hip_check(hipMemsetAsync(word, 0, sizeof(f), s), "hipMemsetAsync(flags)");
      hip_check(hipStreamSynchronize(s), "hipStreamSynchronize");
    }
    *flags = f;
  });
}
