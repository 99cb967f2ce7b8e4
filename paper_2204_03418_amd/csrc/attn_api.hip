// C ABI of attention over token streams: rotary positions, pages, the cache.
// Stateless host side: every call checks its arguments, picks a kernel and
// enqueues it; a negative status means nothing ran.
#include <cmath>

#include "cache.hpp"
#include "launch.hpp"
#include "token_check.hpp"

using namespace coinf;

namespace {

constexpr int32_t kMaxBatch = 65535, kMaxKvHeads = 32767;  // of a grid's second and third axis

bool pages_ok(int32_t batch, int32_t pages, int32_t page_tokens, int32_t stream_pages,
              int32_t kv_heads, int32_t head_dim) {
  return batch > 0 && pages > 0 && stream_pages > 0 && kv_heads > 0 && head_dim > 0 &&
         head_dim <= CO_ATTN_MAX_HEAD && page_tokens >= 16 && page_tokens <= 256 &&
         (page_tokens & (page_tokens - 1)) == 0;
}

// Whether the sizes fit the kernels' indexes: a page below 2^31 bytes, table and pages too.
bool pages_fit(int32_t batch, int32_t pages, int32_t page_tokens, int32_t stream_pages,
               int32_t kv_heads, int32_t head_dim) {
  const PageHead lay{page_tokens, cache_blocks(head_dim)};
  return batch <= kMaxBatch && kv_heads <= kMaxKvHeads && pages < (1 << 30) &&
         mul_to(batch, stream_pages + int64_t(1), 1 << 30) >= 0 &&
         mul_to(lay.bytes(), kv_heads, INT32_MAX) >= 0;
}

co_status pages_desc(const co_pages_desc* d) {
  if (!d || d->layers <= 0 ||
      !pages_ok(d->batch, d->pages, d->page_tokens, d->stream_pages, d->kv_heads, d->head_dim))
    return CO_EINVAL;
  if (!pages_fit(d->batch, d->pages, d->page_tokens, d->stream_pages, d->kv_heads, d->head_dim) ||
      mul_to(mul_to(page_bytes(*d), d->pages, kMaxOffset), d->layers, kMaxOffset) < 0)
    return CO_ENOTSUP;
  return CO_OK;
}

bool state_ok(const co_pages* s) {
  if (!s || !s->pool || !aligned(s->pool, 16) || !s->workspace || !aligned(s->workspace, 16))
    return false;
  for (const int32_t* p : {s->table, s->tokens, s->first, s->refs, s->base, s->granted, s->refused})
    if (!p || !aligned(p, 4)) return false;
  return true;
}

co_status attn_desc(const co_attn_desc* d) {
  if (!d || !dtype_ok(d->dtype) || d->heads <= 0 || d->window < 0 || !std::isfinite(d->scale) ||
      !pages_ok(d->batch, d->pages, d->page_tokens, d->stream_pages, d->kv_heads, d->head_dim) ||
      d->heads % d->kv_heads)
    return CO_EINVAL;
  if (!pages_fit(d->batch, d->pages, d->page_tokens, d->stream_pages, d->kv_heads, d->head_dim) ||
      mul_to(d->heads, d->head_dim, INT32_MAX) < 0)
    return CO_ENOTSUP;
  return CO_OK;
}

bool cache_ok(const co_attn_cache* c) {
  return c && c->pool && aligned(c->pool, 16) && c->table && aligned(c->table, 4) && c->base &&
         aligned(c->base, 4) && aligned(c->granted, 4) && aligned(c->first, 4);
}

// Whether a call's tokens and values are as many as the kernels count.
bool tokens_fit(int32_t batch, int32_t T, int64_t width) {
  return mul_to(mul_to(batch, T, INT32_MAX), width, kMaxValues) >= 0;
}

}  // namespace

extern "C" {

co_status co_rotary_turns(int32_t rotary_dim, double base, const co_rotary_scaling* scaling,
                          uint64_t* turns) {
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > CO_ATTN_MAX_HEAD || !turns ||
      !(base > 0) || !std::isfinite(base))
    return CO_EINVAL;
  const int32_t kind = scaling ? scaling->kind : CO_ROTARY_PLAIN;
  if (kind < CO_ROTARY_PLAIN || kind > CO_ROTARY_PARTS) return CO_EINVAL;
  if (kind != CO_ROTARY_PLAIN && (!(scaling->factor > 0) || !std::isfinite(scaling->factor)))
    return CO_EINVAL;
  if (kind == CO_ROTARY_BASE && rotary_dim == 2) return CO_EINVAL;
  if (kind == CO_ROTARY_PARTS &&
      (!(scaling->original > 0) || !std::isfinite(scaling->original) ||
       !std::isfinite(scaling->low) || !std::isfinite(scaling->high) ||
       !(scaling->low < scaling->high)))
    return CO_EINVAL;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  long double b = base;
  if (kind == CO_ROTARY_BASE)
    b *= powl(scaling->factor, (long double)(rotary_dim) / (rotary_dim - 2));
  for (int i = 0; i < rotary_dim / 2; ++i) {
    long double f = powl(b, -2.0L * i / rotary_dim);  // radians a position
    if (kind == CO_ROTARY_LINEAR) f /= scaling->factor;
    if (kind == CO_ROTARY_PARTS) {
      long double k = (scaling->original * f / two_pi - scaling->low) /
                      ((long double)(scaling->high) - scaling->low);
      k = k < 0 ? 0 : k > 1 ? 1 : k;
      f = k * f + (1 - k) * f / scaling->factor;
    }
    const long double turn = fmodl(f / two_pi, 1.0L);
    if (!(turn >= 0 && turn < 1)) return CO_EINVAL;  // a frequency past the type's range
    const long double v = rintl(turn * 18446744073709551616.0L);
    turns[i] = v < 18446744073709551616.0L ? uint64_t(v) : 0;
  }
  return CO_OK;
}

co_status co_rotary_forward(const co_rotary_desc* d, const co_rotary_call* c, void* stream) {
  if (!d || !c || d->batch <= 0 || d->heads[0] <= 0 || d->heads[1] < 0 || d->head_dim <= 0 ||
      d->rotary_dim < 2 || d->rotary_dim % 2 || d->rotary_dim > d->head_dim ||
      d->rotary_dim > CO_ATTN_MAX_HEAD || !dtype_ok(d->dtype) ||
      (d->layout != CO_ROTARY_HALF && d->layout != CO_ROTARY_INTERLEAVED) ||
      !std::isfinite(d->magnitude) || c->T < 0)
    return CO_EINVAL;
  const int32_t B = d->batch, T = c->T;
  if (T == 0) return CO_OK;
  if (!c->turns || !aligned(c->turns, 8) || !aligned(c->positions, 4) || !aligned(c->lengths, 4))
    return CO_EINVAL;
  if (c->positions && (mul_to(c->position_batch_stride, B, kMaxOffset) < 0 ||
                       mul_to(c->position_token_stride, T, kMaxOffset) < 0))
    return CO_EINVAL;
  co_rotary_call k = *c;
  if (d->heads[1] == 0) k.x[1] = k.y[1] = co_tokens{nullptr, 0, 0};
  for (int i = 0; i < (d->heads[1] ? 2 : 1); ++i) {
    const int64_t width = mul_to(d->heads[i], d->head_dim, INT32_MAX);
    if (width < 0 || !tokens_ok(k.x[i], B, T, d->dtype) ||
        !out_ok(k.y[i], B, T, width, d->dtype))
      return CO_EINVAL;
    if (!tokens_fit(B, T, width)) return CO_ENOTSUP;
    for (int j = 0; j < (d->heads[1] ? 2 : 1); ++j) {
      if (j == i ? !in_place_ok(k.y[i], d->dtype, k.x[i], d->dtype, B, T)
                 : k.y[i].data == k.x[j].data || k.y[i].data == k.y[j].data)
        return CO_EINVAL;
    }
  }
  return done(launch_rotary(*d, k, as_stream(stream)));
}

co_status co_pages_query(const co_pages_desc* desc, co_pages_info* info) {
  if (const co_status st = pages_desc(desc)) return st;
  if (!info) return CO_EINVAL;
  info->page_bytes = page_bytes(*desc);
  info->pool_bytes = info->page_bytes * desc->pages * desc->layers;
  info->workspace_bytes = pages_workspace(*desc);
  return CO_OK;
}

co_status co_pages_reserve(const co_pages_desc* desc, const co_pages* s, int32_t T,
                           const int32_t* lengths, int32_t keep, void* stream) {
  if (const co_status st = pages_desc(desc)) return st;
  if (!state_ok(s) || T < 0 || keep < 0 || !aligned(lengths, 4)) return CO_EINVAL;
  return done(launch_pages_reserve(*desc, *s, T, lengths, keep, as_stream(stream)));
}

co_status co_pages_truncate(const co_pages_desc* desc, const co_pages* s, const int32_t* lengths,
                            void* stream) {
  if (const co_status st = pages_desc(desc)) return st;
  if (!state_ok(s) || !lengths || !aligned(lengths, 4)) return CO_EINVAL;
  return done(launch_pages_truncate(*desc, *s, lengths, as_stream(stream)));
}

co_status co_pages_select(const co_pages_desc* desc, const co_pages* s, const int32_t* source,
                          void* stream) {
  if (const co_status st = pages_desc(desc)) return st;
  if (!state_ok(s) || !source || !aligned(source, 4)) return CO_EINVAL;
  return done(launch_pages_select(*desc, *s, source, as_stream(stream)));
}

co_status co_pages_compact(const co_pages_desc* desc, const co_pages* s, void* stream) {
  if (const co_status st = pages_desc(desc)) return st;
  if (!state_ok(s)) return CO_EINVAL;
  return done(launch_pages_compact(*desc, *s, as_stream(stream)));
}

co_status co_attn_append(const co_attn_desc* desc, const co_attn_cache* cache, const co_tokens* k,
                         const co_tokens* v, int32_t T, void* stream) {
  if (const co_status st = attn_desc(desc)) return st;
  if (!cache_ok(cache) || !k || !v || T < 0) return CO_EINVAL;
  if (T == 0) return CO_OK;
  if (!tokens_ok(*k, desc->batch, T, desc->dtype) || !tokens_ok(*v, desc->batch, T, desc->dtype))
    return CO_EINVAL;
  if (!tokens_fit(desc->batch, T, int64_t(desc->kv_heads) * desc->head_dim)) return CO_ENOTSUP;
  return done(launch_attn_append(*desc, *cache, *k, *v, T, as_stream(stream)));
}

co_status co_attn_read(const co_attn_desc* desc, const co_attn_cache* cache, const int32_t* from,
                       const co_tokens* k, const co_tokens* v, int32_t T, void* stream) {
  if (const co_status st = attn_desc(desc)) return st;
  if (!cache_ok(cache) || !cache->granted || !from || !aligned(from, 4) || !k || !v || T < 0)
    return CO_EINVAL;
  if (T == 0) return CO_OK;
  const int64_t width = int64_t(desc->kv_heads) * desc->head_dim;
  if (!out_ok(*k, desc->batch, T, width, desc->dtype) ||
      !out_ok(*v, desc->batch, T, width, desc->dtype) || k->data == v->data)
    return CO_EINVAL;
  if (!tokens_fit(desc->batch, T, width)) return CO_ENOTSUP;
  return done(launch_attn_read(*desc, *cache, from, *k, *v, T, as_stream(stream)));
}

co_status co_attn_workspace_bytes(const co_attn_desc* desc, int32_t T, int64_t* bytes) {
  if (const co_status st = attn_desc(desc)) return st;
  if (T < 0 || !bytes) return CO_EINVAL;
  if (!tokens_fit(desc->batch, T, int64_t(desc->heads) * desc->head_dim)) return CO_ENOTSUP;
  *bytes = attend_workspace(*desc, T);
  return CO_OK;
}

co_status co_attn_forward_steps(const co_attn_desc* desc, const co_attn_cache* cache,
                                const co_tokens* q, const co_tokens* y, int32_t T,
                                void* workspace, int64_t workspace_bytes, void* stream) {
  if (const co_status st = attn_desc(desc)) return st;
  if (!cache_ok(cache) || !q || !y || T < 0 || workspace_bytes < 0 || !aligned(workspace, 16))
    return CO_EINVAL;
  if (T == 0) return CO_OK;
  const int64_t width = int64_t(desc->heads) * desc->head_dim;
  if (!tokens_ok(*q, desc->batch, T, desc->dtype) ||
      !out_ok(*y, desc->batch, T, width, desc->dtype) || q->data == y->data)
    return CO_EINVAL;
  if (!tokens_fit(desc->batch, T, width)) return CO_ENOTSUP;
  const int64_t need = attend_workspace(*desc, T);
  if (need && (!workspace || workspace_bytes < need)) return CO_ESCRATCH;
  return done(launch_attend(*desc, *cache, *q, *y, T, workspace, as_stream(stream)));
}

}  // extern "C"
