// kt_cache_host.h -- host helpers of the operators on the paged cache: argument checks, and f(format, head size) of a cache.
#pragma once
#include <algorithm>
#include <type_traits>

#include "kt_host.h"
#include "kt_kvcache.h"

namespace kt {

static bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }

// A launch's x has less than 2^32 threads.
static bool grid_fits(int64_t wgs, int threads) { return wgs <= UINT32_MAX / threads; }

// rows of `width` values of `dtype`: leading dimension and 16-byte alignment
static bool rows_ok(const void* p, int64_t ld, int64_t width, kt_dtype dtype) {
  return ld >= width && ld <= ((int64_t)1 << 24) && ld % (dtype == KT_F32 ? 4 : 8) == 0 && !misaligned(p, 16);
}

static int log2_of(int64_t v) {
  int b = 0;
  while (((int64_t)1 << b) < v) ++b;
  return b;
}

// f(integral_constant<KV>, integral_constant<HD>)
template <class F>
static auto with_cache(const kt_kv_cache* c, F f) {
  using std::integral_constant;
  auto hd = [&](auto kv) {
    if (c->head_dim == 64) return f(kv, integral_constant<int, 64>{});
    if (c->head_dim == 128) return f(kv, integral_constant<int, 128>{});
    return f(kv, integral_constant<int, 256>{});
  };
  if (c->format == KT_KV_BF16) return hd(integral_constant<int, kKvBf16>{});
  if (c->format == KT_KV_U8) return hd(integral_constant<int, kKvU8>{});
  return hd(integral_constant<int, kKvU4>{});
}

static kt_status check_cache_shape(const kt_kv_cache* c) {
  if (!c) return fail(KT_ERR_INVALID_ARG, "cache must not be null");
  if (c->format != KT_KV_BF16 && c->format != KT_KV_U8 && c->format != KT_KV_U4)
    return fail(KT_ERR_BAD_DTYPE, "cache format must be KT_KV_BF16, KT_KV_U8 or KT_KV_U4");
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return fail(KT_ERR_NOT_SUPPORTED, "head_dim = %lld: heads of 64, 128 or 256 features", (long long)c->head_dim);
  if (c->n_pages < 1 || c->n_pages > ((int64_t)1 << 31) - 1) return fail(KT_ERR_BAD_SHAPE, "n_pages must be in [1, 2^31)");
  if (c->n_heads < 1 || c->n_heads > 1024) return fail(KT_ERR_BAD_SHAPE, "n_heads must be in [1, 1024]");
  if (c->page_size < 64 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
    return fail(KT_ERR_BAD_SHAPE, "page_size = %lld: a power of two from 64 to 65536", (long long)c->page_size);
  return KT_OK;
}
static kt_status check_cache(const kt_kv_cache* c) {
  if (kt_status s = check_cache_shape(c)) return s;
  if (!c->data) return fail(KT_ERR_INVALID_ARG, "cache data must not be null");
  if (misaligned(c->data, 16)) return fail(KT_ERR_BAD_SHAPE, "cache data must be 16-byte aligned");
  return KT_OK;
}
static KvCache device_cache(const kt_kv_cache* c) {
  return KvCache{static_cast<char*>(c->data), c->n_pages, (int)c->n_heads, log2_of(c->page_size)};
}

}  // namespace kt
