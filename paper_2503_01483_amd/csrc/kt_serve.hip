// kt_serve.hip -- host side of the serving operators: argument checks, workspace layout, launches, and their part of the extern "C"
// boundary of include/kt.h.
#include "kt_attention.h"
#include "kt_attention_tiles.h"
#include "kt_host.h"
#include "kt_norm.h"

#include <algorithm>
#include <type_traits>

namespace kt {

static bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }

// A launch's x has less than 2^32 threads.
static bool grid_fits(int64_t wgs, int threads) { return wgs <= UINT32_MAX / threads; }

// rows of `width` values of `dtype`: leading dimension and 16-byte alignment
static bool rows_ok(const void* p, int64_t ld, int64_t width, kt_dtype dtype) {
  return ld >= width && ld <= ((int64_t)1 << 24) && ld % (dtype == KT_F32 ? 4 : 8) == 0 && !misaligned(p, 16);
}

// ------------------------------------------------------------------ norm ----------
template <typename T, typename TG, int FORMAT>
static kt_status launch_norm(const NormArgs& a, hipStream_t st) {
  const int64_t chunks = ceil_div(a.d, 8);
  auto go = [&](auto tpr, auto ch) {
    constexpr int TPR = decltype(tpr)::value, CH = decltype(ch)::value, ROWS = TPR >= 256 ? 1 : 256 / TPR;
    const int64_t wgs = ceil_div(a.n, ROWS), x = std::min<int64_t>(wgs, 1 << 20);
    add_rmsnorm_quant_kernel<T, TG, FORMAT, TPR, CH><<<dim3((unsigned)x, (unsigned)ceil_div(wgs, x)), TPR > 256 ? TPR : 256, 0, st>>>(a);
  };
  using std::integral_constant;
  // As many threads a row as leave none idle and a thread one or two chunks: 64 rows / 8192 rows, us, bf16 to 8 bits, with a sum:
  //   512  64 threads 3.3 / 7.1;   2048  64 threads 5.9 / 21.1, 256 threads 3.5 / 22.9;   4096  256 threads 4.9 / 40.5;
  //   8192  256 threads 6.2 / 98.0, 1024 threads 4.5 / 87.5;   16384  1024 threads 5.8 / 176;   32768  8.5 / 357
  if (chunks <= 64) go(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (chunks <= 256) go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (chunks <= 512) go(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (chunks <= 1024) go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  else if (chunks <= 2048) go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  else go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
  return launch_ok() ? KT_OK : fail(KT_ERR_DEVICE, "norm kernel launch failed");
}
template <typename T, typename TG>
static kt_status dispatch_norm(const NormArgs& a, int format, hipStream_t st) {
  switch (format) {
    case KT_Q_NONE: return launch_norm<T, TG, kFormatNone>(a, st);
    case KT_Q_INT4: return launch_norm<T, TG, kFormatInt4>(a, st);
    case KT_Q_INT8: return launch_norm<T, TG, kFormatInt8>(a, st);
    default: return launch_norm<T, TG, kFormatE4M3>(a, st);
  }
}

// ------------------------------------------------------------------ cache ---------
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

// ------------------------------------------------------------------ attention -----
constexpr int64_t kWaveWorkers = (int64_t)kNumCUs * 8;  // waves that share the key tiles of few rows: two workgroups of four a CU (heads of 256, bf16 or 8 bits: registers for one, the others follow)
constexpr int64_t kMaxTokens = (int64_t)1 << 30;         // of a sequence's pages, of a prefix
constexpr int64_t kMaxSequences = 4096;                 // their tile counts are listed in LDS
// Waves of a workgroup of kt_attention_tiles.h: two a SIMD; one where a head of 256 features takes all registers.  (Two workgroups of four
// waves instead of one of eight: a prompt of 2 x 8192 tokens, 32 heads of 128, bf16, 938 us instead of 839: every tile is copied twice.)
constexpr int tile_waves(int64_t hd) { return hd == 256 ? 4 : 8; }
constexpr int64_t tile_rows(int64_t hd) { return 32 * tile_waves(hd); }
constexpr int64_t kTileWorkers = kNumCUs;  // as many as are resident (LDS)

// Single tokens and a few at a time take kt_attention.h, whose time grows with every sixteen rows a head; what has more rows takes
// kt_attention_tiles.h, whose tiles of 256 rows are wasted on fewer.  By the rows of a sequence and head, us with the one / the other, 64
// sequences of 4096 tokens (4 of 30000), 8 heads:
//   bf16  64 features   32 rows 161 / 228 (90 / 112), 64 rows 268 / 221;     128 features  16 rows 221 / 326, 32 rows 301 / 315 (182 / 160);
//         256 features  16 rows 408 / 522, 32 rows 559 / 500
//   u8    64 features   64 rows 190 / 303 (103 / 151), 96 rows 314 / 304;    128 features  64 rows 281 / 369 (166 / 186), 96 rows 475 / 375;
//         256 features  32 rows 365 / 506 (208 / 249), 64 rows 586 / 512
//   u4    64 features   64 rows 150 / 294 (87 / 148);                        128 features  64 rows 215 / 372 (114 / 184), 128 rows 417 / 382;
//         256 features  64 rows 343 / 469 (185 / 231), 96 rows 562 / 472
static int64_t most_few_rows(const kt_kv_cache* c) {
  if (c->format == KT_KV_BF16) return c->head_dim == 64 ? 32 : 16;
  return c->format == KT_KV_U8 && c->head_dim == 256 ? 32 : 64;
}

// Tiles of a prefix that single tokens share are split until the launch fills the card (96 tokens, 8192 in front: 16 splits).
static int64_t prefix_splits(int64_t n_tokens, int64_t hq, int64_t n_heads, int64_t hd, int64_t prefix_len) {
  const int64_t items = ceil_div(n_tokens * (hq / n_heads), tile_rows(hd)) * n_heads;
  return std::max<int64_t>(1, std::min(kTileWorkers / items, ceil_div(prefix_len, 64)));
}

struct AttendPlan {
  size_t tiles, list, cuts, part, whole, prefix, bytes;
};
// Offsets in the workspace; sized for either kernel (hq rows a token, at most kMaxSequences).
static AttendPlan plan_attention(int64_t n_tokens, int64_t hq, int64_t hd, int64_t prefix_len) {
  AttendPlan p{};
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t o = at;
    at += (size_t)round_up(bytes, 256);
    return o;
  };
  const int64_t row = (hd + 2) * 4;
  p.tiles = take(4 * (kMaxSequences + 1));
  p.list = take(16 * (n_tokens * hq / tile_rows(hd) + kMaxSequences + 1));
  p.cuts = take(16 * kWaveWorkers);
  p.part = take(2 * std::max(kWaveWorkers * kRows, kTileWorkers * tile_rows(hd)) * row);
  if (prefix_len) {
    p.whole = take(n_tokens * hq * row);
    // splits x rows: at most all rows once, or as many as fill the card
    p.prefix = take(std::max(n_tokens * hq, kTileWorkers * tile_rows(hd)) * row);
  }
  p.bytes = at;
  return p;
}

template <int KV, int HD, bool PREFIX>
static bool launch_tiles(const TileArgs& t, int64_t wgs, hipStream_t st) {
  constexpr size_t lds = sizeof(TileShared<KV, HD, tile_waves(HD)>);
  auto kernel = attend_tiles_kernel<KV, HD, tile_waves(HD), PREFIX>;
  if (!ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), lds)) return false;
  kernel<<<dim3((unsigned)wgs), 64 * tile_waves(HD), lds, st>>>(t);
  return true;
}

}  // namespace kt

using namespace kt;

extern "C" {

kt_status kt_add_rmsnorm_quant(const void* X, int64_t ldx, const void* res, int64_t ldres, const void* gain, int64_t n, int64_t d,
                               kt_dtype dtype, kt_dtype gain_dtype, float eps, float clip_ratio, kt_qformat format, void* res_out,
                               int64_t ldro, void* Y, int64_t ldy, void* codes, int64_t ldc, float* scales, void* stream) {
  clear_error();
  if (!X) return fail(KT_ERR_INVALID_ARG, "X must not be null");
  if (!res_out && !Y && !codes && !scales) return fail(KT_ERR_INVALID_ARG, "no output requested");
  if (n < 1 || n > ((int64_t)1 << 31) - 1) return fail(KT_ERR_INVALID_ARG, "n must be in [1, 2^31)");
  if (d < 8 || d > 32768 || d % 8) return fail(KT_ERR_BAD_SHAPE, "d = %lld: a multiple of 8 up to 32768", (long long)d);
  if (dtype != KT_F32 && dtype != KT_BF16) return fail(KT_ERR_BAD_DTYPE, "dtype must be KT_F32 or KT_BF16");
  if (gain && gain_dtype != KT_F32 && gain_dtype != KT_BF16) return fail(KT_ERR_BAD_DTYPE, "gain_dtype must be KT_F32 or KT_BF16");
  if (format != KT_Q_NONE && format != KT_Q_INT4 && format != KT_Q_INT8 && format != KT_Q_E4M3)
    return fail(KT_ERR_BAD_DTYPE, "format must be KT_Q_NONE, KT_Q_INT4, KT_Q_INT8 or KT_Q_E4M3");
  if (format == KT_Q_NONE && (codes || scales)) return fail(KT_ERR_INVALID_ARG, "KT_Q_NONE has neither codes nor scales");
  if (!(eps >= 0.f) || !(eps <= kHuge)) return fail(KT_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (!(clip_ratio > 0.f) || !(clip_ratio <= 1.f)) return fail(KT_ERR_INVALID_ARG, "clip_ratio must be in (0, 1]");
  if (!rows_ok(X, ldx, d, dtype) || (res && !rows_ok(res, ldres, d, dtype)) || (res_out && !rows_ok(res_out, ldro, d, dtype)) ||
      (Y && !rows_ok(Y, ldy, d, dtype)))
    return fail(KT_ERR_BAD_SHAPE, "leading dimensions must be in [d, 2^24] and keep rows 16-byte aligned");
  if (gain && misaligned(gain, 16)) return fail(KT_ERR_BAD_SHAPE, "gain must be 16-byte aligned");
  if (codes && (ldc < d || ldc > ((int64_t)1 << 24) || ldc % 8 || misaligned(codes, 8)))
    return fail(KT_ERR_BAD_SHAPE, "ldc must be a multiple of 8 in [d, 2^24], codes 8-byte aligned");
  NormArgs a{X, res, gain, res_out, Y, static_cast<uint8_t*>(codes), scales, ldx, ldres, ldro, ldy, ldc, (int)n, (int)d, eps, clip_ratio,
             format == KT_Q_INT4 ? 7.f : format == KT_Q_INT8 ? 127.f : 448.f};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == KT_F32) return gain && gain_dtype == KT_BF16 ? dispatch_norm<float, bf16>(a, format, st) : dispatch_norm<float, float>(a, format, st);
  return gain && gain_dtype == KT_F32 ? dispatch_norm<bf16, float>(a, format, st) : dispatch_norm<bf16, bf16>(a, format, st);
}

size_t kt_kv_cache_bytes(const kt_kv_cache* cache) {
  if (check_cache_shape(cache) != KT_OK) return 0;
  return with_cache(cache, [&](auto kv, auto hd) {
    const size_t block = kv_block_bytes<decltype(kv)::value, decltype(hd)::value>(), blocks = (size_t)cache->n_heads * (cache->page_size / 64);
    // sizes that no address space holds count as bad
    return (size_t)cache->n_pages > (((size_t)1 << 47) / block) / blocks ? (size_t)0 : (size_t)cache->n_pages * blocks * block;
  });
}

kt_status kt_kv_append(const kt_kv_cache* cache, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                       int64_t n, int64_t n_q_heads, kt_dtype dtype, const int64_t* slots, const int32_t* positions, const float* rope,
                       int64_t n_pos, int64_t rot_dim, int32_t interleaved, int32_t hadamard, void* Q_out, int64_t ldqo, void* stream) {
  clear_error();
  if (kt_status s = check_cache(cache)) return s;
  if (!K || !V || !slots) return fail(KT_ERR_INVALID_ARG, "K, V and slots must not be null");
  if (n < 1 || n > ((int64_t)1 << 31) - 1) return fail(KT_ERR_INVALID_ARG, "n must be in [1, 2^31)");
  if (dtype != KT_F32 && dtype != KT_BF16) return fail(KT_ERR_BAD_DTYPE, "dtype must be KT_F32 or KT_BF16");
  if (!Q != !Q_out) return fail(KT_ERR_INVALID_ARG, "Q and Q_out go together");
  if (Q ? n_q_heads < 1 || n_q_heads > 65536 : n_q_heads != 0) return fail(KT_ERR_BAD_SHAPE, "n_q_heads must be in [1, 65536], or 0 without Q");
  const int64_t hd = cache->head_dim;
  if ((Q && (!rows_ok(Q, ldq, n_q_heads * hd, dtype) || !rows_ok(Q_out, ldqo, n_q_heads * hd, dtype))) ||
      !rows_ok(K, ldk, cache->n_heads * hd, dtype) || !rows_ok(V, ldv, cache->n_heads * hd, dtype))
    return fail(KT_ERR_BAD_SHAPE, "leading dimensions must be in [heads * head_dim, 2^24] and keep rows 16-byte aligned");
  if (rope) {
    if (!positions) return fail(KT_ERR_INVALID_ARG, "positions must not be null with a rope table");
    if (rot_dim < 16 || rot_dim > hd || rot_dim % 16) return fail(KT_ERR_BAD_SHAPE, "rot_dim = %lld: a multiple of 16 up to head_dim", (long long)rot_dim);
    if (n_pos < 1) return fail(KT_ERR_INVALID_ARG, "n_pos must be positive");
    if (misaligned(rope, 16)) return fail(KT_ERR_BAD_SHAPE, "rope must be 16-byte aligned");
  }
  if (misaligned(slots, 8) || misaligned(positions, 4)) return fail(KT_ERR_BAD_SHAPE, "slots and positions must be aligned to their type");
  const int64_t rows = 256 / (hd / 8), chunks = ceil_div(n_q_heads + cache->n_heads, rows);
  AppendArgs a{device_cache(cache), Q, K, V, Q_out, ldq, ldk, ldv, ldqo, slots, positions, rope, n_pos, (int)n, (int)n_q_heads,
               rope ? (int)rot_dim : 0, (int)chunks, interleaved != 0, hadamard != 0};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t wgs = n * chunks + ceil_div(n, rows) * cache->n_heads;
  if (!grid_fits(wgs, 256)) return fail(KT_ERR_NOT_SUPPORTED, "too many rows for one call");
  with_cache(cache, [&](auto kv, auto h) {
    constexpr int KV = decltype(kv)::value, HD = decltype(h)::value;
    if (dtype == KT_F32) kv_append_kernel<float, KV, HD><<<dim3((unsigned)wgs), 256, 0, st>>>(a);
    else kv_append_kernel<bf16, KV, HD><<<dim3((unsigned)wgs), 256, 0, st>>>(a);
  });
  return launch_ok() ? KT_OK : fail(KT_ERR_DEVICE, "append kernel launch failed");
}

kt_status kt_kv_gather(const kt_kv_cache* cache, const int64_t* slots, int64_t n, void* K, int64_t ldk, void* V, int64_t ldv, kt_dtype dtype,
                       void* stream) {
  clear_error();
  if (kt_status s = check_cache(cache)) return s;
  if (!slots || (!K && !V)) return fail(KT_ERR_INVALID_ARG, "slots and one of K, V must not be null");
  if (n < 1 || n > ((int64_t)1 << 31) - 1) return fail(KT_ERR_INVALID_ARG, "n must be in [1, 2^31)");
  if (dtype != KT_F32 && dtype != KT_BF16) return fail(KT_ERR_BAD_DTYPE, "dtype must be KT_F32 or KT_BF16");
  const int64_t hd = cache->head_dim;
  if ((K && !rows_ok(K, ldk, cache->n_heads * hd, dtype)) || (V && !rows_ok(V, ldv, cache->n_heads * hd, dtype)))
    return fail(KT_ERR_BAD_SHAPE, "leading dimensions must be in [heads * head_dim, 2^24] and keep rows 16-byte aligned");
  if (misaligned(slots, 8)) return fail(KT_ERR_BAD_SHAPE, "slots must be aligned to their type");
  const int64_t rows = 256 / (hd / 8), chunks = K ? ceil_div(cache->n_heads, rows) : 0;
  GatherArgs a{device_cache(cache), slots, K, V, ldk, ldv, (int)n, (int)chunks};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t wgs = n * chunks + (V ? ceil_div(n, rows) * cache->n_heads : 0);
  if (!grid_fits(wgs, 256)) return fail(KT_ERR_NOT_SUPPORTED, "too many rows for one call");
  with_cache(cache, [&](auto kv, auto h) {
    constexpr int KV = decltype(kv)::value, HD = decltype(h)::value;
    if (dtype == KT_F32) kv_gather_kernel<float, KV, HD><<<dim3((unsigned)wgs), 256, 0, st>>>(a);
    else kv_gather_kernel<bf16, KV, HD><<<dim3((unsigned)wgs), 256, 0, st>>>(a);
  });
  return launch_ok() ? KT_OK : fail(KT_ERR_DEVICE, "gather kernel launch failed");
}

size_t kt_paged_attention_bytes(int64_t n_tokens, int64_t n_q_heads, int64_t head_dim, int64_t prefix_len) {
  if (n_tokens < 1 || n_tokens > INT32_MAX || n_q_heads < 1 || n_q_heads > 65535 || (head_dim != 64 && head_dim != 128 && head_dim != 256) ||
      prefix_len < 0 || prefix_len > kMaxTokens)
    return 0;
  return plan_attention(n_tokens, n_q_heads, head_dim, prefix_len).bytes;
}

kt_status kt_paged_attention(const kt_kv_cache* cache, const void* Q, int64_t ldq, kt_dtype dtype, const int32_t* q_starts, const int32_t* lens,
                             const int32_t* pages, int64_t ldp, int64_t n_seq, int64_t n_tokens, int64_t max_q, int64_t n_q_heads,
                             const int32_t* prefix_pages, int64_t prefix_len, float scale, void* O, int64_t ldo, float* lse,
                             void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  if (kt_status s = check_cache(cache)) return s;
  if (!Q || !lens || !pages || !O) return fail(KT_ERR_INVALID_ARG, "Q, lens, pages and O must not be null");
  if (dtype != KT_BF16) return fail(KT_ERR_BAD_DTYPE, "dtype must be KT_BF16");
  if (n_seq < 1 || n_tokens < 1 || n_tokens > INT32_MAX || max_q < 1) return fail(KT_ERR_INVALID_ARG, "n_seq, n_tokens and max_q must be positive");
  if (n_seq > kMaxSequences) return fail(KT_ERR_NOT_SUPPORTED, "n_seq = %lld: at most %lld sequences a call", (long long)n_seq, (long long)kMaxSequences);
  if (!q_starts && (n_tokens != n_seq || max_q != 1)) return fail(KT_ERR_INVALID_ARG, "without q_starts every sequence has one query");
  const int64_t hd = cache->head_dim;
  if (n_q_heads < 1 || n_q_heads > 65535 || n_q_heads % cache->n_heads)
    return fail(KT_ERR_BAD_SHAPE, "n_q_heads must be a multiple of the cache's heads, at most 65535");
  if (!rows_ok(Q, ldq, n_q_heads * hd, dtype) || ldo < n_q_heads * hd || ldo > ((int64_t)1 << 24) || ldo % 4 || misaligned(O, 8))
    return fail(KT_ERR_BAD_SHAPE, "leading dimensions must be in [heads * head_dim, 2^24], rows of Q 16-byte and of O 8-byte aligned");
  if (ldp < 1 || ldp > kMaxTokens / cache->page_size) return fail(KT_ERR_BAD_SHAPE, "ldp must be positive, ldp * page_size at most 2^30");
  if (prefix_len < 0 || prefix_len > kMaxTokens || (prefix_len && !prefix_pages))
    return fail(KT_ERR_INVALID_ARG, "prefix_len must be in [0, 2^30], with prefix_pages");
  if (!(scale > 0.f) || !(scale <= kHuge)) return fail(KT_ERR_INVALID_ARG, "scale must be positive and finite");
  const size_t need = kt_paged_attention_bytes(n_tokens, n_q_heads, hd, prefix_len);
  if (!workspace || workspace_bytes < need)
    return fail(KT_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  if (misaligned(workspace, 256)) return fail(KT_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (misaligned(q_starts, 4) || misaligned(lens, 4) || misaligned(pages, 4) || misaligned(prefix_pages, 4) || misaligned(lse, 4))
    return fail(KT_ERR_BAD_SHAPE, "index arrays and lse must be aligned to their type");

  const int64_t group = n_q_heads / cache->n_heads;
  const int64_t most = most_few_rows(cache);
  const bool few = max_q <= most && max_q * group <= most;
  const int64_t row_tiles = few ? ceil_div(max_q * group, kRows) : 0;
  const int64_t entries = few ? n_seq * row_tiles : n_tokens * group / tile_rows(hd) + n_seq;
  if (entries > INT32_MAX / 2 / cache->n_heads / (ceil_div(ldp * cache->page_size, 64) + (few ? 0 : ceil_div(prefix_len, 64) + kSegmentCost)))
    return fail(KT_ERR_NOT_SUPPORTED, "too many tiles of 64 keys for one call: hand in a narrower page table or fewer tokens");

  if (few && prefix_len && !grid_fits(ceil_div(n_tokens * n_q_heads, 1024 / hd), 256))
    return fail(KT_ERR_NOT_SUPPORTED, "too many rows of queries for one call");

  const AttendPlan p = plan_attention(n_tokens, n_q_heads, hd, prefix_len);
  char* ws = static_cast<char*>(workspace);
  auto floats = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
  TileArgs t{};
  AttendArgs& a = t.a;
  a.cache = device_cache(cache);
  a.q = static_cast<const bf16*>(Q);
  a.q_starts = q_starts;
  a.lens = lens;
  a.pages = pages;
  a.ldq = ldq;
  a.ldp = ldp;
  a.n_seq = (int)n_seq;
  a.n_tokens = (int)n_tokens;
  a.hq = (int)n_q_heads;
  a.group = (int)group;
  a.row_tiles = (int)row_tiles;
  a.scale = scale;
  a.out = static_cast<bf16*>(O);
  a.ldo = ldo;
  a.lse = lse;
  a.workers = (int)kWaveWorkers;
  a.tiles = reinterpret_cast<int*>(ws + p.tiles);
  t.list = reinterpret_cast<int4*>(ws + p.list);
  a.cuts = t.cuts = reinterpret_cast<int4*>(ws + p.cuts);
  a.part = t.part = floats(p.part);
  a.whole = prefix_len ? floats(p.whole) : nullptr;
  t.prefix_pages = prefix_pages;
  t.prefix_len = (int)prefix_len;
  t.workers = (int)kTileWorkers;
  t.entries = (int)entries;
  t.prefix_part = prefix_len ? floats(p.prefix) : nullptr;
  t.splits = prefix_len ? (int)prefix_splits(n_tokens, n_q_heads, cache->n_heads, hd, prefix_len) : 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool ok = with_cache(cache, [&](auto kv, auto h) {
    constexpr int KV = decltype(kv)::value, HD = decltype(h)::value, kRowsOf = 1024 / HD, ROWS = tile_rows(HD);  // (rows of a workgroup that joins)
    if (!few) {
      plan_tiles_kernel<ROWS><<<1, 1024, 0, st>>>(t);
      if (!launch_tiles<KV, HD, false>(t, t.workers, st)) return false;
      join_tiles_kernel<HD, ROWS><<<dim3((unsigned)t.workers, ROWS / kRowsOf), 256, 0, st>>>(t);
      return true;
    }
    if (prefix_len && !launch_tiles<KV, HD, true>(t, ceil_div(n_tokens * group, ROWS) * cache->n_heads * t.splits, st)) return false;
    attend_rows_kernel<KV, HD><<<dim3(kWaveWorkers / 4), 256, (size_t)(n_seq + 1) * 4, st>>>(a);
    if (prefix_len) join_prefix_kernel<HD><<<dim3((unsigned)ceil_div(n_tokens * n_q_heads, kRowsOf)), 256, 0, st>>>(t);
    else attend_join_kernel<HD><<<dim3(kWaveWorkers, 4), 256, 0, st>>>(a);
    return true;
  });
  if (!ok) return fail(KT_ERR_DEVICE, "attention kernel needs more LDS than the device gives");
  return launch_ok() ? KT_OK : fail(KT_ERR_DEVICE, "attention kernel launch failed");
}

}  // extern "C"
