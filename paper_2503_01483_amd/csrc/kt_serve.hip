// kt_serve.hip -- the serving operators' part of the extern "C" boundary of include/kt.h: argument checks and launches (attention's are in
// kt_attention_host.h; drafted tokens and eviction: kt_draft.hip).
#include "kt_attention_host.h"
#include "kt_norm.h"

namespace kt {

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
  return attend<false>(cache, Q, ldq, dtype, q_starts, lens, pages, ldp, n_seq, n_tokens, max_q, n_q_heads, nullptr, 0, prefix_pages, prefix_len, scale,
                       O, ldo, lse, workspace, workspace_bytes, stream);
}

}  // extern "C"
