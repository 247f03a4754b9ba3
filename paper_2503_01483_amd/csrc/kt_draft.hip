// kt_draft.hip -- the part of the extern "C" boundary of include/kt.h that serves drafted tokens and budgets of cached ones: argument checks and launches.
#include "kt_attention_host.h"
#include "kt_evict.h"
#include "kt_mass.h"

namespace kt {

// Index arrays of a call's sequences.
static kt_status check_sequences(const kt_kv_cache* c, int64_t ldp, int64_t n_seq) {
  if (n_seq < 1) return fail(KT_ERR_INVALID_ARG, "n_seq must be positive");
  if (n_seq > kMaxSequences) return fail(KT_ERR_NOT_SUPPORTED, "n_seq = %lld: at most %lld sequences a call", (long long)n_seq, (long long)kMaxSequences);
  if (ldp < 1 || ldp > kMaxTokens / c->page_size) return fail(KT_ERR_BAD_SHAPE, "ldp must be positive, ldp * page_size at most 2^30");
  return KT_OK;
}

}  // namespace kt

using namespace kt;

extern "C" {

kt_status kt_tree_attention(const kt_kv_cache* cache, const void* Q, int64_t ldq, kt_dtype dtype, const int32_t* q_starts, const int32_t* lens,
                            const int32_t* pages, int64_t ldp, int64_t n_seq, int64_t n_tokens, int64_t max_q, int64_t n_q_heads,
                            const uint64_t* tree, int64_t ldt, const int32_t* prefix_pages, int64_t prefix_len, float scale, void* O, int64_t ldo,
                            float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return attend<true>(cache, Q, ldq, dtype, q_starts, lens, pages, ldp, n_seq, n_tokens, max_q, n_q_heads, tree, ldt, prefix_pages, prefix_len, scale, O,
                      ldo, lse, workspace, workspace_bytes, stream);
}

kt_status kt_attention_mass(const kt_kv_cache* cache, const void* Q, int64_t ldq, kt_dtype dtype, const int32_t* q_starts, const int32_t* lens,
                            const int32_t* pages, int64_t ldp, int64_t n_seq, int64_t n_tokens, int64_t max_q, int64_t n_q_heads, float scale,
                            const float* lse, float decay, float* mass, void* stream) {
  clear_error();
  if (kt_status s = check_cache(cache)) return s;
  if (!Q || !lens || !pages || !lse || !mass) return fail(KT_ERR_INVALID_ARG, "Q, lens, pages, lse and mass must not be null");
  if (dtype != KT_BF16) return fail(KT_ERR_BAD_DTYPE, "dtype must be KT_BF16");
  if (n_tokens < 1 || n_tokens > INT32_MAX || max_q < 1) return fail(KT_ERR_INVALID_ARG, "n_tokens and max_q must be positive");
  if (kt_status s = check_sequences(cache, ldp, n_seq)) return s;
  if (!q_starts && (n_tokens != n_seq || max_q != 1)) return fail(KT_ERR_INVALID_ARG, "without q_starts every sequence has one query");
  const int64_t hd = cache->head_dim;
  if (n_q_heads < 1 || n_q_heads > 65535 || n_q_heads % cache->n_heads)
    return fail(KT_ERR_BAD_SHAPE, "n_q_heads must be a multiple of the cache's heads, at most 65535");
  if (!rows_ok(Q, ldq, n_q_heads * hd, dtype)) return fail(KT_ERR_BAD_SHAPE, "ldq must be in [heads * head_dim, 2^24] and keep rows 16-byte aligned");
  if (!(scale > 0.f) || !(scale <= kHuge)) return fail(KT_ERR_INVALID_ARG, "scale must be positive and finite");
  if (!(decay >= 0.f) || !(decay <= kHuge)) return fail(KT_ERR_INVALID_ARG, "decay must be finite and not negative");
  if (misaligned(q_starts, 4) || misaligned(lens, 4) || misaligned(pages, 4) || misaligned(lse, 4) || misaligned(mass, 4))
    return fail(KT_ERR_BAD_SHAPE, "index arrays, lse and mass must be aligned to their type");
  if (n_seq > INT32_MAX / ceil_div(ldp * cache->page_size, 64)) return fail(KT_ERR_NOT_SUPPORTED, "too many blocks of 64 keys for one call: hand in a narrower page table");
  MassArgs t{};
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
  a.group = (int)(n_q_heads / cache->n_heads);
  a.scale = scale;
  t.lse = lse;
  t.mass = mass;
  t.decay = decay;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int64_t most = std::min(max_q, n_tokens) * a.group;  // rows a head
  const bool ok = with_cache(cache, [&](auto kv, auto h) {
    constexpr int KV = decltype(kv)::value, HD = decltype(h)::value;
    using std::integral_constant;
    const int64_t tokens = ldp * cache->page_size;
    const size_t list = mass_lists(n_seq);
    auto grid = [&](int keys) { return dim3((unsigned)std::min<int64_t>(n_seq * ceil_div(tokens, keys) * cache->n_heads, kNumCUs * 8)); };
    auto go_few = [&](auto ni) {
      mass_few_kernel<KV, HD, decltype(ni)::value><<<grid(256), 256, list, st>>>(t);
      return true;
    };
    if (most <= 4) return go_few(integral_constant<int, 1>{});
    if (most <= 64) return go_few(integral_constant<int, 4>{});
    auto kernel = mass_rows_kernel<KV, HD>;
    if (!ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), sizeof(MassShared<HD>) + mass_lists(kMaxSequences))) return false;
    kernel<<<grid(128), 512, sizeof(MassShared<HD>) + list, st>>>(t);
    return true;
  });
  if (!ok) return fail(KT_ERR_DEVICE, "mass kernel needs more LDS than the device gives");
  return launch_ok() ? KT_OK : fail(KT_ERR_DEVICE, "mass kernel launch failed");
}

kt_status kt_kv_select(const kt_kv_cache* cache, const float* mass, const int32_t* lens, const int32_t* pages, int64_t ldp, int64_t n_seq,
                       const int32_t* keep, int64_t sink, int64_t recent, int32_t* kept, int64_t ldk, int32_t* n_kept, void* stream) {
  clear_error();
  if (kt_status s = check_cache_shape(cache)) return s;
  if (!mass || !lens || !pages || !keep || !kept || !n_kept) return fail(KT_ERR_INVALID_ARG, "mass, lens, pages, keep, kept and n_kept must not be null");
  if (kt_status s = check_sequences(cache, ldp, n_seq)) return s;
  if (n_kept == lens) return fail(KT_ERR_INVALID_ARG, "n_kept must not be lens");
  if (sink < 0 || recent < 0) return fail(KT_ERR_INVALID_ARG, "sink and recent must not be negative");
  if (ldk < 1 || ldk > kMaxTokens) return fail(KT_ERR_BAD_SHAPE, "ldk must be in [1, 2^30]");
  if (misaligned(mass, 4) || misaligned(lens, 4) || misaligned(pages, 4) || misaligned(keep, 4) || misaligned(kept, 4) || misaligned(n_kept, 4))
    return fail(KT_ERR_BAD_SHAPE, "arrays must be aligned to their type");
  const SelectArgs a{mass, lens, pages, keep, cache->n_pages, ldp, ldk, (int)cache->n_heads, log2_of(cache->page_size),
                     (int)std::min(sink, kMaxTokens), (int)std::min(recent, kMaxTokens), kept, n_kept};
  // as many rows of 64 tokens a wave as the page table has room for
  auto go = [&](auto per) {
    kv_select_kernel<decltype(per)::value><<<dim3((unsigned)cache->n_heads, (unsigned)n_seq), 1024, 0, static_cast<hipStream_t>(stream)>>>(a);
  };
  using std::integral_constant;
  const int64_t rows = ceil_div(ldp * cache->page_size, 1024);
  if (rows <= 2) go(integral_constant<int, 2>{});
  else if (rows <= 4) go(integral_constant<int, 4>{});
  else if (rows <= 16) go(integral_constant<int, 16>{});
  else go(integral_constant<int, 64>{});
  return launch_ok() ? KT_OK : fail(KT_ERR_DEVICE, "select kernel launch failed");
}

kt_status kt_kv_compact(const kt_kv_cache* cache, const int32_t* pages, int64_t ldp, int64_t n_seq, const int32_t* src, int64_t lds, int32_t per_head,
                        const int32_t* count, const int32_t* first, const int32_t* to_pages, int64_t ldt, float* mass, void* stream) {
  clear_error();
  if (kt_status s = check_cache(cache)) return s;
  if (!pages || !src || !count) return fail(KT_ERR_INVALID_ARG, "pages, src and count must not be null");
  if (kt_status s = check_sequences(cache, ldp, n_seq)) return s;
  const bool in_place = !to_pages || to_pages == pages;
  if (!in_place && (ldt < 1 || ldt > kMaxTokens / cache->page_size)) return fail(KT_ERR_BAD_SHAPE, "ldt must be positive, ldt * page_size at most 2^30");
  if (to_pages == pages && ldt != ldp) return fail(KT_ERR_BAD_SHAPE, "to_pages is pages: ldt must be ldp");
  if (lds < 1 || lds > kMaxTokens) return fail(KT_ERR_BAD_SHAPE, "lds must be in [1, 2^30]");
  if (misaligned(pages, 4) || misaligned(src, 4) || misaligned(count, 4) || misaligned(first, 4) || misaligned(to_pages, 4) || misaligned(mass, 4))
    return fail(KT_ERR_BAD_SHAPE, "index arrays and mass must be aligned to their type");
  const CompactArgs a{device_cache(cache), pages, in_place ? nullptr : to_pages, ldp, ldt, lds, src, count, first, per_head ? (int)cache->n_heads : 1, mass};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid(in_place ? 1u : (unsigned)std::min<int64_t>(ceil_div(lds, 64) + (first ? 1 : 0), 1024), (unsigned)cache->n_heads, (unsigned)n_seq);
  with_cache(cache, [&](auto kv, auto h) {
    constexpr int KV = decltype(kv)::value, HD = decltype(h)::value;
    if (in_place) kv_compact_kernel<KV, HD, true><<<grid, 256, 0, st>>>(a);
    else kv_compact_kernel<KV, HD, false><<<grid, 256, 0, st>>>(a);
  });
  return launch_ok() ? KT_OK : fail(KT_ERR_DEVICE, "compact kernel launch failed");
}

}  // extern "C"
