// kt_attention_host.h -- host side of attention over the paged cache: argument checks, workspace layout, launches.
#pragma once
#include "kt_attention.h"
#include "kt_attention_tiles.h"
#include "kt_cache_host.h"

namespace kt {

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

// Trees: their workgroups of kt_attention_tiles.h have 128 rows and leave out waves without any (bf16, more than 128 rows: 256).  By the rows of a sequence and
// head, us with waves / with tiles, 64 sequences of up to 4096 tokens (4 of 30000), 8 heads:
//   bf16  64 features   8 rows 72 / 78 (38 / 40), 32 rows 101 / 83;            128 features  8 rows 155 / 146 (68 / 62), 32 rows 213 / 156;
//         256 features  8 rows (of 2048) 181 / 200 (164 / 150), 32 rows 229 / 203
//   u8    64 features   32 rows 73 / 96 (49 / 49), 64 rows 114 / 110;          128 features  32 rows 108 / 126 (71 / 66), 64 rows 173 / 153 (106 / 78);
//         256 features  32 rows 232 / 317 (146 / 143), 64 rows 360 / 334
//   u4    64 features   64 rows 100 / 113 (60 / 60), 128 rows 169 / 138;       128 features  64 rows 125 / 141 (81 / 76), 128 rows 223 / 171;
//         256 features  64 rows 282 / 317 (175 / 148), 128 rows 494 / 348
static int64_t most_few_tree_rows(const kt_kv_cache* c) { return c->format == KT_KV_BF16 ? 0 : c->format == KT_KV_U8 ? 32 : 64; }

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

template <int KV, int HD, int WAVES, bool PREFIX, bool TREE>
static bool launch_tiles(const TileArgs& t, int64_t wgs, hipStream_t st) {
  const size_t lds = tiles_lds<KV, HD, WAVES, TREE>() + (TREE ? (size_t)(t.a.n_seq + 1) * 4 : 0);
  auto kernel = attend_tiles_kernel<KV, HD, WAVES, PREFIX, TREE>;
  if (!ensure_dynamic_lds(reinterpret_cast<const void*>(kernel), tiles_lds<KV, HD, WAVES, TREE>() + (TREE ? (kMaxSequences + 1) * 4 : 0))) return false;
  kernel<<<dim3((unsigned)wgs), 64 * WAVES, lds, st>>>(t);
  return true;
}

// One call of kt_paged_attention, or (TREE, with its masks) of kt_tree_attention.
template <bool TREE>
static kt_status attend(const kt_kv_cache* cache, const void* Q, int64_t ldq, kt_dtype dtype, const int32_t* q_starts, const int32_t* lens,
                        const int32_t* pages, int64_t ldp, int64_t n_seq, int64_t n_tokens, int64_t max_q, int64_t n_q_heads,
                        const uint64_t* tree, int64_t ldt, const int32_t* prefix_pages, int64_t prefix_len, float scale, void* O, int64_t ldo,
                        float* lse, void* workspace, size_t workspace_bytes, void* stream) {
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
  if (TREE && !tree) return fail(KT_ERR_INVALID_ARG, "tree must not be null");
  if (TREE && (ldt < 1 || ldt > ((int64_t)1 << 24) || max_q > 64 * ldt || misaligned(tree, 8)))
    return fail(KT_ERR_BAD_SHAPE, "ldt must be in [ceil(max_q / 64), 2^24], tree 8-byte aligned");
  if (!(scale > 0.f) || !(scale <= kHuge)) return fail(KT_ERR_INVALID_ARG, "scale must be positive and finite");
  const size_t need = kt_paged_attention_bytes(n_tokens, n_q_heads, hd, prefix_len);
  if (!workspace || workspace_bytes < need)
    return fail(KT_ERR_WORKSPACE_TOO_SMALL, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  if (misaligned(workspace, 256)) return fail(KT_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (misaligned(q_starts, 4) || misaligned(lens, 4) || misaligned(pages, 4) || misaligned(prefix_pages, 4) || misaligned(lse, 4))
    return fail(KT_ERR_BAD_SHAPE, "index arrays and lse must be aligned to their type");

  const int64_t group = n_q_heads / cache->n_heads;
  const int64_t most = TREE ? most_few_tree_rows(cache) : most_few_rows(cache);
  const bool few = max_q <= most && max_q * group <= most;
  const int64_t row_tiles = few ? ceil_div(max_q * group, kRows) : 0;
  const int64_t entries = few ? n_seq * row_tiles : n_tokens * group / (TREE ? 128 : tile_rows(hd)) + n_seq;
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
  a.tree = reinterpret_cast<const unsigned long long*>(tree);
  a.ldt = ldt;
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
    if constexpr (!TREE || KV != kKvBf16) {  // (no tree over bf16 has few rows)
      if (few) {
        if (prefix_len && !launch_tiles<KV, HD, tile_waves(HD), true, false>(t, ceil_div(n_tokens * group, ROWS) * cache->n_heads * t.splits, st)) return false;
        attend_rows_kernel<KV, HD, TREE><<<dim3(kWaveWorkers / 4), 256, (size_t)(n_seq + 1) * 4, st>>>(a);
        if (prefix_len) join_prefix_kernel<HD><<<dim3((unsigned)ceil_div(n_tokens * n_q_heads, kRowsOf)), 256, 0, st>>>(t);
        else attend_join_kernel<HD><<<dim3(kWaveWorkers, 4), 256, 0, st>>>(a);
        return true;
      }
    }
    auto go = [&](auto waves) {
      constexpr int WAVES = decltype(waves)::value, R = 32 * WAVES;
      if constexpr (TREE) {
        t.workers = kTileWorkers * ROWS / R;
        a.row_tiles = (int)std::min<int64_t>(ceil_div(max_q * group, R), INT32_MAX);
      } else {
        plan_tiles_kernel<R><<<1, 1024, 0, st>>>(t);
      }
      if (!launch_tiles<KV, HD, WAVES, false, TREE>(t, t.workers, st)) return false;
      join_tiles_kernel<HD, R, TREE><<<dim3((unsigned)t.workers, R / kRowsOf), 256, 0, st>>>(t);
      return true;
    };
    using std::integral_constant;
    if constexpr (TREE && KV != kKvBf16) return go(integral_constant<int, 4>{});
    else if constexpr (TREE) return max_q * group <= 128 ? go(integral_constant<int, 4>{}) : go(integral_constant<int, tile_waves(HD)>{});
    else return go(integral_constant<int, tile_waves(HD)>{});
  });
  if (!ok) return fail(KT_ERR_DEVICE, "attention kernel needs more LDS than the device gives");
  return launch_ok() ? KT_OK : fail(KT_ERR_DEVICE, "attention kernel launch failed");
}

}  // namespace kt
