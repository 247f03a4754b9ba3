// kt_evict.h -- which tokens of the paged cache stay within a budget, and moving tokens together.
#pragma once
#include "kt_kvcache.h"

namespace kt {

struct SelectArgs {
  const float* mass;  // [page][head][token of the page]
  const int *lens, *pages, *keep;
  int64_t n_pages, ldp, ldk;
  int n_heads, log2_page, sink, recent;
  int *kept, *n_kept;
};

// Numbers in the order of the masses: larger is kept before smaller; -0 is 0, a NaN is below all.
__device__ __forceinline__ uint32_t mass_order(float m) {
  const uint32_t b = __float_as_uint(m + 0.f);
  return m != m ? 0u : b >> 31 ? ~b : b | 0x80000000u;
}

// One sequence and head a workgroup of 1024.  Of the tokens between the first `sink` and the last `recent` the k largest stay, the lower index of equal
// ones: the k-th largest number is found digit by digit (11, 11 and 10 bits, counted in LDS), then every wave counts what stays in its piece of
// the tokens, and writes it behind that of the waves in front.
__global__ __launch_bounds__(1024) void kv_select_kernel(SelectArgs a) {
  constexpr int kBins = 2048;
  __shared__ int bins[kBins];
  __shared__ int counts[2][16];
  __shared__ int found[3];  // bin, numbers above it
  const int s = blockIdx.y, head = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int len = min(max(a.lens[s], 0), (int)(a.ldp << a.log2_page));
  const int n = min(min(max(a.keep[s], 0), len), (int)a.ldk);
  const int recent = min(a.recent, n), sink = min(a.sink, n - recent);
  const int first = sink, last = len - recent;  // the tokens to choose from
  int k = n - recent - sink;
  const int* pages = a.pages + s * a.ldp;
  int* kept = a.kept + ((int64_t)s * a.n_heads + head) * a.ldk;
  if (head == 0 && threadIdx.x == 0) a.n_kept[s] = n;
  const int page_mask = (1 << a.log2_page) - 1;
  auto number = [&](int t) {  // (of a page outside the cache: as a NaN's)
    const int page = pages[t >> a.log2_page];
    return page < 0 || page >= a.n_pages ? 0u : mass_order(a.mass[(((int64_t)page * a.n_heads + head) << a.log2_page) + (t & page_mask)]);
  };
  uint32_t limit = 0xffffffffu;  // stays: above it, and the first `ties` equal to it
  int ties = 0;
  if (k > 0 && k < last - first) {
    uint32_t prefix = 0;
    int left = k;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      constexpr int kShift[3] = {21, 10, 0};
      const int shift = kShift[pass], width = pass == 2 ? 10 : 11;
      for (int i = threadIdx.x; i < kBins; i += 1024) bins[i] = 0;
      __syncthreads();
      for (int t = first + threadIdx.x; t < last; t += 1024) {
        const uint32_t v = number(t);
        if (pass == 0 || v >> (shift + width) == prefix) atomicAdd(&bins[v >> shift & ((1u << width) - 1)], 1);
      }
      __syncthreads();
      // the bin that the left-th from the top is in: two bins a thread, the top ones first
      const int hi = kBins - 1 - 2 * threadIdx.x, x = bins[hi], y = bins[hi - 1];
      int upto = x + y;
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const int v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
      }
      if (lane == 63) counts[0][wave] = upto;
      __syncthreads();
      for (int w = 0; w < wave; ++w) upto += counts[0][w];
      const int above = upto - x - y;
      if (above < left && left <= upto) {
        const bool second = above + x < left;
        found[0] = second ? hi - 1 : hi;
        found[1] = second ? above + x : above;
      }
      __syncthreads();
      prefix = prefix << width | found[0];
      left -= found[1];
    }
    limit = prefix;
    ties = left;
  } else if (k > 0) {
    limit = 0u;
    ties = len;
  }
  // pieces of whole waves
  const int piece = ((len + 1023) >> 10) * 64, from = wave * piece, to = min(from + piece, len);
  auto look = [&](int t, bool& stays, bool& equal) {
    const bool in = t < to, middle = in && t >= first && t < last && k > 0;
    const uint32_t v = middle ? number(t) : 0u;
    stays = in && (!middle ? t < first || t >= last : v > limit);
    equal = middle && v == limit;
  };
  int stay = 0, same = 0;
  for (int t = from; t < to; t += 64) {
    bool stays, equal;
    look(t + lane, stays, equal);
    stay += __popcll(__ballot(stays));
    same += __popcll(__ballot(equal));
  }
  if (lane == 0) counts[0][wave] = stay, counts[1][wave] = same;
  __syncthreads();
  int at = 0, seen = 0;  // kept, equal ones, in front of the wave
  for (int w = 0; w < wave; ++w) {
    const int e = counts[1][w];
    at += counts[0][w] + min(e, max(0, ties - seen));
    seen += e;
  }
  const unsigned long long below = (1ull << lane) - 1;
  for (int t = from; t < to; t += 64) {
    bool stays, equal;
    look(t + lane, stays, equal);
    const unsigned long long equals = __ballot(equal);
    stays = stays || (equal && seen + __popcll(equals & below) < ties);
    const unsigned long long all = __ballot(stays);
    if (stays) kept[at + __popcll(all & below)] = t + lane;
    at += __popcll(all);
    seen += __popcll(equals);
  }
}

struct CompactArgs {
  KvCache cache;
  const int *pages, *to_pages;  // to_pages null: in place
  int64_t ldp, ldt, lds;
  const int *src, *count, *first;
  int heads_of_src;             // 1, or one list a head
  float* mass;
};

// Tokens src[j] of a sequence become its tokens first + j.  A workgroup of 256 takes the tokens of one block of where they go: source places of the
// 64 are looked up once, keys move 16 bytes a lane, values token by token of each row of a feature.  Into other pages every block has a workgroup of its
// own; in place one workgroup takes a head's blocks in turn, and reads all of a block's tokens before it writes any: lists ascend, so that no token
// is written that a later block reads.
template <int KV, int HD, bool IN_PLACE>
__global__ __launch_bounds__(256) void kv_compact_kernel(CompactArgs a) {
  constexpr int HALF = kv_half_bytes<KV, HD>(), KEY = HALF / kBlockTokens, PIECES = HALF / 16, KP = (PIECES + 255) / 256;
  constexpr int UNIT = KV == kKvBf16 ? 2 : 1, ROWS = KV == kKvU4 ? HD / 2 : HD, VP = ROWS / 4;
  using unit = std::conditional_t<UNIT == 2, uint16_t, uint8_t>;
  __shared__ const char* from_block[64];  // null: nothing goes here
  __shared__ int from_tok[64];
  const int head = blockIdx.y, s = blockIdx.z, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t count = min((int64_t)max(a.count[s], 0), a.lds), first = a.first ? a.first[s] : 0;
  if (first < 0) return;
  const int* src = a.src + ((int64_t)s * a.heads_of_src + (a.heads_of_src > 1 ? head : 0)) * a.lds;
  const int *pages = a.pages + s * a.ldp, *into = IN_PLACE ? pages : a.to_pages + s * a.ldt;
  const int log2_page = a.cache.log2_page, page_mask = (1 << log2_page) - 1;
  const int64_t most = a.ldp << log2_page, most_to = (IN_PLACE ? a.ldp : a.ldt) << log2_page;
  for (int64_t b = (first >> 6) + blockIdx.x; b * 64 < min(first + count, most_to); b += gridDim.x) {
    const int to_page = into[b * 64 >> log2_page];
    const bool there = to_page >= 0 && to_page < a.cache.n_pages;
    char* to = there ? a.cache.data + kv_block_offset<KV, HD>(a.cache, to_page, head, (int)(b * 64 & page_mask) >> 6) : nullptr;
    if (IN_PLACE) __syncthreads();
    if (threadIdx.x < 64) {
      const int64_t j = b * 64 + lane - first;
      const char* block = nullptr;
      int tok = 0;
      if (there && j >= 0 && j < count) {
        const int t = src[j];
        if (t >= 0 && t < most && !(IN_PLACE && t == j + first)) {
          const int page = pages[t >> log2_page];
          tok = t & 63;
          if (page >= 0 && page < a.cache.n_pages) block = a.cache.data + kv_block_offset<KV, HD>(a.cache, page, head, (t & page_mask) >> 6);
        }
      }
      from_block[lane] = block;
      from_tok[lane] = tok;
    }
    __syncthreads();
    const char* mine = from_block[lane];
    const int tok = from_tok[lane];
    u32x4 k[KP];
    unit v[VP];
    float2 par = {0.f, 0.f};
    float mass = 0.f;
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      const int p = threadIdx.x + 256 * i, of = p * 16 / KEY;
      if (p < PIECES && from_block[of]) k[i] = *reinterpret_cast<const u32x4*>(from_block[of] + from_tok[of] * KEY + p * 16 % KEY);
    }
    if (mine) {
#pragma unroll
      for (int i = 0; i < VP; ++i) v[i] = *reinterpret_cast<const unit*>(mine + HALF + ((4 * i + wave) * kBlockTokens + tok) * UNIT);
      if (KV != kKvBf16 && wave < 2) par = reinterpret_cast<const float2*>(mine + 2 * HALF)[wave * kBlockTokens + tok];
      // (a block's page and head are its number, so that its mass lies where it does)
      if (a.mass && wave == 2) mass = a.mass[(mine - a.cache.data) / kv_block_bytes<KV, HD>() * kBlockTokens + tok];
    }
    if (IN_PLACE) {  // all loads have arrived before any store
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      const int p = threadIdx.x + 256 * i;
      if (p < PIECES && from_block[p * 16 / KEY]) *reinterpret_cast<u32x4*>(to + p * 16) = k[i];
    }
    if (mine) {
#pragma unroll
      for (int i = 0; i < VP; ++i) *reinterpret_cast<unit*>(to + HALF + ((4 * i + wave) * kBlockTokens + lane) * UNIT) = v[i];
      if (KV != kKvBf16 && wave < 2) reinterpret_cast<float2*>(to + 2 * HALF)[wave * kBlockTokens + lane] = par;
      if (a.mass && wave == 2) a.mass[(to - a.cache.data) / kv_block_bytes<KV, HD>() * kBlockTokens + lane] = mass;
    }
    if (!IN_PLACE) __syncthreads();
  }
}

}  // namespace kt
