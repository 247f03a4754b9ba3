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

// Numbers in the order of the masses, from 1 on: larger is kept before smaller; -0 is 0, a NaN is below all.
__device__ __forceinline__ uint32_t mass_order(float m) {
  const uint32_t b = __float_as_uint(m + 0.f);
  return m != m ? 1u : b ^ (uint32_t)((int)b >> 31 | (int)0x80000000u);
}

// How many of a mask's lanes are in front of this one.
__device__ __forceinline__ uint32_t lanes_below(unsigned long long mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// One sequence and head a workgroup of 16 waves.  The n largest tokens stay, the lower index of equal ones, where the first `sink` and the last `recent` count
// as the largest of all: the n-th largest number is found digit by digit (11, 11 and 10 bits, counted in LDS), then every wave counts what stays in its
// piece of the tokens, and writes it behind that of the waves in front.
// A wave has PER neighbouring rows of 64 tokens, whose numbers it keeps in registers: they are read once, all at the same time.  What is longer than 1024 PER tokens
// goes through in as many parts, read again for every digit.  Digits are counted 8 times side by side (few tokens: twice), by lane: the top digit of a float is
// its exponent, which most of a wave's lanes share, and an LDS counter takes its additions one by one.
// Bound by a compute unit's instructions, and barriers where there are few tokens: 8 heads of 2300 tokens 9 us, 256 of up to 16384 18 us, 16 of up to 65536 33 us
// (numbers read again for each digit and counted row by row instead: 11, 49, 157).
template <int PER>
__global__ __launch_bounds__(1024) void kv_select_kernel(SelectArgs a) {
  constexpr int kBins = 2048, kCopies = PER < 16 ? 2 : 8, PART = 1024 * PER;
  constexpr uint32_t kStays = 0xffffffffu;  // of a token that stays in any case; 0: of one that there is not
  __shared__ __align__(16) int bins[kBins * kCopies];
  __shared__ int counts[2][16];
  __shared__ int found[2];  // bin, numbers above it
  const int s = blockIdx.y, head = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int len = min(max(a.lens[s], 0), (int)(a.ldp << a.log2_page));
  const int n = min(min(max(a.keep[s], 0), len), (int)a.ldk);
  const int recent = min(a.recent, n), sink = min(a.sink, n - recent), last = len - recent;
  const int* pages = a.pages + s * a.ldp;
  int* kept = a.kept + ((int64_t)s * a.n_heads + head) * a.ldk;
  if (head == 0 && threadIdx.x == 0) a.n_kept[s] = n;
  const int page_mask = (1 << a.log2_page) - 1, parts = (int)(((int64_t)len + PART - 1) / PART);
  uint32_t v[PER];  // the lane's numbers of a part: tokens part PART + (wave PER + i) 64 + lane
  auto row = [&](int part, int i) { return part * PART + (wave * PER + i) * 64; };
  auto load = [&](int part) {
    // where the rows' masses lie, one a lane
    static_assert(PER <= 64);
    const int mine = row(part, 0) + 64 * (lane < PER ? lane : 0);
    const int page = pages[min(mine, len - 1) >> a.log2_page];
    const bool there = page >= 0 && page < a.n_pages;
    const int64_t place = there ? ((((int64_t)page * a.n_heads + head) << a.log2_page) + (mine & page_mask)) * 4 : 0;
    const unsigned long long not_there = __ballot(!there && mine < len);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int64_t at = (int64_t)__builtin_amdgcn_readlane((int)(place >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)place, i);
      v[i] = reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(a.mass) + at)[lane];  // (behind the last token: of its page, and not looked at)
    }
    const int row0 = row(part, 0);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      v[i] = mass_order(__uint_as_float(v[i]));
      if (row0 + 64 * i < sink || row0 + 64 * i + 64 > last) {
        const int t = row0 + 64 * i + lane;
        v[i] = t >= len ? 0u : t < sink || t >= last ? kStays : v[i];
      }
    }
    if (not_there)
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (not_there >> i & 1ull) v[i] = v[i] == 0u || v[i] == kStays ? v[i] : 1u;
  };

  uint32_t limit = 0u;  // stays: above it, and the first `ties` equal to it
  int ties = 0;
  if (n == 0) return;
  if (parts == 1) load(0);
  if (n < len) {
    uint32_t prefix = 0;
    int left = n;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
#pragma unroll
      for (int i = 0; i < kBins * kCopies / 4096; ++i) reinterpret_cast<int4*>(bins)[threadIdx.x + 1024 * i] = int4{0, 0, 0, 0};
      __syncthreads();
      for (int part = 0; part < parts; ++part) {
        if (parts > 1) load(part);
        if (pass == 0) {
#pragma unroll
          for (int i = 0; i < PER; ++i) atomicAdd(&bins[(v[i] >> 21) * kCopies + (lane & (kCopies - 1))], 1);
        } else {
          const uint32_t from = prefix << (shift + width);
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            const uint32_t x = v[i] - from;
            if (x >> (shift + width) == 0) atomicAdd(&bins[(x >> shift) * kCopies + (lane & (kCopies - 1))], 1);
          }
        }
      }
      __syncthreads();
      // the bin that the left-th from the top is in: two bins a thread, the top ones first
      const int hi = kBins - 1 - 2 * threadIdx.x;
      auto count = [&](int bin) {
        if constexpr (kCopies == 2) {
          const int2 b = *reinterpret_cast<const int2*>(bins + bin * kCopies);
          return b.x + b.y;
        } else {
          const int4* b = reinterpret_cast<const int4*>(bins + bin * kCopies);
          return b[0].x + b[0].y + b[0].z + b[0].w + b[1].x + b[1].y + b[1].z + b[1].w;
        }
      };
      const int x = count(hi), y = count(hi - 1);
      int upto = sum_up_to(x + y);
      if (lane == 63) counts[0][wave] = upto;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 16; ++w) upto += w < wave ? counts[0][w] : 0;
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
  }
  int at = 0, seen = 0;  // kept, equal ones, in front of the part, then of the wave
  for (int part = 0; part < parts; ++part) {
    if (parts > 1) load(part);
    int stay = 0, same = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {  // (a lane's own: a count of lanes waits for the comparison)
      stay += v[i] > limit;
      same += v[i] == limit;
    }
    stay = sum_up_to(stay);
    same = sum_up_to(same);
    __syncthreads();
    if (lane == 63) counts[0][wave] = stay, counts[1][wave] = same;
    __syncthreads();
    int next = at, next_seen = seen;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w == wave) at = next, seen = next_seen;
      const int e = counts[1][w];
      next += counts[0][w] + min(e, max(0, ties - next_seen));
      next_seen += e;
    }
    at = __builtin_amdgcn_readfirstlane(at);
    seen = __builtin_amdgcn_readfirstlane(seen);
    const int row0 = row(part, 0) + lane;
    char* to = reinterpret_cast<char*>(kept);
    auto write = [&](int i, bool stays) {
      const unsigned long long all = __ballot(stays);
      if (stays) *reinterpret_cast<int*>(to + ((uint32_t)at + lanes_below(all)) * 4u) = row0 + 64 * i;
      at += __popcll(all);
    };
    if (next_seen <= ties || seen >= ties) {  // all of the wave's equal ones stay (those of later waves do), or none
      const uint32_t beyond = seen >= ties ? limit : limit - 1;  // (a limit of 0 has no ties)
#pragma unroll
      for (int i = 0; i < PER; ++i) write(i, v[i] > beyond);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const bool equal = v[i] == limit;
        const unsigned long long equals = __ballot(equal);
        write(i, v[i] > limit || (equal && seen + (int)lanes_below(equals) < ties));
        seen += __popcll(equals);
      }
    }
    at = next;
    seen = next_seen;
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

// Bound by fetches of 64 bytes, of which a list that leaves out most tokens wants a few bytes of values: 32 sequences of up to 16384 to 4096 tokens, 8 heads of
// 128, 4 bits, 104 us, 194 MB fetched and 155 written; 2 of up to 65536 to 8192, bf16, 62 us, 151 and 68.
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
