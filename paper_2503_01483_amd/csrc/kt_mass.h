// kt_mass.h -- attention weight that the tokens of the paged cache receive from new queries, accumulated a token and key head.
//
//   mass_j <- decay mass_j (0 of a token that is one of the queries) + sum_r exp(scale q_r . k_j - lse_r),  r over the rows of j's key head that see j
//
// A wave holds 64 keys, one block of the cache, and goes through the rows sixteen at a time, S = Q K^T in 16 x 16 x 32 products with the keys on the
// columns: a lane has four keys and of each the scores of four rows, whose exponentials it adds up; the four quarters of the wave are added once at the
// end.  A token's {step, minimum} are its lane's own, and neighbouring lanes write neighbouring masses.  Every sum has a fixed order and one owner: nothing
// is atomic, no score leaves the registers.  Of a page that sequences share, the first of them that has a token owns its mass (owned_in_front).
// With few rows, row j of sixteen is row 4 (j % 4) + j / 4 of the products, so that the first four (a token's, with four queries a head) lie in one register of
// every quarter, and only that is exponentiated.
#pragma once
#include "kt_attention.h"

namespace kt {

struct MassArgs {
  AttendArgs a;     // cache, q, q_starts, lens, pages, ldq, ldp, n_seq, n_tokens, hq, group, scale, lse (read)
  const float* lse;
  float* mass;      // [page][head][token of the page]
  float decay;
};

// As to_lds_16, 4 bytes a lane.
__device__ __forceinline__ void to_lds_4(uint32_t voffset, const char* base, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(voffset), "s"(base), "s"(lds_addr) : "memory", "m0");
}

// Lists of sequences (LDS): a tag of the page that each begins with [n_seq, rounded up], groups of keys of one head in front of each [n_seq + 1].
constexpr int kTagsAtOnce = 512;  // a wave's 16-byte loads
__host__ __device__ constexpr int64_t mass_tags_bytes(int64_t n_seq) { return (n_seq + kTagsAtOnce - 1) / kTagsAtOnce * kTagsAtOnce * 2; }
constexpr size_t mass_lists(int64_t n_seq) { return (size_t)(mass_tags_bytes(n_seq) + (n_seq + 1) * 4); }
__device__ __forceinline__ uint16_t page_tag(int page) { return (uint16_t)((uint32_t)page * 2654435761u >> 16); }  // (2^32 / golden ratio)

// By a workgroup of THREADS.
template <int THREADS>
__device__ __forceinline__ void list_key_groups(const AttendArgs& a, int keys, int* cum, uint16_t* tags) {
  __shared__ int wave_sum[THREADS / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int carry = 0;
  for (int base = 0; base < a.n_seq; base += THREADS) {
    const int s = base + threadIdx.x;
    int mine = 0;
    if (s < a.n_seq) {
      mine = (int)(((unsigned)sequence_of(a, s).len + keys - 1) / (unsigned)keys);
      tags[s] = page_tag(a.pages[s * a.ldp]);  // (of an empty one whatever it is: it owns no token)
    }
    const int upto = sum_up_to(mine);
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int before = carry;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < wave) before += wave_sum[w];
      carry += wave_sum[w];
    }
    if (s < a.n_seq) cum[s] = before + upto - mine;
    __syncthreads();
  }
  if (threadIdx.x == 0) cum[a.n_seq] = carry;
  __syncthreads();
}

// How many of sequence s' tokens, as far as they lie in `page`, place `place` of its table, belong to sequences in front of it, which share the page: they
// begin with the same page as s and have this one at the same place.  Whoever else names a page is not looked for: each pair of places would have to be compared.
// No more than `enough` are looked for.  All lanes take part; uniform, as the arguments are.
// Beside the loads of keys it costs little (decode, 4 bits: 64 sequences behind up to 16384 103 to 118 us with and without, 32 behind 8000 39 us, without it 38; 256
// behind up to 2000 48 (47), 1024 behind 500 63 (59), 4096 behind 70 134 (106)); 256 that share the first half of their pages take 62.
__device__ __forceinline__ int owned_in_front(const AttendArgs& a, const uint16_t* tags, int s, int place, int page, int enough) {
  const int lane = threadIdx.x & 63;
  const uint32_t both = tags[s] * 0x10001u;
  int most = 0;
  for (int base = 0; base < s; base += kTagsAtOnce) {
    const u32x4 d = reinterpret_cast<const u32x4*>(tags + base)[lane];
    uint32_t same = 0;  // bit i: sequence 2 i of the lane's eight, bit 16 + i: 2 i + 1 (and maybe one behind a match: the tables say)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = d[i] ^ both;
      same |= ((x - 0x10001u) & ~x & 0x80008000u) >> (15 - i);
    }
    for (; same && most < enough; same &= same - 1) {
      const int at = __builtin_ctz(same), o = base + 8 * lane + 2 * (at & 15) + (at >> 4);
      if (o >= s) continue;
      const int64_t row = o * a.ldp;
      const int first = a.pages[row], its = a.pages[row + place], len = sequence_of(a, o).len;  // (asked for together)
      if (first == a.pages[s * a.ldp] && its == page) most = max(most, len);
    }
    if (__any(most >= enough)) return enough;
  }
  return wave_max(most);
}

// Few rows: a wave goes through all of them, 4 NI at a time, with queries straight from memory.  Bound by HBM: 64 tokens behind up to 16384, 32 + 8 heads of 128, 4 bits:
// 101 to 104 us, 4.1 TB/s of keys, parameters and masses.
template <int KV, int HD, int NI>
__global__ __launch_bounds__(256, 2) void mass_few_kernel(MassArgs t) {
  extern __shared__ __align__(16) char lds[];
  constexpr int W = HD / 32, ROWS = 4 * NI;
  constexpr float kInf = __builtin_inff(), kZero = KV == kKvU4 ? 16.f : 0.f;  // codes of 4 bits enter as 16 + c
  using Tile = Tile64<KV, HD>;
  const AttendArgs& a = t.a;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), r = lane & 15, g = lane >> 4, heads = a.cache.n_heads;
  const int page_blocks = a.cache.log2_page - 6;
  const float c = a.scale * 1.44269504f;
  uint16_t* const tags = reinterpret_cast<uint16_t*>(lds);
  int* const cum = reinterpret_cast<int*>(lds + mass_tags_bytes(a.n_seq));
  list_key_groups<256>(a, 256, cum, tags);
  const int64_t total = (int64_t)cum[a.n_seq] * heads;
  const int step_q = ROWS / a.group, step_r = ROWS - step_q * a.group;

  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int at = (int)(u / heads), head = (int)(u - (int64_t)at * heads);
    const int s = uniform(sequence_at(cum, a.n_seq, at));
    const Sequence q = sequence_of(a, s);
    const int tile = (at - uniform(cum[s])) * 4 + wave, ahead = q.len - q.count, key0 = tile * 64;
    const int there = uniform(min(q.len - key0, 64));
    int page = there > 0 ? a.pages[s * a.ldp + (tile >> page_blocks)] : -1;
    if (page >= a.cache.n_pages) page = -1;
    page = uniform(page);
    if (page < 0) continue;
    float sum[4] = {0.f, 0.f, 0.f, 0.f}, old = 0.f;
    float* const mass = t.mass + (((int64_t)page * heads + head) << a.cache.log2_page) + (key0 & ((1 << a.cache.log2_page) - 1));
    Tile k;
    const char* block = a.cache.data + kv_block_offset<KV, HD>(a.cache, page, head, tile & ((1 << page_blocks) - 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) k.load_key(block, 16 * i + r, i, g);
    [[maybe_unused]] float2 par[4];
    if constexpr (KV != kKvBf16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) par[i] = reinterpret_cast<const float2*>(block + 2 * Tile::kHalf)[16 * i + r];
    }
    if (t.decay != 0.f && key0 + lane < ahead) old = mass[lane];
    // rows from the first that sees the first key on; this lane's queries are those of row j of a group of rows
    const int j = (r >> 2) + 4 * (r & 3);
    const int64_t rows = (int64_t)q.count * a.group;
    int64_t row0 = max(0, key0 - ahead) * (int64_t)a.group & ~(int64_t)(ROWS - 1);
    int in_seq = (int)((row0 + j) / a.group), rest = (int)(row0 + j - (int64_t)in_seq * a.group);
    bf16x8 qf[W];
    float lse = 0.f;
    int seen = 0;  // of the block's tokens by row j; 0: it adds nothing
    auto ask = [&] {
      const bool live = j < ROWS && row0 + j < rows;
      const int64_t token = q.first + (live ? in_seq : 0);
      const int qh = head * a.group + (live ? rest : 0);
#pragma unroll
      for (int w = 0; w < W; ++w) qf[w] = *reinterpret_cast<const bf16x8*>(a.q + token * a.ldq + qh * HD + 32 * w + 8 * g);
      lse = t.lse[token * a.hq + qh];
      seen = live ? ahead + in_seq + 1 - key0 : 0;
      in_seq += step_q;
      rest += step_r;
      if (rest >= a.group) rest -= a.group, ++in_seq;
    };
    if (row0 < rows) ask();
    // (beside the loads that are under way, that of `old` among them: of a token that another sequence owns it is not used)
    const int in_front = owned_in_front(a, tags, s, tile >> page_blocks, page, key0 + there);
    if constexpr (KV != kKvBf16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) par[i].x *= c, par[i].y *= c;
    }
    while (row0 < rows) {
      if constexpr (KV != kKvBf16) {  // (codes are expanded anew for every group of rows: kept expanded they would take the registers of other waves)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int w = 0; w < Tile::KD; ++w) asm volatile("" : "+v"(k.k[i][w]));
      }
      f32x4 x[4], qsum = {0.f, 0.f, 0.f, 0.f};
      if constexpr (KV != kKvBf16) {
        bf16x8 one;
#pragma unroll
        for (int e = 0; e < 8; ++e) one[e] = (bf16)1.f;
#pragma unroll
        for (int w = 0; w < W; ++w) qsum = mfma16(qf[w], one, qsum);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = KV == kKvU4 ? -kZero * qsum : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) x[i] = mfma16(qf[w], k.template key<(int)kZero>(i, w), x[i]);
      }
      const bool counts = fabsf(lse) <= kHuge;
      const float mine = counts ? lse * -1.44269504f : -kInf;
      const int mine_seen = counts ? seen : 0;
      const bool edge = __any(j < ROWS && mine_seen < 64);  // (lanes behind the last row have none)
      float base[NI];
      [[maybe_unused]] int sees[NI];
#pragma unroll
      for (int e = 0; e < NI; ++e) base[e] = __shfl(mine, 4 * g + e);
      if (edge)
#pragma unroll
        for (int e = 0; e < NI; ++e) sees[e] = __shfl(mine_seen, 4 * g + e);
      row0 += ROWS;
      if (row0 < rows) ask();
#pragma unroll
      for (int e = 0; e < NI; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y;
          if constexpr (KV == kKvBf16) y = fmaf(x[i][e], c, base[e]);
          else y = fmaf(x[i][e], par[i].x, fmaf(par[i].y, qsum[e], base[e]));
          x[i][e] = __builtin_amdgcn_exp2f(y);
        }
      if (edge)
#pragma unroll
        for (int e = 0; e < NI; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i][e] = 16 * i + r < sees[e] ? x[i][e] : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float add = x[i][0];
#pragma unroll
        for (int e = 1; e < NI; ++e) add += x[i][e];
        sum[i] += add;
      }
    }
    // lane l has key l
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = quarters_sum(sum[i]);
    const float mine = g == 0 ? sum[0] : g == 1 ? sum[1] : g == 2 ? sum[2] : sum[3];
    if (lane < there && key0 + lane >= in_front) mass[lane] = fmaf(t.decay, old, mine);
  }
}

// Many rows: queries go through LDS, 64 rows at a time, double buffered, straight from memory, by lanes that read neighbouring bytes (an operand's
// own lanes read sixteen rows at once, of which the first-level cache finds one a cycle: 690 us instead of 440 to 450 for prompts of up to 2 x 8192, 32 + 8 heads of 128, bf16).  Four of the eight waves share a block and
// take sixteen of the rows each, the two blocks lie next to each other.  Rows go from the last one down to the first that sees the first key:
// workgroups that begin together find each other's queries in the caches.
// Bound by the vector ALU (an exponential, two more instructions a score) and by the workgroup with the most rows, alone on its compute unit at the
// end: 750 to 770 TFLOP/s of Q K^T for those prompts.
template <int HD>
struct alignas(16) MassShared {
  char q[2][64 * HD * 2];  // 16-byte chunks of a row exchanged by its number, so that eight rows' are in all banks
  float lse[2][64];        // as it comes
  float base[2][64];       // -lse in bits; -inf: the row adds nothing
  int sees[2][64];         // tokens of the sequence that a row sees; 0 of one that adds nothing
  int least[2];            // the least of these
};

// What is asked for again behind the rows of a block of keys (LDS: in registers, full of keys, it would push others out to memory).
struct MassBlock {
  int s, tile, page, there, head;
};

template <int KV, int HD>
__global__ __launch_bounds__(512, HD == 256 ? 2 : 4) void mass_rows_kernel(MassArgs t) {
  extern __shared__ __align__(16) char lds[];
  using Shared = MassShared<HD>;
  Shared& sh = *reinterpret_cast<Shared*>(lds);
  __shared__ float joined[8][64];
  __shared__ MassBlock blocks[2];
  constexpr int WK = 2, WR = 4, W = HD / 32, ROWB = HD * 2, PIECES = HD / 64;  // KiB of a wave
  constexpr float kInf = __builtin_inff(), kZero = KV == kKvU4 ? 16.f : 0.f;
  using Tile = Tile64<KV, HD>;
  const AttendArgs& a = t.a;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), r = lane & 15, g = lane >> 4, heads = a.cache.n_heads;
  const int wk = wave / WR, wr = wave % WR, page_blocks = a.cache.log2_page - 6;
  const float c = a.scale * 1.44269504f, per_group = 1.f / (float)a.group;
  const int step_q = 64 / a.group, step_r = 64 - step_q * a.group;
  uint16_t* const tags = reinterpret_cast<uint16_t*>(lds + sizeof(Shared));
  int* const cum = reinterpret_cast<int*>(lds + sizeof(Shared) + mass_tags_bytes(a.n_seq));
  list_key_groups<512>(a, 64 * WK, cum, tags);
  const int64_t total = (int64_t)cum[a.n_seq] * heads;

  auto mass_of = [&](int page, int head, int tile) {
    return t.mass + (((int64_t)page * heads + head) << a.cache.log2_page) + (tile * 64 & ((1 << a.cache.log2_page) - 1)) + lane;
  };

  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int at = (int)(u / heads), head = (int)(u - (int64_t)at * heads);
    const int s = uniform(sequence_at(cum, a.n_seq, at));
    const Sequence q = sequence_of(a, s);
    // a sequence's groups of keys: the first half in order, then from the last one back, so that two on a compute unit have as many rows together
    const int groups = uniform(cum[s + 1] - cum[s]), n = at - uniform(cum[s]), group = n < (groups + 1) / 2 ? n : groups - 1 - (n - (groups + 1) / 2);
    const int tile = group * WK + wk, ahead = q.len - q.count, key0 = tile * 64;
    const int there = uniform(min(q.len - key0, 64));
    int page = there > 0 ? a.pages[s * a.ldp + (tile >> page_blocks)] : -1;
    if (page >= a.cache.n_pages) page = -1;
    page = uniform(page);
    float sum[4] = {0.f, 0.f, 0.f, 0.f}, old = 0.f;
    if (wr == 0 && lane == 0) blocks[wk] = MassBlock{s, tile, page, there, head};
    Tile k;
    const char* block = a.cache.data + (page < 0 ? 0 : kv_block_offset<KV, HD>(a.cache, page, head, tile & ((1 << page_blocks) - 1)));
#pragma unroll
    for (int i = 0; i < 4; ++i) k.load_key(block, 16 * i + r, i, g);
    [[maybe_unused]] float2 par[4];
    if constexpr (KV != kKvBf16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) par[i] = reinterpret_cast<const float2*>(block + 2 * Tile::kHalf)[16 * i + r];
    }
    if (page >= 0 && wr == 0 && t.decay != 0.f && key0 + lane < ahead) old = *mass_of(page, head, tile);
    const int64_t rows = (int64_t)q.count * a.group;
    const int64_t first = max(0, group * WK * 64 - ahead) * (int64_t)a.group >> 6;  // tile of 64 rows
    int64_t rt = ((rows + 63) >> 6) - 1;
    int base_q = (int)(rt * 64 / a.group), base_r = (int)(rt * 64 - (int64_t)base_q * a.group);  // the first row of the tile that is asked for next
    int sees = 0;  // by row `lane` of the tile that was asked for last
    // Row `row` of that tile: its query and head.  (Numbers of less than 2^17: the product is off by one at most.)
    auto find = [&](int row, int& in_seq, int& rest) {
      const int x = base_r + row;
      in_seq = (int)((float)x * per_group);
      rest = x - in_seq * a.group;
      if (rest < 0) rest += a.group, --in_seq;
      if (rest >= a.group) rest -= a.group, ++in_seq;
      in_seq += base_q;
    };
    // The i-th piece that this wave fetches of a tile: this lane's part lies `offset` behind the first row of the tile's first query and of the head.
    const char* const heads_lse = reinterpret_cast<const char*>(t.lse + (int64_t)q.first * a.hq + head * a.group);
    const char* const heads_q = reinterpret_cast<const char*>(a.q) + ((int64_t)q.first * a.ldq + head * a.group * HD) * 2;
    auto offset_of = [&](int i, int lane, int64_t left) {
      const int byte = (wave * PIECES + i) * 1024 + lane * 16, row = byte / ROWB, chunk = byte % ROWB / 16 ^ (row & 7);
      int in_seq, rest;
      find(row, in_seq, rest);
      const bool live = row < left;  // (rows behind the last one: some row of the first query that is there)
      return (live ? (uint32_t)(in_seq - base_q) * (uint32_t)(a.ldq * 2) + (uint32_t)(rest * ROWB) : 0u) + (uint32_t)(chunk * 16);
    };
    auto send = [&](const char* base, uint32_t offset, int i, int at) { to_lds_16(offset, base, uniform((int)(uintptr_t)sh.q[at] + (wave * PIECES + i) * 1024)); };
    auto fetch = [&](int64_t rt, int at) {
      int tid = threadIdx.x;
      asm volatile("" : "+v"(tid));  // (places are worked out anew: kept, they would push the keys out to memory)
      const char* base = heads_q + (int64_t)base_q * a.ldq * 2;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) send(base, offset_of(i, tid & 63, rows - rt * 64), i, at);
      if (wave == 0) {
        int in_seq, rest;
        find(tid, in_seq, rest);
        to_lds_4(rt * 64 + tid < rows ? ((uint32_t)(in_seq - base_q) * (uint32_t)a.hq + (uint32_t)rest) * 4u : 0u, heads_lse + (int64_t)base_q * a.hq * 4,
                 uniform((int)(uintptr_t)sh.lse[at]));
        sees = ahead + in_seq + 1;
      }
      base_q -= step_q;
      base_r -= step_r;
      if (base_r < 0) base_r += a.group, --base_q;
    };
    // Where the query heads of a key head divide 64, rows of neighbouring tiles are whole queries apart: places are those of the tile before.
    const bool even = step_r == 0;
    uint32_t offsets[PIECES] = {}, offset_lse = 0;
    auto place_next = [&] {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) offsets[i] = offset_of(i, lane, 64);
      int in_seq, rest;
      find(lane, in_seq, rest);
      offset_lse = ((uint32_t)(in_seq - base_q) * (uint32_t)a.hq + (uint32_t)rest) * 4u;
    };
    auto fetch_even = [&](int at) {
      const char* base = heads_q + (int64_t)base_q * a.ldq * 2;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) send(base, offsets[i], i, at);
      if (wave == 0) to_lds_4(offset_lse, heads_lse + (int64_t)base_q * a.hq * 4, uniform((int)(uintptr_t)sh.lse[at]));
      sees -= step_q;
      base_q -= step_q;
    };
    auto put = [&](int64_t rt, int at) {
      if (wave == 0) {
        const float lse = sh.lse[at][lane];
        const bool counts = fabsf(lse) <= kHuge && rt * 64 + lane < rows;
        const int mine = counts ? sees : 0;
        sh.base[at][lane] = counts ? lse * -1.44269504f : -kInf;
        sh.sees[at][lane] = mine;
        const int least = -wave_max(-mine);
        if (lane == 0) sh.least[at] = least;
      }
    };
    bf16x8 kf[4][W];
    __syncthreads();  // the buffers are free
    if (rt >= first) {
      fetch(rt, rt & 1);
      if (even && rt > first) place_next();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int w = 0; w < W; ++w) kf[i][w] = k.template key<(int)kZero>(i, w);
    if constexpr (KV != kKvBf16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) par[i].x *= c, par[i].y *= c;
    }
    // keys have arrived before the loop: a wait for them in it would be one for the queries that are on their way
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int w = 0; w < W; ++w) asm volatile("" : "+v"(kf[i][w]));
    for (; rt >= first; --rt) {
      const int at = rt & 1;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's part has arrived
      put(rt, at);
      __syncthreads();
      if (rt > first) {
        if (even) fetch_even(at ^ 1);
        else fetch(rt - 1, at ^ 1);
      }
      const bool edge = uniform(sh.least[at]) < key0 + 64;
      {
        const int row0 = 16 * wr;
        bf16x8 qf[W];
#pragma unroll
        for (int w = 0; w < W; ++w) qf[w] = *reinterpret_cast<const bf16x8*>(sh.q[at] + (row0 + r) * ROWB + (((4 * w + g) ^ (r & 7)) << 4));
        const f32x4 base = *reinterpret_cast<const f32x4*>(&sh.base[at][row0 + 4 * g]);
        f32x4 x[4], qsum = {0.f, 0.f, 0.f, 0.f};
        if constexpr (KV != kKvBf16) {
          bf16x8 one;
#pragma unroll
          for (int e = 0; e < 8; ++e) one[e] = (bf16)1.f;
#pragma unroll
          for (int w = 0; w < W; ++w) qsum = mfma16(qf[w], one, qsum);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = KV == kKvU4 ? -kZero * qsum : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < W; ++w) x[i] = mfma16(qf[w], kf[i][w], x[i]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float y;
            if constexpr (KV == kKvBf16) y = fmaf(x[i][e], c, base[e]);
            else y = fmaf(x[i][e], par[i].x, fmaf(par[i].y, qsum[e], base[e]));
            x[i][e] = __builtin_amdgcn_exp2f(y);
          }
        if (edge) {
          const int4 seen = *reinterpret_cast<const int4*>(&sh.sees[at][row0 + 4 * g]);
          const int see[4] = {seen.x, seen.y, seen.z, seen.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i][e] = key0 + 16 * i + r < see[e] ? x[i][e] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += (x[i][0] + x[i][1]) + (x[i][2] + x[i][3]);
      }
    }
    // lane l has key l
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = quarters_sum(sum[i]);
    joined[wave][lane] = g == 0 ? sum[0] : g == 1 ? sum[1] : g == 2 ? sum[2] : sum[3];
    __syncthreads();
    if (wr == 0) {
      const MassBlock b = blocks[wk];
      const int page = uniform(b.page), tile = uniform(b.tile), there = uniform(b.there);
      if (page >= 0) {
        const int in_front = owned_in_front(a, tags, uniform(b.s), tile >> page_blocks, page, tile * 64 + there);
        if (lane < there && tile * 64 + lane >= in_front) {
          float mine = 0.f;
#pragma unroll
          for (int w = 0; w < WR; ++w) mine += joined[wk * WR + w][lane];
          *mass_of(page, b.head, tile) = fmaf(t.decay, old, mine);
        }
      }
    }
  }
}

}  // namespace kt
