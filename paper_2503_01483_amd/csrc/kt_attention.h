// kt_attention.h -- attention of single tokens and of chunks over the paged cache of kt_kvcache.h.
//
//   out_r = sum_j p_rj v_j / sum_j p_rj,  p_rj = exp(scale q_r . k_j - max),  j over the prefix and the sequence's tokens up to r's own
// The rows of one key / value head (the G query heads that share it, for each query token of a sequence) form row tiles of 16; a row
// tile times a head is a segment, and a segment's keys come in tiles of 64, one block of the cache each.
//
// A WAVE is a worker.  It computes S^T = K Q^T (keys on the rows of the 16 x 16 x 32 products, rows of Q on the columns), so that a lane
// holds the scores of one row and of 16 keys that lie next to each other in its column of V^T: after the exponentials the scores ARE
// the operand of O^T = V^T P^T.  Nothing goes through LDS but the quantisers' parameters, no wave waits for another.
// All key tiles of all segments form one list, and every wave takes an equal piece of it, whatever the lengths: a segment that is
// cut leaves {O, max, sum} of each piece in the workspace, and a second launch puts them together (4 to 9 us).
//
// Bound by HBM: 64 tokens behind up to 16384, 32 + 2 x 8 heads of 128, 4 bits: 159 us, 4.8 TB/s (a large copy: 4.8); 4 behind 131072, 8 bits: 159 us,
// 5.2 TB/s.  One token behind 1027: 11 us, a chain of lookups, loads and products by waves of one or two tiles each.
// More rows than 16 read their keys again, mostly from the caches on the way.
//
// Quantised rows are never expanded: k = s c + b gives q . k = s (q . c) + b sum(q), and v = s c + b gives p v = (p s) c + p b, so that the
// codes themselves, exact in bf16, are the operands.  A 4-bit code becomes 128 + c by OR (0x4300 | c), two at a time; a product of
// the same rounded p s with a constant takes 136 (u8: 128) off again within the tile, which leaves the codes centred and costs no accuracy.
// Held in fp32: scores, running maximum, sum of p, O.  Rounded to bf16: p, 2^-8 of a term, in both signs; p s goes in as the sum of two bf16
// (2^-16): the product has room for it beside the memory.
#pragma once
#include "kt_kvcache.h"

namespace kt {

constexpr int kRows = 16;  // rows of a segment

struct AttendArgs {
  KvCache cache;
  const bf16* q;
  const int *q_starts, *lens, *pages;  // q_starts null: token i is the only query of sequence i
  int64_t ldq, ldp;
  int n_seq, n_tokens, hq, group;
  int row_tiles;  // kt_attention.h: at most this many of a sequence
  float scale;
  bf16* out;
  int64_t ldo;
  float* lse;
  // workspace
  int workers;   // waves that take pieces of the list
  int* tiles;    // [n_seq + 1] key tiles of one head in front of each sequence
  int4* cuts;    // [workers] the segment whose first piece a worker has while others have the rest: {first token, first row * 32 + rows, head, pieces or 0}
  float* part;   // pieces of cut segments: O [2 workers][kRows][HD], then {max in bits, sum} [2 workers][kRows]
  float* whole;  // null: whole segments go to out.  Else something is to be joined: O [n_tokens][hq][HD], then {max, sum} [n_tokens][hq]
  const unsigned long long* tree;  // [n_tokens][ldt] bits: which queries of its sequence a query sees (kernels with TREE; else null)
  int64_t ldt;
};

// Which of the `there` tokens of a tile a query of a tree sees, one a bit: those in front of the sequence's queries, and the queries that its row of words
// names.  behind: the tile's first token less the sequence's first query; a tile has bits of two words.
__device__ __forceinline__ unsigned long long tree_sees(const AttendArgs& a, int64_t token, int behind, int there) {
  const unsigned long long all = there >= 64 ? ~0ull : (1ull << there) - 1;
  if (behind <= -64) return all;
  const unsigned long long* row = a.tree + token * a.ldt;
  auto word = [&](int64_t w) { return w < 0 ? ~0ull : w < a.ldt ? row[w] : 0ull; };
  const int w = behind >> 6, b = behind & 63;
  return all & (b ? word(w) >> b | word(w + 1) << (64 - b) : word(w));
}

// First token and number of a sequence's queries, and its tokens in the cache.
struct Sequence {
  int first, count, len;
};
__device__ __forceinline__ Sequence sequence_of(const AttendArgs& a, int s) {
  Sequence q{s, 1, 0};
  if (a.q_starts) {
    q.first = min(max(a.q_starts[s], 0), a.n_tokens);
    q.count = min(max(a.q_starts[s + 1] - q.first, 0), a.n_tokens - q.first);
  }
  q.len = min(max(a.lens[s], 0), (int)(a.ldp << a.cache.log2_page));
  return q;
}
__device__ __forceinline__ int key_tiles(const Sequence& q) { return max(1, (int)(((unsigned)q.len + 63) >> 6)); }
__device__ __forceinline__ int row_tiles(const AttendArgs& a, const Sequence& q) {
  return (int)min(((int64_t)q.count * a.group + kRows - 1) / kRows, (int64_t)a.row_tiles);
}

// Key tiles of one head in front of each sequence, those of each of its row tiles, `cum` [n_seq + 1] (LDS), by a workgroup of 256.  Of a
// sequence with more rows than the caller's bound the first ones are computed.
__device__ __forceinline__ void list_tiles(const AttendArgs& a, int* cum) {
  __shared__ int wave_sum[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int carry = 0;
  for (int base = 0; base < a.n_seq; base += 256) {
    const int s = base + threadIdx.x;
    int mine = 0;
    if (s < a.n_seq) {
      const Sequence q = sequence_of(a, s);
      mine = row_tiles(a, q) * key_tiles(q);
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int t = __shfl_up(upto, o);
      if (lane >= o) upto += t;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int before = carry;
    for (int w = 0; w < wave; ++w) before += wave_sum[w];
    if (s < a.n_seq) cum[s] = before + upto - mine;
    carry += wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
    if (base + 256 < a.n_seq) __syncthreads();
  }
  if (threadIdx.x == 0) cum[a.n_seq] = carry;
  __syncthreads();
}

// The last sequence that starts at or before place u of the list.
__device__ __forceinline__ int sequence_at(const int* cum, int n_seq, int u) {
  int lo = 0, hi = n_seq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cum[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
// Tiles of a worker's piece of a list of `total` (worker w has [w n, (w + 1) n)).
__device__ __forceinline__ int piece_length(int total, int workers) { return max(1, (int)(((unsigned)total + workers - 1) / (unsigned)workers)); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// 8 codes of 4 bits as bf16 ZERO + c: elements 2 i, 2 i + 1 in dword i.  ZERO: 128 or 16; of sums with the smaller one less is lost when it is taken off.
template <int ZERO = 128>
__device__ __forceinline__ bf16x8 spread_nibbles(uint32_t x) {
  static_assert(ZERO == 128 || ZERO == 16);
  u32x4 t;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (ZERO == 128) t[i] = (x >> (4 * i) & 0x000f000fu) | 0x43004300u;
    else t[i] = ((i ? x >> (4 * i - 3) : x << 3) & 0x00780078u) | 0x41804180u;
  }
  return __builtin_bit_cast(bf16x8, t);
}
// 8 tokens' low or high nibbles as bf16 128 + c, in the order 0 2 1 3 4 6 5 7.
__device__ __forceinline__ bf16x8 spread_rows(uint32_t x, uint32_t y, int shift) {
  const u32x4 t = {(x >> shift & 0x000f000fu) | 0x43004300u, (x >> (8 + shift) & 0x000f000fu) | 0x43004300u,
                   (y >> shift & 0x000f000fu) | 0x43004300u, (y >> (8 + shift) & 0x000f000fu) | 0x43004300u};
  return __builtin_bit_cast(bf16x8, t);
}
__device__ __forceinline__ bf16x8 spread_bytes(uint32_t x, uint32_t y) {
  bf16x8 t;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    t[i] = (bf16)(float)(x >> (8 * i) & 0xffu);
    t[4 + i] = (bf16)(float)(y >> (8 * i) & 0xffu);
  }
  return t;
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// 16 bytes a lane from memory straight into LDS: lane l lands at lds_addr + 16 l (wave-uniform).  Assembly, so that LDS reads of other buffers
// do not wait for them: waits are placed by hand (vmcnt).
__device__ __forceinline__ void to_lds_16(uint32_t voffset, const char* base, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voffset), "s"(base), "s"(lds_addr) : "memory", "m0");
}

// Maximum over the lanes of a wave, by row shifts and broadcasts; uniform.
__device__ __forceinline__ int wave_max(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x111, 0xf, 0xf, false));  // row_shr 1, 2, 4, 8
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x112, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x114, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x118, 0xf, 0xf, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x142, 0xf, 0xf, false));  // row_bcast 15, 31
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x143, 0xf, 0xf, false));
  return __builtin_amdgcn_readlane(v, 63);
}

// Sum and maximum over the four quarters of a wave.
__device__ __forceinline__ float quarters_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ float quarters_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}

// The registers of one tile of 64 keys.  A lane (r = lane % 16, g = lane / 16) holds features 8 g .. of four keys, token(t) for t = 0 .. 3, and
// 16 tokens of HD / 16 features r, r + 16, ... (u4: HD / 32 pairs): those whose scores the products leave in it.
template <int KV, int HD>
struct Tile64 {
  static constexpr int kHalf = kv_half_bytes<KV, HD>();
  static constexpr int KD = HD * kv_bits<KV>() / 128;         // dwords of a lane's features of one key
  static constexpr int VR = KV == kKvU4 ? HD / 32 : HD / 16;  // rows of values of a lane
  static constexpr int VD = KV == kKvBf16 ? 8 : 4;            // dwords of each
  uint32_t k[4][KD], v[VR][VD];
  u32x4 par;

  __device__ __forceinline__ static int token(int t, int r) {
    return KV == kKvBf16 ? 32 * (t >> 1) + 8 * (r >> 2) + 4 * (t & 1) + (r & 3) : 16 * (r >> 2) + 4 * t + (r & 3);
  }
  // token `tok` of a block as the t-th key
  __device__ __forceinline__ void load_key(const char* block, int tok, int t, int g) {
    const char* row = block + tok * (kHalf / kBlockTokens);
    if constexpr (KV == kKvBf16) {
#pragma unroll
      for (int w = 0; w < HD / 32; ++w) *reinterpret_cast<u32x4*>(&k[t][4 * w]) = *reinterpret_cast<const u32x4*>(row + 64 * w + 16 * g);
    } else if constexpr (KD % 4 == 0) {
#pragma unroll
      for (int i = 0; i < KD; i += 4) *reinterpret_cast<u32x4*>(&k[t][i]) = *reinterpret_cast<const u32x4*>(row + 4 * KD * g + 4 * i);
    } else {
      *reinterpret_cast<u32x2*>(&k[t][0]) = *reinterpret_cast<const u32x2*>(row + 4 * KD * g);
    }
  }
  __device__ __forceinline__ void load_keys(const char* block, int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) load_key(block, token(t, r), t, g);
    if constexpr (KV != kKvBf16) par = reinterpret_cast<const u32x4*>(block + 2 * kHalf)[lane];
  }
  __device__ __forceinline__ void load_values(const char* block, int lane) {
    const int r = lane & 15, g = lane >> 4;
    const char* from = block + kHalf;
#pragma unroll
    for (int i = 0; i < VR; ++i) {
      if constexpr (KV == kKvBf16) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          *reinterpret_cast<u32x4*>(&v[i][4 * j]) = *reinterpret_cast<const u32x4*>(from + (16 * i + r) * 128 + 64 * j + 16 * g);
      } else {
        *reinterpret_cast<u32x4*>(&v[i][0]) = *reinterpret_cast<const u32x4*>(from + (16 * i + r) * 64 + 16 * g);
      }
    }
  }
  template <int ZERO = 128>
  __device__ __forceinline__ bf16x8 key(int t, int w) const {
    if constexpr (KV == kKvBf16) return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(&k[t][4 * w]));
    else if constexpr (KV == kKvU8) return spread_bytes(k[t][2 * w], k[t][2 * w + 1]);
    else return spread_nibbles<ZERO>(k[t][w]);
  }
  // features 16 td + r, the 8 tokens of half j
  __device__ __forceinline__ bf16x8 value(int td, int j) const {
    if constexpr (KV == kKvBf16) return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(&v[td][4 * j]));
    else if constexpr (KV == kKvU8) return spread_bytes(v[td][2 * j], v[td][2 * j + 1]);
    else return spread_rows(v[td >> 1][2 * j], v[td >> 1][2 * j + 1], 4 * (td & 1));
  }
};

// Takes values that are not finite, and those of tokens `there` on, out of a dword of the values of tokens `at` and at + 1 (0 NaN = NaN); the former
// are noted in `which`.
__device__ __forceinline__ uint32_t only_finite(uint32_t d, int at, int there, unsigned long long& which) {
  d = at >= there ? 0u : at + 1 >= there ? d & 0xffffu : d;
  if ((d & 0x7f80u) == 0x7f80u) which |= 1ull << at, d &= 0xffff0000u;
  if ((d & 0x7f800000u) == 0x7f800000u) which |= 2ull << at, d &= 0xffffu;
  return d;
}
// The tokens that any lane has noted; uniform.
__device__ __forceinline__ unsigned long long any_lane(unsigned long long which) {
  unsigned long long all = 0ull;
  if (__any(which != 0ull))
    for (int j = 0; j < 64; ++j) all |= (unsigned long long)(__any(which >> j & 1ull) ? 1 : 0) << j;
  return all;
}

// The list's order: sequences, in each its heads, in each its row tiles, in each the key tiles.
// TREE: of its sequence's queries a row sees those that its mask names (tree_sees), not those up to its own.
template <int KV, int HD, bool TREE>
__global__ __launch_bounds__(256, HD == 256 ? 1 : 2) void attend_rows_kernel(AttendArgs a) {
  extern __shared__ int cum[];
  __shared__ float4 params[4][64];
  constexpr int TD = HD / 16;
  // The next tile asked for as registers come free, where it needs no more of them: decode of 64 behind 16384, 4 bits, 172 -> 166 us.  With 8 bits
  // registers spill (4 behind 131072: 138 -> 165), and bf16 tiles take as many as there are.
  constexpr bool kEarly = KV == kKvU4 && HD <= 128;
  constexpr int kZero = TREE ? 16 : 128;  // what codes of 4 bits of keys enter with
  constexpr float kOffset = KV == kKvU4 ? 136.f : 128.f, kCentre = KV == kKvU4 ? 8.f : 128.f;
  constexpr float kNone = -__builtin_inff();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4, heads = a.cache.n_heads;
  list_tiles(a, cum);
  if (blockIdx.x == 0 && a.whole)
    for (int s = threadIdx.x; s <= a.n_seq; s += 256) a.tiles[s] = cum[s];
  const int total = cum[a.n_seq] * heads, per = uniform(piece_length(total, a.workers));
  const int me = uniform(blockIdx.x * 4 + wave), begin = me * per, end = min(begin + per, total);
  const float c = a.scale * 1.44269504f;
  const int page_blocks = a.cache.log2_page - 6;
  int4 cut = {0, 0, 0, 0};

  for (int u = begin; u < end;) {
    // the segment that tile u belongs to, and this wave's tiles of it
    const int s = uniform(sequence_at(cum, a.n_seq, (int)((unsigned)u / (unsigned)heads)));
    const Sequence q = sequence_of(a, s);
    const int tiles = uniform(key_tiles(q)), rel = u - uniform(cum[s]) * heads;
    const int in_head = tiles * row_tiles(a, q), head = uniform((int)((unsigned)rel / (unsigned)in_head)), behind = rel - head * in_head;
    const int row_tile = uniform((int)((unsigned)behind / (unsigned)tiles)), start = u - (behind - row_tile * tiles), row0 = row_tile * kRows;
    const int first = u - start, last = min(tiles, end - start);

    // this lane's row
    const int in_seq = (row0 + r) / a.group, qh = head * a.group + (row0 + r - in_seq * a.group);
    const bool live = in_seq < q.count;
    const int64_t token = q.first + (live ? in_seq : 0);
    const int sees = min(max(q.len - q.count + in_seq + 1, 0), q.len), all_see = q.len - q.count + (TREE ? 0 : row0 / a.group + 1);
    bf16x8 qf[HD / 32];
    float qsum = 0.f;
#pragma unroll
    for (int w = 0; w < HD / 32; ++w) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[w][e] = (bf16)0.f;
      if (live) qf[w] = *reinterpret_cast<const bf16x8*>(a.q + token * a.ldq + qh * HD + 32 * w + 8 * g);
    }
    if constexpr (KV != kKvBf16) {
#pragma unroll
      for (int w = 0; w < HD / 32; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) qsum += (float)qf[w][e];
      qsum = quarters_sum(qsum);
    }

    f32x4 o[TD];
#pragma unroll
    for (int i = 0; i < TD; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNone, l = 0.f, low = 0.f;
    const int* pages = a.pages + s * a.ldp;
    Tile64<KV, HD> t64;

    // Where a tile's block lies, and how many of its tokens there are: none of a page outside the cache (then some block's place is given).
    auto place = [&](int tile, int& there) {
      there = min(q.len - tile * 64, 64);
      const int page = there > 0 ? pages[tile >> page_blocks] : -1;
      if (page < 0 || page >= a.cache.n_pages) {
        there = 0;
        return (int64_t)0;
      }
      return kv_block_offset<KV, HD>(a.cache, page, head, tile & ((1 << page_blocks) - 1));
    };
    int there, there_next = 0;
    int64_t block = place(first, there), block_next = 0;
    if constexpr (kEarly) {
      t64.load_keys(a.cache.data + block, lane);
      t64.load_values(a.cache.data + block, lane);
    }
    for (int tile = first; tile < last; ++tile) {
      // kEarly: the next tile's keys are asked for once these are used up, its values likewise: each has the other's time to arrive in
      const bool more = tile + 1 < last;
      if (more) block_next = place(tile + 1, there_next);
      if constexpr (!kEarly) {
        t64.load_keys(a.cache.data + block, lane);
        t64.load_values(a.cache.data + block, lane);
      }
      f32x4 x[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float x0 = KV == kKvU4 ? -(float)kZero * qsum : 0.f;
        x[t] = f32x4{x0, x0, x0, x0};
#pragma unroll
        for (int w = 0; w < HD / 32; ++w) x[t] = mfma16(t64.template key<kZero>(t, w), qf[w], x[t]);
      }
      // a lane's 16 keys: their {step, minimum}, keys' and values'
      f32x4 vp[4][2];
      if constexpr (KV != kKvBf16) {
        params[wave][lane] = __builtin_bit_cast(float4, t64.par);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const f32x4* kp = reinterpret_cast<const f32x4*>(params[wave]) + 8 * g;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const f32x4 p = kp[2 * t + h];
            x[t][2 * h] = fmaf(x[t][2 * h], p[0], p[1] * qsum);
            x[t][2 * h + 1] = fmaf(x[t][2 * h + 1], p[2], p[3] * qsum);
            vp[t][h] = kp[32 + 2 * t + h];
          }
        __builtin_amdgcn_wave_barrier();
      }
      if (kEarly && more) t64.load_keys(a.cache.data + block_next, lane);
      const bool masked = there < 64 || tile * 64 + 64 > all_see;
      const int seen = min(max(sees - tile * 64, 0), there);
      unsigned long long bits = 0ull;  // TREE: of the tile's tokens, those that are seen
      if (TREE && masked) bits = tree_sees(a, token, tile * 64 - (q.len - q.count), there);
      auto hidden = [&](int j) { return TREE ? !(bits >> j & 1ull) : j >= seen; };
      if (masked) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (hidden(Tile64<KV, HD>::token(t, 4 * g + i))) x[t][i] = kNone;
      }
      float most = m;
#pragma unroll
      for (int t = 0; t < 4; ++t) most = fmaxf(most, fmaxf(fmaxf(x[t][0], x[t][1]), fmaxf(x[t][2], x[t][3])));
      most = quarters_max(most);
      const float mc = most == kNone ? 0.f : most * c;
      if (__any(most > m)) {
        const float shrink = most > m ? __builtin_amdgcn_exp2f(fmaf(m, c, -mc)) : 1.f;  // (1 +- 2^-24 |mc| otherwise: a row's bits go by its own scores)
        l *= shrink;
        low *= shrink;
#pragma unroll
        for (int i = 0; i < TD; ++i) o[i] *= shrink;
        m = most;
      }
      bf16x8 pf[2];
      [[maybe_unused]] bf16x8 rest[2];  // what rounding p s leaves
      float sum[4] = {0.f, 0.f, 0.f, 0.f};  // (of a tile first: fewer roundings at the size of the whole)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float p = __builtin_amdgcn_exp2f(fmaf(x[t][i], c, -mc));
          sum[i] += p;
          const int e = 4 * (t & 1) + i, at = KV == kKvU4 ? (e & 4) | (e & 1) << 1 | (e & 2) >> 1 : e;
          if constexpr (KV != kKvBf16) {
            const float vs = vp[t][i >> 1][2 * (i & 1)], vb = vp[t][i >> 1][2 * (i & 1) + 1];
            const bool off = masked && hidden(Tile64<KV, HD>::token(t, 4 * g + i));  // parameters of keys that are not seen may be anything
            low = off ? low : fmaf(p, fmaf(kCentre, vs, vb), low);
            p = off ? 0.f : p * vs;
            rest[t >> 1][at] = (bf16)(p - (float)(bf16)p);
          }
          pf[t >> 1][at] = (bf16)p;
        }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      if constexpr (KV == kKvBf16) {
        if (masked) {  // what a row does not see may be anything, and 0 NaN = NaN
          unsigned long long odd = 0ull;
#pragma unroll
          for (int i = 0; i < TD; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int w = 0; w < 4; ++w) t64.v[i][4 * j + w] = only_finite(t64.v[i][4 * j + w], 32 * j + 8 * g + 2 * w, there, odd);
          const bf16* v = reinterpret_cast<const bf16*>(a.cache.data + block + kv_half_bytes<KV, HD>()) + 4 * g * kBlockTokens;
#pragma unroll 1
          for (odd = any_lane(odd); odd; odd &= odd - 1) {
            const int j = __builtin_ctzll(odd);
#pragma unroll
            for (int i = 0; i < TD; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float x = (float)v[(16 * i + e) * kBlockTokens + j];
                if (!hidden(j) && !(fabsf(x) <= kHuge)) o[i][e] += x;
              }
          }
        }
#pragma unroll
        for (int i = 0; i < TD; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) o[i] = mfma16(t64.value(i, j), pf[j], o[i]);
      } else {
        bf16x8 off;
#pragma unroll
        for (int e = 0; e < 8; ++e) off[e] = (bf16)-kOffset;
        f32x4 shift = {0.f, 0.f, 0.f, 0.f};  // the same in all its rows
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          shift = mfma16(off, pf[j], shift);
          shift = mfma16(off, rest[j], shift);
        }
#pragma unroll
        for (int i = 0; i < TD; ++i) {
          f32x4 t = shift;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const bf16x8 v = t64.value(i, j);
            t = mfma16(v, pf[j], t);
            t = mfma16(v, rest[j], t);
          }
          o[i] += t;
        }
      }
      if (kEarly && more) t64.load_values(a.cache.data + block_next, lane);
      block = block_next;
      there = there_next;
    }

    l = quarters_sum(l);
    if constexpr (KV != kKvBf16) {
      const float add = quarters_sum(low);
#pragma unroll
      for (int i = 0; i < TD; ++i) o[i] += add;
    }
    const bool whole = first == 0 && last == tiles;
    if (whole && !a.whole) {
      if (live) {
        const float inv = l > 0.f ? 1.f / l : l;  // (NaN stays)
        bf16* to = a.out + token * a.ldo + qh * HD + 4 * g;
#pragma unroll
        for (int i = 0; i < TD; ++i) {
          bf16 t[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) t[e] = (bf16)(l == 0.f ? 0.f : o[i][e] * inv);
          *reinterpret_cast<u32x2*>(to + 16 * i) = __builtin_bit_cast(u32x2, t);
        }
        if (a.lse && g == 0) a.lse[token * a.hq + qh] = l == 0.f ? kNone : (m * c + __log2f(l)) * 0.693147181f;
      }
    } else {
      if (live) {
        const int64_t slot = whole ? token * a.hq + qh : (int64_t)(2 * me + (first ? 0 : 1)) * kRows + r;
        float* base = whole ? a.whole : a.part;
        float* to = base + slot * HD + 4 * g;
#pragma unroll
        for (int i = 0; i < TD; ++i) *reinterpret_cast<f32x4*>(to + 16 * i) = o[i];
        if (g == 0)
          reinterpret_cast<float2*>(base + (whole ? (int64_t)a.n_tokens * a.hq : (int64_t)2 * a.workers * kRows) * HD)[slot] =
              make_float2(l == 0.f ? kNone : m * c, l);
      }
      if (first == 0 && !whole)
        cut = int4{q.first, row0 * 32 + (int)min((int64_t)q.count * a.group - row0, (int64_t)kRows), head, (int)((unsigned)(start + tiles - 1) / (unsigned)per) - me + 1};
    }
    u = start + last;
  }
  if (lane == 0) a.cuts[me] = cut;
}

// The pieces of cut segments put together: one segment a workgroup of 256, HD / 4 threads a piece of a row.
template <int HD>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int TR = HD / 4, AT = 256 / TR;
  constexpr float kNone = -__builtin_inff();
  __shared__ f32x4 sh_o[AT][TR];
  __shared__ float2 sh_ml[AT];
  const int4 cut = a.cuts[blockIdx.x];
  if (cut.w == 0) return;
  const float2* ml = reinterpret_cast<const float2*>(a.part + (int64_t)2 * a.workers * kRows * HD);
  const int t = threadIdx.x % TR, at = threadIdx.x / TR;
  const int row0 = cut.y >> 5, rows = cut.y & 31;
  for (int r = blockIdx.y; r < rows; r += gridDim.y) {
    float m = kNone, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int k = at; k < cut.w; k += AT) {
      const int64_t slot = (2 * ((int64_t)blockIdx.x + k) + (k ? 0 : 1)) * kRows + r;
      const float2 d = ml[slot];
      const f32x4 v = *reinterpret_cast<const f32x4*>(a.part + slot * HD + 4 * t);
      const float most = fmaxf(m, d.x), base = most == kNone ? 0.f : most;
      const float f = __builtin_amdgcn_exp2f(d.x - base), h = __builtin_amdgcn_exp2f(m - base);
      l = fmaf(d.y, f, l * h);
      o = v * f + o * h;
      m = most;
    }
    __syncthreads();
    sh_o[at][t] = o;
    if (t == 0) sh_ml[at] = make_float2(m, l);
    __syncthreads();
    if (at == 0) {
      float most = kNone;
#pragma unroll
      for (int i = 0; i < AT; ++i) most = fmaxf(most, sh_ml[i].x);
      const float base = most == kNone ? 0.f : most;
      l = 0.f;
      o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < AT; ++i) {
        const float f = __builtin_amdgcn_exp2f(sh_ml[i].x - base);
        l = fmaf(sh_ml[i].y, f, l);
        o += sh_o[i][t] * f;
      }
      const int64_t token = cut.x + (row0 + r) / a.group, qh = cut.z * a.group + (row0 + r) % a.group;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      bf16 v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (bf16)(l == 0.f ? 0.f : o[e] * inv);
      *reinterpret_cast<u32x2*>(a.out + token * a.ldo + qh * HD + 4 * t) = __builtin_bit_cast(u32x2, v);
      if (a.lse && t == 0) a.lse[token * a.hq + qh] = l == 0.f ? kNone : (base + __log2f(l)) * 0.693147181f;
    }
  }
}

}  // namespace kt
