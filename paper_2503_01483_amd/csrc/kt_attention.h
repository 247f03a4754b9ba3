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
// cut leaves {O, max, sum} of each piece in the workspace, and attend_join_kernel puts them together.
//
// Quantised rows are never expanded: k = s c + b gives q . k = s (q . c) + b sum(q), and v = s c + b gives p v = (p s) c + p b, so that the
// codes themselves, exact in bf16, are the operands.  A 4-bit code becomes 128 + c by OR (0x4300 | c), two at a time; what the 128
// adds is taken off again with the same rounded p s (a row of ones in V^T), so that it costs no accuracy, and with 8 more the codes
// are centred, which keeps the rounding of p s to bf16 as small as that of p would be against plain values.
// Held in fp32: scores, running maximum, sum of p, O.  Rounded to bf16: p (or p s), 2^-9 of a term each, in both signs.
#pragma once
#include "kt_kvcache.h"

namespace kt {

constexpr int kRows = 16;  // rows of a segment

struct AttendArgs {
  KvCache cache;
  const bf16* q;
  const int *q_starts, *lens, *pages;  // q_starts null: token i is the only query of sequence i; lens null: `fixed_len` for all
  int64_t ldq, ldp, fixed_len;
  int n_seq, n_tokens, hq, group;
  int workers;  // waves that take pieces
  float scale;
  bf16* out;
  int64_t ldo;
  float* lse;
  float* part;   // pieces of cut segments: O [2 workers][kRows][HD], then {max in bits, sum} [2 workers][kRows]
  float* whole;  // null: whole segments go to out.  Else something is to be joined: O [n_tokens][hq][HD], then {max, sum} [n_tokens][hq]
  bool causal;
};

// First token and number of a sequence's queries, and its tokens in the cache.
struct Sequence {
  int first, count;
  int64_t len;
};
__device__ __forceinline__ Sequence sequence_of(const AttendArgs& a, int s) {
  Sequence q;
  if (a.q_starts) {
    const int b = a.q_starts[s], e = a.q_starts[s + 1];
    q.first = min(max(b, 0), a.n_tokens);
    q.count = min(max(e - q.first, 0), a.n_tokens - q.first);
  } else if (a.lens) {
    q.first = s;
    q.count = 1;
  } else {
    q.first = 0;
    q.count = a.n_tokens;
  }
  const int64_t room = a.ldp << a.cache.log2_page;
  q.len = a.lens ? min((int64_t)max(a.lens[s], 0), room) : a.fixed_len;
  return q;
}
__device__ __forceinline__ int64_t key_tiles(const Sequence& q) { return max((int64_t)1, (q.len + 63) >> 6); }
__device__ __forceinline__ int row_tiles(const AttendArgs& a, const Sequence& q) {
  return (int)(((int64_t)q.count * a.group + kRows - 1) / kRows);
}

// Key tiles of the sequences in front of each, into `cum` [n_seq + 1] (LDS), by a workgroup of 256.
__device__ __forceinline__ void list_tiles(const AttendArgs& a, int64_t* cum) {
  __shared__ int64_t wave_sum[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t carry = 0;
  for (int base = 0; base < a.n_seq; base += 256) {
    const int s = base + threadIdx.x;
    int64_t mine = 0;
    if (s < a.n_seq) {
      const Sequence q = sequence_of(a, s);
      mine = key_tiles(q) * row_tiles(a, q) * a.cache.n_heads;
    }
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int64_t t = __shfl_up(upto, o);
      if (lane >= o) upto += t;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int64_t before = carry;
    for (int w = 0; w < wave; ++w) before += wave_sum[w];
    if (s < a.n_seq) cum[s] = before + upto - mine;
    carry += wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
    __syncthreads();
  }
  if (threadIdx.x == 0) cum[a.n_seq] = carry;
  __syncthreads();
}

// The sequence that tile u of the list belongs to.
__device__ __forceinline__ int sequence_at(const int64_t* cum, int n_seq, int64_t u) {
  int lo = 0, hi = n_seq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cum[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)v) |
                   (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32);
}

// 8 codes of 4 bits as bf16 128 + c: elements 2 i, 2 i + 1 in dword i.
__device__ __forceinline__ bf16x8 spread_nibbles(uint32_t x) {
  u32x4 t;
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = (x >> (4 * i) & 0x000f000fu) | 0x43004300u;
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
  __device__ __forceinline__ void load_keys(const char* block, int lane) {
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const char* row = block + token(t, r) * (kHalf / kBlockTokens);
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
  __device__ __forceinline__ bf16x8 key(int t, int w) const {
    if constexpr (KV == kKvBf16) return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(&k[t][4 * w]));
    else if constexpr (KV == kKvU8) return spread_bytes(k[t][2 * w], k[t][2 * w + 1]);
    else return spread_nibbles(k[t][w]);
  }
  // features 16 td + r, the 8 tokens of half j
  __device__ __forceinline__ bf16x8 value(int td, int j) const {
    if constexpr (KV == kKvBf16) return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(&v[td][4 * j]));
    else if constexpr (KV == kKvU8) return spread_bytes(v[td][2 * j], v[td][2 * j + 1]);
    else return spread_rows(v[td >> 1][2 * j], v[td >> 1][2 * j + 1], 4 * (td & 1));
  }
};

template <int KV, int HD>
__global__ __launch_bounds__(256) void attend_rows_kernel(AttendArgs a) {
  extern __shared__ int64_t cum[];
  __shared__ float4 params[4][64];
  constexpr int TD = HD / 16;
  constexpr float kOffset = KV == kKvU4 ? 136.f : 128.f, kCentre = KV == kKvU4 ? 8.f : 128.f;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  list_tiles(a, cum);
  const int64_t total = cum[a.n_seq], workers = min((int64_t)a.workers, total);
  const int64_t me = (int64_t)blockIdx.x * 4 + wave;
  if (me >= workers) return;
  int64_t u = uniform64(me * total / workers);
  const int64_t end = uniform64((me + 1) * total / workers), begin = u;
  const float c = a.scale * 1.44269504f;
  constexpr float kNone = -__builtin_inff();

  while (u < end) {
    // the segment that tile u belongs to, and this wave's tiles of it
    const int s = __builtin_amdgcn_readfirstlane(sequence_at(cum, a.n_seq, u));
    const Sequence q = sequence_of(a, s);
    const int64_t tiles = uniform64(key_tiles(q)), rel = u - cum[s];
    const int64_t segment = uniform64(rel / tiles), start = cum[s] + segment * tiles;
    const int row_tile = (int)(segment / a.cache.n_heads), head = (int)(segment - (int64_t)row_tile * a.cache.n_heads);
    int64_t tile = uniform64(u - start);
    const int64_t last = uniform64(min(tiles, end - start)), first = tile;

    // this lane's row
    const int64_t row = (int64_t)row_tile * kRows + r;
    const int in_seq = (int)(row / a.group), qh = head * a.group + (int)(row - (int64_t)in_seq * a.group);
    const bool live = in_seq < q.count;
    const int64_t token = q.first + (live ? in_seq : 0);
    const int64_t sees = a.causal ? min(max(q.len - q.count + in_seq + 1, (int64_t)0), q.len) : q.len;
    const int64_t all_see = a.causal ? q.len - q.count + (int64_t)row_tile * kRows / a.group + 1 : q.len;  // what every row of the tile sees
    bf16x8 qf[HD / 32];
    float qsum = 0.f;
#pragma unroll
    for (int w = 0; w < HD / 32; ++w) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[w][e] = (bf16)0.f;
      if (live) qf[w] = *reinterpret_cast<const bf16x8*>(a.q + token * a.ldq + (int64_t)qh * HD + 32 * w + 8 * g);
#pragma unroll
      for (int e = 0; e < 8; ++e) qsum += (float)qf[w][e];
    }
    qsum = quarters_sum(qsum);

    f32x4 o[TD], ones_acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < TD; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNone, l = 0.f, low = 0.f;
    const int* pages = a.pages + (a.lens ? s * a.ldp : 0);
    Tile64<KV, HD> t64;

    for (; tile < last; ++tile) {
      if (tile * 64 >= q.len) break;
      const int64_t page = pages[tile >> (a.cache.log2_page - 6)];
      if (page < 0 || page >= a.cache.n_pages) continue;  // a page outside the cache holds nothing to see
      const char* block = a.cache.data + kv_block_offset<KV, HD>(a.cache, page, head, (int)(tile & ((1 << (a.cache.log2_page - 6)) - 1)));
      t64.load_keys(block, lane);
      t64.load_values(block, lane);

      f32x4 x[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float x0 = KV == kKvU4 ? -128.f * qsum : 0.f;
        x[t] = f32x4{x0, x0, x0, x0};
#pragma unroll
        for (int w = 0; w < HD / 32; ++w) x[t] = mfma16(t64.key(t, w), qf[w], x[t]);
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
      const bool masked = tile * 64 + 64 > all_see;
      const int seen = (int)min(max(sees - tile * 64, (int64_t)0), (int64_t)64);
      if (masked) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (Tile64<KV, HD>::token(t, 4 * g + i) >= seen) x[t][i] = kNone;
      }
      float most = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
      most = fmaxf(most, fmaxf(fmaxf(fmaxf(x[2][0], x[2][1]), fmaxf(x[2][2], x[2][3])), fmaxf(fmaxf(x[3][0], x[3][1]), fmaxf(x[3][2], x[3][3]))));
      most = fmaxf(m, quarters_max(most));
      const float mc = most == kNone ? 0.f : most * c;
      const float shrink = __builtin_amdgcn_exp2f(fmaf(m, c, -mc));
      m = most;
      l *= shrink;
      low *= shrink;
      ones_acc *= shrink;
#pragma unroll
      for (int i = 0; i < TD; ++i) o[i] *= shrink;
      bf16x8 pf[2];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float p = __builtin_amdgcn_exp2f(fmaf(x[t][i], c, -mc));
          l += p;
          if constexpr (KV != kKvBf16) {
            const float vs = vp[t][i >> 1][2 * (i & 1)], vb = vp[t][i >> 1][2 * (i & 1) + 1];
            const bool off = masked && Tile64<KV, HD>::token(t, 4 * g + i) >= seen;  // parameters of keys that are not seen may be anything
            low = off ? low : fmaf(p, fmaf(kCentre, vs, vb), low);
            p = off ? 0.f : p * vs;
          }
          const int e = 4 * (t & 1) + i;
          pf[t >> 1][KV == kKvU4 ? (e & 4) | (e & 1) << 1 | (e & 2) >> 1 : e] = (bf16)p;
        }
      if constexpr (KV == kKvBf16) {
        if (tile * 64 + 64 > q.len) {  // what lies behind the last token may be anything, and 0 NaN = NaN
          const int there = (int)(q.len - tile * 64);
#pragma unroll
          for (int i = 0; i < TD; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const int at = 32 * j + 8 * g + 2 * w;
                uint32_t& d = t64.v[i][4 * j + w];
                d = at >= there ? 0u : at + 1 >= there ? d & 0xffffu : d;
              }
        }
      } else {
        bf16x8 one;
#pragma unroll
        for (int e = 0; e < 8; ++e) one[e] = (bf16)1.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) ones_acc = mfma16(one, pf[j], ones_acc);
      }
#pragma unroll
      for (int i = 0; i < TD; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) o[i] = mfma16(t64.value(i, j), pf[j], o[i]);
    }

    l = quarters_sum(l);
    if constexpr (KV != kKvBf16) {
      const float add = quarters_sum(low) - kOffset * ones_acc[0];
#pragma unroll
      for (int i = 0; i < TD; ++i) o[i] += add;
    }
    const bool whole = first == 0 && last == tiles;
    if (whole && !a.whole) {
      if (live) {
        const float inv = l > 0.f ? 1.f / l : l;  // (NaN stays)
        bf16* to = a.out + token * a.ldo + (int64_t)qh * HD + 4 * g;
#pragma unroll
        for (int i = 0; i < TD; ++i) {
          bf16 t[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) t[e] = (bf16)(l == 0.f ? 0.f : o[i][e] * inv);
          *reinterpret_cast<u32x2*>(to + 16 * i) = __builtin_bit_cast(u32x2, t);
        }
        if (a.lse && g == 0) a.lse[token * a.hq + qh] = l == 0.f ? kNone : fmaf(m, a.scale, __logf(l));
      }
    } else if (live) {
      const int64_t slot = whole ? token * a.hq + qh : (2 * me + (start < begin ? 0 : 1)) * kRows + r;
      float* base = whole ? a.whole : a.part;
      float* to = base + slot * HD + 4 * g;
#pragma unroll
      for (int i = 0; i < TD; ++i) *reinterpret_cast<f32x4*>(to + 16 * i) = o[i];
      if (g == 0)
        reinterpret_cast<float2*>(base + (whole ? (int64_t)a.n_tokens * a.hq : (int64_t)2 * a.workers * kRows) * HD)[slot] =
            make_float2(l == 0.f ? kNone : m * c, l);
    }
    u = start + last;
  }
}

struct JoinArgs {
  AttendArgs own, prefix;  // prefix.workers = 0: none
};

// Where the pieces of a row lie: workers [begin, end) have one each.
struct Pieces {
  const float* o;
  const float2* ml;
  int64_t begin, end, start, total, workers, row;  // row: in the segment; of a whole segment (workers = 0): its place in `whole`
  __device__ __forceinline__ int64_t slot(int64_t w) const {
    return workers ? (2 * w + (start < w * total / workers ? 0 : 1)) * kRows + row : row;
  }
};
template <int HD>
__device__ __forceinline__ Pieces pieces_of(const AttendArgs& a, int64_t total, int64_t start, int64_t tiles, int64_t row, int64_t out_row) {
  Pieces p;
  p.total = total;
  p.workers = min((int64_t)a.workers, total);
  p.start = start;
  p.row = row;
  p.begin = ((start + 1) * p.workers - 1) / total;
  p.end = ((start + tiles) * p.workers - 1) / total + 1;
  p.o = a.part;
  p.ml = reinterpret_cast<const float2*>(a.part + (int64_t)2 * a.workers * kRows * HD);
  if (p.end - p.begin == 1 && a.whole) {
    p.workers = 0;
    p.row = out_row;
    p.o = a.whole;
    p.ml = reinterpret_cast<const float2*>(a.whole + (int64_t)a.n_tokens * a.hq * HD);
  }
  return p;
}

// One output row a workgroup of 256: HD / 4 threads hold a row, 1024 / HD pieces at a time.
template <int HD>
__global__ __launch_bounds__(256) void attend_join_kernel(JoinArgs a) {
  extern __shared__ int64_t cum[];
  constexpr int TR = HD / 4, AT = 256 / TR;
  __shared__ float sh_m[4];
  __shared__ f32x4 sh_o[AT][TR];
  const AttendArgs& own = a.own;
  list_tiles(own, cum);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t token = blockIdx.x;
  const int qh = blockIdx.y, head = qh / own.group;
  // the token's sequence
  int s = (int)token;
  if (own.q_starts) {
    int lo = 0, hi = own.n_seq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (own.q_starts[mid] <= token) lo = mid;
      else hi = mid - 1;
    }
    s = lo;
  }
  const Sequence q = sequence_of(own, s);
  if (token < q.first || token >= q.first + q.count) return;
  const int64_t row = (token - q.first) * own.group + (qh - head * own.group), tiles = key_tiles(q);
  const int64_t out_row = token * own.hq + qh;
  Pieces p[2];
  p[0] = pieces_of<HD>(own, cum[own.n_seq], cum[s] + (row / kRows * own.cache.n_heads + head) * tiles, tiles, row % kRows, out_row);
  int sides = 1;
  if (a.prefix.workers) {
    sides = 2;
    const Sequence z = sequence_of(a.prefix, 0);
    const int64_t prow = token * own.group + (qh - head * own.group), ptiles = key_tiles(z);
    p[1] = pieces_of<HD>(a.prefix, ptiles * row_tiles(a.prefix, z) * own.cache.n_heads, (prow / kRows * own.cache.n_heads + head) * ptiles, ptiles,
                         prow % kRows, out_row);
  } else if (p[0].end - p[0].begin == 1) {
    return;  // a whole segment: written already
  }
  constexpr float kNone = -__builtin_inff();
  // the largest maximum, then the sum
  float m = kNone;
  for (int k = 0; k < sides; ++k)
    for (int64_t w = p[k].begin + threadIdx.x; w < p[k].end; w += 256) m = fmaxf(m, p[k].ml[p[k].slot(w)].x);
#pragma unroll
  for (int o = 1; o < 64; o *= 2) m = fmaxf(m, __shfl_xor(m, o));
  if (lane == 0) sh_m[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(sh_m[0], sh_m[1]), fmaxf(sh_m[2], sh_m[3]));
  const float base = m == kNone ? 0.f : m;
  const int t = threadIdx.x % TR, at = threadIdx.x / TR;
  float l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < sides; ++k)
    for (int64_t w = p[k].begin + at; w < p[k].end; w += AT) {
      const int64_t slot = p[k].slot(w);
      const float2 d = p[k].ml[slot];
      const float f = __builtin_amdgcn_exp2f(d.x - base);
      l = fmaf(d.y, f, l);
      o += *reinterpret_cast<const f32x4*>(p[k].o + slot * HD + 4 * t) * f;
    }
  sh_o[at][t] = o;
  __shared__ float sh_s[AT];
  if (t == 0) sh_s[at] = l;
  __syncthreads();
  if (at != 0) return;
  for (int i = 1; i < AT; ++i) o += sh_o[i][t], l += sh_s[i];
  const float inv = l == 0.f ? 0.f : 1.f / l;
  bf16 v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (bf16)(l == 0.f ? 0.f : o[e] * inv);
  *reinterpret_cast<u32x2*>(own.out + token * own.ldo + (int64_t)qh * HD + 4 * t) = __builtin_bit_cast(u32x2, v);
  if (own.lse && t == 0) own.lse[token * own.hq + qh] = l == 0.f ? kNone : (base + __log2f(l)) * 0.693147181f;
}

}  // namespace kt
