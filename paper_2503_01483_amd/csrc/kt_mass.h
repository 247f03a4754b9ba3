// kt_mass.h -- attention weight that the tokens of the paged cache receive from new queries, accumulated a token and key head.
//
//   mass_j <- decay mass_j (0 of a token that is one of the queries) + sum_r exp(scale q_r . k_j - lse_r),  r over the rows of j's key head that see j
//
// A wave holds 64 keys, one block of the cache, in the registers of the 16 x 16 x 32 products' first operand (S^T = K Q^T, as in kt_attention.h) and
// goes through the rows sixteen at a time: a lane adds up the exponentials of one row in sixteen for its 16 keys, and the 16 lanes are added
// once at the end.  Every sum has a fixed order and one owner: nothing is atomic, no score leaves the registers.
#pragma once
#include "kt_attention.h"

namespace kt {

struct MassArgs {
  AttendArgs a;     // cache, q, q_starts, lens, pages, ldq, ldp, n_seq, n_tokens, hq, group, scale, lse (read)
  const float* lse;
  float* mass;      // [page][head][token of the page]
  float decay;
};

// Sum over the 16 lanes of a row of the wave, in all of them.
__device__ __forceinline__ float row16_sum(float v) {
  v += lane_xor<1>(v);
  v += lane_xor<2>(v);
  v += lane_xor<4>(v);
  return v + lane_xor<8>(v);
}

// Groups of keys of one head in front of each sequence, `cum` [n_seq + 1] (LDS), by a workgroup of 256.
__device__ __forceinline__ void list_key_groups(const AttendArgs& a, int keys, int* cum) {
  __shared__ int wave_sum[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int carry = 0;
  for (int base = 0; base < a.n_seq; base += 256) {
    const int s = base + threadIdx.x;
    int mine = 0;
    if (s < a.n_seq) {
      const Sequence q = sequence_of(a, s);
      mine = (int)(((unsigned)q.len + keys - 1) / (unsigned)keys);
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
    __syncthreads();
  }
  if (threadIdx.x == 0) cum[a.n_seq] = carry;
  __syncthreads();
}

// WR of a workgroup's four waves share a block's rows, 4 / WR blocks lie next to each other.
template <int KV, int HD, int WR>
__global__ __launch_bounds__(256, 2) void mass_kernel(MassArgs t) {
  extern __shared__ int cum[];
  __shared__ float joined[WR > 1 ? 4 : 1][64];
  constexpr int WK = 4 / WR;
  constexpr float kInf = __builtin_inff();
  using Tile = Tile64<KV, HD>;
  const AttendArgs& a = t.a;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), r = lane & 15, g = lane >> 4, heads = a.cache.n_heads;
  const int wk = wave / WR, wr = wave % WR, page_blocks = a.cache.log2_page - 6;
  const float c = a.scale * 1.44269504f;
  list_key_groups(a, 64 * WK, cum);
  const int64_t total = (int64_t)cum[a.n_seq] * heads;
  const int step_q = 16 * WR / a.group, step_r = 16 * WR - step_q * a.group;

  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int at = (int)(u / heads), head = (int)(u - (int64_t)at * heads);
    const int s = uniform(sequence_at(cum, a.n_seq, at));
    const Sequence q = sequence_of(a, s);
    const int tile = (at - uniform(cum[s])) * WK + wk, ahead = q.len - q.count, key0 = tile * 64;
    const int there = uniform(min(q.len - key0, 64));
    int page = there > 0 ? a.pages[s * a.ldp + (tile >> page_blocks)] : -1;
    if (page >= a.cache.n_pages) page = -1;
    page = uniform(page);
    float sum[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[i][e] = 0.f;
    if (page >= 0) {
      Tile k;
      const int64_t block = kv_block_offset<KV, HD>(a.cache, page, head, tile & ((1 << page_blocks) - 1));
      k.load_keys(a.cache.data + block, lane);
      [[maybe_unused]] f32x4 par[4][2];  // {step, minimum} of a lane's keys
      if constexpr (KV != kKvBf16) {
        const f32x4* p = reinterpret_cast<const f32x4*>(a.cache.data + block + 2 * Tile::kHalf) + 8 * g;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) par[i][h] = p[2 * i + h];
      }
      // rows from the first that sees the first key on
      const int64_t rows = (int64_t)q.count * a.group;
      int64_t row = (max(0, key0 - ahead) * (int64_t)a.group & ~(int64_t)15) + 16 * wr + r;
      int in_seq = (int)(row / a.group), rest = (int)(row - (int64_t)in_seq * a.group);
      for (; row - r < rows; row += 16 * WR) {
        const bool live = row < rows;
        const int64_t token = q.first + (live ? in_seq : 0);
        const int qh = head * a.group + (live ? rest : 0);
        bf16x8 qf[HD / 32];
#pragma unroll
        for (int w = 0; w < HD / 32; ++w) qf[w] = *reinterpret_cast<const bf16x8*>(a.q + token * a.ldq + qh * HD + 32 * w + 8 * g);
        const float lse = t.lse[token * a.hq + qh];
        const bool counts = live && fabsf(lse) <= kHuge;
        const float base = counts ? lse * 1.44269504f : kInf;
        f32x4 x[4], qsum = {0.f, 0.f, 0.f, 0.f};
        if constexpr (KV != kKvBf16) {
          bf16x8 one;
#pragma unroll
          for (int e = 0; e < 8; ++e) one[e] = (bf16)1.f;
#pragma unroll
          for (int w = 0; w < HD / 32; ++w) qsum = mfma16(one, qf[w], qsum);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = KV == kKvU4 ? -128.f * qsum : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < HD / 32; ++w) x[i] = mfma16(k.key(i, w), qf[w], x[i]);
          if constexpr (KV != kKvBf16) {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] = fmaf(x[i][e], par[i][e >> 1][2 * (e & 1)], par[i][e >> 1][2 * (e & 1) + 1] * qsum[e]);
          }
        }
        const int seen = counts ? ahead + in_seq + 1 - key0 : 0;  // of the block's tokens
        const bool edge = __any(seen < 64);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(fmaf(x[i][e], c, -base));
            sum[i][e] += edge && Tile::token(i, 4 * g + e) >= seen ? 0.f : p;
          }
        in_seq += step_q;
        rest += step_r;
        if (rest >= a.group) rest -= a.group, ++in_seq;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[i][e] = row16_sum(sum[i][e]);
    // lane r of a quarter keeps its r-th key
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) mine = r == i ? sum[i >> 2][i & 3] : mine;
    const int j = Tile::token(r >> 2, 4 * g + (r & 3));
    if constexpr (WR > 1) {
      __syncthreads();
      joined[wave][lane] = mine;
      __syncthreads();
      if (wr != 0) continue;
      mine = 0.f;
#pragma unroll
      for (int w = 0; w < WR; ++w) mine += joined[wk * WR + w][lane];
    }
    if (page >= 0 && j < there) {
      float* to = t.mass + (((int64_t)page * heads + head) << a.cache.log2_page) + ((key0 + j) & ((1 << a.cache.log2_page) - 1));
      if (key0 + j < ahead && t.decay != 0.f) mine = fmaf(t.decay, *to, mine);
      *to = mine;
    }
  }
}

}  // namespace kt
