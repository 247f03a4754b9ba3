// kt_attention_tiles.h -- attention of many rows: prompts, chunks, and a prefix that a whole batch shares.
//
// A workgroup holds 32 rows a wave (kt_attention.h says what rows are) and stages tiles of 64 keys and values through LDS, double buffered.  Products
// are 32 x 32 x 16: S^T = K Q^T, then O^T += V^T P^T with the exponentials of a lane's scores as the operand, as in kt_attention.h; the
// keys' rows are read with bits 2 and 3 of the key's number exchanged, which makes the eight scores that a lane holds of each
// sixteen keys neighbours.
//
// Bound by the matrix cores and the vector ALU side by side: a wave's tile takes 1024 cycles of products and about 900 of
// exponentials and the like (HD = 128), and 32 KiB of LDS reads, 256 cycles of the CU's.
//
// bf16 caches go straight from memory to LDS.  Of quantised ones the keys' codes do, as exact bf16 values, and a score becomes s (q . c) + b sum(q)
// in fp32 as in kt_attention.h; the values are expanded on the way, in fp16: a row s c + b is scaled by a power of two per
// tile, found from the rows' {s, b}, so that its largest value is just below one, and rounded to 11 bits (2^-11 of it or less; bf16 would have 8, little
// more than the codes of 8 bits).  The exponent is carried along with O like the running maximum.  The maximum is raised only
// once a score passes it by 2^8 (p stays below 256 in either type).
//
// All key tiles of all row tiles form one list, heads outermost; each workgroup takes an equal piece, neighbouring pieces on one XCD, whose
// L2 then holds the keys of few heads.  Segments that are cut are joined by a second launch.
#pragma once
#include <type_traits>

#include "kt_attention.h"

namespace kt {

struct TileArgs {
  AttendArgs a;
  const int* prefix_pages;
  int prefix_len;
  int workers;           // workgroups; a multiple of 8
  int entries;           // row tiles of one head, gaps among them
  int *cum, *seq, *row;  // [entries + 1] key tiles in front of each, its sequence and row tile
  int4* cuts;            // [workers] {entry, head, pieces or 0}
  float* part;           // pieces of cut segments: O [2 workers][R][HD], then {max in bits, sum}
  int splits;            // of a prefix of its own (kt_attention.h takes the rest)
  float* prefix_part;    // [splits][n_tokens][hq][HD], then {max in bits, sum}
};

// 16 bytes a lane from memory straight into LDS: lane l lands at lds_addr + 16 l (wave-uniform).  Assembly, so that LDS reads of other buffers
// do not wait for them: waits are placed by hand (vmcnt).
__device__ __forceinline__ void to_lds_16(uint32_t voffset, const char* base, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voffset), "s"(base), "s"(lds_addr) : "memory", "m0");
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

template <class T>
__device__ __forceinline__ const T* uniform_ptr(const T* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const T*>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
                                    (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}

// Row tiles of R rows get numbers floor(first query * group / R) + s + 0, 1, ... (s their sequence): different for every sequence's.
__device__ __forceinline__ int64_t first_entry(const AttendArgs& a, int s, int R) {
  return (int64_t)min(max(a.q_starts ? a.q_starts[s] : s, 0), a.n_tokens) * a.group / R + s;
}

// The list of row tiles.  One workgroup of 1024.
template <int R>
__global__ __launch_bounds__(1024) void plan_tiles_kernel(TileArgs t) {
  __shared__ int wave_sum[16];
  const AttendArgs& a = t.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int prefix_tiles = (int)(((unsigned)t.prefix_len + 63) >> 6);
  int carry = 0;
  for (int base = 0; base < t.entries; base += 1024) {
    const int e = base + threadIdx.x;
    int mine = 0, s = 0;
    int64_t rt = 0;
    if (e < t.entries) {
      int hi = a.n_seq - 1;
      while (s < hi) {
        const int mid = (s + hi + 1) >> 1;
        if (first_entry(a, mid, R) <= e) s = mid;
        else hi = mid - 1;
      }
      const Sequence q = sequence_of(a, s);
      rt = e - first_entry(a, s, R);
      const int64_t rows = (int64_t)q.count * a.group;
      if (rt >= 0 && rt * R < rows) {
        const int last = (int)((min(rows, (rt + 1) * R) - 1) / a.group);
        const int sees = min(max(q.len - q.count + last + 1, 0), q.len);
        mine = max(1, prefix_tiles + (int)(((unsigned)sees + 63) >> 6));
      }
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int v = __shfl_up(upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int before = carry;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += wave_sum[w];
      carry += wave_sum[w];
    }
    if (e < t.entries) {
      t.cum[e] = before + upto - mine;
      t.seq[e] = s;
      t.row[e] = (int)rt;
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) t.cum[t.entries] = carry;
}

template <int KV, int HD, int WAVES>
struct TileShared {
  static constexpr int kKeys = kBlockTokens * HD * 2, kBuffer = 2 * kKeys;
  char data[2][kBuffer];           // keys [64][HD], values [HD][64], 16-byte chunks exchanged within a row (swizzled)
  float2 keys[2][64];              // {step, minimum} of the keys, times the factor of the exponentials
  _Float16 par[WAVES][2][64];      // of the tile that is being expanded: its values' steps and minima
  unsigned odd[2];                 // tokens of a tile with values that are not finite (bf16)
};

// The state of a workgroup's current tile of keys.
struct TileInfo {
  int v_exp;                 // exponent (biased by 126) that the values were scaled down by
  unsigned long long odd;    // tokens whose values are not finite (as 0 in LDS)
};

template <int KV, int HD, int WAVES>
struct TileLoader {
  using Shared = TileShared<KV, HD, WAVES>;
  static constexpr int THREADS = 64 * WAVES, kHalf = kv_half_bytes<KV, HD>(), ROWB = HD * 2;
  static constexpr int KMASK = HD >= 128 ? 15 : 7;
  // quantised: 16-byte (HD = 64, u4: 8-byte) pieces of a thread
  static constexpr int KW = KV == kKvU4 ? HD / 32 : HD / 16;                      // dwords of a (token, quarter)
  static constexpr int KP = 256 / THREADS > 0 ? 256 / THREADS : 1;                // (token, quarter)s of a thread
  static constexpr int VROWS = KV == kKvU4 ? HD / 2 : HD;
  static constexpr int VP = (VROWS * 4 + THREADS - 1) / THREADS;                  // (row, 16 tokens)s of a thread
  uint32_t k[KV == kKvBf16 ? 1 : KP][KV == kKvBf16 ? 1 : KW];
  u32x4 v[KV == kKvBf16 ? 1 : VP];
  float2 kp, vp;

  // Begins loading a block: bf16 into `buf`, else into registers.
  __device__ __forceinline__ void begin(const char* block, char* buf) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if constexpr (KV == kKvBf16) {
      const unsigned at = (unsigned)(uintptr_t)buf;  // (LDS addresses are the low 32 bits)
      constexpr int STEPS = Shared::kKeys / 1024 / WAVES;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int kb = (wave * STEPS + i) * 1024, byte = kb + lane * 16;
        const int row = byte / ROWB, chunk = byte % ROWB / 16;
        to_lds_16(row * ROWB + ((chunk ^ (row & KMASK)) << 4), block, __builtin_amdgcn_readfirstlane(at + kb));
      }
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int kb = (wave * STEPS + i) * 1024, byte = kb + lane * 16;
        const int row = byte / 128, chunk = byte % 128 / 16;
        to_lds_16(kHalf + row * 128 + ((chunk ^ (row & 7)) << 4), block, __builtin_amdgcn_readfirstlane(at + Shared::kKeys + kb));
      }
    } else {
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const char* from = block + (threadIdx.x + i * THREADS) * (KW * 4);
        if (KP * THREADS > 256 && threadIdx.x >= 256) break;
        if constexpr (KW % 4 == 0) {
#pragma unroll
          for (int j = 0; j < KW; j += 4) *reinterpret_cast<u32x4*>(&k[i][j]) = *reinterpret_cast<const u32x4*>(from + 4 * j);
        } else {
          *reinterpret_cast<u32x2*>(&k[i][0]) = *reinterpret_cast<const u32x2*>(from);
        }
      }
#pragma unroll
      for (int i = 0; i < VP; ++i) {
        const int piece = threadIdx.x + i * THREADS;
        if (piece < VROWS * 4) v[i] = *reinterpret_cast<const u32x4*>(block + kHalf + piece * 16);
      }
      kp = reinterpret_cast<const float2*>(block + 2 * kHalf)[lane];
      vp = reinterpret_cast<const float2*>(block + 2 * kHalf)[kBlockTokens + lane];
    }
  }

  // Finishes it: expanded into buffer `at`.  `there`: tokens of the block that exist; c: factor of the exponentials; v_run: exponent of O so far,
  // for a floor.
  __device__ __forceinline__ void finish(Shared& sh, int at, int there, float c, int v_run, TileInfo& info) {
    if constexpr (KV != kKvBf16) {
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
      constexpr float top = KV == kKvU4 ? 15.f : 255.f;
      char* buf = sh.data[at];
      const bool is = lane < there;
      if (wave == 0) sh.keys[at][lane] = is ? make_float2(kp.x * c, kp.y * c) : make_float2(0.f, 0.f);
      float vs = is ? vp.x : 0.f, vb = is ? vp.y : 0.f;
      float most = fmaxf(fabsf(vb), fabsf(fmaf(top, vs, vb)));
      const bool bad = !(most <= kHuge) || vs != vs;
      info.odd = __ballot(bad);
      if (bad) vs = vb = most = 0.f;
      info.v_exp = max(min(wave_max((int)(__float_as_uint(most) >> 23)), 252), v_run - 60);
      const float vf = __uint_as_float((unsigned)(253 - info.v_exp) << 23);
      sh.par[wave][0][lane] = (_Float16)(vs * vf);
      sh.par[wave][1][lane] = (_Float16)(vb * vf);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const f16x2 bias = {(_Float16)-1024.f, (_Float16)-1024.f};
      auto half2 = [](uint32_t x) { return __builtin_bit_cast(f16x2, x); };
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const int unit = threadIdx.x + i * THREADS, token = unit >> 2, g = unit & 3;
        if (KP * THREADS > 256 && threadIdx.x >= 256) break;
#pragma unroll
        for (int w = 0; w < HD / 32; ++w) {
          bf16x8 out;
          if constexpr (KV == kKvU4) out = spread_nibbles(k[i][w]);
          else out = spread_bytes(k[i][2 * w], k[i][2 * w + 1]);
          *reinterpret_cast<bf16x8*>(buf + token * ROWB + (((4 * w + g) ^ (token & KMASK)) << 4)) = out;
        }
      }
#pragma unroll
      for (int i = 0; i < VP; ++i) {
        const int piece = threadIdx.x + i * THREADS, row = piece >> 2, g = piece & 3;
        if (piece >= VROWS * 4) break;
        const u32x4* vs4 = reinterpret_cast<const u32x4*>(&sh.par[wave][0][16 * g]);
        const u32x4* vb4 = reinterpret_cast<const u32x4*>(&sh.par[wave][1][16 * g]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // 8 tokens
          const u32x4 s8 = vs4[h], b8 = vb4[h];
#pragma unroll
          for (int n = 0; n < (KV == kKvU4 ? 2 : 1); ++n) {
            u32x4 out;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t x = v[i][2 * h + (j >> 1)];
              if constexpr (KV == kKvU4) x = (n ? x >> 4 : x) & 0x0f0f0f0fu;
              x = __builtin_amdgcn_perm(0x64646464u, x, j & 1 ? 0x07030702u : 0x07010700u);
              out[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(half2(x) + bias, half2(s8[j]), half2(b8[j])));
            }
            const int f = KV == kKvU4 ? (row >> 4) * 32 + 16 * n + (row & 15) : row;
            *reinterpret_cast<u32x4*>(buf + Shared::kKeys + f * 128 + (((2 * g + h) ^ (f & 7)) << 4)) = out;
          }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
};

// N products in order, `product(n, operand)`, each with an operand from LDS, `read(n)`, that is asked for kAhead products earlier: left to itself
// the compiler waits for every read in front of its product.
template <int N, class Read, class Product>
__device__ __forceinline__ void pipelined(Read read, Product product) {
  constexpr int kAhead = 4;
  decltype(read(0)) ring[kAhead];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) ring[n] = read(n);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    product(n, ring[n % kAhead]);
    if (n + kAhead < N) ring[n % kAhead] = read(n + kAhead);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// PREFIX: the rows of all tokens over the prefix alone, split over its tiles, to prefix_part; else the list.
template <int KV, int HD, int WAVES, bool PREFIX>
__global__ __launch_bounds__(64 * WAVES, HD == 256 && WAVES == 4 ? 1 : 2) void attend_tiles_kernel(TileArgs t) {
  constexpr int R = 32 * WAVES, TD = HD / 32, KS = HD / 16;
  constexpr bool Q16 = KV != kKvBf16;  // quantised: p and the values in fp16
  using frag = std::conditional_t<Q16, f16x8, bf16x8>;
  using elem = std::conditional_t<Q16, _Float16, bf16>;
  using Loader = TileLoader<KV, HD, WAVES>;
  using Shared = typename Loader::Shared;
  extern __shared__ __align__(16) char lds[];
  Shared& sh = *reinterpret_cast<Shared*>(lds);
  constexpr float kNone = -__builtin_inff();
  const AttendArgs& a = t.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5, heads = a.cache.n_heads;
  const int page_blocks = a.cache.log2_page - 6, prefix_tiles = (int)(((unsigned)t.prefix_len + 63) >> 6);
  const float c = a.scale * 1.44269504f;

  int me, begin, end, per = 0, one = 0;
  if constexpr (PREFIX) {
    me = blockIdx.x;
    begin = 0;
    end = 1;
  } else {
    me = (blockIdx.x & 7) * (t.workers >> 3) + (blockIdx.x >> 3);
    one = t.cum[t.entries];
    per = piece_length(one * heads, t.workers);
    begin = me * per;
    end = min(begin + per, one * heads);
  }
  int4 cut = {0, 0, 0, 0};

  for (int u = begin; u < end;) {
    int head, entry = 0, tiles, first, last, row_tile, split = 0;
    Sequence q;
    const int* pages = nullptr;
    if constexpr (PREFIX) {
      const int row_tiles = (int)(((int64_t)a.n_tokens * a.group + R - 1) / R);
      split = me / (row_tiles * heads);
      const int rest = me - split * row_tiles * heads;
      head = rest / row_tiles;
      row_tile = rest - head * row_tiles;
      q = Sequence{0, a.n_tokens, 0};
      tiles = prefix_tiles;
      first = (int)((int64_t)tiles * split / t.splits);
      last = (int)((int64_t)tiles * (split + 1) / t.splits);
    } else {
      head = (int)((unsigned)u / (unsigned)one);
      const int in = u - head * one;
      entry = uniform(sequence_at(t.cum, t.entries, in));
      const int s = uniform(t.seq[entry]);
      row_tile = uniform(t.row[entry]);
      q = sequence_of(a, s);
      pages = a.pages + s * a.ldp;
      const int at = uniform(t.cum[entry]);
      tiles = uniform(t.cum[entry + 1]) - at;
      first = in - at;
      last = min(tiles, first + (end - u));
    }
    // this lane's row
    const int64_t row = (int64_t)row_tile * R + 32 * wave + r;
    const bool live = row < (int64_t)q.count * a.group;
    const int in_seq = live ? (int)(row / a.group) : 0, qh = head * a.group + (live ? (int)(row - (int64_t)in_seq * a.group) : 0);
    const int64_t token = q.first + in_seq;
    const int sees = min(max(q.len - q.count + in_seq + 1, 0), q.len);                                    // of its own tokens
    const int all_see = q.len - q.count + 1 + (int)((int64_t)row_tile * R / a.group);                     // what every row of the workgroup sees
    bf16x8 qf[KS];
    float qsum = 0.f;
#pragma unroll
    for (int w = 0; w < KS; ++w) {
      qf[w] = *reinterpret_cast<const bf16x8*>(a.q + token * a.ldq + qh * HD + 16 * w + 8 * h);
      if constexpr (Q16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) qsum += (float)qf[w][i];
      }
    }
    if constexpr (Q16) qsum += __shfl_xor(qsum, 32);
    // arrived before the loop: a wait for them in it would wait for the tiles that are on their way to LDS as well
#pragma unroll
    for (int w = 0; w < KS; ++w) asm volatile("" : "+v"(qf[w]));

    f32x16 o[TD];
#pragma unroll
    for (int i = 0; i < TD; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m = kNone, l = 0.f;  // m: in bits (times c)
    int v_run = 0;             // exponent of O
    Loader ld;
    TileInfo info = {0, 0ull}, info_next = {0, 0ull};

    PageWindow window;
    const int* window_of = nullptr;
    // the block of tile `tile` and how many of its tokens exist; null: none that can be seen
    auto block_of = [&](int tile, int& there) -> const char* {
      const bool own = tile >= prefix_tiles;
      const int k = own ? tile - prefix_tiles : tile, len = own ? q.len : t.prefix_len;
      there = min(len - k * 64, 64);
      if (there <= 0) return nullptr;
      const int* table = own ? pages : t.prefix_pages;
      if (window_of != table) window.count = 0;
      window_of = table;
      const int64_t page = window.get(table, k >> page_blocks, (len + 63 >> 6) + (1 << page_blocks) - 1 >> page_blocks);
      if (page < 0 || page >= a.cache.n_pages) return nullptr;
      return uniform_ptr(a.cache.data + kv_block_offset<KV, HD>(a.cache, page, head, k & ((1 << page_blocks) - 1)));
    };

    int there = 0, there_next = 0;
    const char* block = block_of(first, there);
    __syncthreads();  // the buffers are free (the last segment's tile was read)
    if (block) {
      ld.begin(block, sh.data[0]);
      ld.finish(sh, 0, there, c, v_run, info);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    for (int tile = first; tile < last; ++tile) {
      const int buf = (tile - first) & 1;
      const char* next = nullptr;
      if (tile + 1 < last) {
        next = block_of(tile + 1, there_next);
        if (next) ld.begin(next, sh.data[buf ^ 1]);
      }
      const bool own = tile >= prefix_tiles;
      const int base = own ? (tile - prefix_tiles) * 64 : 0;
      const bool masked = own ? base + 64 > all_see : there < 64;
      const int seen = own ? min(max(sees - base, 0), there) : there;
      if (block) {
        char* kb = sh.data[buf];
        unsigned long long odd = info.odd;
        if constexpr (!Q16) {
          if (masked) {  // what a row does not see may be anything, and 0 NaN = NaN
            if (threadIdx.x < 2) sh.odd[threadIdx.x] = 0u;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < HD * 8 / (64 * WAVES); ++i) {
              const int piece = threadIdx.x + i * 64 * WAVES, f = piece >> 3, chunk = (piece & 7) ^ (f & 7);
              u32x4* p = reinterpret_cast<u32x4*>(kb + Shared::kKeys + piece * 16);
              u32x4 d = *p;
              unsigned which = 0u;
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const int at = 8 * chunk + 2 * w;
                d[w] = at >= there ? 0u : at + 1 >= there ? d[w] & 0xffffu : d[w];
                if ((d[w] & 0x7f80u) == 0x7f80u) which |= 1u << (2 * w), d[w] &= 0xffff0000u;
                if ((d[w] & 0x7f800000u) == 0x7f800000u) which |= 2u << (2 * w), d[w] &= 0xffffu;
              }
              *p = d;
              if (which) atomicOr(&sh.odd[chunk >> 2], which << (8 * (chunk & 3)));
            }
            __syncthreads();
            odd = (unsigned long long)sh.odd[1] << 32 | sh.odd[0];
          }
        }
        f32x16 x[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[k][e] = KV == kKvU4 ? -128.f * qsum : 0.f;  // (codes of 4 bits enter as 128 + c)
        {
          // (keys 32 further on have the same low bits)
          const int key = (r & 0x13) | (r & 4) << 1 | (r & 8) >> 1;
          const char* from = kb + key * Loader::ROWB;
          pipelined<2 * KS>(
              [&](int n) {
                return *reinterpret_cast<const bf16x8*>(from + (n & 1) * (32 * Loader::ROWB) + (((2 * (n >> 1) + h) ^ (key & Loader::KMASK)) << 4));
              },
              [&](int n, bf16x8 f) { x[n & 1] = mfma32(f, qf[n >> 1], x[n & 1]); });
        }
        if constexpr (Q16) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              const float4 kp = *reinterpret_cast<const float4*>(&sh.keys[buf][32 * k + 16 * (e >> 3) + 8 * h + (e & 7)]);
              x[k][e] = fmaf(x[k][e], kp.x, kp.y * qsum);
              x[k][e + 1] = fmaf(x[k][e + 1], kp.z, kp.w * qsum);
            }
        }
        if (masked) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (32 * k + 16 * (e >> 3) + 8 * h + (e & 7) >= seen) x[k][e] = kNone;
        }
        int shift = 0;
        if constexpr (Q16) {
          if (info.v_exp > v_run) {
            const float f = v_run - info.v_exp > -126 ? __uint_as_float((unsigned)(127 + v_run - info.v_exp) << 23) : 0.f;
#pragma unroll
            for (int i = 0; i < TD; ++i) o[i] *= f;
            v_run = info.v_exp;
          }
          shift = info.v_exp - v_run;  // at least -60
        }
        float most = fmaxf(x[0][0], x[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) most = fmaxf(most, fmaxf(x[0][e], x[1][e]));
        most = fmaxf(most, __shfl_xor(most, 32));
        if constexpr (!Q16) most *= c;
        if (__any(most > m + 8.f)) {
          const float raised = fmaxf(m, most), shrink = raised == kNone ? 1.f : __builtin_amdgcn_exp2f(m - raised);
          l *= shrink;
#pragma unroll
          for (int i = 0; i < TD; ++i) o[i] *= shrink;
          m = raised;
        }
        const float mb = (m == kNone ? 0.f : m) - (float)shift;
        frag pf[4];
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float p = __builtin_amdgcn_exp2f(Q16 ? x[k][e] - mb : fmaf(x[k][e], c, -mb));
            sum[e & 3] += p;
            pf[2 * k + (e >> 3)][e & 7] = (elem)p;
          }
        const float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        l += Q16 ? all * __uint_as_float((unsigned)(127 - shift) << 23) : all;
        {
          const char* from = kb + Shared::kKeys + r * 128;  // (features 32 further on have the same low bits)
          pipelined<4 * TD>([&](int n) { return *reinterpret_cast<const frag*>(from + n % TD * (32 * 128) + (((2 * (n / TD) + h) ^ (r & 7)) << 4)); },
                            [&](int n, frag f) { o[n % TD] = mfma32(f, pf[n / TD], o[n % TD]); });
        }
        if (odd) {
          const unsigned long long mine = seen >= 64 ? ~0ull : (1ull << seen) - 1;
          if constexpr (Q16) {
            const float add = odd & mine ? __builtin_nanf("") : 0.f;
#pragma unroll
            for (int i = 0; i < TD; ++i) o[i] += add;
          } else {
            const bf16* v = reinterpret_cast<const bf16*>(block + Loader::kHalf) + 4 * h * kBlockTokens;
#pragma unroll 1
            for (unsigned long long left = odd; left; left &= left - 1) {
              const int j = __builtin_ctzll(left);
#pragma unroll
              for (int i = 0; i < TD; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const float y = (float)v[(32 * i + (e & 3) + 8 * (e >> 2)) * kBlockTokens + j];
                  if (j < seen && !(fabsf(y) <= kHuge)) o[i][e] += y;
                }
            }
          }
        }
      }
      if (next) ld.finish(sh, buf ^ 1, there_next, c, v_run, info_next);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      block = next;
      info = info_next;
      there = there_next;
    }

    l += __shfl_xor(l, 32);
    if constexpr (Q16) {
      const float f = __uint_as_float((unsigned)(v_run + 1) << 23);
#pragma unroll
      for (int i = 0; i < TD; ++i) o[i] *= f;
    }
    const bool whole = !PREFIX && first == 0 && last == tiles;
    if (live) {
      if (whole) {
        const float inv = l > 0.f ? 1.f / l : l;  // (NaN stays)
        bf16* to = a.out + token * a.ldo + qh * HD + 4 * h;
#pragma unroll
        for (int i = 0; i < TD; ++i)
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            bf16 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = (bf16)(l == 0.f ? 0.f : o[i][e + k] * inv);
            *reinterpret_cast<u32x2*>(to + 32 * i + 2 * e) = __builtin_bit_cast(u32x2, v);
          }
        if (a.lse && h == 0) a.lse[token * a.hq + qh] = l == 0.f ? kNone : (m + __log2f(l)) * 0.693147181f;
      } else {
        const int64_t slot = PREFIX ? (split * (int64_t)a.n_tokens + token) * a.hq + qh : (int64_t)(2 * me + (first ? 0 : 1)) * R + 32 * wave + r;
        float* to = (PREFIX ? t.prefix_part : t.part) + slot * HD + 4 * h;
#pragma unroll
        for (int i = 0; i < TD; ++i)
#pragma unroll
          for (int e = 0; e < 16; e += 4) *reinterpret_cast<f32x4*>(to + 32 * i + 2 * e) = f32x4{o[i][e], o[i][e + 1], o[i][e + 2], o[i][e + 3]};
        const int64_t slots = PREFIX ? (int64_t)t.splits * a.n_tokens * a.hq : (int64_t)2 * t.workers * R;
        if (h == 0) reinterpret_cast<float2*>((PREFIX ? t.prefix_part : t.part) + slots * HD)[slot] = make_float2(l == 0.f ? kNone : m, l);
      }
    }
    if constexpr (PREFIX) break;
    if (first == 0 && !whole) cut = int4{entry, head, (int)((unsigned)(u + tiles - 1) / (unsigned)per) - me + 1, 0};
    u += last - first;
  }
  if (!PREFIX && threadIdx.x == 0) t.cuts[me] = cut;
}

// Running {max, sum, O} of a row's pieces, four features a lane.
struct Joined {
  float m = -__builtin_inff(), l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  __device__ __forceinline__ void add(float2 d, f32x4 v) {
    const float most = fmaxf(m, d.x), base = most == -__builtin_inff() ? 0.f : most;
    const float f = __builtin_amdgcn_exp2f(d.x - base), h = __builtin_amdgcn_exp2f(m - base);
    l = fmaf(d.y, f, l * h);
    o = v * f + o * h;
    m = most;
  }
  __device__ __forceinline__ void store(const AttendArgs& a, int64_t token, int qh, int hd, int lane4) const {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16 v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (bf16)(l == 0.f ? 0.f : o[e] * inv);
    *reinterpret_cast<u32x2*>(a.out + token * a.ldo + (int64_t)qh * hd + lane4) = __builtin_bit_cast(u32x2, v);
    if (a.lse && lane4 == 0) a.lse[token * a.hq + qh] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.693147181f;
  }
};

// The cut segments of the list: HD / 4 threads a row, grid (workers, R HD / 1024).
template <int HD, int R>
__global__ __launch_bounds__(256) void join_tiles_kernel(TileArgs t) {
  constexpr int TR = HD / 4;
  const int me = blockIdx.x;
  const int4 cut = t.cuts[me];
  if (cut.z == 0) return;
  const AttendArgs& a = t.a;
  const Sequence q = sequence_of(a, t.seq[cut.x]);
  const int r = blockIdx.y * (256 / TR) + threadIdx.x / TR, lane4 = 4 * (threadIdx.x % TR);
  const int64_t row = (int64_t)t.row[cut.x] * R + r;
  if (row >= (int64_t)q.count * a.group) return;
  const float2* ml = reinterpret_cast<const float2*>(t.part + (int64_t)2 * t.workers * R * HD);
  Joined j;
  for (int k = 0; k < cut.z; ++k) {
    const int64_t slot = (2 * ((int64_t)me + k) + (k ? 0 : 1)) * R + r;
    j.add(ml[slot], *reinterpret_cast<const f32x4*>(t.part + slot * HD + lane4));
  }
  const int in_seq = (int)(row / a.group);
  j.store(a, q.first + in_seq, cut.y * a.group + (int)(row - (int64_t)in_seq * a.group), HD, lane4);
}

// Every row of a batch of single tokens behind a prefix: its own pieces (kt_attention.h) and those over the prefix.  HD / 4 threads a row.
template <int HD>
__global__ __launch_bounds__(256) void join_prefix_kernel(TileArgs t) {
  constexpr int TR = HD / 4;
  const AttendArgs& a = t.a;
  const int64_t out_row = (int64_t)blockIdx.x * (256 / TR) + threadIdx.x / TR;
  if (out_row >= (int64_t)a.n_tokens * a.hq) return;
  const int lane4 = 4 * (threadIdx.x % TR);
  const int token = (int)(out_row / a.hq), qh = (int)(out_row - (int64_t)token * a.hq), head = qh / a.group;
  int s = token;
  if (a.q_starts) {
    int lo = 0, hi = a.n_seq - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.q_starts[mid] <= token) lo = mid;
      else hi = mid - 1;
    }
    s = lo;
  }
  const Sequence q = sequence_of(a, s);
  const int r = (token - q.first) * a.group + qh - head * a.group;
  if (token < q.first || token >= q.first + q.count || r >= kRows) return;
  const int total = a.tiles[a.n_seq] * a.cache.n_heads, per = piece_length(total, a.workers);
  const int tiles = key_tiles(q), start = a.tiles[s] * a.cache.n_heads + head * tiles;
  const int w0 = (int)((unsigned)start / (unsigned)per), w1 = (int)((unsigned)(start + tiles - 1) / (unsigned)per);
  Joined j;
  const int64_t rows = (int64_t)a.n_tokens * a.hq;
  const float2* pml = reinterpret_cast<const float2*>(t.prefix_part + t.splits * rows * HD);
  for (int z = 0; z < t.splits; ++z) j.add(pml[z * rows + out_row], *reinterpret_cast<const f32x4*>(t.prefix_part + (z * rows + out_row) * HD + lane4));
  if (w0 == w1) {
    j.add(reinterpret_cast<const float2*>(a.whole + rows * HD)[out_row], *reinterpret_cast<const f32x4*>(a.whole + out_row * HD + lane4));
  } else {
    const float2* ml = reinterpret_cast<const float2*>(a.part + (int64_t)2 * a.workers * kRows * HD);
    for (int w = w0; w <= w1; ++w) {
      const int64_t slot = (2 * (int64_t)w + (w == w0 ? 1 : 0)) * kRows + r;
      j.add(ml[slot], *reinterpret_cast<const f32x4*>(a.part + slot * HD + lane4));
    }
  }
  j.store(a, token, qh, HD, lane4);
}

}  // namespace kt
