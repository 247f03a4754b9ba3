// kt_attention_tiles.h -- attention of many rows: prompts, chunks, and a prefix that a whole batch shares.
//
// A workgroup holds 32 rows a wave (kt_attention.h says what rows are) and stages tiles of 64 keys and values through LDS, double buffered.  Products
// are 32 x 32 x 16: S^T = K Q^T, then O^T += V^T P^T with the exponentials of a lane's scores as the operand, as in kt_attention.h; the
// keys' rows are read with bits 2 and 3 of the key's number exchanged, which makes the eight scores that a lane holds of each
// sixteen keys neighbours.
//
// A wave's tile takes the matrix cores 1024 cycles (HD = 128) and the vector ALU about as long, most of it exponentials: three quarters of them are
// worked out beside the products of the values that need the others, the rest beside the other wave of the SIMD.
// 2 x 8192 tokens, 32 + 2 x 8 heads of 128, bf16: 808 to 838 us, 806 to 835 TFLOP/s (a matrix product of 8192: 1143); 8 x 300 behind 8000, 4 bits: 262 to 292 us,
// 530 to 590, by the card.  No unit is the bound: of the cycles (at 1.9 to 2.0 GHz, counted) the matrix cores are busy 40 % / 30 %, the vector ALU 63 % in both, the LDS
// 30 % / 37 %, a third / a quarter of that for bank conflicts.  What is missing is overlap: quantised tiles are expanded between the last product and
// the barrier, by all waves at once, and a segment's ends cost 19000 cycles.
//
// bf16 caches go straight from memory to LDS.  Of quantised ones the keys' codes do, as exact bf16 values, and a score becomes s (q . c) + b sum(q)
// in fp32 as in kt_attention.h; the values are expanded on the way, in fp16: a row s c + b is scaled by a power of two, one a
// tile, found from the rows' {s, b}, so that its largest value is just below one (one a token, entering with p, in tiles that some row does not see all of, so
// that no row depends on what it does not see, and where sizes differ by more than 2^6), and computed in fp16 as s (c - middle) + (b + s middle): the roundings
// of both parts and of the sum are 1.5 x 2^-11 of that largest value together (uncentred, s c is off by up to 2^-11 of the row's whole width
// more; bf16 would have 2^-8, little more than the codes of 8 bits).  A row has two running maxima, of the
// scores for its sum of p and of score and exponent together for O, so that large values of little weight leave the others their bits.  They are raised only
// once they are passed by 2^8 (p, and p times the power of two, stay below 256).  In fp16 p goes in times 2^7: it is rounded to 2^-31 of the row's largest
// p |v| at worst, and a million tokens of it do not show in a result.
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
  int4* list;            // [entries + 1] {tiles of the keys (and cost) in front, sequence, row tile, tiles and cost}
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

// Row tiles of R rows get numbers floor(first query * group / R) + s + 0, 1, ... (s their sequence): different for every sequence's.
__device__ __forceinline__ int64_t first_entry(const AttendArgs& a, int s, int R) {
  return (int64_t)min(max(a.q_starts ? a.q_starts[s] : s, 0), a.n_tokens) * a.group / R + s;
}

// What a segment costs beside its tiles, in tiles: its queries, the first tiles' way to LDS, its output (19000 cycles, a tile 4400).  Counted in the
// list, in front of them, so that pieces take equally long.
constexpr int kSegmentCost = 4;

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
        mine = kSegmentCost + max(1, prefix_tiles + (int)(((unsigned)sees + 63) >> 6));
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
      t.list[e] = int4{before + upto - mine, s, (int)rt, mine};
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) t.list[t.entries] = int4{carry, 0, 0, 0};
}

template <int KV, int HD, int WAVES>
struct TileShared {
  static constexpr int kTile = kBlockTokens * HD * 2;
  // 16-byte chunks exchanged within a row (swizzled)
  char keys[2][kTile];          // [64][HD]
  char values[2][kTile];        // [HD][64]
  float2 par[2][64];            // {step, minimum} of the keys, times the factor of the exponentials
  _Float16 expand[WAVES][2][64];  // steps of the values that are being expanded, and what their middle code stands for
  float power[2][64];             // exponents of the tokens' values, where each has its own
  unsigned long long odd[2][WAVES];  // bf16: tokens of a masked tile with values that are not finite, those in the pieces of each wave
};

// Moves tiles of keys and of values into LDS.
template <int KV, int HD, int WAVES>
struct TileLoader {
  using Shared = TileShared<KV, HD, WAVES>;
  static constexpr int THREADS = 64 * WAVES, kHalf = kv_half_bytes<KV, HD>(), ROWB = HD * 2;
  // The chunks of key row `row` are exchanged with this: eight lanes that read together, rows 0 .. 3 and 8 .. 11 or the like, take eight
  // different ones of the eight places that 32 banks have.  Linear: of rows without a common bit it is that of each, exclusive or.
  __host__ __device__ static constexpr int exchange(int row) { return (row & 3) | (row & 8) >> 1 | (HD >= 128 ? (row & 4) << 1 : 0); }
  static constexpr int STEPS = Shared::kTile / 1024 / WAVES;                      // bf16: KiB of a wave, keys and values each
  // quantised: pieces of a thread
  static constexpr int KW = KV == kKvU4 ? HD / 32 : HD / 16;                      // dwords of a (token, quarter)
  static constexpr int VROWS = KV == kKvU4 ? HD / 2 : HD;
  static constexpr int VP = (VROWS * 4 + THREADS - 1) / THREADS;                  // (row, 16 tokens)s of a thread
  // (where keys and values are 256 pieces each, of 512 threads half take the ones, half the others)
  __device__ __forceinline__ static int piece(int tid, int i) { return (VROWS * 4 == 256 && THREADS == 512 ? tid ^ 256 : tid) + i * THREADS; }
  // the thread's number, and with it every address, worked out anew: kept over the loop they would push others out to memory
  __device__ __forceinline__ static int thread() {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    return tid;
  }
  static_assert(THREADS >= 256);                                                  // (256 (token, quarter)s: at most one a thread)
  uint32_t k[KV == kKvBf16 ? 1 : KW];
  u32x4 v[KV == kKvBf16 ? 1 : VP];
  float2 kp, vp;

  // bf16: where in a block lane and wave of the first of STEPS pieces of keys, of values, begin to read
  __device__ __forceinline__ static int key_source() {
    const int tid = thread(), byte = (tid >> 6) * (STEPS * 1024) + (tid & 63) * 16, row = byte / ROWB;
    return row * ROWB + ((byte % ROWB / 16 ^ exchange(row)) << 4);
  }
  __device__ __forceinline__ static int value_source() {
    const int tid = thread(), byte = (tid >> 6) * (STEPS * 1024) + (tid & 63) * 16, row = byte / 128;
    return kHalf + row * 128 + ((byte % 128 / 16 ^ (row & 7)) << 4);
  }
  // what the exchange adds to the source of the i-th piece of keys: a KiB further on the row's number has other bits, without a carry
  __device__ __forceinline__ static constexpr int key_turn(int i) { return exchange(1024 / ROWB * i) << 4; }
  // quantised: asks for keys and for values
  __device__ __forceinline__ void ask_keys(const char* block) {
    const int tid = thread();
    const char* from = block + tid * (KW * 4);
    if (tid < 256) {
      if constexpr (KW % 4 == 0) {
#pragma unroll
        for (int j = 0; j < KW; j += 4) *reinterpret_cast<u32x4*>(&k[j]) = *reinterpret_cast<const u32x4*>(from + 4 * j);
      } else {
        *reinterpret_cast<u32x2*>(&k[0]) = *reinterpret_cast<const u32x2*>(from);
      }
    }
    kp = reinterpret_cast<const float2*>(block + 2 * kHalf)[tid & 63];
  }
  __device__ __forceinline__ void ask_values(const char* block) {
    const int tid = thread();
#pragma unroll
    for (int i = 0; i < VP; ++i) {
      if (piece(tid, i) < VROWS * 4) v[i] = *reinterpret_cast<const u32x4*>(block + kHalf + piece(tid, i) * 16);
    }
    vp = reinterpret_cast<const float2*>(block + 2 * kHalf)[kBlockTokens + (tid & 63)];
  }

  // Keys into buffer `at`.  `there`: tokens of the block that exist; c: factor of the exponentials.
  __device__ __forceinline__ void put_keys(Shared& sh, int at, int there, float c) const {
    const int tid = thread(), token = tid >> 2, g = tid & 3;
    if (tid < 64) sh.par[at][tid] = tid < there ? make_float2(kp.x * c, kp.y * c) : make_float2(0.f, 0.f);
    if (tid < 256) {
#pragma unroll
      for (int w = 0; w < HD / 32; ++w) {
        bf16x8 out;
        if constexpr (KV == kKvU4) out = spread_nibbles(k[w]);
        else out = spread_bytes(k[2 * w], k[2 * w + 1]);
        *reinterpret_cast<bf16x8*>(sh.keys[at] + token * ROWB + (((4 * w + g) ^ exchange(token)) << 4)) = out;
      }
    }
  }
  // The largest value of token `lane`; 0 of one that does not exist or has a value that is not finite (bad).
  __device__ __forceinline__ float largest_value(int lane, int there, bool& bad) const {
    constexpr float top = KV == kKvU4 ? 15.f : 255.f;
    const float vs = lane < there ? vp.x : 0.f, vb = lane < there ? vp.y : 0.f, most = fmaxf(fabsf(vb), fabsf(fmaf(top, vs, vb)));
    bad = !(most <= kHuge) || vs != vs;
    return bad ? 0.f : most;
  }
  __device__ __forceinline__ static int power_of(float most) { return min((int)(__float_as_uint(most) >> 23), 252); }
  // Looks at the sizes of the values that were asked for: returns the exponent (biased by 126) that they are to be scaled down by.  each: every token by one of
  // its own (0 is returned), as asked for, or because a token's is more than 2^6 below the largest.
  __device__ __forceinline__ int look(int there, bool& each) const {
    bool bad;
    const float most = largest_value(thread() & 63, there, bad);
    const int mine = power_of(most), v_exp = wave_max(mine);
    each = each || __any(most > 0.f && mine + 6 < v_exp);
    return each ? 0 : v_exp;
  }
  // Values, expanded, into buffer `at`, scaled as `look` has found; odd: the tokens whose values are not finite (as 0).
  __device__ __forceinline__ void put_values(Shared& sh, int at, int there, int v_exp, bool each, unsigned long long& odd) const {
    const int tid = thread(), lane = tid & 63, wave = uniform(tid >> 6);
    constexpr float centre = KV == kKvU4 ? 8.f : 128.f;
    bool bad;
    const float most = largest_value(lane, there, bad);
    odd = __ballot(bad);
    const float vs = bad || lane >= there ? 0.f : vp.x, vb = bad || lane >= there ? 0.f : vp.y;
    if (each) {
      v_exp = power_of(most);
      if (wave == 0) sh.power[at][lane] = (float)v_exp;
    }
    const float f = __uint_as_float((unsigned)(253 - v_exp) << 23);
    sh.expand[wave][0][lane] = (_Float16)(vs * f);
    sh.expand[wave][1][lane] = (_Float16)(fmaf(centre, vs, vb) * f);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const f16x2 bias = {(_Float16)(-1024.f - centre), (_Float16)(-1024.f - centre)};  // (1024 + c - 1024 - centre: exact)
    auto half2 = [](uint32_t x) { return __builtin_bit_cast(f16x2, x); };
#pragma unroll
    for (int i = 0; i < VP; ++i) {
      const int row = piece(tid, i) >> 2, g = piece(tid, i) & 3;
      if (piece(tid, i) >= VROWS * 4) break;
      const u32x4* s4 = reinterpret_cast<const u32x4*>(&sh.expand[wave][0][16 * g]);
      const u32x4* b4 = reinterpret_cast<const u32x4*>(&sh.expand[wave][1][16 * g]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // 8 tokens
        const u32x4 s8 = s4[h], b8 = b4[h];
#pragma unroll
        for (int n = 0; n < (KV == kKvU4 ? 2 : 1); ++n) {
          u32x4 out;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t x = v[i][2 * h + (j >> 1)];
            if constexpr (KV == kKvU4) x = (n ? x >> 4 : x) & 0x0f0f0f0fu;
            x = __builtin_amdgcn_perm(0x64646464u, x, j & 1 ? 0x07030702u : 0x07010700u);  // two bytes as fp16 1024 + c
            out[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(half2(x) + bias, half2(s8[j]), half2(b8[j])));
          }
          const int f = KV == kKvU4 ? (row >> 4) * 32 + 16 * n + (row & 15) : row;
          *reinterpret_cast<u32x4*>(sh.values[at] + f * 128 + (((2 * g + h) ^ (f & 7)) << 4)) = out;
        }
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
};

// N products in order, `product(n, operand)`, each with an operand from LDS, `read(n)`, that is asked for kAhead products earlier: left to itself
// the compiler waits for every read in front of its product.  beside(n): other work, done while the matrix cores are at it.
template <int N, class Read, class Product, class Beside>
__device__ __forceinline__ void pipelined(Read read, Product product, Beside beside) {
  constexpr int kAhead = 3;
  decltype(read(0)) ring[kAhead];
#pragma unroll
  for (int n = 0; n < kAhead; ++n) ring[n] = read(n);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    product(n, ring[n % kAhead]);
    if (n + kAhead < N) ring[n % kAhead] = read(n + kAhead);
    beside(n);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Two neighbours of p in fp16, to nearest (2^-11 of each at most): cut off, the sums would be 2^-12 or so too small beside that of p itself.
__device__ __forceinline__ void put_pair(f16x8& f, int at, float a, float b) {
  const f16x2 both = __builtin_convertvector((f32x2){a, b}, f16x2);
  f[at] = both[0];
  f[at + 1] = both[1];
}
__device__ __forceinline__ void put_pair(bf16x8&, int, float, float) {}

// A workgroup's tile of keys.
struct TileState {
  int64_t block;  // offset of its block in the cache; some block where there is none
  int there;      // tokens of it that exist
  int base;       // the sequence's first token in it; negative: of the prefix
};

// PREFIX: the rows of all tokens over the prefix alone, split over its tiles, to prefix_part; else the list.
template <int KV, int HD, int WAVES, bool PREFIX>
__global__ __launch_bounds__(64 * WAVES, HD == 256 && WAVES == 4 ? 1 : 2) void attend_tiles_kernel(TileArgs t) {
  constexpr int R = 32 * WAVES, TD = HD / 32, KS = HD / 16;
  constexpr bool Q16 = KV != kKvBf16;  // quantised: p and the values in fp16
  constexpr int kUp = Q16 ? 7 : 0;     // p enters times 2^kUp: at most 2^15
  using frag = std::conditional_t<Q16, f16x8, bf16x8>;
  using Loader = TileLoader<KV, HD, WAVES>;
  using Shared = typename Loader::Shared;
  extern __shared__ __align__(16) char lds[];
  Shared& sh = *reinterpret_cast<Shared*>(lds);
  constexpr float kNone = -__builtin_inff();
  const AttendArgs& a = t.a;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), r = lane & 31, h = lane >> 5, heads = a.cache.n_heads;
  const int page_blocks = a.cache.log2_page - 6, prefix_tiles = (int)(((unsigned)t.prefix_len + 63) >> 6);
  const float c = a.scale * 1.44269504f;

  int me, begin, end, per = 0, one = 0;
  if constexpr (PREFIX) {
    me = blockIdx.x;
    begin = 0;
    end = 1;
  } else {
    me = (blockIdx.x & 7) * (t.workers >> 3) + (blockIdx.x >> 3);
    one = t.list[t.entries].x;
    per = piece_length(one * heads, t.workers);
    begin = me * per;
    end = min(begin + per, one * heads);
  }
  int4 cut = {0, 0, 0, 0};
  int entry = -1;

  for (int u = begin; u < end;) {
    int head, tiles, first, last, row_tile, split = 0, units = 0, in = 0;
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
      in = u - head * one;
      // the entry that place `in` of a head's list is in: looked for once, then the next ones in turn
      if (entry < 0) {
        int lo = 0, hi = t.entries - 1;
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (t.list[mid].x <= in) lo = mid;
          else hi = mid - 1;
        }
        entry = uniform(lo);
      }
      int4 item = t.list[entry];
      while (item.x + item.w <= in) item = t.list[++entry];
      entry = uniform(entry);
      const int s = uniform(item.y), at = uniform(item.x), all = uniform(item.w);
      row_tile = uniform(item.z);
      q = sequence_of(a, s);
      pages = a.pages + s * a.ldp;
      tiles = all - kSegmentCost;
      units = min(all - (in - at), end - u);
      first = max(0, in - at - kSegmentCost);
      last = max(0, in - at + units - kSegmentCost);
      if (first >= last) {  // nothing but the cost
        u += units;
        if (in + units == one) entry = 0;
        continue;
      }
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

    f32x16 o[TD];
#pragma unroll
    for (int i = 0; i < TD; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m = kNone, l = 0.f;  // m: in bits (times c)
    int v_run = 0, v_exp = 0;  // exponents of O (of this lane's row), of the values at hand
    bool each = false;         // these have one a token
    unsigned long long odd = 0ull;
    Loader ld;

    // Offsets of 64 tiles' blocks, one a lane, looked up together; those of tiles without a block are negative.
    int64_t window = -1;
    int window_from = first, window_end = first;
    const int64_t head_at = kv_block_offset<KV, HD>(a.cache, 0, head, 0), page_bytes = kv_block_offset<KV, HD>(a.cache, 1, 0, 0);
    auto state_of = [&](int tile) {
      if (tile >= window_end) {
        window_from = tile;
        window_end = tile + 64;
        const int at = tile + lane;
        const bool own = at >= prefix_tiles;
        const int k = own ? at - prefix_tiles : at;
        window = -1;
        if (at < last && k * 64 < (own ? q.len : t.prefix_len)) {
          const int page = (own ? pages : t.prefix_pages)[k >> page_blocks];
          if (page >= 0 && page < a.cache.n_pages)
            window = head_at + page * page_bytes + (k & ((1 << page_blocks) - 1)) * (int64_t)kv_block_bytes<KV, HD>();
        }
      }
      TileState x;
      const int hi = __builtin_amdgcn_readlane((int)(window >> 32), tile - window_from);
      x.block = (int64_t)hi << 32 | (uint32_t)__builtin_amdgcn_readlane((int)window, tile - window_from);
      const int k = tile - prefix_tiles;
      x.base = k >= 0 ? k * 64 : -1;
      x.there = min((k >= 0 ? q.len : t.prefix_len) - (k >= 0 ? k : tile) * 64, 64);
      if (hi < 0) x.there = 0, x.block = 0;
      return x;
    };
    auto masked_of = [&](const TileState& x) { return x.there < 64 || (x.base >= 0 && x.base + 64 > all_see); };
    auto seen_of = [&](const TileState& x) { return x.base >= 0 ? min(max(sees - x.base, 0), x.there) : x.there; };
    // operands in LDS: the exchange puts n into bits of the address that only an exclusive or reaches.  Where a lane reads is worked out anew for
    // each half tile: kept in registers, it would push others out to memory, and a wait for those is one for the copies under way
    auto key_place = [&] {
      const int l = Loader::thread() & 63, k = (l & 0x13) | (l & 4) << 1 | (l & 8) >> 1;
      return k * Loader::ROWB + (((l >> 5) ^ Loader::exchange(k)) << 4);
    };
    auto value_place = [&] {
      const int l = Loader::thread() & 63;
      return (l & 31) * 128 + (((l >> 5) ^ (l & 7)) << 4);
    };
    auto key_operand = [&](int place, int at, int n) {  // (keys 32 further on have the same low bits)
      return *reinterpret_cast<const bf16x8*>(sh.keys[at] + (place ^ (n >> 1) << 5) + (n & 1) * (32 * Loader::ROWB));
    };
    auto value_operand = [&](int place, int at, int n) {  // (features too)
      return *reinterpret_cast<const frag*>(sh.values[at] + (place ^ (n / TD) << 5) + n % TD * (32 * 128));
    };
    auto clear = [&](f32x16(&x)[2]) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[k][e] = KV == kKvU4 ? -128.f * qsum : 0.f;  // (codes of 4 bits enter as 128 + c)
    };
    // scores 2 i, 2 i + 1, in bits, from products
    auto finish_scores = [&](f32x16(&x)[2], int at, int i) {
      const int k = i >> 3, e = 2 * (i & 7);
      if constexpr (Q16) {
        const float4 p = *reinterpret_cast<const float4*>(&sh.par[at][32 * k + 16 * (e >> 3) + 8 * h + (e & 7)]);
        x[k][e] = fmaf(x[k][e], p.x, p.y * qsum);
        x[k][e + 1] = fmaf(x[k][e + 1], p.z, p.w * qsum);
      } else {
        x[k][e] *= c;
        x[k][e + 1] *= c;
      }
    };
    auto mask = [&](f32x16(&x)[2], int seen) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (32 * k + 16 * (e >> 3) + 8 * h + (e & 7) >= seen) x[k][e] = kNone;
    };
    auto largest = [&](const f32x16(&x)[2]) {
      float most = fmaxf(x[0][0], x[1][0]);
#pragma unroll
      for (int e = 1; e < 16; ++e) most = fmaxf(most, fmaxf(x[0][e], x[1][e]));
      return most;
    };

    // bf16: the i-th of 2 STEPS pieces that a wave copies of a tile, keys first
    const int copy_at = uniform(wave * Loader::STEPS * 1024);
    auto copy = [&](int64_t block, int at, int i) {
      const bool key = i < Loader::STEPS;
      const int j = key ? i : i - Loader::STEPS, from = key ? Loader::key_source() ^ Loader::key_turn(j) : Loader::value_source();
      to_lds_16(from + 1024 * j, a.cache.data + block, uniform((int)(uintptr_t)(key ? sh.keys[at] : sh.values[at]) + copy_at + 1024 * j));
    };
    // bf16: in a tile that not all rows see all of, what a wave has copied of the values (arrived, in buffer `at`) is gone through: 0 NaN = NaN, so what
    // is not finite goes in as 0 (and is noted), and so does what lies behind the last token
    auto clean = [&](const TileState& x, int at) {
      unsigned long long which = 0ull;
#pragma unroll
      for (int i = 0; i < Loader::STEPS; ++i) {
        const int piece = (copy_at + 1024 * i) / 16 + lane, chunk = (piece & 7) ^ (piece >> 3 & 7);
        u32x4* from = reinterpret_cast<u32x4*>(sh.values[at]) + piece;
        u32x4 d = *from;
#pragma unroll
        for (int w = 0; w < 4; ++w) d[w] = only_finite(d[w], 8 * chunk + 2 * w, x.there, which);
        *from = d;
      }
      const unsigned long long all = any_lane(which);
      if (lane == 0) sh.odd[at][wave] = all;
    };

    TileState now = state_of(first);
    __syncthreads();  // the buffers are free (the last segment's tiles were read)
    if constexpr (Q16) {
      ld.ask_keys(a.cache.data + now.block);
      ld.ask_values(a.cache.data + now.block);
      ld.put_keys(sh, 0, now.there, c);
      each = masked_of(now);
      v_exp = ld.look(now.there, each);
      ld.put_values(sh, 0, now.there, v_exp, each, odd);
    } else {
#pragma unroll
      for (int i = 0; i < 2 * Loader::STEPS; ++i) copy(now.block, 0, i);
    }
    // queries arrived before the loop: a wait for them in it would wait for the tiles that are on their way to LDS as well
#pragma unroll
    for (int w = 0; w < KS; ++w) asm volatile("" : "+v"(qf[w]));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (!Q16 && masked_of(now)) clean(now, 0);
    __syncthreads();

    for (int tile = first; tile < last; ++tile) {
      const int at = tile - first & 1;
      const TileState next = state_of(tile + 1);
      if constexpr (Q16) {
        ld.ask_keys(a.cache.data + next.block);
        ld.ask_values(a.cache.data + next.block);
      }
      [[maybe_unused]] int v_next = 0;
      [[maybe_unused]] bool each_next = false;
      f32x16 x[2];
      clear(x);
      {
        const int place = key_place();
        pipelined<2 * KS>([&](int n) { return key_operand(place, at, n); }, [&](int n, bf16x8 f) { x[n & 1] = mfma32(f, qf[n >> 1], x[n & 1]); },
                          [&](int n) {
                            if constexpr (!Q16) {
                              constexpr int EVERY = KS / Loader::STEPS;
                              if (n % EVERY == 0) copy(next.block, at ^ 1, n / EVERY);
                            } else if (n == 2 * KS - 5) {  // (the chunk: 290 us four products from the end, 280 five, 282 six, 285 eight)
                              each_next = masked_of(next);
                              v_next = ld.look(next.there, each_next);
                            }
                          });
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) finish_scores(x, at, i);
      if (masked_of(now)) mask(x, seen_of(now));
      float most = largest(x);
      auto of_halves = [](float v) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
      };
      most = of_halves(most);
      int shift = 0;
      if constexpr (Q16) {
        // O is held relative to 2^(m + v_run), the largest p |v| of the row so far, so that a large value of little weight takes no bits off the
        // others; both parts of it are raised by the row's own scores alone.
        // (In differences of scores throughout: a large score added to an exponent would swallow it.)
        const float up = most - m;  // not a number where nothing has been seen yet
        float size = (float)v_exp, alone = 0.f;
        if (each) {  // p alone for its sum, and with the token's exponent
          const float* power = &sh.power[at][8 * h];
          const float base = most == kNone ? 0.f : most;
          size = kNone;
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float s = x[i >> 4][i & 15] - base, with = s + power[32 * (i >> 4) + 16 * (i >> 3 & 1) + (i & 7)];
            alone += __builtin_amdgcn_exp2f(s);
            size = fmaxf(size, with);
            x[i >> 4][i & 15] = with;
          }
          size = of_halves(size);
        }
        const bool higher = up > 8.f, raise = higher || size + up > (float)v_run + 8.f;
        if (__any(raise)) {
          const int run = max(v_run - (higher ? (int)fminf(up, 1024.f) : 0), (int)ceilf(fmaxf(higher ? size : size + up, -1024.f)));
          const float shrink = raise ? __builtin_amdgcn_exp2f((float)(v_run - run) - (higher ? up : 0.f)) : 1.f;
          l *= higher ? __builtin_amdgcn_exp2f(-up) : 1.f;
#pragma unroll
          for (int i = 0; i < TD; ++i) o[i] *= shrink;
          if (higher) m = most;
          if (raise) v_run = run;
        }
        shift = max(v_exp - v_run, each ? -1000 : -60);  // (p is nothing in fp16 from 2^-60 on)
        if (each) l += alone * (m == kNone ? 1.f : __builtin_amdgcn_exp2f(most - m + (float)kUp));
      } else if (__any(most > m + 8.f)) {
        const bool raise = most > m + 8.f;  // (of a row by its own scores alone)
        const float shrink = raise ? __builtin_amdgcn_exp2f(m - most) : 1.f;
        l *= shrink;
#pragma unroll
        for (int i = 0; i < TD; ++i) o[i] *= shrink;
        if (raise) m = most;
      }
      const float mb = (m == kNone ? 0.f : Q16 && each ? m - most : m) - (float)(shift + kUp);
      frag pf[4];
      float sum[2] = {0.f, 0.f}, even = 0.f;
      auto exponential = [&](int i) {
        const int k = i >> 4, e = i & 15;
        const float v = __builtin_amdgcn_exp2f(x[k][e] - mb);
        sum[e & 1] += v;
        if constexpr (!Q16) pf[2 * k + (e >> 3)][e & 7] = (bf16)v;
        else if (e & 1) put_pair(pf[2 * k + (e >> 3)], e & 6, even, v);
        else even = v;
      };
#pragma unroll
      for (int i = 0; i < 8; ++i) exponential(i);
      {
        const int place = value_place();
        pipelined<4 * TD>([&](int n) { return value_operand(place, at, n); }, [&](int n, frag f) { o[n % TD] = mfma32(f, pf[n / TD], o[n % TD]); },
                          [&](int n) {  // for the next sixteen keys
                            if (n < 3 * TD) {
#pragma unroll
                              for (int i = 8 + 8 * n / TD; i < 8 + 8 * (n + 1) / TD; ++i) exponential(i);
                            }
                          });
      }
      const float all = sum[0] + sum[1];
      if constexpr (!Q16) l += all;
      else if (!each) l += ldexpf(all, -shift);
      if constexpr (!Q16) {
        odd = 0ull;
        if (masked_of(now)) {
#pragma unroll
          for (int w = 0; w < WAVES; ++w) odd |= sh.odd[at][w];
          odd = (unsigned long long)(uint32_t)uniform((int)(odd >> 32)) << 32 | (uint32_t)uniform((int)odd);
        }
      }
      if (odd) {
        const int seen = seen_of(now);
        const unsigned long long mine = seen >= 64 ? ~0ull : (1ull << seen) - 1;
        if constexpr (Q16) {
          const float add = odd & mine ? __builtin_nanf("") : 0.f;
#pragma unroll
          for (int i = 0; i < TD; ++i) o[i] += add;
        } else {
          const bf16* v = reinterpret_cast<const bf16*>(a.cache.data + now.block + Loader::kHalf) + 4 * h * kBlockTokens;
#pragma unroll 1
          for (; odd; odd &= odd - 1) {
            const int j = __builtin_ctzll(odd);
#pragma unroll
            for (int i = 0; i < TD; ++i)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float w = (float)v[(32 * i + (e & 3) + 8 * (e >> 2)) * kBlockTokens + j];
                if (j < seen && !(fabsf(w) <= kHuge)) o[i][e] += w;
              }
          }
        }
      }
      if constexpr (Q16) {
        ld.put_keys(sh, at ^ 1, next.there, c);
        each = each_next;
        v_exp = v_next;
        ld.put_values(sh, at ^ 1, next.there, v_exp, each, odd);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      if (!Q16 && masked_of(next)) clean(next, at ^ 1);
      __syncthreads();
      now = next;
    }

    l += __shfl_xor(l, 32);
    if constexpr (Q16) {
      const int over = max(v_run - 200, 0);  // so that sums of the largest values stay in range
      m += (float)over;
      l = ldexpf(l, -kUp - over);
#pragma unroll
      for (int i = 0; i < TD; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = ldexpf(o[i][e], v_run - 126 - kUp - over);
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
    if (first == 0 && !whole) cut = int4{entry, head, (int)((unsigned)(u + (tiles - first) + (units - (last - first)) - 1) / (unsigned)per) - me + 1, 0};
    u += units;
    if (in + units == one) entry = 0;
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
  const int4 entry = t.list[cut.x];
  const Sequence q = sequence_of(a, entry.y);
  const int r = blockIdx.y * (256 / TR) + threadIdx.x / TR, lane4 = 4 * (threadIdx.x % TR);
  const int64_t row = (int64_t)entry.z * R + r;
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
  if (token < q.first || token >= q.first + q.count || r >= a.row_tiles * kRows) return;
  const int total = a.tiles[a.n_seq] * a.cache.n_heads, per = piece_length(total, a.workers);
  const int tiles = key_tiles(q), start = a.tiles[s] * a.cache.n_heads + (head * row_tiles(a, q) + r / kRows) * tiles;
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
      const int64_t slot = (2 * (int64_t)w + (w == w0 ? 1 : 0)) * kRows + r % kRows;
      j.add(ml[slot], *reinterpret_cast<const f32x4*>(a.part + slot * HD + lane4));
    }
  }
  j.store(a, token, qh, HD, lane4);
}

}  // namespace kt
