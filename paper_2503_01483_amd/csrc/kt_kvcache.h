// kt_kvcache.h -- the paged key / value cache: where its bytes lie, and writing and reading single tokens.
//
// A page holds page_size tokens of every key / value head, [page][head][page_size / 64] blocks.  A block is 64 tokens of one head in
// one piece of memory: keys by token, values by FEATURE, then {step, minimum} of each key and of each value (not in bf16).  Both halves
// are in the order in which the attention kernels multiply them: the 16 bytes that a lane of a matrix instruction takes are
// neighbours, so that a wave reads a block with plain 16-byte loads straight into operands, without LDS and without a transpose.  The
// price is paid once per token when it is written (bytes 64 or 128 apart), not each time it is read.
//   keys, feature 32 w + 8 g + e (w step of a product over the features, g lane quarter, e < 8):
//     bf16  as they come
//     u8    byte g (hd / 4) + 8 w + e
//     u4    dword g (hd / 32) + w, nibble e / 2 for even e, 4 + e / 2 for odd e: (dword >> 4 i) & 0x000f000f is elements 2 i, 2 i + 1
//   values: row of 64 tokens per feature; u4: features f and f + 16 of every 32 share a row, f in the low nibbles
// A byte belongs to one token in every format, so that tokens can be written side by side without reading.
#pragma once
#include "kt_serve_util.h"

namespace kt {

constexpr int kBlockTokens = 64;
enum { kKvBf16 = 0, kKvU8 = 1, kKvU4 = 2 };

template <int KV>
__host__ __device__ constexpr int kv_bits() { return KV == kKvBf16 ? 16 : KV == kKvU8 ? 8 : 4; }
// bytes of a block's keys (its values take as many), and of the block
template <int KV, int HD>
__host__ __device__ constexpr int kv_half_bytes() { return kBlockTokens * HD * kv_bits<KV>() / 8; }
template <int KV, int HD>
__host__ __device__ constexpr int kv_block_bytes() { return 2 * kv_half_bytes<KV, HD>() + (KV == kKvBf16 ? 0 : 2 * kBlockTokens * 8); }

struct KvCache {
  char* data;
  int64_t n_pages;
  int n_heads, log2_page;  // tokens of a page: 2^log2_page >= 64
};

template <int KV, int HD>
__device__ __forceinline__ int64_t kv_block_offset(const KvCache& c, int64_t page, int head, int block) {
  return (((page * c.n_heads + head) << (c.log2_page - 6)) + block) * (int64_t)kv_block_bytes<KV, HD>();
}

struct AppendArgs {
  KvCache cache;
  const void *q, *k, *v;
  void* q_out;
  int64_t ldq, ldk, ldv, ldqo;
  const int64_t* slots;
  const int* positions;
  const float* rope;  // [n_pos][rot]: cosines, then sines
  int64_t n_pos;
  int n, hq, rot;
  int chunks;  // workgroups of a token's queries and keys
  bool interleaved, hadamard;
};

// Value of lane `lane ^ O`, on the vector ALU for distances up to 8 (a row of 16 lanes), where every lane is in use.
template <int O>
__device__ __forceinline__ float lane_xor(float x) {
  const int v = __float_as_int(x);
  if constexpr (O == 1) return __int_as_float(__builtin_amdgcn_mov_dpp(v, 0xb1, 0xf, 0xf, true));        // quad_perm 1 0 3 2
  else if constexpr (O == 2) return __int_as_float(__builtin_amdgcn_mov_dpp(v, 0x4e, 0xf, 0xf, true));   // quad_perm 2 3 0 1
  else if constexpr (O == 4)                                                                             // 7 - lane, then 3 - lane
    return __int_as_float(__builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true));
  else if constexpr (O == 8) return __int_as_float(__builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true));  // row_ror 8
  else return __shfl_xor(x, O);
}

// Position rotation of the first `rot` of a row's 8 LPR features, 8 of which this lane holds (l-th lane of the row).
// fp32, one rounding an operation.
template <int LPR>
__device__ __forceinline__ void rotate_position(float (&y)[8], const float* row, int rot, bool interleaved, int l) {
#pragma clang fp contract(off)
  const int half = rot / 2, lanes = rot / 16;  // lanes of each half
  if (interleaved) {
    if (8 * l >= rot) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float c = row[4 * l + i], s = row[half + 4 * l + i], a = y[2 * i], b = y[2 * i + 1];
      y[2 * i] = a * c - b * s;
      y[2 * i + 1] = b * c + a * s;
    }
    return;
  }
  const bool second = l >= lanes;
  float z[8];
  if (rot == 8 * LPR) {
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = lane_xor<LPR / 2>(y[e]);
  } else {
    const int other = (threadIdx.x & 63) + (l >= 2 * lanes ? 0 : second ? -lanes : lanes);
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], other);
  }
  if (l >= 2 * lanes) return;
  const int at = 8 * (second ? l - lanes : l);
  float c[8], s[8];
  load8(row + at, c);
  load8(row + half + at, s);
  const float sign = second ? 1.f : -1.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = y[e] * c[e], r = z[e] * s[e];
    y[e] = fmaf(r, sign, p);  // p + r or p - r: the product is exact
  }
}

// H / sqrt(8 LPR) on the row, butterflies by distances 1, 2, 4, ...; fp32, one rounding an operation.  Across lanes the second of a pair takes
// y - p for p - y, which makes a step one instruction on its neighbour's value; the sign (of the parity of the lane's number) is put right at the end.
// (Assembly: the compiler makes it a move, a wait and a multiply-add.  A value that the vector ALU has written, or its mask of lanes, may be read across
// lanes two and five instructions later.)
// One step: y += sign * (y of the neighbour at distance S).
template <int S>
__device__ __forceinline__ void add_neighbours(float (&y)[8], float sign) {
#define KT_EIGHT(how)                                                                                                        \
  asm volatile("s_nop 4\n\tv_fmac_f32_dpp %0, %0, %8 " how "\n\tv_fmac_f32_dpp %1, %1, %8 " how "\n\tv_fmac_f32_dpp %2, %2, %8 " how      \
      "\n\tv_fmac_f32_dpp %3, %3, %8 " how "\n\tv_fmac_f32_dpp %4, %4, %8 " how "\n\tv_fmac_f32_dpp %5, %5, %8 " how              \
      "\n\tv_fmac_f32_dpp %6, %6, %8 " how "\n\tv_fmac_f32_dpp %7, %7, %8 " how                                                \
      : "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]), "+v"(y[4]), "+v"(y[5]), "+v"(y[6]), "+v"(y[7])                       \
      : "v"(sign))
  if constexpr (S == 1) KT_EIGHT("quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf");
  else if constexpr (S == 2) KT_EIGHT("quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf");
  else if constexpr (S == 8) KT_EIGHT("row_ror:8 row_mask:0xf bank_mask:0xf");
  else
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fmaf(lane_xor<S>(y[e]), sign, y[e]);
#undef KT_EIGHT
}
template <int LPR, int S>
__device__ __forceinline__ void butterfly(float (&y)[8], int l) {
  if constexpr (S < LPR) {
    const float sign = l & S ? -1.f : 1.f;  // (a product with it is exact)
    add_neighbours<S>(y, sign);
    butterfly<LPR, 2 * S>(y, l);
  }
}
template <int LPR>
__device__ __forceinline__ void rotate_hadamard(float (&y)[8], int l) {
#pragma clang fp contract(off)
#pragma unroll
  for (int s = 1; s < 8; s *= 2)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!(e & s)) {
        const float a = y[e], b = y[e + s];
        y[e] = a + b;
        y[e + s] = a - b;
      }
  butterfly<LPR, 1>(y, l);
  constexpr float root = LPR == 8 ? 0.125f : LPR == 16 ? 0.08838834764831845f : 0.0625f;
  const float norm = __popc(l) & 1 ? -root : root;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= norm;
}

template <int LPR, int S, class F>
__device__ __forceinline__ float row_reduce(float v, F f) {
  if constexpr (S < LPR) return row_reduce<LPR, 2 * S>(f(v, lane_xor<S>(v)), f);
  else return v;
}

// Codes and {step, minimum} of the row (LPR lanes of 8 values); a row with a value that is not finite gets NaN for both and codes 0.
// A code is the quotient ((y - min) top) / width, rounded to fp32, rounded half to even.  A product with the reciprocal is within 2^-14 of it, so that
// only one that near to the middle of two codes is divided (of 512 values about one in ten waves has one; ties of bf16 inputs are common).
template <int LPR>
__device__ __forceinline__ void quantise_row(const float (&y)[8], float top, uint32_t (&code)[8], float& step, float& low) {
#pragma clang fp contract(off)
  float lo = y[0], hi = y[0], bad = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) lo = fminf(lo, y[e]), hi = fmaxf(hi, y[e]), bad += y[e] * 0.f;
  lo = row_reduce<LPR, 1>(lo, [](float a, float b) { return fminf(a, b); });
  hi = row_reduce<LPR, 1>(hi, [](float a, float b) { return fmaxf(a, b); });
  const int shift = threadIdx.x & 63 & ~(LPR - 1);
  const bool all_finite = (__ballot(!(bad == 0.f)) >> shift & ((1ull << LPR) - 1)) == 0ull;
  const float width = hi - lo;
  step = width / top;
  low = lo;
  if (step < kTiny) step = 0.f;
  const bool finite = all_finite && width * top <= kHuge, some = finite && step > 0.f;
  const float inv = 1.f / width;  // (finite where step > 0)
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float num = (y[e] - lo) * top;
    float q = num * inv, n = rintf(q);
    if (__any(some && fabsf(q - n) > 0.4999f)) n = rintf(num / width);
    code[e] = some ? (uint32_t)n : 0u;
  }
  if (!finite) step = low = __builtin_nanf("");
}

// Where token `slot` of a head lies: its block and number in it; null if the cache has no such slot.
template <int KV, int HD>
__device__ __forceinline__ char* place_of(const KvCache& c, int64_t slot, int head, int& tok) {
  const int64_t page = slot >> c.log2_page;
  if (slot < 0 || page >= c.n_pages) return nullptr;
  const int in_page = (int)(slot & ((1ll << c.log2_page) - 1));
  tok = in_page & 63;
  return c.data + kv_block_offset<KV, HD>(c, page, head, in_page >> 6);
}

// HD / 8 lanes a row of 8 values each.  The first n * chunks workgroups take the queries and keys of a token: rotated, then to q_out or into
// their pages.  The others take the values of one head and of as many tokens as the workgroup has rows: these cross over to rows by feature in LDS,
// so that the bytes of neighbouring slots are written together.
// 8192 tokens of 32 + 2 x 8 heads of 128, rotated twice, to 4 bits: 71 us, 2.6 TB/s, bound by the vector ALU (issuing 98 % of the cycles; the
// 182 MB alone would take 38); 64 tokens 5.1 us; 1537 of heads of 64, to 8 bits, 10 us.  A row takes HD / 8 lanes, so that a lane's loads are 16 bytes and the
// exchanges of both rotations stay within a row of 16 lanes (vector ALU, no LDS) up to 128 features.
template <typename T, int KV, int HD>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  constexpr int LPR = HD / 8, ROWS = 256 / LPR, HALF = kv_half_bytes<KV, HD>();
  constexpr float top = KV == kKvU8 ? 255.f : 15.f;
  const int l = threadIdx.x % LPR, in_wg = threadIdx.x / LPR, w = l >> 2, g = l & 3, hkv = a.cache.n_heads;
  const int64_t rotated = (int64_t)a.n * a.chunks;
  float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  int tok = 0;
  if (blockIdx.x < rotated) {
    const int token = blockIdx.x / (unsigned)a.chunks, r = (blockIdx.x - token * a.chunks) * ROWS + in_wg;
    const bool is_q = r < a.hq, live = r < a.hq + hkv;  // (lanes behind the last row stay for the exchanges and write nothing)
    const int head = is_q ? r : r - a.hq;
    // (asked for together with slot and position, whatever these say)
    if (live) load8(static_cast<const T*>(is_q ? a.q : a.k) + token * (is_q ? a.ldq : a.ldk) + head * HD + 8 * l, y);
    const int64_t slot = a.slots[token];
    const int pos = a.rope ? a.positions[token] : 0;
    // a token without a slot or position of its own is passed over
    if (!place_of<KV, HD>(a.cache, slot, 0, tok) || (a.rope && (pos < 0 || pos >= a.n_pos))) return;
    if (a.rope) rotate_position<LPR>(y, a.rope + pos * (int64_t)a.rot, a.rot, a.interleaved, l);
    if (a.hadamard) rotate_hadamard<LPR>(y, l);
    [[maybe_unused]] uint32_t code[8];
    [[maybe_unused]] float step, low;
    if constexpr (KV != kKvBf16) {
      if (r - in_wg + ROWS > a.hq) quantise_row<LPR>(y, top, code, step, low);  // (a workgroup with keys)
    }
    if (!live) return;
    if (is_q) {
      store8(static_cast<T*>(a.q_out) + token * a.ldqo + head * HD + 8 * l, y);
      return;
    }
    char* block = place_of<KV, HD>(a.cache, slot, head, tok);
    if constexpr (KV == kKvBf16) {
      store8(reinterpret_cast<bf16*>(block) + tok * HD + 8 * l, y);
    } else {
      if constexpr (KV == kKvU8) {
        const u32x2 t = {code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24, code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24};
        *reinterpret_cast<u32x2*>(block + tok * HD + g * (HD / 4) + 8 * w) = t;
      } else {
        const uint32_t t = code[0] | code[2] << 4 | code[4] << 8 | code[6] << 12 | code[1] << 16 | code[3] << 20 | code[5] << 24 | code[7] << 28;
        *reinterpret_cast<uint32_t*>(block + tok * (HD / 2) + (g * (HD / 32) + w) * 4) = t;
      }
      if (l == 0) reinterpret_cast<float2*>(block + 2 * HALF)[tok] = make_float2(step, low);
    }
    return;
  }
  // ---- values
  constexpr int BYTES = KV == kKvBf16 ? 2 : 1, FEATURES = KV == kKvU4 ? HD / 2 : HD;  // of a token's entry in a row, rows
  __shared__ __align__(16) char turned[FEATURES][ROWS * BYTES + (ROWS * BYTES < 16 ? 0 : 4)];
  __shared__ int64_t slots[ROWS];
  const int64_t index = blockIdx.x - rotated;
  const int group = (int)(index / hkv), head = (int)(index - (int64_t)group * hkv);
  const int64_t token = (int64_t)group * ROWS + in_wg;
  if (token < a.n) load8(static_cast<const T*>(a.v) + token * a.ldv + head * HD + 8 * l, y);
  const int64_t slot = token < a.n ? a.slots[token] : -1;
  const int pos = a.rope && token < a.n ? a.positions[token] : 0;
  char* block = place_of<KV, HD>(a.cache, slot, head, tok);
  const bool live = block && (!a.rope || (pos >= 0 && pos < a.n_pos));
  if (l == 0) slots[in_wg] = live ? slot : -1;
  if constexpr (KV == kKvBf16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) reinterpret_cast<bf16*>(turned[8 * l + e])[in_wg] = (bf16)y[e];
  } else {
    uint32_t code[8];
    float step, low;
    quantise_row<LPR>(y, top, code, step, low);
    if constexpr (KV == kKvU8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) turned[8 * l + e][in_wg] = (char)code[e];
    } else {  // (the lanes of the first 16 of 32 features write both nibbles)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t other = (uint32_t)__float_as_int(lane_xor<2>(__int_as_float((int)code[e])));
        if (g < 2) turned[16 * w + 8 * g + e][in_wg] = (char)(code[e] | other << 4);
      }
    }
    if (live && l == 0) reinterpret_cast<float2*>(block + 2 * HALF)[kBlockTokens + tok] = make_float2(step, low);
  }
  __syncthreads();
  // eight entries of a feature at a time: together where their slots are neighbours in a block and the first is a multiple of eight
  constexpr int RUN = 8;
  static_assert(ROWS % RUN == 0);
  for (int i = threadIdx.x; i < FEATURES * (ROWS / RUN); i += 256) {
    const int f = i / (ROWS / RUN), first = i % (ROWS / RUN) * RUN;
    bool run = slots[first] >= 0 && (slots[first] & (RUN - 1)) == 0;
#pragma unroll
    for (int k = 1; k < RUN; ++k) run = run && slots[first + k] == slots[first] + k;
    if (run) {
      char* to = place_of<KV, HD>(a.cache, slots[first], head, tok) + HALF + (f * kBlockTokens + tok) * BYTES;
#pragma unroll
      for (int k = 0; k < 2 * BYTES; ++k) reinterpret_cast<uint32_t*>(to)[k] = *reinterpret_cast<const uint32_t*>(&turned[f][first * BYTES + 4 * k]);
    } else {
#pragma unroll
      for (int k = 0; k < RUN; ++k) {
        char* to = place_of<KV, HD>(a.cache, slots[first + k], head, tok);
        if (!to) continue;
        to += HALF + (f * kBlockTokens + tok) * BYTES;
        if constexpr (BYTES == 2) *reinterpret_cast<uint16_t*>(to) = *reinterpret_cast<const uint16_t*>(&turned[f][(first + k) * 2]);
        else *to = turned[f][first + k];
      }
    }
  }
}

struct GatherArgs {
  KvCache cache;
  const int64_t* slots;
  void *k, *v;
  int64_t ldk, ldv;
  int n, chunks;  // workgroups of a token's keys (0: no keys)
};

// Keys and values of single slots as values: the same workgroups the other way round.  Bound by waits: 8192 tokens of 8 heads of 128, 4 bits, 18.7 us
// (43 MB, most of it written: 2.3 TB/s, half of a copy's), the vector ALU 54 % of the cycles; rows of values are read 8 bytes at a time.  64 tokens 4.7.
template <typename T, int KV, int HD>
__global__ __launch_bounds__(256) void kv_gather_kernel(GatherArgs a) {
#pragma clang fp contract(off)
  constexpr int LPR = HD / 8, ROWS = 256 / LPR, HALF = kv_half_bytes<KV, HD>();
  const int l = threadIdx.x % LPR, in_wg = threadIdx.x / LPR, w = l >> 2, g = l & 3, hkv = a.cache.n_heads;
  const int64_t with_keys = (int64_t)a.n * a.chunks;
  float y[8];
  int tok = 0;
  if (blockIdx.x < with_keys) {
    const int token = blockIdx.x / (unsigned)a.chunks, head = (blockIdx.x - token * a.chunks) * ROWS + in_wg;
    const char* block = head < hkv ? place_of<KV, HD>(a.cache, a.slots[token], head, tok) : nullptr;
    if (!block) return;
    if constexpr (KV == kKvBf16) {
      load8(reinterpret_cast<const bf16*>(block) + tok * HD + 8 * l, y);
    } else {
      const float2 p = reinterpret_cast<const float2*>(block + 2 * HALF)[tok];
      if constexpr (KV == kKvU8) {
        const u32x2 t = *reinterpret_cast<const u32x2*>(block + tok * HD + g * (HD / 4) + 8 * w);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (float)(t[e / 4] >> (8 * (e & 3)) & 0xffu) * p.x + p.y;
      } else {
        const uint32_t t = *reinterpret_cast<const uint32_t*>(block + tok * (HD / 2) + (g * (HD / 32) + w) * 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (float)(t >> (4 * (e / 2 + 4 * (e & 1))) & 15u) * p.x + p.y;
      }
    }
    store8(static_cast<T*>(a.k) + token * a.ldk + head * HD + 8 * l, y);
    return;
  }
  // ---- values
  constexpr int BYTES = KV == kKvBf16 ? 2 : 1, FEATURES = KV == kKvU4 ? HD / 2 : HD, RUN = 8;
  __shared__ __align__(16) char turned[FEATURES][ROWS * BYTES + (ROWS * BYTES < 16 ? 0 : 4)];
  __shared__ int64_t slots[ROWS];
  const int64_t index = blockIdx.x - with_keys;
  const int group = (int)(index / hkv), head = (int)(index - (int64_t)group * hkv);
  const int64_t token = (int64_t)group * ROWS + in_wg;
  if (l == 0) slots[in_wg] = token < a.n ? a.slots[token] : -1;
  __syncthreads();
  for (int i = threadIdx.x; i < FEATURES * (ROWS / RUN); i += 256) {
    const int f = i / (ROWS / RUN), first = i % (ROWS / RUN) * RUN;
    bool run = (slots[first] & (RUN - 1)) == 0;
#pragma unroll
    for (int k = 1; k < RUN; ++k) run = run && slots[first + k] == slots[first] + k;
    if (run) {
      const char* from = place_of<KV, HD>(a.cache, slots[first], head, tok);
      if (!from) continue;
      from += HALF + (f * kBlockTokens + tok) * BYTES;
#pragma unroll
      for (int k = 0; k < 2 * BYTES; ++k) *reinterpret_cast<uint32_t*>(&turned[f][first * BYTES + 4 * k]) = reinterpret_cast<const uint32_t*>(from)[k];
    } else {
#pragma unroll
      for (int k = 0; k < RUN; ++k) {
        const char* from = place_of<KV, HD>(a.cache, slots[first + k], head, tok);
        if (!from) continue;
        from += HALF + (f * kBlockTokens + tok) * BYTES;
        if constexpr (BYTES == 2) *reinterpret_cast<uint16_t*>(&turned[f][(first + k) * 2]) = *reinterpret_cast<const uint16_t*>(from);
        else turned[f][first + k] = *from;
      }
    }
  }
  __syncthreads();
  const char* block = place_of<KV, HD>(a.cache, slots[in_wg], head, tok);
  if (!block) return;
  if constexpr (KV == kKvBf16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (float)reinterpret_cast<const bf16*>(turned[8 * l + e])[in_wg];
  } else {
    const float2 p = reinterpret_cast<const float2*>(block + 2 * HALF)[kBlockTokens + tok];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t c = (uint8_t)turned[KV == kKvU8 ? 8 * l + e : 16 * w + 8 * (g & 1) + e][in_wg];
      y[e] = (float)(KV == kKvU8 ? c : c >> (g & 2 ? 4 : 0) & 15u) * p.x + p.y;
    }
  }
  store8(static_cast<T*>(a.v) + token * a.ldv + head * HD + 8 * l, y);
}

}  // namespace kt
