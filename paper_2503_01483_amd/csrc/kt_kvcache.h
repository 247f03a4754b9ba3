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
  bool interleaved, hadamard;
};

// Value of lane `lane ^ O` (O < 8 LPR; rows of lanes lie next to each other).
template <int O>
__device__ __forceinline__ float lane_xor(float x) { return __shfl_xor(x, O); }

// Position rotation of the first `rot` of a row's features, 8 of which this lane holds (l-th lane of the row).
// fp32, one rounding an operation.
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
  const int other = (threadIdx.x & 63) + (l >= 2 * lanes ? 0 : second ? -lanes : lanes);
  float z[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], other);
  if (l >= 2 * lanes) return;
  const int at = 8 * (second ? l - lanes : l);
  float c[8], s[8];
  load8(row + at, c);
  load8(row + half + at, s);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = y[e] * c[e], r = z[e] * s[e];
    y[e] = second ? p + r : p - r;
  }
}

// H / sqrt(8 LPR) on the row, butterflies by distances 1, 2, 4, ...; fp32, one rounding an operation.
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
#pragma unroll
  for (int s = 1; s < LPR; s *= 2)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __shfl_xor(y[e], s);
      y[e] = l & s ? p - y[e] : y[e] + p;
    }
  constexpr float norm = LPR == 8 ? 0.125f : LPR == 16 ? 0.08838834764831845f : 0.0625f;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] *= norm;
}

// Codes and {step, minimum} of the row (LPR lanes of 8 values); a row with a value that is not finite gets NaN for both and codes 0.
template <int LPR>
__device__ __forceinline__ void quantise_row(const float (&y)[8], float top, uint32_t (&code)[8], float& step, float& low) {
#pragma clang fp contract(off)
  float lo = y[0], hi = y[0], bad = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) lo = fminf(lo, y[e]), hi = fmaxf(hi, y[e]), bad += y[e] * 0.f;
#pragma unroll
  for (int s = 1; s < LPR; s *= 2) {
    lo = fminf(lo, __shfl_xor(lo, s));
    hi = fmaxf(hi, __shfl_xor(hi, s));
    bad += __shfl_xor(bad, s);
  }
  const float width = hi - lo;
  step = width / top;
  low = lo;
  if (step < kTiny) step = 0.f;
  const bool finite = bad == 0.f && width * top <= kHuge;
#pragma unroll
  for (int e = 0; e < 8; ++e) code[e] = finite && step > 0.f ? (uint32_t)rintf(((y[e] - lo) * top) / width) : 0u;
  if (!finite) step = low = __builtin_nanf("");
}

// One row of queries, keys or values by LPR = HD / 8 lanes of 8 values each: rotated, then to q_out or into its page.
template <typename T, int KV, int HD>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  constexpr int LPR = HD / 8, ROWS = 256 / LPR, HALF = kv_half_bytes<KV, HD>();
  const int l = threadIdx.x % LPR, hkv = a.cache.n_heads, rows = a.hq + 2 * hkv;
  const int64_t index = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR;
  const int64_t token = index / rows;
  const int r = (int)(index - token * rows);
  // a token without a slot or position of its own is passed over: its lanes stay for the exchanges and write nothing
  const int64_t slot = token < a.n ? a.slots[token] : -1;
  const int pos = a.rope && token < a.n ? a.positions[token] : 0;
  const bool live = slot >= 0 && slot >> a.cache.log2_page < a.cache.n_pages && (!a.rope || (pos >= 0 && pos < a.n_pos));
  const bool is_q = r < a.hq, is_k = !is_q && r < a.hq + hkv;
  const int head = is_q ? r : is_k ? r - a.hq : r - a.hq - hkv;
  const T* from = static_cast<const T*>(is_q ? a.q : is_k ? a.k : a.v);
  float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (live) load8(from + token * (is_q ? a.ldq : is_k ? a.ldk : a.ldv) + head * HD + 8 * l, y);
  {
    float z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = y[e];
    if (a.rope) rotate_position(z, a.rope + (live ? pos : 0) * (int64_t)a.rot, a.rot, a.interleaved, l);
    if (a.hadamard) rotate_hadamard<LPR>(z, l);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = is_q || is_k ? z[e] : y[e];
  }
  uint32_t code[8];
  float step = 0.f, low = 0.f;
  if constexpr (KV != kKvBf16) quantise_row<LPR>(y, KV == kKvU8 ? 255.f : 15.f, code, step, low);
  [[maybe_unused]] uint32_t other[8];
  if constexpr (KV == kKvU4) {
#pragma unroll
    for (int e = 0; e < 8; ++e) other[e] = (uint32_t)__shfl_xor((int)code[e], 2);
  }
  if (!live) return;
  if (is_q) {
    store8(static_cast<T*>(a.q_out) + token * a.ldqo + head * HD + 8 * l, y);
    return;
  }
  const int64_t page = slot >> a.cache.log2_page;
  const int in_page = (int)(slot & ((1ll << a.cache.log2_page) - 1)), tok = in_page & 63;
  char* block = a.cache.data + kv_block_offset<KV, HD>(a.cache, page, head, in_page >> 6);
  const int w = l >> 2, g = l & 3;
  if constexpr (KV == kKvBf16) {
    if (is_k) {
      store8(reinterpret_cast<bf16*>(block) + tok * HD + 8 * l, y);
    } else {
      bf16* v = reinterpret_cast<bf16*>(block + HALF) + tok;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[(8 * l + e) * kBlockTokens] = (bf16)y[e];
    }
  } else {
    if (is_k) {
      if constexpr (KV == kKvU8) {
        const u32x2 t = {code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24, code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24};
        *reinterpret_cast<u32x2*>(block + tok * HD + g * (HD / 4) + 8 * w) = t;
      } else {
        const uint32_t t = code[0] | code[2] << 4 | code[4] << 8 | code[6] << 12 | code[1] << 16 | code[3] << 20 | code[5] << 24 | code[7] << 28;
        *reinterpret_cast<uint32_t*>(block + tok * (HD / 2) + (g * (HD / 32) + w) * 4) = t;
      }
    } else {
      uint8_t* v = reinterpret_cast<uint8_t*>(block + HALF) + tok;
      if constexpr (KV == kKvU8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[(8 * l + e) * kBlockTokens] = (uint8_t)code[e];
      } else if (g < 2) {  // (the lanes of the first 16 of 32 features write both nibbles)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[(16 * w + 8 * g + e) * kBlockTokens] = (uint8_t)(code[e] | other[e] << 4);
      }
    }
    if (l == 0) reinterpret_cast<float2*>(block + 2 * HALF)[(is_k ? 0 : kBlockTokens) + tok] = make_float2(step, low);
  }
}

struct GatherArgs {
  KvCache cache;
  const int64_t* slots;
  void *k, *v;
  int64_t ldk, ldv;
  int n;
};

// Keys and values of single slots as values; a row of one head by HD / 8 lanes.
template <typename T, int KV, int HD>
__global__ __launch_bounds__(256) void kv_gather_kernel(GatherArgs a) {
#pragma clang fp contract(off)
  constexpr int LPR = HD / 8, ROWS = 256 / LPR, HALF = kv_half_bytes<KV, HD>();
  const int l = threadIdx.x % LPR, hkv = a.cache.n_heads;
  const int64_t index = (int64_t)blockIdx.x * ROWS + threadIdx.x / LPR;
  const int64_t token = index / (2 * hkv);
  if (token >= a.n) return;
  const int r = (int)(index - token * (2 * hkv));
  const bool is_k = r < hkv;
  const int head = is_k ? r : r - hkv;
  const int64_t slot = a.slots[token], page = slot >> a.cache.log2_page;
  if (slot < 0 || page >= a.cache.n_pages) return;
  if (is_k ? !a.k : !a.v) return;
  const int in_page = (int)(slot & ((1ll << a.cache.log2_page) - 1)), tok = in_page & 63;
  const char* block = a.cache.data + kv_block_offset<KV, HD>(a.cache, page, head, in_page >> 6);
  const int w = l >> 2, g = l & 3;
  float y[8];
  if constexpr (KV == kKvBf16) {
    if (is_k) {
      load8(reinterpret_cast<const bf16*>(block) + tok * HD + 8 * l, y);
    } else {
      const bf16* v = reinterpret_cast<const bf16*>(block + HALF) + tok;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (float)v[(8 * l + e) * kBlockTokens];
    }
  } else {
    uint32_t code[8];
    if (is_k) {
      if constexpr (KV == kKvU8) {
        const u32x2 t = *reinterpret_cast<const u32x2*>(block + tok * HD + g * (HD / 4) + 8 * w);
#pragma unroll
        for (int e = 0; e < 8; ++e) code[e] = t[e / 4] >> (8 * (e & 3)) & 0xffu;
      } else {
        const uint32_t t = *reinterpret_cast<const uint32_t*>(block + tok * (HD / 2) + (g * (HD / 32) + w) * 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) code[e] = t >> (4 * (e / 2 + 4 * (e & 1))) & 15u;
      }
    } else {
      const uint8_t* v = reinterpret_cast<const uint8_t*>(block + HALF) + tok;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        code[e] = KV == kKvU8 ? v[(8 * l + e) * kBlockTokens] : v[(16 * w + 8 * (g & 1) + e) * kBlockTokens] >> (g & 2 ? 4 : 0) & 15;
    }
    const float2 p = reinterpret_cast<const float2*>(block + 2 * HALF)[(is_k ? 0 : kBlockTokens) + tok];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (float)code[e] * p.x + p.y;
  }
  if (is_k) store8(static_cast<T*>(a.k) + token * a.ldk + head * HD + 8 * l, y);
  else store8(static_cast<T*>(a.v) + token * a.ldv + head * HD + 8 * l, y);
}

}  // namespace kt
