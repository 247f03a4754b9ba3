// kt_norm.h -- residual addition, RMS norm and per-token codes of token rows.
//
//   h = x + res,  u = h gain,  y = u rstd with rstd = 1 / sqrt(mean h^2 + eps)
// The codes of y with the step clip max|y| / L are those of u with the step t = clip max|u| / L: rstd cancels, so both statistics
// of a row, sum h^2 and max |u|, come from one pass over registers, and the codes do not depend on how the sum is rounded.
// A row stays in the registers of its threads, so that memory is read and written once: HBM-bound.  16384 rows of 4096, bf16, residual in
// and out, 4-bit codes as values: 99 us, 5.4 TB/s.  Small calls are bound by the launch: one row of 2048 takes 3.0 us, 193 of 4096 4.8.
// The arithmetic of the codes is part of the interface (fp32, one rounding an operation): contraction is off.
#pragma once
#include "kt_serve_util.h"

namespace kt {

enum { kFormatNone = 0, kFormatInt4 = 1, kFormatInt8 = 2, kFormatE4M3 = 3 };

struct NormArgs {
  const void *x, *res, *gain;
  void *res_out, *y;
  uint8_t* codes;
  float* scales;
  int64_t ldx, ldres, ldro, ldy, ldc;
  int n, d;
  float eps, clip, qmax;
};

// Sum and maximum over the TPR threads of a row.  The magnitudes are compared as bit patterns, which puts a NaN above everything.
template <int TPR>
__device__ __forceinline__ void row_sum_max(float& sum, uint32_t& most, float (*sh)[2]) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    sum += __shfl_xor(sum, o);
    most = max(most, (uint32_t)__shfl_xor((int)most, o));
  }
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6][0] = sum, sh[threadIdx.x >> 6][1] = __uint_as_float(most);
    __syncthreads();
    sum = sh[0][0];
    most = __float_as_uint(sh[0][1]);
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w) sum += sh[w][0], most = max(most, __float_as_uint(sh[w][1]));
  }
}

// TPR threads a row, CH chunks of 8 values a thread (8 TPR CH >= d), 256 or TPR threads a workgroup.
template <typename T, typename TG, int FORMAT, int TPR, int CH>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void add_rmsnorm_quant_kernel(NormArgs a) {
#pragma clang fp contract(off)
  constexpr int ROWS = TPR >= 256 ? 1 : 256 / TPR;
  __shared__ float sh[TPR / 64][2];
  const int lane = threadIdx.x % TPR;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + threadIdx.x / TPR;
  if (row >= a.n) return;  // (a whole wave; rows that share a workgroup need no barrier)
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* res = a.res ? static_cast<const T*>(a.res) + row * a.ldres : nullptr;
  const TG* gain = static_cast<const TG*>(a.gain);
  float u[CH][8];
  float sum = 0.f;
  uint32_t top = 0u;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = 8 * (lane + TPR * c);
    if (at < a.d) {
      load8(x + at, u[c]);
      if (res) {
        float r[8];
        load8(res + at, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[c][e] += r[e];
      }
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = 8 * (lane + TPR * c);
    if (at < a.d) {
      if (a.res_out) store8(static_cast<T*>(a.res_out) + row * a.ldro + at, u[c]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(u[c][e], u[c][e], sum);
      if (gain) {
        float g[8];
        load8(gain + at, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[c][e] *= g[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(u[c][e]) & 0x7fffffffu);
    }
  }
  row_sum_max<TPR>(sum, top, sh);
  const float most = __uint_as_float(top);
  const float rstd = 1.f / sqrtf(sum / (float)a.d + a.eps);
  const float t = (a.clip * most) / a.qmax;
  const bool finite = sum <= kHuge && most <= kHuge;  // false for NaN as well
  float r = 0.f, scale = 0.f;
  if (t >= kTiny) r = 1.f / t, scale = t * rstd;
  if (!finite) scale = __builtin_nanf("");
  if constexpr (FORMAT == kFormatNone) scale = sum <= kHuge ? rstd : __builtin_nanf("");  // (1 / inf would pass for a row of zeros)
  if (FORMAT != kFormatNone && a.scales && lane == 0) a.scales[row] = scale;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = 8 * (lane + TPR * c);
    if (at >= a.d) continue;
    if constexpr (FORMAT == kFormatNone) {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[c][e] *= scale;
    } else {
      uint32_t code[2] = {0u, 0u};
#pragma unroll
      for (int e = 0; e < 8; ++e) u[c][e] = finite ? fminf(fmaxf(u[c][e] * r, -a.qmax), a.qmax) : 0.f;
      if constexpr (FORMAT == kFormatE4M3) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          code[w] = __builtin_amdgcn_cvt_pk_fp8_f32(u[c][4 * w], u[c][4 * w + 1], 0, false);
          code[w] = __builtin_amdgcn_cvt_pk_fp8_f32(u[c][4 * w + 2], u[c][4 * w + 3], code[w], true);
          u[c][4 * w] = __builtin_amdgcn_cvt_f32_fp8(code[w], 0);
          u[c][4 * w + 1] = __builtin_amdgcn_cvt_f32_fp8(code[w], 1);
          u[c][4 * w + 2] = __builtin_amdgcn_cvt_f32_fp8(code[w], 2);
          u[c][4 * w + 3] = __builtin_amdgcn_cvt_f32_fp8(code[w], 3);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[c][e] = rintf(u[c][e]);
          code[e / 4] |= ((uint32_t)(int)u[c][e] & 0xffu) << (8 * (e & 3));
        }
      }
      if (a.codes) *reinterpret_cast<u32x2*>(a.codes + row * a.ldc + at) = u32x2{code[0], code[1]};
#pragma unroll
      for (int e = 0; e < 8; ++e) u[c][e] *= scale;
    }
    if (a.y) store8(static_cast<T*>(a.y) + row * a.ldy + at, u[c]);
  }
}

}  // namespace kt
