// Shared by the linears with 4-bit weights: activations as scaled fp16 terms, codes as fp16, the epilogue.
#pragma once

#include "kernels.h"
#include "kv4.cuh"

namespace chimera {

// 2^(14 - floor(log2 top)) for the bits of a largest magnitude (1 when it is 0 or not finite).
__device__ __forceinline__ float token_scale(uint32_t top) {
  const int e = static_cast<int>(top >> 23 & 255u);
  const int k = e == 0 || e == 255 ? 127 : min(268 - e, 253);
  return __uint_as_float(static_cast<uint32_t>(k) << 23);
}

// Eight activations of one token from column k.
__device__ __forceinline__ void load8(const W4Params& p, int m, int k, float (&x)[8]) {
  const size_t at = static_cast<size_t>(m) * p.ldx + k;
  if (p.x_f32) {
    const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(p.X) + at);
    *reinterpret_cast<float4*>(x) = src[0];
    *reinterpret_cast<float4*>(x + 4) = src[1];
    return;
  }
  uint4 u = *reinterpret_cast<const uint4*>(static_cast<const bf16*>(p.X) + at);
  const uint32_t h[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(h[i] << 16);
    x[2 * i + 1] = __uint_as_float(h[i] & 0xffff0000u);
  }
  if (p.X_lo) {
    u = *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(p.X_lo) + at);
    const uint32_t l[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] += __uint_as_float(l[i] << 16);
      x[2 * i + 1] += __uint_as_float(l[i] & 0xffff0000u);
    }
  }
}

__device__ __forceinline__ uint32_t top_bits(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  return top;
}

// The eight codes of a word less their zero, exact in fp16, paired as by nibbles_f16; off is
// 1024 + zero and off16 -(64 + zero), each twice.
__device__ __forceinline__ void w4_codes_f16(uint32_t w, uint32_t off, uint32_t off16, uint32_t (&r)[4]) {
  const __half2 sixteenth = __halves2half2(__ushort_as_half(0x2c00), __ushort_as_half(0x2c00));
  uint32_t u[4];
  nibbles_f16(w, u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __half2 x = *reinterpret_cast<__half2*>(&u[i]);
    x = (i & 1) ? __hfma2(x, sixteenth, *reinterpret_cast<__half2*>(&off16)) : __hsub2(x, *reinterpret_cast<__half2*>(&off));
    r[i] = *reinterpret_cast<uint32_t*>(&x);
  }
}
__device__ __forceinline__ uint32_t zero_off(uint32_t z) { return 0x64006400u + z * 0x00010001u; }
__device__ __forceinline__ uint32_t zero_off16(uint32_t z) { return 0xd400d400u + z * 0x00100010u; }

__device__ __forceinline__ void store_y(const W4Params& p, int m, int n, float y) {
  const size_t at = static_cast<size_t>(m) * p.ldy + n;
  if (p.epi == EPI_RESID) {
    static_cast<float*>(p.Y)[at] += y;
    return;
  }
  if (p.epi == EPI_SILU) y = silu_f(y);
  if (p.out_f32)
    static_cast<float*>(p.Y)[at] = y;
  else
    static_cast<bf16*>(p.Y)[at] = __float2bfloat16_rn(y);
}

}  // namespace chimera
