// The 4-bit KV cache: layout of a page, 4-bit codes as fp16, and fp16 matrix products.
//
// A row (one position of one kv head) of head_dim values is held as 4-bit codes with a step
// and a base of its own, x = base + step * code:
//   base = bf16(min x), step = bf16((max x - min x) fp32(1 / 15)), code = clamp(rint((x - base) / step), 0, 15)
// (a row of equal values has step 0 and codes 0; a row with a value that is not finite, a range past
// fp32's or a minimum past bf16's is kept as base NaN, step 0).  One step per row and head, not one per group of channels: then
//   q . k      = step (q . code) + base (sum of q)
//   sum p_j v_j = sum (p_j step_j) code_j + sum p_j base_j
// and the codes enter the matrix products as whole numbers, exact in fp16, with no arithmetic
// per value but their conversion.
//
// Pool: [blocks][kv heads][page], a page holds 16 rows in 16 head_dim + 128 contiguous bytes (one
// bulk copy):
//   K codes  [16 rows][head_dim / 8 words], channel 8 w + i at bits 4 i of word w
//   V codes  [8 row pairs][8 chunks][head_dim / 32 words]: word w of the chunk of channels
//            [C g, C g + C), C = head_dim / 8, holds channels C g + 4 w + i of row 2 pair at bits 4 i and of
//            row 2 pair + 1 at bits 16 + 4 i (the two rows that share a register of the second
//            matrix product); chunk g sits at place g ^ swizzle(pair), so that the eight
//            lanes of a shared-memory wavefront read different banks
//   K steps and bases [16 x (step bf16, base bf16)], V steps and bases
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace chimera {

constexpr int KV4_ROWS = 16;

template <int HD>
struct Kv4 {
  static constexpr int ROW = HD / 2;            // bytes of a row's codes
  static constexpr int CHUNK = HD / 8;          // bytes of a chunk of V, and its channels
  static constexpr int V = KV4_ROWS * ROW;      // offsets in the page
  static constexpr int KS = 2 * KV4_ROWS * ROW;
  static constexpr int VS = KS + 4 * KV4_ROWS;
  static constexpr int BYTES = VS + 4 * KV4_ROWS;
  __host__ __device__ static constexpr int place(int pair, int g) {
    return g ^ (HD == 128 ? 2 * (pair & 3) : 4 * ((pair >> 1) & 1));
  }
  // Offset of the halfword with channels 4 w4 .. 4 w4 + 3 of a V row.
  __host__ __device__ static constexpr int v_half(int row, int w4) {
    const int pair = row >> 1, per = CHUNK / 4;
    return V + pair * 2 * ROW + place(pair, w4 / per) * CHUNK + (w4 % per) * 4 + (row & 1) * 2;
  }
};

inline int kv4_page_bytes(int hd) { return KV4_ROWS * hd + 128; }

// (step, base) of a row, packed as two bf16.
__device__ __forceinline__ float kv4_step(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float kv4_base(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// (x & mask) | bits in one instruction (the compiler makes two of it when both are constants).
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "r"(mask), "r"(bits));
  return r;
}
// The nibbles of a word as fp16 pairs (0,4), (1,5), (2,6), (3,7): 1024 + c in pairs 0 and 2, 1024 + 16 c in
// 1 and 3 (ten bits of mantissa hold a nibble at either place).  The method, whole numbers put into the mantissa of a
// power of two, is published in Kim, Henry, Fahim and Awadalla, "Who Says Elephants Can't Run: Bringing Large Scale
// MoE Models into Cloud Scale Production" (2022).
__device__ __forceinline__ void nibbles_f16(uint32_t w, uint32_t (&u)[4]) {
  const uint32_t h = w >> 8;
  u[0] = and_or(w, 0x000f000fu, 0x64006400u);
  u[1] = and_or(w, 0x00f000f0u, 0x64006400u);
  u[2] = and_or(h, 0x000f000fu, 0x64006400u);
  u[3] = and_or(h, 0x00f000f0u, 0x64006400u);
}

// The eight codes of a word less 8, exact in fp16, paired as above.
__device__ __forceinline__ void kv4_codes(uint32_t w, uint32_t (&r)[4]) {
  const __half2 off = __halves2half2(__ushort_as_half(0x6408), __ushort_as_half(0x6408));    // 1032
  const __half2 sixteenth = __halves2half2(__ushort_as_half(0x2c00), __ushort_as_half(0x2c00));
  const __half2 off16 = __halves2half2(__ushort_as_half(0xd480), __ushort_as_half(0xd480));  // -72
  uint32_t u[4];
  nibbles_f16(w, u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __half2 x = *reinterpret_cast<__half2*>(&u[i]);
    x = (i & 1) ? __hfma2(x, sixteenth, off16) : __hsub2(x, off);
    r[i] = *reinterpret_cast<uint32_t*>(&x);
  }
}

// d += A B: 16 x 16 by 16 x 8, fp16 in, fp32 sums.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same with d = A B.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                              uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Two fp32 values as a pair of fp16 and the pair of what that rounding left.
__device__ __forceinline__ void split_f16(float x, float y, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(x, y);
  const float2 f = __half22float2(h);
  const __half2 l = __floats2half2_rn(x - f.x, y - f.y);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  lo = *reinterpret_cast<const uint32_t*>(&l);
}

// Untiled bulk copy of a multiple of 16 bytes into shared memory (both sides 16-byte aligned).
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

}  // namespace chimera
