// Linear with 4-bit weights: Y[M][N] (epilogue)= X[M][K] . W^T with
// W[n][k] = scale[n][k / group] (code[n][k] - zero[n][k / group]), codes 0..15.
//
// code - zero is a whole number of at most 4 bits and a sign, exact in bf16, so a group's
// products with bf16 activations are exact and are summed in fp32 by the matrix units;
// the group's scale multiplies the sum, in fp32.  fp32 activations enter as three bf16 terms
// (24 bits), hi + lo ones as their two.
//
// The weights are the A operand (16 features) straight from the packed words: thread
// (r, t) of a warp takes the word of 8 codes at t of a 32-code block of features r and r + 8, and
// the activations are staged in shared memory in the order in which the nibbles come out.  Eight
// warps share 16 features, each with every eighth block of K, and their sums are added
// in the order of the warps.
#include "kernels.h"
#include "kv4.cuh"
#include "launch.cuh"

namespace chimera {
namespace {

constexpr int WARPS = 8, FEATURES = 16;
constexpr int KC = 1024;                // K per staged chunk
constexpr int XROW = KC * 2 + 64;       // bytes of a token's chunk: 64 past a multiple of 128 keeps the
                                        // reads of two tokens in different banks

// The eight codes of a word less the zero, exact in bf16: pairs of nibbles (0,4) .. (3,7).
// 0x4300 | c is 128 + c; off holds 128 + zero twice.
__device__ __forceinline__ void w4_codes(uint32_t w, __nv_bfloat162 off, uint32_t (&r)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t u = (w >> (4 * i) & 0x000f000fu) | 0x43004300u;
    __nv_bfloat162 x = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&u), off);
    r[i] = *reinterpret_cast<uint32_t*>(&x);
  }
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&x);
}

// TT tiles of 8 tokens, TERMS bf16 terms per activation (1, 2: X and X_lo; 3: fp32 X).
template <int TT, int TERMS>
__global__ void __launch_bounds__(WARPS * 32) w4_kernel(const __grid_constant__ W4Params p) {
  extern __shared__ __align__(128) unsigned char smem[];  // [TERMS][8 TT][XROW], later the warps' sums
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, r = lane / 4, t = lane & 3;
  pdl_wait();
  pdl_trigger();
  const int n0 = blockIdx.x * FEATURES, m0 = blockIdx.y * 8 * TT;
  const int groups = (p.K + p.group - 1) / p.group;
  const int na = min(n0 + r, p.N - 1), nb = min(n0 + r + 8, p.N - 1);
  const unsigned char* wa = p.W + static_cast<size_t>(na) * (p.K / 2) + 4 * t;
  const unsigned char* wb = p.W + static_cast<size_t>(nb) * (p.K / 2) + 4 * t;
  const bf16* scale = reinterpret_cast<const bf16*>(p.scale);
  float acc[TT][4] = {};
  for (int k0 = 0; k0 < p.K; k0 += KC) {
    const int kc = min(KC, p.K - k0);
    __syncthreads();
    for (int i = tid; i < 8 * TT * (kc / 8); i += WARPS * 32) {
      const int col = i / (kc / 8), at = i % (kc / 8), m = m0 + col;
      uint4 v[TERMS];
#pragma unroll
      for (int s = 0; s < TERMS; ++s) v[s] = make_uint4(0, 0, 0, 0);
      if (m < p.M) {
        const size_t x0 = static_cast<size_t>(m) * p.ldx + k0 + 8 * at;
        if (TERMS == 3) {
          float x[8];
          const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(p.X) + x0);
          *reinterpret_cast<float4*>(x) = src[0];
          *reinterpret_cast<float4*>(x + 4) = src[1];
#pragma unroll
          for (int s = 0; s < TERMS; ++s) {
            uint32_t* u = reinterpret_cast<uint32_t*>(&v[s]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              u[j] = pack_bf16(x[j], x[j + 4]);
              x[j] -= __uint_as_float(u[j] << 16);
              x[j + 4] -= __uint_as_float(u[j] & 0xffff0000u);
            }
          }
        } else {
#pragma unroll
          for (int s = 0; s < TERMS; ++s) {
            const uint4 w = *reinterpret_cast<const uint4*>((s ? reinterpret_cast<const bf16*>(p.X_lo) : static_cast<const bf16*>(p.X)) + x0);
            v[s] = make_uint4(__byte_perm(w.x, w.z, 0x5410), __byte_perm(w.x, w.z, 0x7632), __byte_perm(w.y, w.w, 0x5410),
                              __byte_perm(w.y, w.w, 0x7632));
          }
        }
      }
#pragma unroll
      for (int s = 0; s < TERMS; ++s) *reinterpret_cast<uint4*>(smem + (s * 8 * TT + col) * XROW + at * 16) = v[s];
    }
    __syncthreads();
    for (int kb = warp; kb < kc / 32; kb += WARPS) {
      const int k = k0 + kb * 32, gi = k / p.group;
      const uint32_t a = *reinterpret_cast<const uint32_t*>(wa + k / 2), b = *reinterpret_cast<const uint32_t*>(wb + k / 2);
      const size_t ga = static_cast<size_t>(na) * groups + gi, gb = static_cast<size_t>(nb) * groups + gi;
      const float sa = __bfloat162float(scale[ga]), sb = __bfloat162float(scale[gb]);
      const float za = p.zero ? p.zero[ga] : 8.f, zb = p.zero ? p.zero[gb] : 8.f;
      uint32_t ua[4], ub[4];
      w4_codes(a, __float2bfloat162_rn(128.f + za), ua);
      w4_codes(b, __float2bfloat162_rn(128.f + zb), ub);
#pragma unroll
      for (int i = 0; i < TT; ++i) {
        float d[4] = {};
#pragma unroll
        for (int s = 0; s < TERMS; ++s) {
          const uint4 x = *reinterpret_cast<const uint4*>(smem + (s * 8 * TT + 8 * i + r) * XROW + kb * 64 + t * 16);
          mma_bf16(d, ua[0], ub[0], ua[1], ub[1], x.x, x.y);
          mma_bf16(d, ua[2], ub[2], ua[3], ub[3], x.z, x.w);
        }
        acc[i][0] = fmaf(sa, d[0], acc[i][0]);
        acc[i][1] = fmaf(sa, d[1], acc[i][1]);
        acc[i][2] = fmaf(sb, d[2], acc[i][2]);
        acc[i][3] = fmaf(sb, d[3], acc[i][3]);
      }
    }
  }
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);  // [warp][token][16 features]
#pragma unroll
  for (int i = 0; i < TT; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[(warp * 8 * TT + 8 * i + 2 * t + (j & 1)) * FEATURES + r + 8 * (j >> 1)] = acc[i][j];
  }
  __syncthreads();
  for (int i = tid; i < 8 * TT * FEATURES; i += WARPS * 32) {
    const int m = m0 + i / FEATURES, n = n0 + i % FEATURES;
    if (m >= p.M || n >= p.N) continue;
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) y += sums[w * 8 * TT * FEATURES + i];
    const size_t at = static_cast<size_t>(m) * p.ldy + n;
    if (p.epi == EPI_RESID) {
      static_cast<float*>(p.Y)[at] += y;
      continue;
    }
    if (p.epi == EPI_SILU) y = silu_f(y);
    if (p.out_f32)
      static_cast<float*>(p.Y)[at] = y;
    else
      static_cast<bf16*>(p.Y)[at] = __float2bfloat16_rn(y);
  }
}

template <int TT, int TERMS>
cudaError_t launch(const W4Params& p, cudaStream_t s) {
  const int x = TERMS * 8 * TT * XROW, sums = WARPS * 8 * TT * FEATURES * 4;
  const int smem = x > sums ? x : sums;
  const cudaError_t e = cudaFuncSetAttribute(w4_kernel<TT, TERMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const dim3 grid((p.N + FEATURES - 1) / FEATURES, (p.M + 8 * TT - 1) / (8 * TT));
  return launch_pdl(w4_kernel<TT, TERMS>, grid, dim3(WARPS * 32), smem, s, p);
}

template <int TT>
cudaError_t launch_terms(const W4Params& p, cudaStream_t s) {
  return p.x_f32 ? launch<TT, 3>(p, s) : p.X_lo ? launch<TT, 2>(p, s) : launch<TT, 1>(p, s);
}

}  // namespace

cudaError_t linear_w4(const W4Params& p, cudaStream_t s) {
  return p.M <= 8 ? launch_terms<1>(p, s) : p.M <= 16 ? launch_terms<2>(p, s) : launch_terms<3>(p, s);
}

}  // namespace chimera
