// Linear with 4-bit weights for many tokens, on the 5th-generation tensor cores.
//
//   Y[M][N] (epilogue)= sum over groups g of K: scale[n][g] (codes[n] - zero[n][g]) . X16[m],
//   X16 the activations as one or two fp16 terms scaled by a power of two per token.
//
// The weights are the MMA's A operand (M = 128 features) and come from tensor memory: a thread of the eight
// unpacking warps owns one feature, reads its codes from shared memory (TMA, 256 columns per row and
// stage), turns a group of them into fp16 whole numbers and stores them to its TMEM lane, two
// per column.  Shared memory holds only what TMA wrote, and no swizzle has to be undone.
// The products of a group go to an accumulator of their own, which the same thread reads
// back and adds to its sums in fp32, times the group's scale: the scale costs one FMA per feature, token and
// group and is never rounded into a weight, and no chain of (truncating) tensor-core sums is
// longer than a group.  A CTA takes 256 features (two A tiles share the tokens' B tile) and up to 64 tokens;
// two TMEM buffers of A and D let the MMAs of a group run while the next is unpacked.
//
// Work split: stream-K over (tile, 256 columns of K), one CTA per SM; tiles cut between CTAs
// are joined by the last to arrive, in CTA order (deterministic).
//
// Roles (384 threads): warp 0 TMA of the tokens, warp 1 the MMAs, warp 2 TMA of the weights, warps 4..11 unpack
// and sum (warp w: TMEM lanes 32 (w % 4) .., feature tile w / 4 - 1).
#include <algorithm>

#include "kernels.h"
#include "kv4.cuh"
#include "launch.cuh"
#include "linear_w4.cuh"

namespace chimera {
namespace {

constexpr int BM = 128, FEATURES = 2 * BM;
constexpr int WK = 256;                    // columns per weight stage: 128 bytes of a row
constexpr int XK = 128;                    // columns per token stage: two 128-byte atoms
constexpr int W_STAGE = FEATURES * WK / 2, W_STAGES = 3, X_STAGES = 3;
constexpr int THREADS = 384, UNPACK_WARP = 4, UNPACK = 256;
constexpr int A_COLS = 64;                 // TMEM columns of a group's codes (128 of them)
constexpr uint32_t TMEM_COLS = 512;        // A [tile][2], D [tile][2]
constexpr unsigned long long WAIT_NS = 2000000000ull;

struct ManyParams {
  CUtensorMap tmW;    // codes: [N][K / 2] bytes, box 128 x 128 bytes, 128-byte swizzle
  CUtensorMap tmX;    // X16: [terms * M][K] fp16, box TN x 64
  W4Params w;
  const float* down;  // [M]: what undoes a token's scale
  int groups, terms, kstages, tok_tiles;
  uint32_t units;     // tiles * kstages
};

// D[tmem] (+)= A[tmem] B[smem]^T, fp16 in, fp32 sums.
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
                                          uint32_t elected) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(elected)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_ld16_async(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
// The wait names the registers, so that no use of them is moved above it.
__device__ __forceinline__ void tmem_wait16(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}

__device__ __forceinline__ int cta_of_unit(uint32_t u, uint32_t U, uint32_t G) { return static_cast<int>(((u + 1) * G - 1) / U); }
__device__ __forceinline__ uint32_t unit_begin(uint32_t c, uint32_t U, uint32_t G) { return c * U / G; }

// Does any thread of the barrier say so?
__device__ __forceinline__ bool any_of(int id, int nthreads, bool pred) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred pi, po;\n\t"
      "setp.ne.u32 pi, %1, 0;\n\t"
      "bar.red.or.pred po, %2, %3, pi;\n\t"
      "selp.u32 %0, 1, 0, po;\n\t}"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(pred)), "r"(id), "r"(nthreads)
      : "memory");
  return r != 0;
}

// TN: tokens of a tile (16, 32 or 64).
size_t many_smem(int tn, int terms) { return 1024 + W_STAGES * W_STAGE + static_cast<size_t>(X_STAGES) * terms * 2 * tn * 128; }

template <int G, int TN>
__global__ void __launch_bounds__(THREADS, 1) w4_many_kernel(const __grid_constant__ ManyParams p) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t w_full[W_STAGES], w_empty[W_STAGES], x_full[X_STAGES], x_empty[X_STAGES];
  __shared__ uint64_t a_full[2][2], mma_done[2][2], drain;  // [tile][buffer]
  __shared__ uint32_t tmem_slot;
  __shared__ int s_abort, s_last, s_w_asked, s_x_asked;
  unsigned char* smem = smem_raw + (1024 - (smem_u32(smem_raw) & 1023u)) % 1024;
  unsigned char* x_smem = smem + W_STAGES * W_STAGE;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  volatile int* abort = &s_abort;
  const W4Params& w = p.w;
  if (threadIdx.x == 0) {
    for (int i = 0; i < W_STAGES; ++i) {
      mbar_init(w_full + i, 1);
      mbar_init(w_empty + i, UNPACK / 32);
    }
    for (int i = 0; i < X_STAGES; ++i) {
      mbar_init(x_full + i, 1);
      mbar_init(x_empty + i, 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(a_full[i / 2] + i % 2, BM);
      mbar_init(mma_done[i / 2] + i % 2, 1);
    }
    mbar_init(&drain, 1);
    mbar_fence_init();
    s_abort = s_w_asked = s_x_asked = 0;
  }
  if (warp == 1) tmem_alloc(&tmem_slot, TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  const uint32_t U = p.units, CTAS = gridDim.x, KS = p.kstages;
  const uint32_t u_begin = unit_begin(blockIdx.x, U, CTAS), u_end = unit_begin(blockIdx.x + 1, U, CTAS);
  constexpr int PER_X = XK / G;            // groups of a token stage
  constexpr int X_ATOM = TN * 128;         // bytes of 64 columns of the tokens' tile
  // token stages of a weight stage that starts at column k0 (the last may be short)
  auto x_stages_of = [&](int ks) { return min(WK, w.K - ks * WK) > XK ? 2 : 1; };

  if (warp == 2) {
    // ---------------- TMA of the weights ----------------
    // Every kernel before the one that wrote X16 is complete (it lets its dependents launch after its own
    // wait), so the weights may be read before this kernel's wait.
    if (lane == 0) {
      const uint64_t policy = policy_evict_first();
      bool ok = true;
      for (uint32_t u = u_begin; ok && u < u_end; ++u) {
        const int i = static_cast<int>(u - u_begin), stage = i % W_STAGES;
        if (i >= W_STAGES) ok = mbar_wait(w_empty + stage, (i / W_STAGES - 1) & 1, abort, WAIT_NS);
        if (!ok) break;
        const int row = static_cast<int>(u / KS) / p.tok_tiles * FEATURES, ks = static_cast<int>(u % KS);
        mbar_arrive_expect_tx(w_full + stage, W_STAGE);
#pragma unroll
        for (int tile = 0; tile < 2; ++tile)
          tma_load_2d_hint(smem + stage * W_STAGE + tile * (W_STAGE / 2), &p.tmW, ks * (WK / 4), row + tile * BM, w_full + stage, policy);
        s_w_asked = i + 1;
      }
    }
    __syncwarp();
  } else if (warp == 0) {
    // ---------------- TMA of the tokens ----------------
    if (lane == 0) {
      pdl_wait();
      int xi = 0;
      bool ok = true;
      for (uint32_t u = u_begin; ok && u < u_end; ++u) {
        const int m0 = static_cast<int>(u / KS) % p.tok_tiles * TN, ks = static_cast<int>(u % KS);
        for (int x = 0; x < x_stages_of(ks); ++x) {
          const int stage = xi % X_STAGES;
          if (xi >= X_STAGES) ok = mbar_wait(x_empty + stage, (xi / X_STAGES - 1) & 1, abort, WAIT_NS);
          if (!ok) break;
          unsigned char* dst = x_smem + stage * p.terms * 2 * X_ATOM;
          mbar_arrive_expect_tx(x_full + stage, p.terms * 2 * X_ATOM);
          for (int i = 0; i < 2 * p.terms; ++i)
            tma_load_2d(dst + i * X_ATOM, &p.tmX, ks * WK + x * XK + i % 2 * 64, m0 + i / 2 * w.M, x_full + stage);
          s_x_asked = ++xi;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------- MMA (the whole warp, one elected lane issues) ----------------
    const uint32_t elected = elect_one();
    const uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(TN >> 3) << 17) | (static_cast<uint32_t>(BM >> 4) << 24);  // fp16, fp32 sums
    const uint64_t desc0 = sw128_desc(smem_u32(x_smem));
    int xi = 0;
    uint32_t n = 0;  // groups so far
    bool ok = true;
    for (uint32_t u = u_begin; ok && u < u_end; ++u) {
      const int ks = static_cast<int>(u % KS);
      for (int x = 0; ok && x < x_stages_of(ks); ++x, ++xi) {
        const int stage = xi % X_STAGES;
        ok = mbar_wait_warp(x_full + stage, xi / X_STAGES & 1, abort, WAIT_NS);
        const int g0 = (ks * WK + x * XK) / G;
        for (int i = 0; ok && i < min(PER_X, p.groups - g0); ++i, ++n) {
          const int buf = n & 1;
#pragma unroll
          for (int tile = 0; tile < 2; ++tile) {
            ok = ok && mbar_wait_warp(a_full[tile] + buf, n >> 1 & 1, abort, WAIT_NS);
            if (!ok) break;
            tc_fence_after();
            const uint32_t a = tmem + (tile * 2 + buf) * A_COLS, d = tmem + 4 * A_COLS + (tile * 2 + buf) * TN;
            uint32_t acc = 0;
            for (int s = 0; s < p.terms; ++s) {
              const uint64_t b0 = desc0 + ((static_cast<uint64_t>(stage) * p.terms + s) * 2 * X_ATOM >> 4);
#pragma unroll
              for (int k = 0; k < G / 16; ++k) {
                const int col = i * G + k * 16;  // in the token stage
                tc_mma_ts(d, a + k * 8, b0 + static_cast<uint64_t>((col / 64 * X_ATOM + col % 64 * 2) >> 4), idesc, acc, elected);
                acc = 1;
              }
            }
            tc_commit(mma_done[tile] + buf, elected);
          }
        }
        if (ok) tc_commit(x_empty + stage, elected);
      }
    }
    __syncwarp();
  } else if (warp >= UNPACK_WARP) {
    // ---------------- unpack, and sum ----------------
    const int tile = (warp - UNPACK_WARP) / 4, row = warp % 4 * 32 + lane;  // feature of the tile
    const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
    const uint32_t a_base = tmem + lanes + tile * 2 * A_COLS, d_base = tmem + lanes + 4 * A_COLS + tile * 2 * TN;
    const uint16_t* scales = reinterpret_cast<const uint16_t*>(w.scale);
    float acc[TN];
    float scale_of[2] = {};  // of the groups whose products are on their way
    uint32_t stored = 0, summed = 0;
    bool ok = true;
    auto add = [&]() {  // the oldest group's products
      const int buf = summed & 1;
      ok = ok && mbar_wait_warp(mma_done[tile] + buf, summed >> 1 & 1, abort, WAIT_NS);
      ++summed;
      if (!ok) return;
      tc_fence_after();
      const float s = buf ? scale_of[1] : scale_of[0];
      constexpr int AT_ONCE = TN < 32 ? 1 : 2;
#pragma unroll
      for (int i0 = 0; i0 < TN / 16; i0 += AT_ONCE) {
        uint32_t d[AT_ONCE][16];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) tmem_ld16_async(d_base + buf * TN + 16 * (i0 + i), d[i]);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          tmem_wait16(d[i]);
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[16 * (i0 + i) + j] = fmaf(s, __uint_as_float(d[i][j]), acc[16 * (i0 + i) + j]);
        }
      }
      tc_fence_before();
    };
    int wi = 0;
    for (uint32_t u = u_begin; ok && u < u_end;) {
      const int t = static_cast<int>(u / KS);
      const uint32_t part_end = min(u_end, static_cast<uint32_t>(t + 1) * KS);
      const int n = t / p.tok_tiles * FEATURES + tile * BM + row, m0 = t % p.tok_tiles * TN;
      const size_t gn = static_cast<size_t>(min(n, w.N - 1)) * p.groups;
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[j] = 0.f;
      const int g_end = min(p.groups, static_cast<int>(part_end - static_cast<uint32_t>(t) * KS) * (WK / G));
      int g = static_cast<int>(u % KS) * (WK / G);
      uint32_t next_scale = scales[gn + g], next_zero = w.zero ? w.zero[gn + g] : 8;
      for (; ok && u < part_end; ++u, ++wi) {
        const int stage = wi % W_STAGES;
        ok = mbar_wait_warp(w_full + stage, wi / W_STAGES & 1, abort, WAIT_NS);
        const unsigned char* codes = smem + stage * W_STAGE + tile * (W_STAGE / 2) + row * 128;
        for (int i = 0; ok && i < WK / G && g < g_end; ++i, ++g) {
          const float scale = __uint_as_float(next_scale << 16);
          const uint32_t off = zero_off(next_zero), off16 = zero_off16(next_zero);
          if (g + 1 < g_end) {
            next_scale = scales[gn + g + 1];
            next_zero = w.zero ? w.zero[gn + g + 1] : 8;
          }
          if (stored - summed == 2) add();
          if (!ok) break;
          const int buf = stored & 1;
#pragma unroll
          for (int c = 0; c < G / 32; ++c) {  // 32 codes: 16 bytes, 16 columns
            const int chunk = i * (G / 32) + c;
            const uint4 v = *reinterpret_cast<const uint4*>(codes + ((chunk ^ (row & 7)) << 4));
            uint32_t r[16];
            w4_codes_f16(v.x, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r));
            w4_codes_f16(v.y, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r + 4));
            w4_codes_f16(v.z, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r + 8));
            w4_codes_f16(v.w, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r + 12));
            tmem_st16(a_base + buf * A_COLS + 16 * c, r);
          }
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          tc_fence_before();
          mbar_arrive(a_full[tile] + buf);
          if (buf)
            scale_of[1] = scale;
          else
            scale_of[0] = scale;
          ++stored;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(w_empty + stage);
      }
      while (summed < stored) add();
      const uint32_t tu0 = static_cast<uint32_t>(t) * KS;
      const int c_first = cta_of_unit(tu0, U, CTAS), c_last = cta_of_unit(tu0 + KS - 1, U, CTAS), parts = c_last - c_first + 1;
      pdl_wait();  // Y, the workspace and its counters are shared with earlier kernels
      ok = !any_of(2, UNPACK, !ok);  // all of them leave together
      bool mine = ok;
      if (ok && parts > 1) {
        // slot 0 of a CTA holds its first tile's part, slot 1 its last one's
        const int slot = 2 * blockIdx.x + (u_begin / KS == static_cast<uint32_t>(t) ? 0 : 1);
        float* part = w.ws + static_cast<size_t>(slot) * FEATURES * TN + tile * BM + row;
#pragma unroll
        for (int j = 0; j < TN; ++j) __stcg(part + j * FEATURES, acc[j]);
        __threadfence();
        named_bar(1, UNPACK);
        if (threadIdx.x == UNPACK_WARP * 32) {
          s_last = atomicAdd(w.counters + t, 1) == parts - 1;
          if (s_last) w.counters[t] = 0;
        }
        named_bar(1, UNPACK);
        mine = s_last;
        if (mine) {
          __threadfence();
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[j] = 0.f;
          for (int c = c_first; c <= c_last; ++c) {
            const int from = 2 * c + (unit_begin(c, U, CTAS) / KS == static_cast<uint32_t>(t) ? 0 : 1);
            const float* src = w.ws + static_cast<size_t>(from) * FEATURES * TN + tile * BM + row;
            float v[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) v[j] = __ldcg(src + j * FEATURES);
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[j] += v[j];
          }
        }
        named_bar(1, UNPACK);  // s_last has been read
      }
      if (mine && n < w.N) {
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[j] = m0 + j < w.M ? acc[j] * p.down[m0 + j] : 0.f;
        if (w.epi == EPI_RESID) {
          float* y = static_cast<float*>(w.Y) + static_cast<size_t>(m0) * w.ldy + n;
#pragma unroll
          for (int j = 0; j < TN; ++j)
            if (m0 + j < w.M) acc[j] += y[static_cast<size_t>(j) * w.ldy];
#pragma unroll
          for (int j = 0; j < TN; ++j)
            if (m0 + j < w.M) y[static_cast<size_t>(j) * w.ldy] = acc[j];
        } else {
#pragma unroll
          for (int j = 0; j < TN; ++j)
            if (m0 + j < w.M) store_y(w, m0 + j, n, acc[j]);
        }
      }
    }
    if (!ok && lane == 0) atomicOr(w.err, ERR_TIMEOUT);
  }

  pdl_wait();
  pdl_trigger();
  tc_fence_before();
  __syncthreads();
  // A role gave up: copies in flight land before the CTA leaves, and the MMAs end before the tensor memory goes.
  if (s_abort) {
    if (threadIdx.x == 0) {
      atomicOr(w.err, ERR_TIMEOUT);
      for (int i = max(0, s_w_asked - W_STAGES); i < s_w_asked; ++i)
        mbar_wait_plain(w_full + i % W_STAGES, i / W_STAGES & 1, WAIT_NS);
      for (int i = max(0, s_x_asked - X_STAGES); i < s_x_asked; ++i)
        mbar_wait_plain(x_full + i % X_STAGES, i / X_STAGES & 1, WAIT_NS);
    } else if (warp == 1) {
      tc_commit(&drain, elect_one());
      mbar_wait_plain(&drain, 0, WAIT_NS);
    }
    __syncthreads();
  }
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
}

// One block per token: its fp16 terms, in the order of the codes, and what undoes its scale.
__global__ void __launch_bounds__(256) w4_tokens_kernel(W4Params p, int terms, unsigned char* x16, float* down) {
  __shared__ uint32_t sh_top;
  if (threadIdx.x == 0) sh_top = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();  // after the wait: the linear may read the weights before its own
  const int m = blockIdx.x, lane = threadIdx.x & 31;
  uint32_t top = 0;
  for (int i = threadIdx.x; i < p.K / 8; i += 256) {
    float x[8];
    load8(p, m, 8 * i, x);
    top = max(top, top_bits(x));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if (lane == 0) atomicMax(&sh_top, top);
  __syncthreads();
  const float up = token_scale(sh_top);
  if (threadIdx.x == 0) down[m] = 1.f / up;
  for (int i = threadIdx.x; i < p.K / 8; i += 256) {
    float x[8];
    load8(p, m, 8 * i, x);
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) split_f16(x[j] * up, x[j + 4] * up, hi[j], lo[j]);
    unsigned char* dst = x16 + static_cast<size_t>(m) * p.K * 2 + 16 * i;
    *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    if (terms == 2) *reinterpret_cast<uint4*>(dst + static_cast<size_t>(p.M) * p.K * 2) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

template <int G, int TN>
cudaError_t launch(const ManyParams& p, int grid, cudaStream_t s) {
  const cudaError_t e =
      cudaFuncSetAttribute(w4_many_kernel<G, TN>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(many_smem(TN, 2)));
  return e != cudaSuccess ? e : launch_pdl(w4_many_kernel<G, TN>, dim3(grid), dim3(THREADS), many_smem(TN, p.terms), s, p);
}
template <int G>
cudaError_t launch_tile(const ManyParams& p, int tn, int grid, cudaStream_t s) {
  return tn == 16 ? launch<G, 16>(p, grid, s) : tn == 32 ? launch<G, 32>(p, grid, s) : launch<G, 64>(p, grid, s);
}

}  // namespace

cudaError_t linear_w4_many(const W4Params& all, cudaStream_t s) {
  const int terms = all.x_f32 || all.X_lo ? 2 : 1;
  // passes of as many tokens as the scratch holds
  const size_t per_token = static_cast<size_t>(all.K) * 2 * terms + 4;
  const size_t room = all.scratch_bytes / per_token;
  if (room < 1) return cudaErrorInvalidValue;
  int pass = static_cast<int>(std::min<size_t>(room, static_cast<size_t>(all.M)));
  if (pass < all.M && pass > 64) pass = pass / 64 * 64;
  for (int m0 = 0; m0 < all.M; m0 += pass) {
    W4Params w = all;
    w.M = std::min(pass, all.M - m0);
    const size_t xs = static_cast<size_t>(m0) * w.ldx, ys = static_cast<size_t>(m0) * w.ldy;
    w.X = static_cast<const char*>(w.X) + xs * (w.x_f32 ? 4 : 2);
    if (w.X_lo) w.X_lo = reinterpret_cast<const bf16_raw*>(reinterpret_cast<const char*>(w.X_lo) + xs * 2);
    w.Y = static_cast<char*>(w.Y) + ys * (w.out_f32 ? 4 : 2);
    unsigned char* x16 = static_cast<unsigned char*>(w.scratch);
    float* down = reinterpret_cast<float*>(x16 + static_cast<size_t>(w.M) * w.K * 2 * terms);
    ManyParams p{};
    p.w = w;
    p.down = down;
    p.terms = terms;
    p.groups = (w.K + w.group - 1) / w.group;
    p.kstages = (w.K + WK - 1) / WK;
    const int tn = w.M <= 16 ? 16 : w.M <= 32 ? 32 : 64;
    p.tok_tiles = (w.M + tn - 1) / tn;
    const long long tiles = static_cast<long long>((w.N + FEATURES - 1) / FEATURES) * p.tok_tiles;
    const long long units = tiles * p.kstages;
    if (tiles > tc_max_tiles() || units * tc_num_sms() >= (1LL << 32)) return cudaErrorInvalidValue;
    p.units = static_cast<uint32_t>(units);
    if (encode_2d_bf16(&p.tmW, w.W, w.K / 4, w.N, w.K / 4, 64, BM) != 0 ||
        encode_2d_bf16(&p.tmX, x16, w.K, static_cast<uint64_t>(terms) * w.M, w.K, 64, tn) != 0)
      return cudaErrorInvalidValue;
    cudaError_t e = launch_pdl(w4_tokens_kernel, dim3(w.M), dim3(256), 0, s, w, terms, x16, down);
    if (e != cudaSuccess) return e;
    const int grid = static_cast<int>(std::min<long long>(units, tc_num_sms()));
    e = w.group == 128 ? launch_tile<128>(p, tn, grid, s) : w.group == 64 ? launch_tile<64>(p, tn, grid, s) : launch_tile<32>(p, tn, grid, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace chimera
