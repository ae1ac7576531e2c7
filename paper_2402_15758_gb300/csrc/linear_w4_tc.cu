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
// Work split: stream-K over (tile, 256 columns of K), one CTA per SM; the parts of tiles cut between CTAs go to the
// workspace and are added by a second kernel in CTA order (deterministic).
//
// Measured (GB300, 22016 x 4096, group 128): 16 tokens 22.7 us, 64 29.2, 64 in two terms 32 (alone, the tokens'
// kernel 4, the products 26, the join 9), 256 tokens 83 in one term, 90 in two; 4096 x 4096, 16 tokens 11.8.  Bound by the
// unpacking warps, each group's codes after the sums of the one before: 0.7 us for 256 features x 128 columns (the tensor
// pipe is active 45 % of the time, an instruction is issued in 42 %, DRAM works at 22 %).  From 256 tokens on the 16-bit
// linear is faster, 81 us in one term and 68 in two (128 tokens: 50 and 49 here): a CTA takes 64 tokens, so 256
// unpack the weights four times.
//
// Roles: warp 0 TMA of the tokens, warps 1 and 3 the MMAs of a tile each (one warp for both was the bottleneck: an MMA
// takes 28 cycles to issue and a wait 200), warp 2 TMA of the weights, the others unpack and sum (warp w: TMEM
// lanes 32 (w % 4) ..).
#include <algorithm>

#include "kernels.h"
#include "kv4.cuh"
#include "launch.cuh"
#include "linear_w4.cuh"

namespace chimera {
namespace {

constexpr int BM = 128;                    // features of a tile
constexpr int WK = 256;                    // columns per weight stage: 128 bytes of a row
constexpr int XK = 128;                    // columns per token stage: two 128-byte atoms
constexpr int W_TILE = BM * WK / 2, W_BYTES = 6 * W_TILE, MAX_X_STAGES = 8;
constexpr int UNPACK_WARP = 4;
// Eight warps unpack, whether a CTA has one tile or two (sixteen for two tiles: 16 tokens of 22016 x 4096 26.6 us
// instead of 25.5, 64 tokens 41 instead of 35): warps that share the features of a tile.
__host__ __device__ constexpr int halves(int ft) { return 2 / ft; }
// Parts of a 256-feature tile up to which a CTA takes two tiles of 128 features, which share their tokens; with more the
// join costs more than that saves.  64 tokens in two terms, 22016 x 4096 (2 parts): two tiles 31.1 us, one 39.8; 4096 x
// 11008 (9 parts): two 27.2, one 25.0; 64 tokens in one, 12288 x 4096 (3 parts): two 20.6, one 22.7; 4096 x 4096 (9):
// two 15.7, one 12.6.
constexpr int FEW_PARTS = 4;
constexpr int A_COLS = 64;                 // TMEM columns of a group's codes (128 of them)
constexpr unsigned long long WAIT_NS = 2000000000ull;

struct ManyParams {
  CUtensorMap tmW;    // codes: [N][K / 2] bytes, box 128 x 128 bytes, 128-byte swizzle
  CUtensorMap tmX;    // X16: [terms * M][K] fp16, box TN x 64
  W4Params w;
  const float* down;  // [M]: what undoes a token's scale
  int groups, terms, kstages, tok_tiles;
  int x_stages;
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
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
// N consecutive columns of this thread's lane (8, 16 or 32), without a wait; and the wait, which names the
// registers, so that no use of them is moved above it.
template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 8) tmem_ld8(taddr + i, r + i);
}
template <int N>
__device__ __forceinline__ void tmem_wait_cols(uint32_t (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}

// a += s x, b += s y in one instruction.
__device__ __forceinline__ void fma2(float s, float x, float y, float& a, float& b) {
  asm("{\n\t.reg .b64 s, v, t;\n\t"
      "mov.b64 s, {%2, %2};\n\tmov.b64 v, {%3, %4};\n\tmov.b64 t, {%0, %1};\n\t"
      "fma.rn.f32x2 t, s, v, t;\n\tmov.b64 {%0, %1}, t;\n\t}"
      : "+f"(a), "+f"(b)
      : "f"(s), "f"(x), "f"(y));
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

// The epilogue of one feature and 8 tokens from m0 on.  The kind is decided outside the loops, so that loads,
// divisions and stores of the tokens overlap.
__device__ __forceinline__ void store_feature(const W4Params& w, int m0, int n, float (&v)[8]) {
  const size_t at = static_cast<size_t>(m0) * w.ldy + n;
  const int rows = w.M - m0;
  if (w.epi == EPI_RESID) {
    // every load before the first sum, and none behind a branch (the last row again for those past it)
    const float* y = static_cast<const float*>(w.Y) + at;
    float old[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) old[j] = y[static_cast<size_t>(min(j, rows - 1)) * w.ldy];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += old[j];
  } else if (w.epi == EPI_SILU) {
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = 1.f + expf(-v[j]);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] /= e[j];
  }
  if (w.out_f32) {
    float* y = static_cast<float*>(w.Y) + at;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < rows) y[static_cast<size_t>(j) * w.ldy] = v[j];
  } else {
    bf16* y = static_cast<bf16*>(w.Y) + at;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < rows) y[static_cast<size_t>(j) * w.ldy] = __float2bfloat16_rn(v[j]);
  }
}

// Stages of the tokens' ring: what the weights' leaves (a request for tokens waits in the copy engine behind those
// for weights: with three stages the MMAs of 16 tokens waited for half of the time).
int many_x_stages(int tn, int terms) { return std::min(MAX_X_STAGES, (226 * 1024 - 1024 - W_BYTES) / (terms * 2 * tn * 128)); }
size_t many_smem(int tn, int terms) { return 1024 + W_BYTES + static_cast<size_t>(many_x_stages(tn, terms)) * terms * 2 * tn * 128; }

// FT: tiles of a CTA.
template <int G, int TN, int FT>
__global__ void __launch_bounds__(UNPACK_WARP * 32 + FT * halves(FT) * BM, 1) w4_many_kernel(const __grid_constant__ ManyParams p) {
  constexpr int HALVES = halves(FT), FEATURES = FT * BM, UNPACK = FT * HALVES * BM, W_STAGE = FT * W_TILE, W_STAGES = W_BYTES / W_STAGE;
  constexpr uint32_t D_COL = FT * 2 * A_COLS;  // tensor memory: codes [tile][2], sums [tile][2]
  constexpr uint32_t TMEM_COLS = FT == 2 ? 512 : 256;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t w_full[W_STAGES], w_empty[W_STAGES], x_full[MAX_X_STAGES], x_empty[MAX_X_STAGES];
  __shared__ uint64_t a_full[FT][2], mma_done[FT][2], drain[2];  // [tile][buffer]
  __shared__ uint32_t tmem_slot;
  __shared__ int s_abort, s_w_asked, s_x_asked;
  unsigned char* smem = smem_raw + (1024 - (smem_u32(smem_raw) & 1023u)) % 1024;
  unsigned char* x_smem = smem + W_BYTES;
  const int warp = threadIdx.x / 32, lane = threadIdx.x & 31;
  volatile int* abort = &s_abort;
  const W4Params& w = p.w;
  if (threadIdx.x == 0) {
    for (int i = 0; i < W_STAGES; ++i) {
      mbar_init(w_full + i, 1);
      mbar_init(w_empty + i, UNPACK / 32);
    }
    for (int i = 0; i < p.x_stages; ++i) {
      mbar_init(x_full + i, 1);
      mbar_init(x_empty + i, FT);
    }
    for (int i = 0; i < 2 * FT; ++i) {
      mbar_init(a_full[i / 2] + i % 2, 4 * HALVES);
      mbar_init(mma_done[i / 2] + i % 2, 1);
    }
    mbar_init(drain, 1);
    mbar_init(drain + 1, 1);
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
  auto x_stages_of = [&](int ks) { return (min(WK, w.K - ks * WK) + XK - 1) / XK; };

  if (warp == 2) {
    // ---------------- TMA of the weights ----------------
    // Every kernel before the one that wrote X16 is complete (it lets its dependents launch after its own
    // wait), so the weights may be read before this kernel's wait.
    if (lane == 0) {
      const uint64_t policy = policy_evict_first();
      bool ok = true;
      int t = static_cast<int>(u_begin / KS), ks = static_cast<int>(u_begin % KS), i = 0;
      int row = t / p.tok_tiles * FEATURES;
      for (uint32_t u = u_begin; ok && u < u_end; ++u, ++i) {
        const int stage = i % W_STAGES;
        if (i >= W_STAGES) ok = mbar_wait(w_empty + stage, (i / W_STAGES - 1) & 1, abort, WAIT_NS);
        if (!ok) break;
        mbar_arrive_expect_tx(w_full + stage, W_STAGE);
#pragma unroll
        for (int tile = 0; tile < FT; ++tile)
          tma_load_2d_hint(smem + stage * W_STAGE + tile * W_TILE, &p.tmW, ks * (WK / 4), row + tile * BM, w_full + stage, policy);
        s_w_asked = i + 1;
        if (++ks == static_cast<int>(KS)) {
          ks = 0;
          row = ++t / p.tok_tiles * FEATURES;
        }
      }
    }
    __syncwarp();
  } else if (warp == 0) {
    // ---------------- TMA of the tokens ----------------
    if (lane == 0) {
      pdl_wait();
      int stage = 0, asked = 0;
      uint32_t phase = 1;  // parity of the stage's last release
      int t = static_cast<int>(u_begin / KS), ks = static_cast<int>(u_begin % KS);
      int m0 = t % p.tok_tiles * TN;
      bool ok = true;
      for (uint32_t u = u_begin; ok && u < u_end; ++u) {
        const int steps = x_stages_of(ks);
        for (int x = 0; x < steps; ++x) {
          if (asked >= p.x_stages) ok = mbar_wait(x_empty + stage, phase, abort, WAIT_NS);
          if (!ok) break;
          unsigned char* dst = x_smem + stage * p.terms * 2 * X_ATOM;
          mbar_arrive_expect_tx(x_full + stage, p.terms * 2 * X_ATOM);
          for (int i = 0; i < 2 * p.terms; ++i)
            tma_load_2d(dst + i * X_ATOM, &p.tmX, ks * WK + x * XK + i % 2 * 64, m0 + i / 2 * w.M, x_full + stage);
          s_x_asked = ++asked;
          if (++stage == p.x_stages) {
            stage = 0;
            phase ^= 1;
          }
        }
        if (++ks == static_cast<int>(KS)) {
          ks = 0;
          m0 = ++t % p.tok_tiles * TN;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1 || (FT == 2 && warp == 3)) {
    // ---------------- MMA of a tile (the whole warp, one elected lane issues) ----------------
    const int tile = warp / 2;
    const uint32_t elected = elect_one();
    const uint32_t idesc = (1u << 4) | (static_cast<uint32_t>(TN >> 3) << 17) | (static_cast<uint32_t>(BM >> 4) << 24);  // fp16, fp32 sums
    const uint64_t desc0 = sw128_desc(smem_u32(x_smem));
    // (counters instead of divisions: three of them took this warp 800 cycles per group)
    int stage = 0, ks = static_cast<int>(u_begin % KS);
    uint32_t phase = 0, n = 0;  // n: groups so far
    bool ok = true;
    for (uint32_t u = u_begin; ok && u < u_end; ++u) {
      const int steps = x_stages_of(ks);
      for (int x = 0; ok && x < steps; ++x) {
        ok = mbar_wait_warp(x_full + stage, phase, abort, WAIT_NS);
        const int here = min(PER_X, p.groups - (ks * WK + x * XK) / G);
        const uint64_t b_stage = desc0 + static_cast<uint64_t>(stage * p.terms * 2 * X_ATOM >> 4);
        for (int i = 0; ok && i < here; ++i, ++n) {
          const int buf = n & 1;
          ok = mbar_wait_warp(a_full[tile] + buf, n >> 1 & 1, abort, WAIT_NS);
          if (!ok) break;
          tc_fence_after();
          const uint32_t a = tmem + (tile * 2 + buf) * A_COLS, d = tmem + D_COL + (tile * 2 + buf) * TN;
          uint32_t acc = 0;
          for (int s = 0; s < p.terms; ++s) {
            const uint64_t b0 = b_stage + static_cast<uint64_t>(s * 2 * X_ATOM >> 4);
#pragma unroll
            for (int k = 0; k < G / 16; ++k) {
              const int col = i * G + k * 16;  // in the token stage
              tc_mma_ts(d, a + k * 8, b0 + static_cast<uint64_t>((col / 64 * X_ATOM + col % 64 * 2) >> 4), idesc, acc, elected);
              acc = 1;
            }
          }
          tc_commit(mma_done[tile] + buf, elected);
        }
        if (ok) tc_commit(x_empty + stage, elected);
        if (++stage == p.x_stages) {
          stage = 0;
          phase ^= 1;
        }
      }
      if (++ks == static_cast<int>(KS)) ks = 0;
    }
    __syncwarp();
  } else if (warp >= UNPACK_WARP) {
    // ---------------- unpack, and sum ----------------
    // Two warps share 32 features of a tile: each takes half of a group's codes and half of the tokens' sums.
    constexpr int COLS = TN / HALVES;
    const int tile = (warp - UNPACK_WARP) / 4 % FT, half = (warp - UNPACK_WARP) / (4 * FT), row = warp % 4 * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(warp % 4 * 32) << 16;
    const uint32_t a_base = tmem + lanes + tile * 2 * A_COLS + half * (G / 4);
    const uint32_t d_base = tmem + lanes + D_COL + tile * 2 * TN + half * COLS;
    const uint16_t* scales = reinterpret_cast<const uint16_t*>(w.scale);
    float acc[COLS];
    float scale_of[2] = {};  // of the groups whose products are on their way
    uint32_t stored = 0, summed = 0;
    bool ok = true;
    // the oldest group's products: waited for; asked for and added, up to 16 columns at a time
    constexpr int ONCE = COLS < 16 ? COLS : 16;
    uint32_t d[ONCE];
    auto products_there = [&]() {
      ok = ok && mbar_wait_warp(mma_done[tile] + (summed & 1), summed >> 1 & 1, abort, WAIT_NS);
      if (ok) tc_fence_after();
      return ok;
    };
    auto ask = [&](int at) { tmem_ld_cols<ONCE>(d_base + (summed & 1) * TN + at, d); };
    auto add = [&](int at) {
      const float s = summed & 1 ? scale_of[1] : scale_of[0];
      tmem_wait_cols<ONCE>(d);
#pragma unroll
      for (int j = 0; j < ONCE; j += 2) fma2(s, __uint_as_float(d[j]), __uint_as_float(d[j + 1]), acc[at + j], acc[at + j + 1]);
    };
    // Slot 0 of a CTA holds its first tile's part, slot 1 its last one's.
    auto slot_of = [&](int c, int t) { return 2 * c + (unit_begin(c, U, CTAS) / KS == static_cast<uint32_t>(t) ? 0 : 1); };
    auto part_of = [&](int slot) {
      return w.ws + (static_cast<size_t>(slot) * TN + half * COLS) * FEATURES + tile * BM + row;
    };
    int wi = 0;
    for (uint32_t u = u_begin; ok && u < u_end;) {
      const int t = static_cast<int>(u / KS);
      const uint32_t t0 = static_cast<uint32_t>(t) * KS, part_end = min(u_end, t0 + KS);
      const bool whole = u == t0 && part_end == t0 + KS;
      const int n = t / p.tok_tiles * FEATURES + tile * BM + row;
      const size_t gn = static_cast<size_t>(min(n, w.N - 1)) * p.groups;
#pragma unroll
      for (int j = 0; j < COLS; ++j) acc[j] = 0.f;
      const int g_end = min(p.groups, static_cast<int>(part_end - t0) * (WK / G));
      int g = static_cast<int>(u - t0) * (WK / G);
      uint32_t next_scale = scales[gn + g], next_zero = w.zero ? w.zero[gn + g] : 8;
      for (; ok && u < part_end; ++u, ++wi) {
        const int stage = wi % W_STAGES;
        ok = mbar_wait_warp(w_full + stage, wi / W_STAGES & 1, abort, WAIT_NS);
        const unsigned char* codes = smem + stage * W_STAGE + tile * W_TILE + row * 128;
        for (int i = 0; ok && i < WK / G && g < g_end; ++i, ++g) {
          const float scale = __uint_as_float(next_scale << 16);
          const uint32_t off = zero_off(next_zero), off16 = zero_off16(next_zero);
          if (g + 1 < g_end) {
            next_scale = scales[gn + g + 1];
            next_zero = w.zero ? w.zero[gn + g + 1] : 8;
          }
          const int buf = stored & 1;
          const bool full = stored - summed == 2;  // the buffer's last products are read back on the way
          if (full && !products_there()) break;
          // between the codes' chunks of 16 bytes (8 with groups of 32 and two halves)
          constexpr int CHUNKS = G / 32 / HALVES > 0 ? G / 32 / HALVES : 1, STEPS = COLS / ONCE;
#pragma unroll
          for (int c = 0; c < CHUNKS || c < STEPS; ++c) {
            if (full && c < STEPS) ask(c * ONCE);
            if (c < CHUNKS) {
              if constexpr (G / HALVES < 32) {
                const uint2 v = *reinterpret_cast<const uint2*>(codes + ((i ^ (row & 7)) << 4) + half * 8);
                uint32_t r[8];
                w4_codes_f16(v.x, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r));
                w4_codes_f16(v.y, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r + 4));
                tmem_st8(a_base + buf * A_COLS, r);
              } else {
                const int chunk = (HALVES * i + half) * CHUNKS + c;
                const uint4 v = *reinterpret_cast<const uint4*>(codes + ((chunk ^ (row & 7)) << 4));
                uint32_t r[16];
                w4_codes_f16(v.x, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r));
                w4_codes_f16(v.y, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r + 4));
                w4_codes_f16(v.z, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r + 8));
                w4_codes_f16(v.w, off, off16, *reinterpret_cast<uint32_t(*)[4]>(r + 12));
                tmem_st16(a_base + buf * A_COLS + 16 * c, r);
              }
            }
            if (full && c < STEPS) add(c * ONCE);
          }
          if (full) ++summed;
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(a_full[tile] + buf);
          if (buf)
            scale_of[1] = scale;
          else
            scale_of[0] = scale;
          ++stored;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(w_empty + stage);
      }
      for (; summed < stored && products_there(); ++summed) {
#pragma unroll
        for (int at = 0; at < COLS; at += ONCE) ask(at), add(at);
      }
      tc_fence_before();
      pdl_wait();  // Y and the workspace are shared with earlier kernels
      ok = !any_of(2, UNPACK, !ok);  // all of them leave together
      if (!ok) break;
      // The part goes to the workspace, and the join of a cut tile to a kernel of its own, over all SMs.
      float* part = part_of(slot_of(blockIdx.x, t));
#pragma unroll
      for (int j = 0; j < COLS; ++j) __stcg(part + j * FEATURES, acc[j]);
      if (!whole || n >= w.N) continue;
      const int m0 = t % p.tok_tiles * TN + half * COLS;
#pragma unroll 1
      for (int at = 0; at < COLS && m0 + at < w.M; at += 8) {  // (a loop: straight-line code waits for its fetches)
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __ldcg(part + (at + j) * FEATURES) * p.down[min(m0 + at + j, w.M - 1)];
        store_feature(w, m0 + at, n, v);
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
      for (int i = max(0, s_x_asked - p.x_stages); i < s_x_asked; ++i)
        mbar_wait_plain(x_full + i % p.x_stages, i / p.x_stages & 1, WAIT_NS);
    } else if (warp == 1 || warp == 3) {  // (the lanes that issued them: the election is deterministic)
      tc_commit(drain + warp / 2, elect_one());
      mbar_wait_plain(drain + warp / 2, 0, WAIT_NS);
    }
    __syncthreads();
  }
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
}

// Joins the tiles that were cut between CTAs: a thread adds the parts of one feature and 8 tokens, in the CTAs'
// order, and runs the epilogue.  In the linear itself, by the last CTA to arrive, it took 12 us after the last
// product (64 tokens of 22016 x 4096): one SM read all parts of a tile.
__global__ void __launch_bounds__(256) w4_join_kernel(const __grid_constant__ ManyParams p, int tn, int features, int ctas) {
  pdl_wait();
  pdl_trigger();
  const W4Params& w = p.w;
  const uint32_t U = p.units, KS = p.kstages;
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  const int row = static_cast<int>(i % features), per_tile = tn / 8;
  const long long chunk = i / features;
  const int t = static_cast<int>(chunk / per_tile), at = static_cast<int>(chunk % per_tile) * 8;
  if (static_cast<uint32_t>(t) >= U / KS) return;
  const int n = t / p.tok_tiles * features + row, m0 = t % p.tok_tiles * tn + at;
  const uint32_t t0 = static_cast<uint32_t>(t) * KS;
  const int c0 = cta_of_unit(t0, U, ctas), c1 = cta_of_unit(t0 + KS - 1, U, ctas);
  if (c0 == c1 || n >= w.N || m0 >= w.M) return;
  const float* first = w.ws + (static_cast<size_t>(2 * c0 + (unit_begin(c0, U, ctas) / KS == static_cast<uint32_t>(t) ? 0 : 1)) * tn + at) * features + row;
  float sum[8] = {};
  for (int c = c0; c <= c1; c += 4) {  // the loads of four parts in flight
    float v[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // only the first CTA may end in the tile; the others begin in it
      const float* x = c + k == c0 ? first : w.ws + (static_cast<size_t>(2 * min(c + k, c1)) * tn + at) * features + row;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[k][j] = c + k <= c1 ? __ldcg(x + j * features) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += v[k][j];
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] *= p.down[min(m0 + j, w.M - 1)];
  store_feature(w, m0, n, sum);
}

// One block per token: its fp16 terms, in the order of the codes, and what undoes its scale.  A row of up to 8192
// columns stays in registers between the search for its largest value and its conversion.
constexpr int TOKEN_THREADS = 256, TOKEN_VECS = 4;
__global__ void __launch_bounds__(TOKEN_THREADS) w4_tokens_kernel(W4Params p, int terms, unsigned char* x16, float* down) {
  __shared__ uint32_t sh_top[TOKEN_THREADS / 32];
  pdl_wait();
  pdl_trigger();  // after the wait: the linear may read the weights before its own
  const int m = blockIdx.x, vecs = p.K / 8;
  float x[TOKEN_VECS][8];
  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < TOKEN_VECS; ++v)
    if (threadIdx.x + v * TOKEN_THREADS < vecs) load8(p, m, 8 * (threadIdx.x + v * TOKEN_THREADS), x[v]);
#pragma unroll
  for (int v = 0; v < TOKEN_VECS; ++v)
    if (threadIdx.x + v * TOKEN_THREADS < vecs) top = max(top, top_bits(x[v]));
  for (int i = threadIdx.x + TOKEN_VECS * TOKEN_THREADS; i < vecs; i += TOKEN_THREADS) {
    float y[8];
    load8(p, m, 8 * i, y);
    top = max(top, top_bits(y));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) sh_top[threadIdx.x / 32] = top;
  __syncthreads();
  top = __reduce_max_sync(0xffffffffu, sh_top[threadIdx.x % (TOKEN_THREADS / 32)]);
  const float up = token_scale(top);
  if (threadIdx.x == 0) down[m] = 1.f / up;
  auto write = [&](int i, const float (&y)[8]) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) split_f16(y[j] * up, y[j + 4] * up, hi[j], lo[j]);
    unsigned char* dst = x16 + static_cast<size_t>(m) * p.K * 2 + 16 * static_cast<size_t>(i);
    *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    if (terms == 2) *reinterpret_cast<uint4*>(dst + static_cast<size_t>(p.M) * p.K * 2) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  };
#pragma unroll
  for (int v = 0; v < TOKEN_VECS; ++v)
    if (threadIdx.x + v * TOKEN_THREADS < vecs) write(threadIdx.x + v * TOKEN_THREADS, x[v]);
  for (int i = threadIdx.x + TOKEN_VECS * TOKEN_THREADS; i < vecs; i += TOKEN_THREADS) {
    float y[8];
    load8(p, m, 8 * i, y);
    write(i, y);
  }
}

template <int G, int TN, int FT>
cudaError_t launch(const ManyParams& p, int grid, cudaStream_t s) {
  const cudaError_t e = allow_smem<w4_many_kernel<G, TN, FT>>(many_smem(TN, 2));
  return e != cudaSuccess ? e : launch_pdl(w4_many_kernel<G, TN, FT>, dim3(grid), dim3(UNPACK_WARP * 32 + FT * halves(FT) * BM), many_smem(TN, p.terms), s, p);
}
template <int G, int TN>
cudaError_t launch_tiles(const ManyParams& p, int ft, int grid, cudaStream_t s) {
  return ft == 2 ? launch<G, TN, 2>(p, grid, s) : launch<G, TN, 1>(p, grid, s);
}
template <int G>
cudaError_t launch_tokens(const ManyParams& p, int tn, int ft, int grid, cudaStream_t s) {
  return tn == 16 ? launch_tiles<G, 16>(p, ft, grid, s) : tn == 32 ? launch_tiles<G, 32>(p, ft, grid, s) : launch_tiles<G, 64>(p, ft, grid, s);
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
    p.x_stages = many_x_stages(tn, terms);
    // one tile per CTA when two would be cut into many parts, which cost their join
    const int ft = (w.N + 2 * BM - 1) / (2 * BM) * p.tok_tiles * FEW_PARTS < tc_num_sms() ? 1 : 2;
    const long long tiles = static_cast<long long>((w.N + ft * BM - 1) / (ft * BM)) * p.tok_tiles;
    const long long units = tiles * p.kstages;
    if (units * tc_num_sms() >= (1LL << 32)) return cudaErrorInvalidValue;
    p.units = static_cast<uint32_t>(units);
    if (encode_2d_bf16(&p.tmW, w.W, w.K / 4, w.N, w.K / 4, 64, BM) != 0 ||
        encode_2d_bf16(&p.tmX, x16, w.K, static_cast<uint64_t>(terms) * w.M, w.K, 64, tn) != 0)
      return cudaErrorInvalidValue;
    cudaError_t e = launch_pdl(w4_tokens_kernel, dim3(w.M), dim3(TOKEN_THREADS), 0, s, w, terms, x16, down);
    if (e != cudaSuccess) return e;
    const int grid = static_cast<int>(std::min<long long>(units, tc_num_sms()));
    e = w.group == 128 ? launch_tokens<128>(p, tn, ft, grid, s)
                       : w.group == 64 ? launch_tokens<64>(p, tn, ft, grid, s) : launch_tokens<32>(p, tn, ft, grid, s);
    if (e != cudaSuccess) return e;
    const long long threads = tiles * (tn / 8) * ft * BM;
    e = launch_pdl(w4_join_kernel, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, s, p, tn, ft * BM, grid);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace chimera
