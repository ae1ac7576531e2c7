// Linear with 4-bit weights: Y[M][N] (epilogue)= X[M][K] . W^T with
// W[n][k] = scale[n][k / group] (code[n][k] - zero[n][k / group]), codes 0..15.
//
// code - zero is a whole number, exact in fp16; a group's products are summed in fp32 by the matrix units, and the
// group's scale multiplies the sum, in fp32.
// The activations enter as fp16, scaled by a power of two per token, hi + lo or fp32 ones as two fp16 terms (2^-23).
#include <algorithm>

#include "kernels.h"
#include "kv4.cuh"
#include "launch.cuh"
#include "linear_w4.cuh"

namespace chimera {
namespace {

constexpr int WARPS = 24, THREADS = WARPS * 32, FEATURES = 16;
// ---------------------------------------------------------------------------
// up to 8 tokens: one pass over the weights at the speed of memory
// ---------------------------------------------------------------------------
// One CTA of 24 warps per SM.  A tile is 16 features (the MMA's rows); KS warps share its K by spans of four groups
// and join their sums after `join` tiles or at the end.  A lane copies (cp.async) into shared memory exactly what it
// will read itself, so a warp runs ahead of its loads with no barrier at all.  The activations stay in shared memory
// for the whole launch.
//
// TINY, where the result is rounded to bf16 and groups are longer than 32: a nibble is used where it lies.  At the end of
// a mantissa with exponent 0 it is a (subnormal) fp16 number, so 8 codes cost 5 instructions instead of 9; nibbles at bit
// 4 count 16 times, in sums of their own; the zero follows in fp32, from the group's sum of the activations.  Sums of
// codes without their zero are longer: the error is 2e-6 of the result instead of 2e-7, which fp32 results do without
// (and sums of 32 cost more than they save: 23.1 us instead of 22.4).
//
// Measured (GB300, 22016 x 4096, group 128, 47 MB): one token 14.3 us, 3.3 TB/s, fp32 out 15.2, in two terms 17.8, group
// 32 22.3; 8 tokens 19; 4096 x 4096 5.9 us (16-bit weights: one token 31.6, 8 tokens 32, 4096 x 4096 10.7).  Three CTAs of
// 8 warps, each with its own copy of the activations: 8 tokens 23 to 26, 4096 x 4096 6.7.  Rings of bulk copies of 256 to 1024 bytes took 19.5 to 23, spans held in registers 17.7.  About
// 4.5 us of every call are the launch, the activations and the join.  Over the whole launch an instruction is issued in
// 51 % of the cycles, the ALUs are as busy, and the warps wait for a slot, the math pipe and shared memory in turn: no
// single limit shows.  80 registers, of which groups of 128 spill 8 bytes.
// From 9 tokens on, which would be a second column of matrices, the tensor cores' kernel: 22016 x 4096, 8 tokens 18.8 us
// here, 22.0 there (1 token 14.3 and 21.9); 4096 x 4096 10.0 and 11.5; 8 tokens in two terms 23.9 in both.
constexpr int FEW_TOKENS = 8;

struct FewParams {
  W4Params w;
  int groups, spans, tiles, ks;
  int stages;          // of a warp's ring
  int join;            // tiles whose sums are held
  int x_pitch;         // of a token's term
  int pairs;           // ceil(M / 2): lanes of a row that hold tokens
  int at_x, at_sums_x, at_sums;  // offsets in shared memory
};

// The scale of a token whose largest magnitude is 2^-6 to 2^7 is 2^8 without asking, so one pass over
// the activations will do: a bf16 value is exact down to 2^-22 and what is lost below stays under
// 2^-27 of the largest.  Other tokens are converted again with a scale of their own: 8 tokens of 22016 x 4096 with an outlier of 500
// each 22.7 us instead of 19.1, one 14.8 instead of 14.4 (4096 x 11008: 12.0, 11.0).
constexpr float USUAL_SCALE = 256.f;
__device__ __forceinline__ bool usual(uint32_t top) { return top >= 0x3c800000u && top < 0x43000000u; }

// A span is four groups of a tile's K, BLOCKS blocks of 128 columns; a stage of the ring is one block or two.
template <int G>
struct Span {
  static constexpr int BLOCKS = G / 32, PER_STAGE = BLOCKS > 1 ? 2 : 1;
  static constexpr int STAGE = PER_STAGE * 2 * 512;  // bytes: [block][rows r, r + 8][lane] 16 bytes
};

// The rows of a tile that a lane reads, and where its share of their codes starts.
struct Rows {
  size_t a, b;  // rows r and r + 8 (the last row for those past it, which are not stored)
  __device__ __forceinline__ Rows(const FewParams& p, int tile, int r)
      : a(min(tile * FEATURES + r, p.w.N - 1)), b(min(tile * FEATURES + r + 8, p.w.N - 1)) {}
};

// The eight codes of a word in pairs (0,4), (1,5), (2,6), (3,7) as the smallest fp16 numbers, without a conversion: a
// nibble c at the end of a mantissa with exponent 0 is c CODE_UNIT, one at bit 4 is 16 c CODE_UNIT.
constexpr float CODE_UNIT = 1.f / 16777216.f;
__device__ __forceinline__ void codes_tiny(uint32_t w, uint32_t (&u)[4]) {
  const uint32_t h = w >> 8;
  u[0] = w & 0x000f000fu;
  u[1] = w & 0x00f000f0u;
  u[2] = h & 0x000f000fu;
  u[3] = h & 0x00f000f0u;
}
__device__ __forceinline__ uint32_t bf16_bits(uint32_t z) { return __float_as_uint(static_cast<float>(z)) & 0xffff0000u; }
__device__ __forceinline__ float2 half2_f(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

// Copies a lane's share of one stage: what a lane copies it alone reads, so the ring needs no barrier.
template <int G>
__device__ __forceinline__ void copy_stage(const FewParams& p, const Rows& rows, int block, int t, unsigned char* dst) {
  const int half = p.w.K / 2;
#pragma unroll
  for (int i = 0; i < Span<G>::PER_STAGE; ++i) {
    const int at = min((block + i) * 64 + t * 16, half - 16);  // past the end the activations are 0
    cp_async16(dst + i * 1024, p.w.W + rows.a * half + at);
    cp_async16(dst + i * 1024 + 512, p.w.W + rows.b * half + at);
  }
}

// Scale and zero of group lane % 4 of a span, both rows, as loaded (arithmetic here would wait for the load).
struct Scales {
  uint32_t sa, sb, za, zb;
  __device__ __forceinline__ void load(const FewParams& p, const Rows& rows, int span, int t) {
    const int g = min(span * 4 + t, p.groups - 1);
    const size_t ga = rows.a * p.groups + g, gb = rows.b * p.groups + g;
    sa = reinterpret_cast<const uint16_t*>(p.w.scale)[ga];
    sb = reinterpret_cast<const uint16_t*>(p.w.scale)[gb];
    za = zb = 8;
    if (p.w.zero) {
      za = p.w.zero[ga];
      zb = p.w.zero[gb];
    }
  }
};

// Words of 4 lanes (lane % 4 = t), 4 each, transposed in two halves: with both steps lane t gets word t of
// every lane's four, with the first alone (far) words 2 (t / 2), 2 (t / 2) + 1 of lanes t % 2 and t % 2 + 2.
__device__ __forceinline__ void swap_far(uint4& v, int t) {
  const bool up = t & 2;
  const uint32_t x = __shfl_xor_sync(0xffffffffu, up ? v.x : v.z, 2), y = __shfl_xor_sync(0xffffffffu, up ? v.y : v.w, 2);
  v = up ? make_uint4(x, y, v.z, v.w) : make_uint4(v.x, v.y, x, y);
}
__device__ __forceinline__ void swap_near(uint4& v, int t) {
  const bool up = t & 1;
  const uint32_t x = __shfl_xor_sync(0xffffffffu, up ? v.x : v.y, 1), y = __shfl_xor_sync(0xffffffffu, up ? v.z : v.w, 1);
  v = up ? make_uint4(x, v.y, y, v.w) : make_uint4(v.x, x, v.z, y);
}

template <int G, int TERMS, bool TINY>
__global__ void __launch_bounds__(THREADS, 1) w4_few_kernel(const __grid_constant__ FewParams p) {
  extern __shared__ __align__(128) unsigned char smem[];  // the warps' rings, activations, sums
  __shared__ uint32_t sh_top[FEW_TOKENS];
  constexpr int BLOCKS = Span<G>::BLOCKS;
  const W4Params& w = p.w;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, r = lane / 4, t = lane & 3;
  // this warp's stream: spans part, part + KS, .. of tiles first, first + step, ..
  const int part = warp % p.ks, per_cta = WARPS / p.ks, step = gridDim.x * per_cta;
  const int first = blockIdx.x + warp / p.ks * gridDim.x;
  // The launch before may still be writing the weights, so what comes first is only asked into L2.
  if (part == 0 && lane < FEATURES && first < p.tiles)
    prefetch_l2(w.W + static_cast<size_t>(min(first * FEATURES + lane, w.N - 1)) * (w.K / 2), w.K / 2);
  if (tid < FEW_TOKENS) sh_top[tid] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  unsigned char* ring = smem + warp * p.stages * Span<G>::STAGE + lane * 16;
  int ask_tile = first, ask_span = part, ask_sub = 0, ask_stage = 0;  // the next stage to copy
  auto ask = [&]() {
    if (ask_tile < p.tiles && ask_span < p.spans) {
      copy_stage<G>(p, Rows(p, ask_tile, r), ask_span * BLOCKS + ask_sub * Span<G>::PER_STAGE, t, ring + ask_stage * Span<G>::STAGE);
      ask_stage = ask_stage + 1 == p.stages ? 0 : ask_stage + 1;
      if (++ask_sub == BLOCKS / Span<G>::PER_STAGE) {
        ask_sub = 0;
        ask_span += p.ks;
        if (ask_span >= p.spans) {
          ask_span = part;
          ask_tile += step;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int i = 1; i < p.stages; ++i) ask();
  Scales next;
  if (first < p.tiles) next.load(p, Rows(p, first, r), part, t);

  // The activations, in the order in which the codes are multiplied: 128-column block, word of a thread,
  // thread, 8 values; zeros past the end.
  const int vecs = p.spans * 4 * G / 8;
  float* sums_x = reinterpret_cast<float*>(smem + p.at_sums_x);  // [group][token]
  auto place = [&](int m, int i, const float (&x)[8], float up) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) split_f16(x[j] * up, x[j + 4] * up, hi[j], lo[j]);
    const int from = i / 4 % 4, word = i % 4;  // the lane that loads this word, and its place there
    int th, at;                                // the lane that multiplies it, and its place there
    if (G == 128) {
      th = from, at = word;
    } else if (G == 64) {
      th = (from & 1) | (word & 2), at = (from & 2) | (word & 1);
    } else {
      th = word, at = from;
    }
    unsigned char* dst = smem + p.at_x + m * TERMS * p.x_pitch + i / 16 * 256 + (at * 4 + th) * 16;
    *reinterpret_cast<uint4*>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    if (TERMS == 2) *reinterpret_cast<uint4*>(dst + p.x_pitch) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    if (!TINY) return;
    // the group's sum, of what the matrix units will be given
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float2 f = half2_f(hi[j]);
      sum += f.x + f.y;
      if (TERMS == 2) {
        f = half2_f(lo[j]);
        sum += f.x + f.y;
      }
    }
    constexpr int LANES = G / 8;
    const uint32_t mask = ((1u << LANES) - 1u) << (lane & -LANES);
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor_sync(mask, sum, d);
    if (lane % LANES == 0) sums_x[i / LANES * FEW_TOKENS + m] = sum * CODE_UNIT;
  };
  // all tokens' in one sequence, AHEAD loads of a thread in flight
  constexpr int AHEAD = 2;
  for (int q0 = tid; q0 - lane < w.M * vecs; q0 += AHEAD * THREADS) {
    float x[AHEAD][8];
    int m[AHEAD], i[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const int q = q0 + a * THREADS;
      m[a] = q / vecs;
      i[a] = q - m[a] * vecs;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[a][j] = 0.f;
      if (m[a] < w.M && 8 * i[a] < w.K) load8(w, m[a], 8 * i[a], x[a]);
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const bool there = m[a] < w.M;
      if (there) place(m[a], i[a], x[a], USUAL_SCALE);
      const uint32_t mask = vecs % 32 == 0 ? 0xffffffffu : 0xffffu << (lane & 16);
      const uint32_t top = __reduce_max_sync(mask, there ? top_bits(x[a]) : 0u);
      if (there && (lane & (vecs % 32 == 0 ? 31 : 15)) == 0) atomicMax(sh_top + m[a], top);
    }
  }
  __syncthreads();
  bool again = false;
  for (int m = 0; m < w.M; ++m)
    if (!usual(sh_top[m])) {
      const float up = token_scale(sh_top[m]);
      for (int i = tid; i < vecs; i += THREADS) {
        float x[8] = {};
        if (8 * i < w.K) load8(w, m, 8 * i, x);
        place(m, i, x, up);
      }
      again = true;
    }
  if (again) __syncthreads();
  float down[2];  // of this thread's tokens
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t top = sh_top[min(2 * t + i, FEW_TOKENS - 1)];
    down[i] = 1.f / (usual(top) ? USUAL_SCALE : token_scale(top));
  }

  // columns past the last token repeat it, and are not stored
  const unsigned char* xs = smem + p.at_x + min(r, w.M - 1) * TERMS * p.x_pitch + t * 16;
  float4* sums = reinterpret_cast<float4*>(smem + p.at_sums);  // [tile][warp][row][pair of tokens]
  const int mine = r * p.pairs + t, line = 8 * p.pairs;
  int held = 0, first_tile = first;  // tiles whose sums are held, the first of them
  // joins the sums of the held tiles: warp j of the KS takes tiles j, j + KS, ..
  auto meet = [&]() {  // of the warps that share tiles
    if (p.ks > 1)
      named_bar(1 + warp / p.ks, p.ks * 32);
    else
      __syncwarp();
  };
  auto join = [&]() {
    meet();
    for (int j = part; j < held && t < p.pairs; j += p.ks) {
      const float4* from = sums + (j * WARPS + warp - part) * line + mine;
      float4 y = from[0];
      for (int i = 1; i < p.ks; ++i) {
        const float4 o = from[i * line];
        y = make_float4(y.x + o.x, y.y + o.y, y.z + o.z, y.w + o.w);
      }
      const int n = (first_tile + j * step) * FEATURES + r;
      const float v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (2 * t + (i & 1) < w.M && n + 8 * (i >> 1) < w.N) store_y(w, 2 * t + (i & 1), n + 8 * (i >> 1), v[i] * (TINY ? 1.f / CODE_UNIT : 1.f) * down[i & 1]);
    }
    meet();
    first_tile += held * step;
    held = 0;
  };
  int stage = 0;
  for (int tile = first; tile < p.tiles; tile += step) {
    float acc[4] = {};
    for (int span = part; span < p.spans; span += p.ks) {
      const Scales now = next;
      if (span + p.ks < p.spans)
        next.load(p, Rows(p, tile, r), span + p.ks, t);
      else if (tile + step < p.tiles)
        next.load(p, Rows(p, tile + step, r), part, t);
      const unsigned char* xb = xs + span * BLOCKS * 256;
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) {
        const unsigned char* src = ring + stage * Span<G>::STAGE + i % Span<G>::PER_STAGE * 1024;
        if (i % Span<G>::PER_STAGE == 0) {
          ask();
          // all but the stages asked for after this one
          if (p.stages >= 6) asm volatile("cp.async.wait_group 5;" ::: "memory");
          else if (p.stages >= 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
          else if (p.stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
          else asm volatile("cp.async.wait_group 1;" ::: "memory");
        }
        uint4 va = *reinterpret_cast<const uint4*>(src), vb = *reinterpret_cast<const uint4*>(src + 512);
        if (i % Span<G>::PER_STAGE == Span<G>::PER_STAGE - 1) stage = stage + 1 == p.stages ? 0 : stage + 1;
        if (G < 128) swap_far(va, t), swap_far(vb, t);
        if (G < 64) swap_near(va, t), swap_near(vb, t);
        const uint32_t a[4] = {va.x, va.y, va.z, va.w}, b[4] = {vb.x, vb.y, vb.z, vb.w};
        const uint32_t both_a = (TINY ? bf16_bits(now.za) : now.za << 16) | now.sa, both_b = (TINY ? bf16_bits(now.zb) : now.zb << 16) | now.sb;
        float sa, sb, za, zb, low[4], high[4];  // sums of products; with nibbles as they lie, high: of those that count 16 times
        float2 sum_x;
        uint32_t oa, oa16, ob, ob16;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          if (v % BLOCKS == 0) {  // a new group
            const int g = i * (4 / BLOCKS) + v / BLOCKS;
            const uint32_t ga = __shfl_sync(0xffffffffu, both_a, (lane & ~3) | g), gb = __shfl_sync(0xffffffffu, both_b, (lane & ~3) | g);
            sa = __uint_as_float(ga << 16), sb = __uint_as_float(gb << 16);
            if constexpr (TINY) {
              za = __uint_as_float(ga & 0xffff0000u), zb = __uint_as_float(gb & 0xffff0000u);
              sum_x = *reinterpret_cast<const float2*>(sums_x + (span * 4 + g) * FEW_TOKENS + 2 * t);
            } else {
              oa = zero_off(ga >> 16), oa16 = zero_off16(ga >> 16), ob = zero_off(gb >> 16), ob16 = zero_off16(gb >> 16);
            }
          }
          uint32_t ua[4], ub[4];
          if constexpr (TINY) {
            codes_tiny(a[v], ua);
            codes_tiny(b[v], ub);
          } else {
            w4_codes_f16(a[v], oa, oa16, ua);
            w4_codes_f16(b[v], ob, ob16, ub);
          }
#pragma unroll
          for (int s = 0; s < TERMS; ++s) {
            const uint4 x = *reinterpret_cast<const uint4*>(xb + i * 256 + s * p.x_pitch + v * 64);
            const bool fresh = v % BLOCKS == 0 && s == 0;
            if constexpr (TINY) {
              if (fresh) {
                mma_f16_first(low, ua[0], ub[0], ua[2], ub[2], x.x, x.z);
                mma_f16_first(high, ua[1], ub[1], ua[3], ub[3], x.y, x.w);
              } else {
                mma_f16(low, ua[0], ub[0], ua[2], ub[2], x.x, x.z);
                mma_f16(high, ua[1], ub[1], ua[3], ub[3], x.y, x.w);
              }
            } else {
              if (fresh)
                mma_f16_first(low, ua[0], ub[0], ua[1], ub[1], x.x, x.y);
              else
                mma_f16(low, ua[0], ub[0], ua[1], ub[1], x.x, x.y);
              mma_f16(low, ua[2], ub[2], ua[3], ub[3], x.z, x.w);
            }
          }
          if (v % BLOCKS == BLOCKS - 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (TINY) low[j] = fmaf(high[j], 0.0625f, fmaf(j < 2 ? -za : -zb, j & 1 ? sum_x.y : sum_x.x, low[j]));
              acc[j] = fmaf(j < 2 ? sa : sb, low[j], acc[j]);
            }
          }
        }
      }
    }
    if (t < p.pairs) sums[(held * WARPS + warp) * line + mine] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (++held == p.join) join();
  }
  if (held) join();
}

template <int G, int TERMS, bool TINY>
cudaError_t launch_few(const FewParams& p, size_t smem, int grid, cudaStream_t s) {
  const cudaError_t e = allow_smem<w4_few_kernel<G, TERMS, TINY>>(226 * 1024);
  return e != cudaSuccess ? e : launch_pdl(w4_few_kernel<G, TERMS, TINY>, dim3(grid), dim3(THREADS), smem, s, p);
}
template <int G>
cudaError_t launch_few_terms(const FewParams& p, size_t smem, int grid, cudaStream_t s) {
  const bool two = p.w.x_f32 || p.w.X_lo;
  if constexpr (G > 32)
    if (!p.w.out_f32) return two ? launch_few<G, 2, true>(p, smem, grid, s) : launch_few<G, 1, true>(p, smem, grid, s);
  return two ? launch_few<G, 2, false>(p, smem, grid, s) : launch_few<G, 1, false>(p, smem, grid, s);
}

// Shared memory of the plan, 0 when the activations do not fit.
size_t few_plan(FewParams* p, const W4Params& w, int* grid) {
  p->w = w;
  p->groups = (w.K + w.group - 1) / w.group;
  p->spans = (p->groups + 3) / 4;
  p->tiles = (w.N + FEATURES - 1) / FEATURES;
  p->x_pitch = p->spans * 4 * w.group * 2 + 64;  // two tokens' reads in different banks
  const int terms = w.x_f32 || w.X_lo ? 2 : 1, stage = WARPS * (w.group == 32 ? 1024 : 2048);
  p->pairs = (w.M + 1) / 2;
  *grid = std::min(p->tiles, tc_num_sms());
  // Warps per tile: as the spans of the busiest warp have it; the most of those that are equal (a tile's rows are
  // read at once: 22016 x 4096 15.2 us with 8, 16.6 with 2).
  const int mine = (p->tiles + *grid - 1) / *grid;  // tiles of a CTA
  int best = 1 << 30;
  for (int ks = 1; ks <= WARPS; ++ks) {
    if (WARPS % ks != 0) continue;
    const int rounds = (mine + WARPS / ks - 1) / (WARPS / ks);
    const int cost = rounds * ((p->spans + ks - 1) / ks);
    if (cost <= best) {
      best = cost;
      p->ks = ks;
      p->join = std::min(rounds, 8 / p->pairs);
    }
  }
  const int x_bytes = (w.M * terms * p->x_pitch + 127) / 128 * 128, sums_x = p->spans * 4 * FEW_TOKENS * 4, sums = p->join * WARPS * 8 * p->pairs * 16;
  const int fit = (226 * 1024 - x_bytes - sums_x - sums) / stage;
  if (fit < 2) return 0;
  p->stages = fit >= 6 ? 6 : fit >= 4 ? 4 : fit;
  p->at_x = p->stages * stage;
  p->at_sums_x = p->at_x + x_bytes;
  p->at_sums = p->at_sums_x + sums_x;
  return p->at_sums + sums;
}

}  // namespace

cudaError_t linear_w4(const W4Params& p, cudaStream_t s) {
  if (p.M <= FEW_TOKENS) {
    FewParams f{};
    int grid = 0;
    const size_t smem = few_plan(&f, p, &grid);
    if (smem) {
      return p.group == 128 ? launch_few_terms<128>(f, smem, grid, s)
                            : p.group == 64 ? launch_few_terms<64>(f, smem, grid, s) : launch_few_terms<32>(f, smem, grid, s);
    }
  }
  return linear_w4_many(p, s);
}

}  // namespace chimera
