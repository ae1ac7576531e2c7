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
#include <algorithm>

#include "kernels.h"
#include "kv4.cuh"
#include "launch.cuh"
#include "linear_w4.cuh"

namespace chimera {
namespace {

constexpr int WARPS = 8, FEATURES = 16;
// ---------------------------------------------------------------------------
// up to 8 tokens: one pass over the weights at the speed of memory
// ---------------------------------------------------------------------------
// A tile is 16 features; KS warps of a CTA share its K, by spans of four groups, and join their sums after
// JOIN tiles or at the end.  A lane copies (cp.async) into shared memory exactly what it will read itself, so a
// warp runs ahead of its loads with no barrier at all.  The activations stay in shared memory for
// the whole launch, as fp16 scaled by a power of two, hi + lo or fp32 ones as two fp16 terms
// (2^-23).  fp16 rather than bf16 because its ten bits of mantissa take a nibble in two
// places: 9 instructions for 8 codes, not 11.
//
// Measured (GB300, 22016 x 4096, group 128, one token, 47 MB): 16.3 us, 2.9 TB/s; the first kernel of this
// file 40.  Rings of bulk copies of 256 to 1024 bytes took 19.5 to 23, spans held in registers 17.7 (16
// warps per SM instead of 24).  Bound by the instructions that turn codes into numbers.
constexpr int FEW_TOKENS = 8, JOIN = 8;

struct FewParams {
  W4Params w;
  int groups, spans, tiles, ks;
  int stages;          // of a warp's ring
  int x_pitch;         // of a token's term
  int pairs;           // ceil(M / 2): lanes of a row that hold tokens
  int at_x, at_sums;   // offsets in shared memory
};

// The scale of a token whose largest magnitude is 2^-6 to 2^7 is 2^8 without asking, so one pass over
// the activations will do: a bf16 value is exact down to 2^-22 and what is lost below stays under
// 2^-27 of the largest.  Other tokens are converted again with a scale of their own.
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

template <int G, int TERMS>
__global__ void __launch_bounds__(WARPS * 32, 3) w4_few_kernel(const __grid_constant__ FewParams p) {
  extern __shared__ __align__(128) unsigned char smem[];  // the warps' rings, activations, sums
  __shared__ uint32_t sh_top[FEW_TOKENS];
  constexpr int BLOCKS = Span<G>::BLOCKS;
  const W4Params& w = p.w;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, r = lane / 4, t = lane & 3;
  if (tid < FEW_TOKENS) sh_top[tid] = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  // this warp's stream: spans part, part + KS, .. of tiles first, first + step, ..
  const int part = warp % p.ks, per_cta = WARPS / p.ks, step = gridDim.x * per_cta;
  const int first = blockIdx.x * per_cta + warp / p.ks;
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
  auto convert = [&](int m, float up, bool look) {
    uint32_t top = 0;
    for (int i = tid; i < vecs; i += WARPS * 32) {
      float x[8] = {};
      if (8 * i < w.K) load8(w, m, 8 * i, x);
      top = max(top, top_bits(x));
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
    }
    if (!look) return;
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) atomicMax(sh_top + m, top);
  };
  for (int m = 0; m < w.M; ++m) convert(m, USUAL_SCALE, true);
  __syncthreads();
  bool again = false;
  for (int m = 0; m < w.M; ++m)
    if (!usual(sh_top[m])) {
      convert(m, token_scale(sh_top[m]), false);
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
  float4* sums = reinterpret_cast<float4*>(smem + p.at_sums);  // [JOIN tiles][warp][row][pair of tokens]
  const int mine = r * p.pairs + t, line = 8 * p.pairs;
  int held = 0, first_tile = first;  // tiles whose sums are held, the first of them
  // joins the sums of the held tiles: warp j of the KS takes tiles j, j + KS, ..
  auto join = [&]() {
    named_bar(1 + warp / p.ks, p.ks * 32);
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
        if (2 * t + (i & 1) < w.M && n + 8 * (i >> 1) < w.N) store_y(w, 2 * t + (i & 1), n + 8 * (i >> 1), v[i] * down[i & 1]);
    }
    named_bar(1 + warp / p.ks, p.ks * 32);
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
        const uint32_t both_a = now.sa | now.za << 16, both_b = now.sb | now.zb << 16;
        uint32_t oa, oa16, ob, ob16;
        float sa, sb, d[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          if (v % BLOCKS == 0) {  // a new group
            const int g = i * (4 / BLOCKS) + v / BLOCKS;
            const uint32_t ga = __shfl_sync(0xffffffffu, both_a, (lane & ~3) | g), gb = __shfl_sync(0xffffffffu, both_b, (lane & ~3) | g);
            oa = zero_off(ga >> 16), oa16 = zero_off16(ga >> 16), ob = zero_off(gb >> 16), ob16 = zero_off16(gb >> 16);
            sa = __uint_as_float(ga << 16), sb = __uint_as_float(gb << 16);
          }
          uint32_t ua[4], ub[4];
          w4_codes_f16(a[v], oa, oa16, ua);
          w4_codes_f16(b[v], ob, ob16, ub);
#pragma unroll
          for (int s = 0; s < TERMS; ++s) {
            const uint4 x = *reinterpret_cast<const uint4*>(xb + i * 256 + s * p.x_pitch + v * 64);
            if (v % BLOCKS == 0 && s == 0)
              mma_f16_first(d, ua[0], ub[0], ua[1], ub[1], x.x, x.y);
            else
              mma_f16(d, ua[0], ub[0], ua[1], ub[1], x.x, x.y);
            mma_f16(d, ua[2], ub[2], ua[3], ub[3], x.z, x.w);
          }
          if (v % BLOCKS == BLOCKS - 1) {
            acc[0] = fmaf(sa, d[0], acc[0]);
            acc[1] = fmaf(sa, d[1], acc[1]);
            acc[2] = fmaf(sb, d[2], acc[2]);
            acc[3] = fmaf(sb, d[3], acc[3]);
          }
        }
      }
    }
    if (t < p.pairs) sums[(held * WARPS + warp) * line + mine] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (++held == JOIN) join();
  }
  if (held) join();
}

template <int G, int TERMS>
cudaError_t launch_few(const FewParams& p, size_t smem, int grid, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(w4_few_kernel<G, TERMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024);
  return e != cudaSuccess ? e : launch_pdl(w4_few_kernel<G, TERMS>, dim3(grid), dim3(WARPS * 32), smem, s, p);
}
template <int G>
cudaError_t launch_few_terms(const FewParams& p, size_t smem, int grid, cudaStream_t s) {
  return p.w.x_f32 || p.w.X_lo ? launch_few<G, 2>(p, smem, grid, s) : launch_few<G, 1>(p, smem, grid, s);
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
  const int x_bytes = (w.M * terms * p->x_pitch + 127) / 128 * 128, sums = JOIN * WARPS * 8 * p->pairs * 16;
  int per_sm = 3;
  for (; per_sm >= 1; --per_sm) {
    const int room = (per_sm == 3 ? 74 : per_sm == 2 ? 112 : 225) * 1024 - x_bytes - sums;
    const int fit = room > 0 ? room / stage : 0;
    p->stages = fit >= 6 ? 6 : fit >= 4 ? 4 : fit;
    if (p->stages >= (per_sm == 1 ? 2 : 3)) break;
  }
  if (per_sm < 1) return 0;
  p->at_x = p->stages * stage;
  p->at_sums = p->at_x + x_bytes;
  const size_t smem = p->at_sums + sums;
  const int slots = per_sm * tc_num_sms();
  // warps per tile: rounds of the launch times spans of a warp
  double best = 1e30;
  for (int ks = 1; ks <= WARPS; ks *= 2) {
    const int rounds = (p->tiles + slots * (WARPS / ks) - 1) / (slots * (WARPS / ks));
    const double cost = rounds * ((p->spans + ks - 1) / ks + 0.1);
    if (cost < best) {
      best = cost;
      p->ks = ks;
    }
  }
  const int per_cta = WARPS / p->ks;
  *grid = std::min((p->tiles + per_cta - 1) / per_cta, slots);
  return smem;
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
