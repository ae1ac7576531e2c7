// Attention over the 4-bit paged cache, and the attention weight that each cached row draws.
//
// With a row's codes c, step s and base b (kv4.cuh), and c' = c - 8, b' = b + 8 s:
//   z_j = q . k_j / sqrt(hd) = (s_j (q . c'_j) + b'_j sum(q)) / sqrt(hd)
//   o   = sum_j p_j v_j      = sum_j (p_j s_j) c'_j + sum_j p_j b'_j
// so both matrix products take the codes as whole fp16 numbers straight from the packed words.
// The factors that are no whole numbers enter as two fp16 terms, hi + lo (22 bits): a query row is
// first scaled by a power of two to a largest value in [16, 32), and p s by the largest step seen so
// far (a power of two above it).  The 16 rows of a matrix product are the hi and the lo terms of
// 8 query rows, and both terms of a row end in the same thread.
//
// A warp takes whole pages (16 keys).  Its copies are one bulk copy per page into a ring of its
// own, so no barrier joins the warps until the end; the shared-memory reads of the fragments
// have no bank conflicts by the page's layout.  Rows of all heads of a group and all queries are one
// list, cut into tiles of 8; the keys of a tile are cut into `splits` ranges, whose results
// the last block to finish merges in their order (no sum depends on who comes first).
#include "kernels.h"
#include "kv4.cuh"
#include "launch.cuh"

namespace chimera {
namespace {

constexpr int WARPS = 8, STAGES = 4, ROWS = 8;
constexpr float NONE = -1e30f;  // the reference of a row that has seen no key
constexpr float LOG2E = 1.4426950408889634f;
// Probabilities are taken relative to a reference 2^11 below a row's maximum, which is raised when a
// logit exceeds it by more than 15: weights of up to 2^15 leave the fp16 pairs an absolute error
// of 2^-36 of the largest (many keys of little weight add up to the result).
constexpr float BELOW = 11.f, SLACK = 15.f;
constexpr unsigned long long WAIT_NS = 2000000000ull;

template <int HD>
struct Smem {
  static constexpr int PAGE = Kv4<HD>::BYTES;
  static constexpr int RING = STAGES * PAGE;  // of a warp; later its 8 x HD sums
  static constexpr int BARS = WARPS * RING;
  static constexpr int ML = BARS + WARPS * STAGES * 8;  // maximum and sum of each warp's rows
  static constexpr int BYTES = ML + WARPS * ROWS * 8;
  static_assert(RING >= ROWS * HD * 4, "the sums reuse the ring");
};

__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}

// A fragments of 8 query rows: thread (r, t) = (lane / 4, lane % 4) holds channels
// [t HD/4, (t + 1) HD/4) of row r, paired as the K words' nibbles are.  scale: by what q . c'
// is multiplied to give base-2 logits; sum: of the row, times the same without the power of two.
template <int HD, typename TQ>
__device__ __forceinline__ void load_rows(const TQ* q, bool there, float softmax_scale, uint32_t (&f)[HD / 16][4], float& scale,
                                          float& sum) {
  constexpr int C = HD / 4;
  float x[C];
  float top = 0.f, s = 0.f;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    x[i] = there ? to_f<TQ>(q[i]) : 0.f;
    top = fmaxf(top, fabsf(x[i]));
    s += x[i];
  }
  top = quad_max(top);
  s = quad_sum(s);
  // 2^(4 - floor(log2 top)), at most 2^126
  const int e = static_cast<int>(__float_as_uint(top) >> 23);
  const int k = e == 0 || e == 255 ? 127 : min(254 - e + 4, 253);
  const float up = __uint_as_float(static_cast<uint32_t>(k) << 23);
  scale = softmax_scale / up;
  sum = s * softmax_scale;
#pragma unroll
  for (int j = 0; j < HD / 16; ++j) {
    const int at = j / 2 * 8 + 2 * (j & 1);
    split_f16(x[at] * up, x[at + 4] * up, f[j][0], f[j][1]);
    split_f16(x[at + 1] * up, x[at + 5] * up, f[j][2], f[j][3]);
  }
}

// q . c' of 8 rows (hi and lo) with the 16 keys of a page: s0 keys 2t, 2t + 1, s1 keys 8 + those.
template <int HD>
__device__ __forceinline__ void page_dots(const unsigned char* page, const uint32_t (&f)[HD / 16][4], int r, int t, float (&s0)[4],
                                          float (&s1)[4]) {
  constexpr int NW = HD / 32;  // words of a key per thread
  const uint32_t* k0 = reinterpret_cast<const uint32_t*>(page + r * Kv4<HD>::ROW) + t * NW;
  const uint32_t* k1 = k0 + 8 * Kv4<HD>::ROW / 4;
  uint32_t a[NW], b[NW];
  if (NW == 4) {
    *reinterpret_cast<uint4*>(a) = *reinterpret_cast<const uint4*>(k0);
    *reinterpret_cast<uint4*>(b) = *reinterpret_cast<const uint4*>(k1);
  } else {
    *reinterpret_cast<uint2*>(a) = *reinterpret_cast<const uint2*>(k0);
    *reinterpret_cast<uint2*>(b) = *reinterpret_cast<const uint2*>(k1);
  }
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    uint32_t u[4];
    kv4_codes(a[w], u);
    mma_f16(s0, f[2 * w][0], f[2 * w][1], f[2 * w][2], f[2 * w][3], u[0], u[1]);
    mma_f16(s0, f[2 * w + 1][0], f[2 * w + 1][1], f[2 * w + 1][2], f[2 * w + 1][3], u[2], u[3]);
    kv4_codes(b[w], u);
    mma_f16(s1, f[2 * w][0], f[2 * w][1], f[2 * w][2], f[2 * w][3], u[0], u[1]);
    mma_f16(s1, f[2 * w + 1][0], f[2 * w + 1][1], f[2 * w + 1][2], f[2 * w + 1][3], u[2], u[3]);
  }
}

// (step, base + 8 step) of the keys 2t, 2t + 1, 2t + 8, 2t + 9 of a page.
__device__ __forceinline__ void key_scales(const unsigned char* at, int t, float (&step)[4], float (&base)[4]) {
  const uint2 a = reinterpret_cast<const uint2*>(at)[t], b = reinterpret_cast<const uint2*>(at)[t + 4];
  const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    step[i] = kv4_step(w[i]);
    base[i] = fmaf(8.f, step[i], kv4_base(w[i]));
  }
}

// What a sequence's rows may see.
struct Seen {
  int n, total;  // committed rows, and all that hold a key
  unsigned long long local;  // the row's ancestors among the local rows
  __device__ __forceinline__ bool operator()(int slot) const {
    return slot < n || (slot < total && (local >> (slot - n) & 1));
  }
};

__device__ __forceinline__ Seen what_is_seen(const Kv4AttnParams& p, int b) {
  Seen s;
  int n = p.n_ctx[b];
  const int cap = p.c.max_pages * KV4_ROWS;
  if (n < 0 || n + p.n_local > cap) {
    if (threadIdx.x == 0) atomicOr(p.c.err, ERR_CAPACITY);
    n = min(max(n, 0), max(cap - p.n_local, 0));
  }
  s.n = n;
  s.total = min(n + p.n_local, cap);
  s.local = 0;
  return s;
}

// Block of the pool for page `at` of the sequence (block 0, with the error flagged, when the
// table names none).
__device__ __forceinline__ int block_of(const Kv4AttnParams& p, const int* table, int at) {
  const int block = table[at];
  if (block >= 0 && block < p.c.n_blocks) return block;
  atomicOr(p.c.err, ERR_BAD_INDEX);
  return 0;
}

template <typename T>
__device__ __forceinline__ void store_out(const Kv4AttnParams& p, size_t at, T v) {
  if (p.out_f32) {
    static_cast<float*>(p.out)[at] = v;
    return;
  }
  store_act(static_cast<bf16*>(p.out), reinterpret_cast<bf16*>(p.out_lo), at, v);
}

template <int HD, typename TQ>
__global__ void __launch_bounds__(WARPS * 32) attn_kv4_kernel(const __grid_constant__ Kv4AttnParams p) {
  extern __shared__ __align__(128) unsigned char smem[];
  using S = Smem<HD>;
  using P = Kv4<HD>;
  __shared__ int sh_abort, sh_last;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, r = lane / 4, t = lane & 3;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::BARS) + warp * STAGES;
  unsigned char* ring = smem + warp * S::RING;
  if (tid == 0) sh_abort = 0;
  if (lane == 0) {
    for (int i = 0; i < STAGES; ++i) mbar_init(bars + i, 1);
    mbar_fence_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  const int group = p.H / p.c.G, n_rows = p.nq * group, tiles = (n_rows + ROWS - 1) / ROWS;
  const int bg = blockIdx.y / tiles, tile = blockIdx.y % tiles, b = bg / p.c.G, g = bg % p.c.G;
  Seen seen = what_is_seen(p, b);
  const int row = tile * ROWS + r;
  const bool there = row < n_rows;
  const int qi = there ? row / group : 0, head = g * group + (there ? row % group : 0);
  if (there && p.n_local) seen.local = p.anc[p.q_local0 + qi];

  // the pages of this block, dealt to its warps in turn
  const int pages = (seen.total + KV4_ROWS - 1) / KV4_ROWS;
  const int split = blockIdx.x, splits = gridDim.x;
  const int p0 = static_cast<int>(static_cast<long long>(pages) * split / splits);
  const int p1 = static_cast<int>(static_cast<long long>(pages) * (split + 1) / splits);
  const int mine = max(0, (p1 - p0 - warp + WARPS - 1) / WARPS);
  const int* table = p.c.table + static_cast<size_t>(b) * p.c.max_pages;
  auto request = [&](int k) {  // lane 0: page p0 + warp + k WARPS into its place of the ring
    const int block = block_of(p, table, p0 + warp + k * WARPS);
    uint64_t* bar = bars + k % STAGES;
    mbar_arrive_expect_tx(bar, P::BYTES);
    bulk_load(ring + k % STAGES * P::BYTES, p.c.pool + (static_cast<size_t>(block) * p.c.G + g) * P::BYTES, P::BYTES, bar);
  };
  if (lane == 0)
    for (int k = 0; k < min(mine, STAGES); ++k) request(k);

  uint32_t qf[HD / 16][4];
  float q_scale, q_sum;
  load_rows<HD, TQ>(static_cast<const TQ*>(p.q) + (static_cast<size_t>(b) * p.q_rows + qi) * p.ldq + head * HD + t * (HD / 4), there,
                    p.scale * LOG2E, qf, q_scale, q_sum);

  float o[HD / 8][4] = {};
  float m = NONE, l = 0.f, bs = 0.f;     // l and bs: this thread's keys alone
  float top = 0x1p-126f, inv_top = 0x1p126f;  // power of two above every V step so far
  for (int k = 0; k < mine; ++k) {
    if (!mbar_wait_warp(bars + k % STAGES, k / STAGES & 1, &sh_abort, WAIT_NS)) {
      // pages still in flight land before the block leaves
      for (int i = k; i < min(mine, k + STAGES); ++i) mbar_wait_plain(bars + i % STAGES, i / STAGES & 1, WAIT_NS);
      if (lane == 0) atomicOr(p.c.err, ERR_TIMEOUT);
      break;
    }
    const unsigned char* page = ring + k % STAGES * P::BYTES;
    float s0[4] = {}, s1[4] = {};
    page_dots<HD>(page, qf, r, t, s0, s1);
    float step[4], base[4], z[4];
    key_scales(page + P::KS, t, step, base);
    z[0] = fmaf(step[0] * q_scale, s0[0] + s0[2], base[0] * q_sum);
    z[1] = fmaf(step[1] * q_scale, s0[1] + s0[3], base[1] * q_sum);
    z[2] = fmaf(step[2] * q_scale, s1[0] + s1[2], base[2] * q_sum);
    z[3] = fmaf(step[3] * q_scale, s1[1] + s1[3], base[3] * q_sum);
    key_scales(page + P::VS, t, step, base);
    const int slot0 = (p0 + warp + k * WARPS) * KV4_ROWS;
    if (slot0 + KV4_ROWS > seen.n) {  // a hidden key counts nothing, whatever its codes and steps are
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!seen(slot0 + 2 * t + (i & 1) + 8 * (i >> 1))) {
          z[i] = -INFINITY;
          step[i] = 0.f;
          base[i] = 0.f;
        }
    }
    const float zmax = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
    const float smax = fmaxf(fmaxf(step[0], step[1]), fmaxf(step[2], step[3]));
    if (__any_sync(0xffffffffu, zmax > m + SLACK || smax > top)) {
      float wide = smax;
#pragma unroll
      for (int s = 16; s; s >>= 1) wide = fmaxf(wide, __shfl_xor_sync(0xffffffffu, wide, s));
      float shrink = 1.f;
      if (wide > top) {
        const uint32_t e = min((__float_as_uint(wide) >> 23) + 1, 252u);
        const float was = top;
        top = __uint_as_float(e << 23);
        inv_top = __uint_as_float((254 - e) << 23);
        shrink = was * inv_top;
      }
      const float raised = fmaxf(m, quad_max(zmax) - BELOW);
      const float a = exp2f(m - raised);
      m = raised;
      l *= a;
      bs *= a;
#pragma unroll
      for (int j = 0; j < HD / 8; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][i] *= a * shrink;
      }
    }
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float e = exp2f(z[i] - m);
      l += e;
      bs = fmaf(e, base[i], bs);
      w[i] = e * (step[i] * inv_top);
    }
    uint32_t h0, l0, h1, l1;
    split_f16(w[0], w[1], h0, l0);
    split_f16(w[2], w[3], h1, l1);
    // V: row pairs t and t + 4, channels [CHUNK r, CHUNK (r + 1))
    constexpr int NV = HD / 32;
    uint32_t va[NV], vb[NV];
    const unsigned char* v0 = page + P::V + t * 2 * P::ROW + P::place(t, r) * P::CHUNK;
    const unsigned char* v1 = page + P::V + (t + 4) * 2 * P::ROW + P::place(t + 4, r) * P::CHUNK;
    if (NV == 4) {
      *reinterpret_cast<uint4*>(va) = *reinterpret_cast<const uint4*>(v0);
      *reinterpret_cast<uint4*>(vb) = *reinterpret_cast<const uint4*>(v1);
    } else {
      *reinterpret_cast<uint2*>(va) = *reinterpret_cast<const uint2*>(v0);
      *reinterpret_cast<uint2*>(vb) = *reinterpret_cast<const uint2*>(v1);
    }
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      uint32_t u[4], x[4];
      kv4_codes(va[c], u);
      kv4_codes(vb[c], x);
#pragma unroll
      for (int i = 0; i < 4; ++i) mma_f16(o[4 * c + i], h0, l0, h1, l1, u[i], x[i]);
    }
    __syncwarp();
    if (lane == 0 && k + STAGES < mine) request(k + STAGES);
  }

  // rows of the warp: column c of sums [r][HD], over the ring (all of its pages have been read)
  l = quad_sum(l);
  bs = quad_sum(bs);
  float* sums = reinterpret_cast<float*>(ring);
  float* ml = reinterpret_cast<float*>(smem + S::ML);
  __syncwarp();
#pragma unroll
  for (int j = 0; j < HD / 8; ++j) {
    sums[r * HD + 2 * t * P::CHUNK + j] = fmaf(o[j][0] + o[j][2], top, bs);
    sums[r * HD + (2 * t + 1) * P::CHUNK + j] = fmaf(o[j][1] + o[j][3], top, bs);
  }
  if (t == 0) {
    ml[(warp * ROWS + r) * 2] = m;
    ml[(warp * ROWS + r) * 2 + 1] = l;
  }
  __syncthreads();

  // the block's rows: warp r merges row r over the warps
  const int my = warp;
  const int mrow = tile * ROWS + my;
  float M = NONE, L = 0.f, f[WARPS];
#pragma unroll
  for (int w = 0; w < WARPS; ++w) M = fmaxf(M, ml[(w * ROWS + my) * 2]);
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    f[w] = exp2f(ml[(w * ROWS + my) * 2] - M);
    L = fmaf(f[w], ml[(w * ROWS + my) * 2 + 1], L);
  }
  float acc[HD / 32];
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    acc[i] = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w)
      acc[i] = fmaf(f[w], reinterpret_cast<const float*>(smem + w * S::RING)[my * HD + lane + 32 * i], acc[i]);
  }
  if (splits > 1) {
    constexpr int LINE = HD + 2;
    float* ws = p.ws + (static_cast<size_t>(blockIdx.y) * splits * ROWS) * LINE;
    float* line = ws + (split * ROWS + my) * LINE;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) line[lane + 32 * i] = acc[i];
    if (lane == 0) {
      line[HD] = M;
      line[HD + 1] = L;
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      const int seen_before = atomicAdd(p.counters + blockIdx.y, 1);
      sh_last = seen_before == splits - 1;
      if (sh_last) p.counters[blockIdx.y] = 0;
    }
    __syncthreads();
    if (!sh_last) return;
    __threadfence();
    M = NONE;
    for (int s = 0; s < splits; ++s) M = fmaxf(M, __ldcg(ws + (s * ROWS + my) * LINE + HD));
    L = 0.f;
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) acc[i] = 0.f;
    for (int s = 0; s < splits; ++s) {
      const float* part = ws + (s * ROWS + my) * LINE;
      const float e = exp2f(__ldcg(part + HD) - M);
      L = fmaf(e, __ldcg(part + HD + 1), L);
#pragma unroll
      for (int i = 0; i < HD / 32; ++i) acc[i] = fmaf(e, __ldcg(part + lane + 32 * i), acc[i]);
    }
  }
  if (mrow >= n_rows) return;
  const int oi = mrow / group, oh = g * group + mrow % group;
  const size_t orow = static_cast<size_t>(b) * p.q_rows + oi;
  const float inv = L == 0.f ? 0.f : 1.f / L;  // a row that sees nothing gives zeros
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) store_out(p, orow * p.ldo + oh * HD + lane + 32 * i, acc[i] * inv);
  if (p.lse && lane == 0) p.lse[orow * p.H + oh] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------
// attention weight per cached row
// ---------------------------------------------------------------------------
constexpr int SCORE_TILES = 8;  // row tiles whose fragments are held in shared memory at a time

template <int HD>
struct ScoreSmem {
  static constexpr int PAGE = KV4_ROWS * HD / 2 + 4 * KV4_ROWS;  // K codes and scales
  static constexpr int RING = STAGES * PAGE;
  static constexpr int BARS = WARPS * RING;
  static constexpr int FRAGS = BARS + WARPS * STAGES * 8;     // [tile][HD / 16][lane] 16 bytes
  static constexpr int ROWF = FRAGS + SCORE_TILES * HD / 16 * 32 * 16;  // [tile][8 rows] (scale, sum, lse, weight)
  static constexpr int LOCAL = ROWF + SCORE_TILES * ROWS * 16;          // [tile][8 rows] ancestors
  static constexpr int BYTES = LOCAL + SCORE_TILES * ROWS * 8;
};

template <int HD, typename TQ>
__global__ void __launch_bounds__(WARPS * 32) score_kv4_kernel(const __grid_constant__ Kv4AttnParams p) {
  extern __shared__ __align__(128) unsigned char smem[];
  using S = ScoreSmem<HD>;
  using P = Kv4<HD>;
  __shared__ int sh_abort;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, r = lane / 4, t = lane & 3;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + S::BARS) + warp * STAGES;
  unsigned char* ring = smem + warp * S::RING;
  if (tid == 0) sh_abort = 0;
  if (lane == 0) {
    for (int i = 0; i < STAGES; ++i) mbar_init(bars + i, 1);
    mbar_fence_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  const int group = p.H / p.c.G, n_rows = p.nq * group, tiles = (n_rows + ROWS - 1) / ROWS;
  const int bg = blockIdx.y, b = bg / p.c.G, g = bg % p.c.G;
  const Seen all = what_is_seen(p, b);
  const int pages = (min(all.total, p.ld_scores) + KV4_ROWS - 1) / KV4_ROWS;
  if (all.total > p.ld_scores && tid == 0) atomicOr(p.c.err, ERR_CAPACITY);
  const int split = blockIdx.x, splits = gridDim.x;
  const int p0 = static_cast<int>(static_cast<long long>(pages) * split / splits);
  const int p1 = static_cast<int>(static_cast<long long>(pages) * (split + 1) / splits);
  const int mine = max(0, (p1 - p0 - warp + WARPS - 1) / WARPS);
  const int* table = p.c.table + static_cast<size_t>(b) * p.c.max_pages;
  float* scores = p.scores + static_cast<size_t>(bg) * p.ld_scores;
  int used = 0;  // stages taken since the start
  bool ok = true;
  for (int tile0 = 0; tile0 < tiles; tile0 += SCORE_TILES) {
    const int held = min(SCORE_TILES, tiles - tile0);
    auto request = [&](int k) {
      const int block = block_of(p, table, p0 + warp + k * WARPS);
      uint64_t* bar = bars + (used + k) % STAGES;
      unsigned char* dst = ring + (used + k) % STAGES * S::PAGE;
      const unsigned char* src = p.c.pool + (static_cast<size_t>(block) * p.c.G + g) * P::BYTES;
      mbar_arrive_expect_tx(bar, S::PAGE);
      bulk_load(dst, src, P::V, bar);
      bulk_load(dst + P::V, src + P::KS, 4 * KV4_ROWS, bar);
    };
    if (lane == 0 && ok)
      for (int k = 0; k < min(mine, STAGES); ++k) request(k);
    __syncthreads();  // every warp has left the fragments of the tiles before
    for (int i = warp; i < held; i += WARPS) {
      const int row = (tile0 + i) * ROWS + r;
      const bool there = row < n_rows;
      const int qi = there ? row / group : 0, head = g * group + (there ? row % group : 0);
      uint32_t f[HD / 16][4];
      float scale, sum;
      load_rows<HD, TQ>(static_cast<const TQ*>(p.q) + (static_cast<size_t>(b) * p.q_rows + qi) * p.ldq + head * HD + t * (HD / 4),
                        there, p.scale * LOG2E, f, scale, sum);
#pragma unroll
      for (int j = 0; j < HD / 16; ++j)
        reinterpret_cast<uint4*>(smem + S::FRAGS)[(i * (HD / 16) + j) * 32 + lane] = make_uint4(f[j][0], f[j][1], f[j][2], f[j][3]);
      if (t == 0) {
        const size_t qrow = static_cast<size_t>(b) * p.q_rows + qi;
        const float lse = there ? p.lse[qrow * p.H + head] * LOG2E : 0.f;
        const float weight = there ? (p.weight ? p.weight[qrow] : 1.f) : 0.f;
        reinterpret_cast<float4*>(smem + S::ROWF)[i * ROWS + r] = make_float4(scale, sum, lse, weight);
        reinterpret_cast<unsigned long long*>(smem + S::LOCAL)[i * ROWS + r] = there && p.n_local ? p.anc[p.q_local0 + qi] : 0;
      }
    }
    __syncthreads();
    for (int k = 0; ok && k < mine; ++k) {
      const int at = used + k;
      if (!mbar_wait_warp(bars + at % STAGES, at / STAGES & 1, &sh_abort, WAIT_NS)) {
        for (int i = at; i < used + min(mine, k + STAGES); ++i) mbar_wait_plain(bars + i % STAGES, i / STAGES & 1, WAIT_NS);
        if (lane == 0) atomicOr(p.c.err, ERR_TIMEOUT);
        ok = false;
        break;
      }
      const unsigned char* page = ring + at % STAGES * S::PAGE;
      float step[4], base[4], sum[4] = {};
      key_scales(page + P::V, t, step, base);
      const int slot0 = (p0 + warp + k * WARPS) * KV4_ROWS;
      const bool whole = slot0 + KV4_ROWS <= all.n;
      for (int i = 0; i < held; ++i) {
        uint32_t f[HD / 16][4];
#pragma unroll
        for (int j = 0; j < HD / 16; ++j)
          *reinterpret_cast<uint4*>(f[j]) = reinterpret_cast<const uint4*>(smem + S::FRAGS)[(i * (HD / 16) + j) * 32 + lane];
        float s0[4] = {}, s1[4] = {};
        page_dots<HD>(page, f, r, t, s0, s1);
        const float4 rf = reinterpret_cast<const float4*>(smem + S::ROWF)[i * ROWS + r];
        Seen seen = all;
        if (!whole) seen.local = reinterpret_cast<const unsigned long long*>(smem + S::LOCAL)[i * ROWS + r];
        const float d[4] = {s0[0] + s0[2], s0[1] + s0[3], s1[0] + s1[2], s1[1] + s1[3]};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float z = fmaf(step[x] * rf.x, d[x], base[x] * rf.y);
          if (rf.w != 0.f && (whole || seen(slot0 + 2 * t + (x & 1) + 8 * (x >> 1)))) sum[x] = fmaf(rf.w, exp2f(z - rf.z), sum[x]);
        }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) sum[x] += __shfl_xor_sync(0xffffffffu, sum[x], s);
        const int slot = slot0 + 2 * t + (x & 1) + 8 * (x >> 1);
        if (r == x && slot < all.total && slot < p.ld_scores) scores[slot] += sum[x];
      }
      __syncwarp();
      if (lane == 0 && k + STAGES < mine) request(k + STAGES);
    }
    used += mine;
  }
}

template <typename K>
cudaError_t launch_sized(K kernel, size_t smem, dim3 grid, const Kv4AttnParams& p, cudaStream_t s) {
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  return e != cudaSuccess ? e : launch_pdl(kernel, grid, dim3(WARPS * 32), smem, s, p);
}

}  // namespace

int kv4_attn_row_tiles(int nq, int H, int G) { return (nq * (H / G) + ROWS - 1) / ROWS; }

int kv4_attn_splits(const Kv4AttnParams& p) {
  const int tiles = kv4_attn_row_tiles(p.nq, p.H, p.c.G) * p.c.B * p.c.G;
  const int want = (2 * tc_num_sms() + tiles - 1) / tiles;
  const int most = (p.c.max_pages + WARPS - 1) / WARPS;
  return want < 1 ? 1 : want > most ? most : want > 64 ? 64 : want;
}

size_t kv4_attn_ws_floats(const Kv4AttnParams& p) {
  return static_cast<size_t>(kv4_attn_row_tiles(p.nq, p.H, p.c.G)) * p.c.B * p.c.G * p.splits * ROWS * (p.c.hd + 2);
}

cudaError_t attention_kv4(const Kv4AttnParams& p, cudaStream_t s) {
  const dim3 grid(p.splits, kv4_attn_row_tiles(p.nq, p.H, p.c.G) * p.c.B * p.c.G);
  if (p.c.hd == 128)
    return p.q_f32 ? launch_sized(attn_kv4_kernel<128, float>, Smem<128>::BYTES, grid, p, s)
                   : launch_sized(attn_kv4_kernel<128, bf16>, Smem<128>::BYTES, grid, p, s);
  return p.q_f32 ? launch_sized(attn_kv4_kernel<64, float>, Smem<64>::BYTES, grid, p, s)
                 : launch_sized(attn_kv4_kernel<64, bf16>, Smem<64>::BYTES, grid, p, s);
}

cudaError_t kv4_score(const Kv4AttnParams& p, cudaStream_t s) {
  const int bg = p.c.B * p.c.G;
  int splits = (2 * tc_num_sms() + bg - 1) / bg;
  const int most = (p.c.max_pages + WARPS - 1) / WARPS;
  splits = splits > most ? most : splits;
  const dim3 grid(splits, bg);
  if (p.c.hd == 128)
    return p.q_f32 ? launch_sized(score_kv4_kernel<128, float>, ScoreSmem<128>::BYTES, grid, p, s)
                   : launch_sized(score_kv4_kernel<128, bf16>, ScoreSmem<128>::BYTES, grid, p, s);
  return p.q_f32 ? launch_sized(score_kv4_kernel<64, float>, ScoreSmem<64>::BYTES, grid, p, s)
                 : launch_sized(score_kv4_kernel<64, bf16>, ScoreSmem<64>::BYTES, grid, p, s);
}

}  // namespace chimera
