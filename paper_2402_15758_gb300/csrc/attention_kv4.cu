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
#include <algorithm>

#include "kernels.h"
#include "kv4.cuh"
#include "launch.cuh"

namespace chimera {
namespace {

constexpr int WARPS = 4;
constexpr float NONE = -1e30f;  // the reference of a row that has seen no key
constexpr float LOG2E = 1.4426950408889634f;
// Probabilities are taken relative to a reference 2^11 below a row's maximum, which is raised when a
// logit exceeds it by more than 15: weights of up to 2^15 leave the fp16 pairs an absolute error
// of 2^-36 of the largest (many keys of little weight add up to the result).
constexpr float BELOW = 11.f, SLACK = 15.f;
constexpr unsigned long long WAIT_NS = 2000000000ull;

// 2^x, relative error 2^-22; results below 2^-126 are 0.
__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}

// 2^(4 - floor(log2 top)), at most 2^126 (1 for 0 and what is not finite).
__device__ __forceinline__ float row_scale(float top) {
  const int e = static_cast<int>(__float_as_uint(top) >> 23);
  return __uint_as_float(static_cast<uint32_t>(e == 0 || e == 255 ? 127 : min(258 - e, 253)) << 23);
}

// HD / 4 consecutive values, 16 bytes at a time where they are aligned.
template <int HD>
__device__ __forceinline__ void load_quarter(const float* q, float (&x)[HD / 4]) {
  if ((reinterpret_cast<uintptr_t>(q) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) *reinterpret_cast<float4*>(x + 4 * i) = reinterpret_cast<const float4*>(q)[i];
  } else {
#pragma unroll
    for (int i = 0; i < HD / 4; ++i) x[i] = q[i];
  }
}
template <int HD>
__device__ __forceinline__ void load_quarter(const bf16* q, float (&x)[HD / 4]) {
#pragma unroll
  for (int i = 0; i < HD / 4; ++i) x[i] = __bfloat162float(q[i]);
}

// A thread's quarter of a query row (channels [t HD/4, (t + 1) HD/4), t = lane % 4).  scale: by what the products of
// the scaled row are multiplied to give base-2 logits; sum: of the row, times the same without the power of two.
template <int HD, typename TQ>
__device__ __forceinline__ void load_row(const TQ* q, bool there, float softmax_scale, float (&x)[HD / 4], float& scale, float& sum) {
  float top = 0.f, s[4] = {};
  if (there) load_quarter<HD>(q, x);
#pragma unroll
  for (int i = 0; i < HD / 4; ++i) {
    x[i] = there ? x[i] : 0.f;
    top = fmaxf(top, fabsf(x[i]));
    s[i % 4] += x[i];
  }
  const float up = row_scale(quad_max(top));
  scale = softmax_scale / up;
  sum = quad_sum((s[0] + s[1]) + (s[2] + s[3])) * softmax_scale;
#pragma unroll
  for (int i = 0; i < HD / 4; ++i) x[i] *= up;
}

// A fragments of 8 query rows, hi and lo terms (the 16 rows of a product): thread (r, t) holds row r, paired
// as the K words' nibbles are.
template <int HD, typename TQ>
__device__ __forceinline__ void load_rows(const TQ* q, bool there, float softmax_scale, uint32_t (&f)[HD / 16][4], float& scale,
                                          float& sum) {
  float x[HD / 4];
  load_row<HD, TQ>(q, there, softmax_scale, x, scale, sum);
#pragma unroll
  for (int j = 0; j < HD / 16; ++j) {
    const int at = j / 2 * 8 + 2 * (j & 1);
    split_f16(x[at], x[at + 4], f[j][0], f[j][1]);
    split_f16(x[at + 1], x[at + 5], f[j][2], f[j][3]);
  }
}

__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
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
  for (int i = 0; i < 4; ++i) s0[i] = s1[i] = 0.f;
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

// Writes a merged row (of the rows of a sequence and kv head) from its sums in shared memory.
template <int HD>
__device__ __forceinline__ void store_row(const Kv4AttnParams& p, int bg, int row, int lane, float M, float L, const float* sums) {
  const int group = p.H / p.c.G, head = bg % p.c.G * group + row % group;
  const size_t out = static_cast<size_t>(bg / p.c.G) * p.q_rows + row / group;
  const float inv = L == 0.f ? 0.f : 1.f / L;  // a row that sees nothing gives zeros
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    const int c = lane + 32 * i;
    store_out(p, out * p.ldo + head * HD + c, sums[c % Kv4<HD>::CHUNK * 8 + c / Kv4<HD>::CHUNK] * inv);
  }
  if (p.lse && lane == 0) p.lse[out * p.H + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

// What a block's warps do: RTW tiles of rows times WARPS / RTW slices of the pages.  PRECISE: tiles of 8 rows in two
// terms; else 16 rows in one (2^-12 of a query and of a weight, a tenth of the rounding of a bf16 result).
template <int HD, bool PRECISE, int RTW>
struct Shape {
  static constexpr int TILE = PRECISE ? 8 : 16, ROWS = TILE * RTW, SLICES = WARPS / RTW;
  static constexpr int STAGES = 8;  // pages of a slice: four pairs
  static constexpr int RING = STAGES * Kv4<HD>::BYTES;
  static constexpr int PITCH = HD + 8;  // of a row of sums: in the order of the products' columns
  static constexpr int SUMS = WARPS * TILE * PITCH * 4;  // over the rings
  static constexpr int BARS = SLICES * RING > SUMS ? SLICES * RING : SUMS;
  static constexpr int ML = BARS + SLICES * STAGES * 16;  // reference and sum of each warp's rows
  static constexpr int BYTES = ML + WARPS * TILE * 8;
};

template <int HD, typename TQ, bool PRECISE, int RTW>
__global__ void __launch_bounds__(WARPS * 32, 3) attn_kv4_kernel(const __grid_constant__ Kv4AttnParams p) {
  extern __shared__ __align__(128) unsigned char smem[];
  using S = Shape<HD, PRECISE, RTW>;
  using P = Kv4<HD>;
  constexpr int TILE = S::TILE, NR = PRECISE ? 1 : 2, STAGES = S::STAGES;  // NR: rows of a thread
  __shared__ int sh_abort;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31, r = lane / 4, t = lane & 3;
  const int rt = warp % RTW, slice = warp / RTW;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::BARS) + slice * 2 * STAGES;
  uint64_t* empty = full + STAGES;
  unsigned char* ring = smem + slice * S::RING;
  if (tid == 0) sh_abort = 0;
  if (lane == 0 && rt == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, RTW);
    }
    mbar_fence_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();

  const int group = p.H / p.c.G, n_rows = p.nq * group, blocks = (n_rows + S::ROWS - 1) / S::ROWS;
  const int bg = blockIdx.y / blocks, row0 = blockIdx.y % blocks * S::ROWS, b = bg / p.c.G, g = bg % p.c.G;
  const Seen all = what_is_seen(p, b);

  // the pages of this block, dealt to its slices in turn
  const int pages = (all.total + KV4_ROWS - 1) / KV4_ROWS;
  const int split = blockIdx.x, splits = gridDim.x;
  const int p0 = static_cast<int>(static_cast<long long>(pages) * split / splits);
  const int p1 = static_cast<int>(static_cast<long long>(pages) * (split + 1) / splits);
  const int mine = max(0, (p1 - p0 - slice + S::SLICES - 1) / S::SLICES);
  const int* table = p.c.table + static_cast<size_t>(b) * p.c.max_pages;
  int asked = 0;
  auto request = [&]() {  // one lane: the next page into its place of the ring
    const int block = block_of(p, table, p0 + slice + asked * S::SLICES), stage = asked % STAGES;
    mbar_arrive_expect_tx(full + stage, P::BYTES);
    bulk_load(ring + stage * P::BYTES, p.c.pool + (static_cast<size_t>(block) * p.c.G + g) * P::BYTES, P::BYTES, full + stage);
    ++asked;
  };
  if (lane == 0 && rt == 0)
    while (asked < min(mine, STAGES - 2)) request();

  uint32_t qf[HD / 16][4];
  float q_scale[NR], q_sum[NR];
  unsigned long long local[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int row = row0 + rt * TILE + r + 8 * i;
    const bool there = row < n_rows;
    const int qi = there ? row / group : 0, head = g * group + (there ? row % group : 0);
    local[i] = there && p.n_local ? p.anc[p.q_local0 + qi] : 0;
    const TQ* q = static_cast<const TQ*>(p.q) + (static_cast<size_t>(b) * p.q_rows + qi) * p.ldq + head * HD + t * (HD / 4);
    if constexpr (PRECISE) {
      load_rows<HD, TQ>(q, there, p.scale * LOG2E, qf, q_scale[i], q_sum[i]);
    } else {
      float x[HD / 4];
      load_row<HD, TQ>(q, there, p.scale * LOG2E, x, q_scale[i], q_sum[i]);
#pragma unroll
      for (int j = 0; j < HD / 16; ++j) {
        const int at = j / 2 * 8 + 2 * (j & 1);
        qf[j][i] = pack_f16(x[at], x[at + 4]);
        qf[j][2 + i] = pack_f16(x[at + 1], x[at + 5]);
      }
    }
  }

  float o[HD / 8][4] = {};
  float m[NR], l[NR], bs[NR];  // l and bs: this thread's keys alone
#pragma unroll
  for (int i = 0; i < NR; ++i) m[i] = NONE, l[i] = bs[i] = 0.f;
  float top = 0x1p-126f, inv_top = 0x1p126f;  // power of two above every V step so far
  // The products of a pair with the queries are taken one pair ahead, so that they overlap the softmax before.
  int stage = 0;  // of the pair whose products come next
  uint32_t phase = 0;
  float dots[2][2][4], ahead[2][2][4];  // [page][keys 0..7, 8..15]
  bool ok = true;
  auto products = [&](int k, float (&d)[2][2][4]) {
    const bool two = k + 1 < mine;
    ok = mbar_wait_warp(full + stage, phase, &sh_abort, WAIT_NS) && (!two || mbar_wait_warp(full + stage + 1, phase, &sh_abort, WAIT_NS));
    if (!ok) return;
    page_dots<HD>(ring + stage * P::BYTES, qf, r, t, d[0][0], d[0][1]);
    page_dots<HD>(ring + (stage + (two ? 1 : 0)) * P::BYTES, qf, r, t, d[1][0], d[1][1]);
    stage += 2;
    if (stage == STAGES) {
      stage = 0;
      phase ^= 1;
    }
  };
  if (mine > 0) products(0, dots);
  for (int k = 0; ok && k < mine; k += 2) {
    const bool two = k + 1 < mine;
    const int now = k % STAGES;  // stage of this pair
    if (k + 2 < mine) products(k + 2, ahead);
    if (!ok) break;
    const unsigned char* page[2] = {ring + now * P::BYTES, ring + (now + (two ? 1 : 0)) * P::BYTES};
    float z[2][NR][4], step[2][4], base[2][4];
    float zmax[NR], smax = 0.f;
#pragma unroll
    for (int i = 0; i < NR; ++i) zmax[i] = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      key_scales(page[h] + P::KS, t, step[h], base[h]);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float* s = dots[h][j / 2];
          const float d = PRECISE ? s[j % 2] + s[2 + j % 2] : s[2 * i + j % 2];
          z[h][i][j] = fmaf(step[h][j] * q_scale[i], d, base[h][j] * q_sum[i]);
        }
      }
      key_scales(page[h] + P::VS, t, step[h], base[h]);
      const int slot0 = (p0 + slice + (k + h) * S::SLICES) * KV4_ROWS;
      if (slot0 + KV4_ROWS > all.n || (h && !two)) {  // a hidden key counts nothing, whatever its codes and steps are
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int slot = slot0 + 2 * t + (j & 1) + 8 * (j >> 1);
          const bool held = slot < all.total && !(h && !two);
          if (!held) step[h][j] = base[h][j] = 0.f;
#pragma unroll
          for (int i = 0; i < NR; ++i)
            if (!held || (slot >= all.n && !(local[i] >> (slot - all.n) & 1))) z[h][i][j] = -INFINITY;
        }
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) zmax[i] = fmaxf(zmax[i], fmaxf(fmaxf(z[h][i][0], z[h][i][1]), fmaxf(z[h][i][2], z[h][i][3])));
      smax = fmaxf(smax, fmaxf(fmaxf(step[h][0], step[h][1]), fmaxf(step[h][2], step[h][3])));
    }
    bool raise = smax > top;
#pragma unroll
    for (int i = 0; i < NR; ++i) raise = raise || zmax[i] > m[i] + SLACK;
    if (__any_sync(0xffffffffu, raise)) {
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
      float a[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float raised = fmaxf(m[i], quad_max(zmax[i]) - BELOW);
        a[i] = exp2f(m[i] - raised);
        m[i] = raised;
        l[i] *= a[i];
        bs[i] *= a[i];
        a[i] *= shrink;
      }
#pragma unroll
      for (int j = 0; j < HD / 8; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][i] *= a[PRECISE ? 0 : i / 2];
      }
    }
    uint32_t wf[2][4];  // the weights as A fragments
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float e = pow2(z[h][i][j] - m[i]);
          l[i] += e;
          bs[i] = fmaf(e, base[h][j], bs[i]);
          w[j] = e * (step[h][j] * inv_top);
        }
        if (PRECISE) {
          split_f16(w[0], w[1], wf[h][0], wf[h][1]);
          split_f16(w[2], w[3], wf[h][2], wf[h][3]);
        } else {
          wf[h][i] = pack_f16(w[0], w[1]);
          wf[h][2 + i] = pack_f16(w[2], w[3]);
        }
      }
    }
    // V: row pairs t and t + 4, channels [CHUNK r, CHUNK (r + 1))
    constexpr int NV = HD / 32;
    uint32_t v[2][2][NV];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const unsigned char* at = page[h] + P::V + (t + 4 * i) * 2 * P::ROW + P::place(t + 4 * i, r) * P::CHUNK;
        if (NV == 4)
          *reinterpret_cast<uint4*>(v[h][i]) = *reinterpret_cast<const uint4*>(at);
        else
          *reinterpret_cast<uint2*>(v[h][i]) = *reinterpret_cast<const uint2*>(at);
      }
    }
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      uint32_t u[4], x[4];
      float d[4][4];
      kv4_codes(v[0][0][c], u);
      kv4_codes(v[0][1][c], x);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // the tensor cores round their sums toward zero: in a chain over all pages that is a bias
        if (PRECISE)
          mma_f16_first(d[i], wf[0][0], wf[0][1], wf[0][2], wf[0][3], u[i], x[i]);
        else
          mma_f16(o[4 * c + i], wf[0][0], wf[0][1], wf[0][2], wf[0][3], u[i], x[i]);
      }
      kv4_codes(v[1][0][c], u);
      kv4_codes(v[1][1][c], x);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (PRECISE) {
          mma_f16(d[i], wf[1][0], wf[1][1], wf[1][2], wf[1][3], u[i], x[i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) o[4 * c + i][j] += d[i][j];
        } else {
          mma_f16(o[4 * c + i], wf[1][0], wf[1][1], wf[1][2], wf[1][3], u[i], x[i]);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < 8; ++i) dots[h][i / 4][i % 4] = ahead[h][i / 4][i % 4];
    }
    __syncwarp();
    if (RTW > 1 && lane == 0) {
      mbar_arrive(empty + now);
      mbar_arrive(empty + now + 1);
    }
    // the pair after the next two, into the places of the pair before this one
    if (lane == 0 && rt == 0 && asked < mine) {
      for (int i = 0; i < 2 && asked < mine; ++i) {
        const int at = asked % STAGES;
        if (RTW > 1 && asked >= STAGES && !mbar_wait(empty + at, (asked / STAGES - 1) & 1, &sh_abort, WAIT_NS)) break;
        request();
      }
    }
    __syncwarp();
  }
  if (!ok && lane == 0) atomicOr(p.c.err, ERR_TIMEOUT);

  // the block's sums, over the rings: channel CHUNK n + j of a row at 8 j + n
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    l[i] = quad_sum(l[i]);
    bs[i] = quad_sum(bs[i]);
  }
  if (lane == 0 && rt == 0 && sh_abort)  // copies still in flight land before the rings are used again
    for (int i = max(0, asked - STAGES); i < asked; ++i) mbar_wait_plain(full + i % STAGES, i / STAGES & 1, WAIT_NS);
  float* ml = reinterpret_cast<float*>(smem + S::ML);
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem) + warp * TILE * S::PITCH;
#pragma unroll
  for (int j = 0; j < HD / 8; ++j) {
#pragma unroll
    for (int i = 0; i < NR; ++i)
      *reinterpret_cast<float2*>(sums + (r + 8 * i) * S::PITCH + 8 * j + 2 * t) =
          make_float2(fmaf(PRECISE ? o[j][0] + o[j][2] : o[j][2 * i], top, bs[i]),
                      fmaf(PRECISE ? o[j][1] + o[j][3] : o[j][2 * i + 1], top, bs[i]));
  }
#pragma unroll
  for (int i = 0; i < NR; ++i)
    if (t == 0) {
      ml[(warp * TILE + r + 8 * i) * 2] = m[i];
      ml[(warp * TILE + r + 8 * i) * 2 + 1] = l[i];
    }
  __syncthreads();

  constexpr int LINE = HD + 4;
  float* ws = p.ws + static_cast<size_t>(blockIdx.y) * splits * S::ROWS * LINE;
  const int here = min(S::ROWS, n_rows - row0);
  for (int my = warp; my < here; my += WARPS) {  // a warp merges a row over the slices
    const int w0 = my / TILE, at = my % TILE;
    constexpr int W = HD / 32;
    float M = NONE, L = 0.f, f[S::SLICES], acc[W] = {};
    float* mine = reinterpret_cast<float*>(smem) + (w0 * TILE + at) * S::PITCH + W * lane;
#pragma unroll
    for (int w = 0; w < S::SLICES; ++w) M = fmaxf(M, ml[((w0 + w * RTW) * TILE + at) * 2]);
#pragma unroll
    for (int w = 0; w < S::SLICES; ++w) {
      f[w] = exp2f(ml[((w0 + w * RTW) * TILE + at) * 2] - M);
      L = fmaf(f[w], ml[((w0 + w * RTW) * TILE + at) * 2 + 1], L);
#pragma unroll
      for (int i = 0; i < W; ++i) acc[i] = fmaf(f[w], mine[w * RTW * TILE * S::PITCH + i], acc[i]);
    }
    if (splits == 1) {
#pragma unroll
      for (int i = 0; i < W; ++i) mine[i] = acc[i];
      __syncwarp();
      store_row<HD>(p, bg, row0 + my, lane, M, L, mine - W * lane);
      continue;
    }
    float* line = ws + (split * S::ROWS + my) * LINE;
    if constexpr (W == 4)
      *reinterpret_cast<float4*>(line + W * lane) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    else
      *reinterpret_cast<float2*>(line + W * lane) = make_float2(acc[0], acc[1]);
    if (lane == 0) {
      line[HD] = M;
      line[HD + 1] = L;
    }
  }
}

// Merges the splits of a row: four warps take every fourth split, and their sums are added in the warps' order.  (By the
// last block of the tile to arrive, 64 rows of 15 splits took longer than the attention itself.)
template <int HD>
__global__ void __launch_bounds__(128) join_kv4_kernel(const __grid_constant__ Kv4AttnParams p, int rows, int blocks) {
  constexpr int LINE = HD + 4, W = HD / 32;  // W: columns of a lane
  __shared__ float sh_acc[4][HD];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, n_rows = p.nq * (p.H / p.c.G);
  const int bg = static_cast<int>(blockIdx.x / n_rows), row = static_cast<int>(blockIdx.x % n_rows), splits = p.splits;
  const float* ws = p.ws + (static_cast<size_t>(bg * blocks + row / rows) * splits * rows + row % rows) * LINE;
  const size_t step = static_cast<size_t>(rows) * LINE;
  // reference and sum of split lane, and of split 32 + lane
  float m[2], l[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bool there = lane + 32 * i < splits;
    m[i] = there ? ws[(lane + 32 * i) * step + HD] : NONE;
    l[i] = there ? ws[(lane + 32 * i) * step + HD + 1] : 0.f;
  }
  float acc[W] = {};
  constexpr int ONCE = 4;
  float v[ONCE][W];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int i = 0; i < ONCE; ++i) {
      const float* part = ws + min(s0 + 4 * i, splits - 1) * step + W * lane;
      if constexpr (W == 4)
        *reinterpret_cast<float4*>(v[i]) = *reinterpret_cast<const float4*>(part);
      else
        *reinterpret_cast<float2*>(v[i]) = *reinterpret_cast<const float2*>(part);
    }
  };
  fetch(warp);
  float M = fmaxf(m[0], m[1]);
#pragma unroll
  for (int s = 16; s; s >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, s));
  const float f[2] = {exp2f(m[0] - M), exp2f(m[1] - M)};
  float L = fmaf(f[0], l[0], f[1] * l[1]);
#pragma unroll
  for (int s = 16; s; s >>= 1) L += __shfl_xor_sync(0xffffffffu, L, s);
  for (int s0 = warp; s0 < splits; s0 += 4 * ONCE) {
    if (s0 != warp) fetch(s0);
#pragma unroll
    for (int i = 0; i < ONCE; ++i) {
      const int s = s0 + 4 * i;
      const float e = __shfl_sync(0xffffffffu, s & 32 ? f[1] : f[0], s & 31);
      if (s >= splits) break;
#pragma unroll
      for (int j = 0; j < W; ++j) acc[j] = fmaf(e, v[i][j], acc[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < W; ++j) sh_acc[warp][W * lane + j] = acc[j];
  __syncthreads();
  if (warp) return;
#pragma unroll
  for (int j = 0; j < W; ++j)
    sh_acc[0][lane + 32 * j] = (sh_acc[0][lane + 32 * j] + sh_acc[1][lane + 32 * j]) + (sh_acc[2][lane + 32 * j] + sh_acc[3][lane + 32 * j]);
  __syncwarp();
  store_row<HD>(p, bg, row, lane, M, L, sh_acc[0]);
}

// ---------------------------------------------------------------------------
// attention weight per cached row
// ---------------------------------------------------------------------------
constexpr int STAGES = 4, ROWS = 8;
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
  __shared__ int sh_abort, sh_queries, sh_query[64];
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

  const int group = p.H / p.c.G, bg = blockIdx.y, b = bg / p.c.G, g = bg % p.c.G;
  // the queries that count
  if (warp == 0) {
    int found = 0;
    for (int i = lane; i < (p.nq + 31) / 32 * 32; i += 32) {
      const bool counts = i < p.nq && (!p.weight || p.weight[static_cast<size_t>(b) * p.q_rows + i] != 0.f);
      const uint32_t all = __ballot_sync(0xffffffffu, counts);
      if (counts) sh_query[found + __popc(all & ((1u << lane) - 1))] = i;
      found += __popc(all);
    }
    if (lane == 0) sh_queries = found;
  }
  __syncthreads();
  const int n_rows = sh_queries * group, tiles = (n_rows + ROWS - 1) / ROWS;
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
      const int qi = there ? sh_query[row / group] : 0, head = g * group + (there ? row % group : 0);
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
      // the page's codes, unpacked once for all tiles
      constexpr int NW = HD / 32;
      uint32_t codes[2][NW][4];
      {
        uint32_t k[2][NW];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const unsigned char* at = page + (r + 8 * h) * P::ROW + t * 4 * NW;
          if (NW == 4)
            *reinterpret_cast<uint4*>(k[h]) = *reinterpret_cast<const uint4*>(at);
          else
            *reinterpret_cast<uint2*>(k[h]) = *reinterpret_cast<const uint2*>(at);
#pragma unroll
          for (int w = 0; w < NW; ++w) kv4_codes(k[h][w], codes[h][w]);
        }
      }
#pragma unroll 2
      for (int i = 0; i < held; ++i) {
        float s[2][4];
#pragma unroll
        for (int j = 0; j < HD / 16; ++j) {
          const uint4 f = reinterpret_cast<const uint4*>(smem + S::FRAGS)[(i * (HD / 16) + j) * 32 + lane];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (j == 0)
              mma_f16_first(s[h], f.x, f.y, f.z, f.w, codes[h][0][0], codes[h][0][1]);
            else
              mma_f16(s[h], f.x, f.y, f.z, f.w, codes[h][j / 2][j % 2 * 2], codes[h][j / 2][j % 2 * 2 + 1]);
          }
        }
        const float4 rf = reinterpret_cast<const float4*>(smem + S::ROWF)[i * ROWS + r];
        Seen seen = all;
        if (!whole) seen.local = reinterpret_cast<const unsigned long long*>(smem + S::LOCAL)[i * ROWS + r];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float z = fmaf(step[x] * rf.x, s[x / 2][x % 2] + s[x / 2][2 + x % 2], base[x] * rf.y);
          if (rf.w != 0.f && (whole || seen(slot0 + 2 * t + (x & 1) + 8 * (x >> 1)))) sum[x] = fmaf(rf.w, pow2(z - rf.z), sum[x]);
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

// How a call's rows are cut: one term per query where the result is rounded to bf16 alone and there are rows
// enough to fill its tiles, and warps that share pages when there are several tiles.
namespace {
struct Cut {
  bool precise;
  int rtw, rows;  // tiles at a time, rows of a block
};
Cut cut_of(const Kv4AttnParams& p) {
  const int rows = p.nq * (p.H / p.c.G);
  const bool precise = rows <= 8 || p.out_f32 || p.out_lo || p.lse;
  const int tile = precise ? 8 : 16, tiles = (rows + tile - 1) / tile;
  const int rtw = tiles == 1 ? 1 : tiles == 2 ? 2 : 4;
  return Cut{precise, rtw, tile * rtw};
}
int blocks_of(const Kv4AttnParams& p) {
  const Cut c = cut_of(p);
  return (p.nq * (p.H / p.c.G) + c.rows - 1) / c.rows * p.c.B * p.c.G;
}
}  // namespace

int kv4_attn_blocks(const Kv4AttnParams& p) { return blocks_of(p); }

int kv4_attn_splits(const Kv4AttnParams& p) {
  const Cut c = cut_of(p);
  const int blocks = blocks_of(p), pairs = (p.c.max_pages + 2 * WARPS / c.rtw - 1) / (2 * WARPS / c.rtw);
  const int want = 3 * tc_num_sms() / blocks;  // three blocks per SM, and none left for a second wave
  return std::max(1, std::min(std::min(want, pairs), 64));
}

size_t kv4_attn_ws_floats(const Kv4AttnParams& p) {
  return static_cast<size_t>(blocks_of(p)) * p.splits * cut_of(p).rows * (p.c.hd + 4);
}

namespace {
template <int HD, typename TQ, bool PRECISE, int RTW>
cudaError_t launch_attn(const Kv4AttnParams& p, cudaStream_t s) {
  const int blocks = blocks_of(p);
  const cudaError_t e = launch_sized(attn_kv4_kernel<HD, TQ, PRECISE, RTW>, Shape<HD, PRECISE, RTW>::BYTES, dim3(p.splits, blocks), p, s);
  if (e != cudaSuccess || p.splits == 1) return e;
  const long long rows = static_cast<long long>(p.nq) * p.c.B * p.H;
  return launch_pdl(join_kv4_kernel<HD>, dim3(static_cast<unsigned>(rows)), dim3(128), 0, s, p, Shape<HD, PRECISE, RTW>::ROWS,
                    blocks / (p.c.B * p.c.G));
}
template <int HD, typename TQ>
cudaError_t launch_cut(const Kv4AttnParams& p, cudaStream_t s) {
  const Cut c = cut_of(p);
  if (c.precise)
    return c.rtw == 1 ? launch_attn<HD, TQ, true, 1>(p, s) : c.rtw == 2 ? launch_attn<HD, TQ, true, 2>(p, s) : launch_attn<HD, TQ, true, 4>(p, s);
  return c.rtw == 1 ? launch_attn<HD, TQ, false, 1>(p, s) : c.rtw == 2 ? launch_attn<HD, TQ, false, 2>(p, s) : launch_attn<HD, TQ, false, 4>(p, s);
}
}  // namespace

cudaError_t attention_kv4(const Kv4AttnParams& p, cudaStream_t s) {
  if (p.c.hd == 128) return p.q_f32 ? launch_cut<128, float>(p, s) : launch_cut<128, bf16>(p, s);
  return p.q_f32 ? launch_cut<64, float>(p, s) : launch_cut<64, bf16>(p, s);
}

cudaError_t kv4_score(const Kv4AttnParams& p, cudaStream_t s) {
  const int bg = p.c.B * p.c.G;
  const int most = (p.c.max_pages + WARPS - 1) / WARPS;
  const dim3 grid(std::max(1, std::min(4 * tc_num_sms() / bg, most)), bg);  // four blocks per SM
  if (p.c.hd == 128)
    return p.q_f32 ? launch_sized(score_kv4_kernel<128, float>, ScoreSmem<128>::BYTES, grid, p, s)
                   : launch_sized(score_kv4_kernel<128, bf16>, ScoreSmem<128>::BYTES, grid, p, s);
  return p.q_f32 ? launch_sized(score_kv4_kernel<64, float>, ScoreSmem<64>::BYTES, grid, p, s)
                 : launch_sized(score_kv4_kernel<64, bf16>, ScoreSmem<64>::BYTES, grid, p, s);
}

}  // namespace chimera
