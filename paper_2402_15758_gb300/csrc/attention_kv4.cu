// Attention over the 4-bit paged cache, and the attention weight that each cached row draws.
//
// With a row's codes c, step s and base b (kv4.cuh), and c' = c - 8, b' = b + 8 s:
//   z_j = q . k_j / sqrt(hd) = (s_j (q . c'_j) + b'_j sum(q)) / sqrt(hd)
//   o   = sum_j p_j v_j      = sum_j (p_j s_j) c'_j + sum_j p_j b'_j
// so both matrix products take the codes as whole fp16 numbers straight from the packed words.
// The factors that are no whole numbers enter as fp16 terms: a query row is first scaled by a power of two to a largest
// value in [16, 32) and is two terms, hi + lo (22 bits); p s is divided by a power of two of the row's own (UNITS below)
// and is two terms, or one where the result is rounded to bf16 anyway (Shape).  Of two terms, the 16 rows of
// a matrix product are those of 8 query rows, and both terms of a row end in the same thread.
//
// A warp takes whole pages (16 keys).  Its copies are one bulk copy per page into a ring of its own (or of the
// warps that share the pages), so no barrier joins the warps until the end; the shared-memory reads of the fragments
// have no bank conflicts by the page's layout.  Rows of all heads of a group and all queries are one list,
// cut into blocks of 8 to 64; the pages are cut into parts, whose results the parts' cluster or a second kernel adds in
// their order (no sum depends on who comes first).
//
// Measured (GB300, hd 128, times of calls in a graph): 1 query of 32 heads over 512 rows 6.7 us (the launch, one trip to
// memory after another, the join); over 16384 rows 30 us, 2.4 TB/s of 71 MB, bound by the instructions that turn codes
// into numbers; 64 queries of 32 heads over 16384 rows 105 us, with weights in two terms 153: the tensor pipe is active
// 45 % of the time (40 %) and an instruction issued in 41 % (48 %); two warps per scheduler, 250 registers each, wait for
// one another's results.  The attention over a hi + lo cache in 16 bits takes 84 us for these 64 queries (540 MB); the 4-bit one
// is the faster up to 16 queries: 30 us and 80 for 1, 41 to 45 and 81 for 16.
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
// UNITS.  A row's sums are held in a power of two of its own, at least LEAST_UNIT.  It is above every step that the row
// has seen (then p s stays below 2^15), unless that is more than 16 times its largest p s: a key of little weight takes
// the others no bits, however large its values are.  What a row does not see takes no part in it.  Bases count as steps 2^-40
// times as large, which only those of equal or enormous values notice.
constexpr float LEAST_UNIT = 0x1p-96f;  // (weights over units stay within fp32)
__device__ __forceinline__ float step_size(float step, float base) { return fmaxf(step, 0x1p-40f * fabsf(base)); }
constexpr unsigned long long WAIT_NS = 2000000000ull;

// 2^x, relative error 2^-22; results below 2^-126 are 0.
__device__ __forceinline__ float pow2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 1 / x of a power of two from 2^-126 to 2^126.
__device__ __forceinline__ float one_over(uint32_t bits) { return __uint_as_float(0x7f000000u - bits); }
__device__ __forceinline__ float one_over(float x) { return one_over(__float_as_uint(x)); }
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

// Of sequence b, within what its page table holds; `fits` says whether n_ctx was.
__device__ __forceinline__ Seen rows_of(const Kv4AttnParams& p, int b, bool& fits) {
  const int cap = p.c.max_pages * KV4_ROWS, n = p.n_ctx[b];
  Seen s;
  fits = n >= 0 && n <= cap - p.n_local;  // (a sum with any n_ctx could pass 32 bits)
  s.n = fits ? n : min(max(n, 0), max(cap - p.n_local, 0));
  s.total = min(s.n + p.n_local, cap);
  s.local = 0;
  return s;
}
__device__ __forceinline__ Seen what_is_seen(const Kv4AttnParams& p, int b) {
  bool fits;
  const Seen s = rows_of(p, b, fits);
  if (!fits && threadIdx.x == 0) atomicOr(p.c.err, ERR_CAPACITY);
  return s;
}

// How a batch of sequences of different lengths is cut (p.slots > 0): the slots of the grid go to the sequences by
// their pages, in parts of about as many pages each.  Lane b holds sequence b's parts and its first slot.  Where all
// have the same number of parts the longest sequence sets the time (8 sequences, 1 query, 32 kv heads of 128,
// 100 to 4000 rows: 63.7 us, dealt 38.8; 32 sequences of 8 kv heads 51.4, dealt 36.5); batches of equal lengths
// lose what the dealing takes (8 of 2000 rows: 39.7 us, dealt 42.7).
constexpr int DEAL_MOST = 32, PARTS_MOST = 64;  // sequences, parts of one
constexpr int CLUSTER_MOST = 8;  // parts that meet in a cluster
struct Deal {
  int parts, first;
};
__device__ __forceinline__ Deal deal_slots(const Kv4AttnParams& p, int lane) {
  int pages = 0;
  bool inside;
  if (lane < p.c.B) pages = (rows_of(p, lane, inside).total + KV4_ROWS - 1) / KV4_ROWS;
  const int total = __reduce_add_sync(0xffffffffu, pages);
  // lane c tries the c-th size of a part; the smallest with slots enough for all is taken (or one part each)
  const float size = fmaxf(static_cast<float>(total) / p.slots, static_cast<float>(p.least_pages)) * (1.f + lane / 16.f + lane * lane / 64.f);
  float inverse = 1.f / size;
  auto parts_of = [](int pages, float inverse) { return min(max(__float2int_ru(pages * inverse), 1), PARTS_MOST); };
  int sum = 0;
#pragma unroll 8
  for (int b = 0; b < p.c.B; ++b) sum += parts_of(__shfl_sync(0xffffffffu, pages, b), inverse);
  const uint32_t fits = __ballot_sync(0xffffffffu, sum <= p.slots);
  inverse = fits ? __shfl_sync(0xffffffffu, inverse, __ffs(fits) - 1) : 0.f;
  Deal d;
  d.parts = lane < p.c.B ? parts_of(pages, inverse) : 0;
  d.first = d.parts;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int before = __shfl_up_sync(0xffffffffu, d.first, o);
    if (lane >= o) d.first += before;
  }
  d.first -= d.parts;
  return d;
}

// The sequence of a slot of the grid, which becomes its part of the sequence's `splits`.
__device__ __forceinline__ int sequence_of(const Deal& d, int& slot, int& splits) {
  const int b = __popc(__ballot_sync(0xffffffffu, d.parts > 0 && d.first <= slot)) - 1;
  slot -= __shfl_sync(0xffffffffu, d.first, b);
  splits = __shfl_sync(0xffffffffu, d.parts, b);
  return b;
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

// What a block's warps do: RTW tiles of rows times WARPS / RTW slices of the pages.  A warp multiplies NM matrices of 16
// rows with every page that it unpacks: the hi and lo terms of 8 rows (PRECISE), or 16 rows whose queries take two
// products and whose weights have one term (2^-12 of a weight, a sixteenth of the rounding of a bf16 result; a
// query in one term would cost 2^-12 of a logit, which for logits of 20 is as much as that rounding).
template <int HD, bool PRECISE, int NM, int RTW>
struct Shape {
  static constexpr int TILE = NM * (PRECISE ? 8 : 16), ROWS = TILE * RTW, SLICES = WARPS / RTW;
  static constexpr int PAGES = NM == 1 ? 2 : 1;  // of a round: with one matrix two pages, for the overlap
  static constexpr int STAGES = 6;               // pages of a slice
  static constexpr int RING = STAGES * Kv4<HD>::BYTES;
  static constexpr int PITCH = HD + 8;  // of a row of sums: in the order of the products' columns
  static constexpr int SUMS = WARPS * TILE * PITCH * 4;  // over the rings
  static constexpr int BARS = SLICES * RING > SUMS ? SLICES * RING : SUMS;
  static constexpr int ML = BARS + SLICES * STAGES * 16;  // reference and sum of each warp's rows
  // The queries stay in registers, or in shared memory: [tile][matrix][term][HD / 16][lane] 16 bytes.
  static constexpr bool HELD = PRECISE && NM == 1;
  static constexpr int TERMS = PRECISE ? 1 : 2;
  static constexpr int FRAGS = ML + WARPS * TILE * 8;
  static constexpr int PEAKS = FRAGS + (HELD ? 0 : RTW * NM * TERMS * (HD / 16) * 512);
  static constexpr int BYTES = PEAKS + WARPS * 32 * NM * (PRECISE ? 1 : 2) * 4;  // of a thread's rows
};

// Where the parts of a sequence meet: in a second kernel (and there are as many of each sequence, or they are dealt by
// length), or, up to eight whose blocks are resident at once, in the cluster that these form: 1 query over 512 rows
// 6.7 us instead of 7.3 on the device, and with one launch less 6.8 instead of 8.4 in the host's call.
enum Parts { EQUAL, DEALT, CLUSTER };

template <int HD, typename TQ, bool PRECISE, int NM, int RTW, Parts PARTS>
__global__ void __launch_bounds__(WARPS * 32, NM == 1 && PRECISE && PARTS != CLUSTER ? 3 : 2) attn_kv4_kernel(const __grid_constant__ Kv4AttnParams p) {
  extern __shared__ __align__(128) unsigned char smem[];
  using S = Shape<HD, PRECISE, NM, RTW>;
  using P = Kv4<HD>;
  constexpr int TILE = S::TILE, STAGES = S::STAGES, PAGES = S::PAGES, TERMS = S::TERMS, NW = HD / 32;
  constexpr int RM = PRECISE ? 1 : 2, NR = NM * RM;  // rows of a thread: of a matrix, in all
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
  const int bg0 = blockIdx.y / blocks, row0 = blockIdx.y % blocks * S::ROWS, g = bg0 % p.c.G;
  int b = bg0 / p.c.G, split = blockIdx.x, splits = gridDim.x;
  if (PARTS == DEALT) {
    const Deal d = deal_slots(p, lane);
    b = sequence_of(d, split, splits);
    if (split >= splits) return;  // (the whole block; a slot that is left over)
  }
  const int bg = b * p.c.G + g;
  const Seen all = what_is_seen(p, b);

  // the pages of this block, dealt to its slices in turn
  const int pages = (all.total + KV4_ROWS - 1) / KV4_ROWS;
  const int p0 = static_cast<int>(static_cast<long long>(pages) * split / splits);
  const int p1 = static_cast<int>(static_cast<long long>(pages) * (split + 1) / splits);
  const int mine = max(0, (p1 - p0 - slice + S::SLICES - 1) / S::SLICES);
  // The blocks of the next 32 pages, one per lane, and of the 32 after them: a request that read its own table entry
  // would hold its warp for a trip to L2.
  const int* table = p.c.table + static_cast<size_t>(b) * p.c.max_pages + p0 + slice;
  auto entries = [&](int k) { return k + lane < mine ? block_of(p, table, (k + lane) * S::SLICES) : 0; };
  int blocks_now = 0, blocks_next = 0;
  if (rt == 0) blocks_now = entries(0), blocks_next = entries(32);
  int asked = 0, ask_stage = 0;
  uint32_t ask_phase = 1;  // parity of the stage's last release
  auto request = [&]() {   // the warp: the next page into its place of the ring
    const int block = __shfl_sync(0xffffffffu, blocks_now, asked & 31);
    if (lane == 0) {
      mbar_arrive_expect_tx(full + ask_stage, P::BYTES);
      bulk_load(ring + ask_stage * P::BYTES, p.c.pool + (static_cast<size_t>(block) * p.c.G + g) * P::BYTES, P::BYTES, full + ask_stage);
    }
    if ((++asked & 31) == 0) {
      blocks_now = blocks_next;
      blocks_next = entries(asked + 32);
    }
    if (++ask_stage == STAGES) {
      ask_stage = 0;
      ask_phase ^= 1;
    }
  };
  if (rt == 0)
    while (asked < min(mine, STAGES - PAGES)) request();

  uint32_t qf[S::HELD ? HD / 16 : 1][4];
  uint4* frags = reinterpret_cast<uint4*>(smem + S::FRAGS) + rt * NM * TERMS * (HD / 16) * 32 + lane;
  float q_scale[NR], q_sum[NR];
  unsigned long long local[NR];
#pragma unroll
  for (int x = 0; x < NM; ++x) {
    uint32_t f[TERMS][HD / 16][4];
#pragma unroll
    for (int i = 0; i < RM; ++i) {
      const int row = row0 + rt * TILE + x * (PRECISE ? 8 : 16) + r + 8 * i;
      const bool there = row < n_rows;
      const int qi = there ? row / group : 0, head = g * group + (there ? row % group : 0), at = x * RM + i;
      local[at] = there && p.n_local ? p.anc[p.q_local0 + qi] : 0;
      const TQ* q = static_cast<const TQ*>(p.q) + (static_cast<size_t>(b) * p.q_rows + qi) * p.ldq + head * HD + t * (HD / 4);
      if constexpr (PRECISE) {
        load_rows<HD, TQ>(q, there, p.scale * LOG2E, f[0], q_scale[at], q_sum[at]);
      } else {
        float v[HD / 4];
        load_row<HD, TQ>(q, there, p.scale * LOG2E, v, q_scale[at], q_sum[at]);
#pragma unroll
        for (int j = 0; j < HD / 16; ++j) {
          const int c = j / 2 * 8 + 2 * (j & 1);
          split_f16(v[c], v[c + 4], f[0][j][i], f[TERMS - 1][j][i]);
          split_f16(v[c + 1], v[c + 5], f[0][j][2 + i], f[TERMS - 1][j][2 + i]);
        }
      }
    }
#pragma unroll
    for (int y = 0; y < TERMS; ++y) {
#pragma unroll
      for (int j = 0; j < HD / 16; ++j) {
        if constexpr (S::HELD) {
#pragma unroll
          for (int i = 0; i < 4; ++i) qf[j][i] = f[y][j][i];
        } else if (slice == 0) {
          frags[((x * TERMS + y) * (HD / 16) + j) * 32] = make_uint4(f[y][j][0], f[y][j][1], f[y][j][2], f[y][j][3]);
        }
      }
    }
  }
  if (!S::HELD) __syncthreads();

  float o[NM][HD / 8][4] = {};
  float m[NR], l[NR], bs[NR];  // l and bs: of p and p b', this thread's keys alone
#pragma unroll
  for (int i = 0; i < NR; ++i) m[i] = NONE, l[i] = bs[i] = 0.f;
  float inv_unit[NR];  // one over the row's unit
  float* peak = reinterpret_cast<float*>(smem + S::PEAKS) + tid;  // the largest p s of a row's raises (registers are short)
#pragma unroll
  for (int i = 0; i < NR; ++i) inv_unit[i] = 1.f / LEAST_UNIT, peak[i * WARPS * 32] = 0.f;
  float least_unit = LEAST_UNIT;  // of this thread's rows
  int stage = 0;
  uint32_t phase = 0;
  for (int k = 0; k < mine; k += PAGES) {
    const bool two = PAGES == 2 && k + 1 < mine;
    if (!mbar_wait_warp(full + stage, phase, &sh_abort, WAIT_NS) ||
        (two && !mbar_wait_warp(full + stage + 1, phase, &sh_abort, WAIT_NS))) {
      if (lane == 0) atomicOr(p.c.err, ERR_TIMEOUT);
      break;
    }
    const unsigned char* page[PAGES];
    float z[PAGES][NR][4], step[PAGES][4], base[PAGES][4];
    float zmax[NR], smax = 0.f;
#pragma unroll
    for (int i = 0; i < NR; ++i) zmax[i] = -INFINITY;
#pragma unroll
    for (int h = 0; h < PAGES; ++h) {
      page[h] = ring + (stage + (h && two ? 1 : 0)) * P::BYTES;
      // q . c' of the rows with the 16 keys of the page: s[.][0] keys 2t, 2t + 1, s[.][1] keys 8 + those
      float s[NM][2][4];
      uint32_t kw[2][NW];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const unsigned char* at = page[h] + (r + 8 * i) * P::ROW + t * 4 * NW;
        if (NW == 4)
          *reinterpret_cast<uint4*>(kw[i]) = *reinterpret_cast<const uint4*>(at);
        else
          *reinterpret_cast<uint2*>(kw[i]) = *reinterpret_cast<const uint2*>(at);
      }
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        uint32_t u[2][4];
        kv4_codes(kw[0][w], u[0]);
        kv4_codes(kw[1][w], u[1]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int x = 0; x < NM; ++x) {
#pragma unroll
            for (int y = 0; y < TERMS; ++y) {
              uint32_t f[4];
              if constexpr (S::HELD) {
#pragma unroll
                for (int i = 0; i < 4; ++i) f[i] = qf[2 * w + j][i];
              } else {
                *reinterpret_cast<uint4*>(f) = frags[((x * TERMS + y) * (HD / 16) + 2 * w + j) * 32];
              }
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                if (w == 0 && j == 0 && y == 0)
                  mma_f16_first(s[x][i], f[0], f[1], f[2], f[3], u[i][2 * j], u[i][2 * j + 1]);
                else
                  mma_f16(s[x][i], f[0], f[1], f[2], f[3], u[i][2 * j], u[i][2 * j + 1]);
              }
            }
          }
        }
      }
      key_scales(page[h] + P::KS, t, step[h], base[h]);
#pragma unroll
      for (int x = 0; x < NM; ++x) {
#pragma unroll
        for (int i = 0; i < RM; ++i) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float* d = s[x][j / 2];
            z[h][x * RM + i][j] = fmaf(step[h][j] * q_scale[x * RM + i], PRECISE ? d[j % 2] + d[2 + j % 2] : d[2 * i + j % 2],
                                       base[h][j] * q_sum[x * RM + i]);
          }
        }
      }
      key_scales(page[h] + P::VS, t, step[h], base[h]);
      const int slot0 = (p0 + slice + (k + h) * S::SLICES) * KV4_ROWS;
      if (slot0 + KV4_ROWS > all.n || (h && !two)) {
        // A hidden key counts nothing, whatever its codes, steps and bases are.  A row of V without numbers has the weight 0
        // in the products, and makes those sums that see it no number.
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int slot = slot0 + 2 * t + (j & 1) + 8 * (j >> 1);
          const bool held = slot < all.total && !(h && !two), number = isfinite(step[h][j]) && isfinite(base[h][j]);
#pragma unroll
          for (int i = 0; i < NR; ++i) {
            if (!held || (slot >= all.n && !(local[i] >> (slot - all.n) & 1)))
              z[h][i][j] = -INFINITY;
            else if (!number)
              bs[i] = NAN;
          }
          if (!held || !number) step[h][j] = base[h][j] = 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) smax = fmaxf(smax, step_size(step[h][j], base[h][j]));
#pragma unroll
      for (int i = 0; i < NR; ++i) zmax[i] = fmaxf(zmax[i], fmaxf(fmaxf(z[h][i][0], z[h][i][1]), fmaxf(z[h][i][2], z[h][i][3])));
    }
    bool raise = smax > least_unit;
#pragma unroll
    for (int i = 0; i < NR; ++i) raise = raise || zmax[i] > m[i] + SLACK;
    if (__any_sync(0xffffffffu, raise)) {
      least_unit = INFINITY;
#pragma unroll
      for (int x = 0; x < NM; ++x) {
        float a[RM];
#pragma unroll
        for (int i = 0; i < RM; ++i) {
          const int at = x * RM + i;
          const float raised = fmaxf(m[at], quad_max(zmax[at]) - BELOW), unit = one_over(inv_unit[at]);
          float wide = 0.f, most = 0.f;  // the largest step that the row sees, and p s
#pragma unroll
          for (int h = 0; h < PAGES; ++h) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float size = step_size(step[h][j], base[h][j]);
              if (z[h][at][j] > -INFINITY) wide = fmaxf(wide, size);
              most = fmaxf(most, pow2(z[h][at][j] - raised) * size);
            }
          }
          wide = quad_max(wide);
          a[i] = exp2f(m[at] - raised);
          m[at] = raised;
          most = fmaxf(peak[at * WARPS * 32] * a[i], quad_max(most));
          peak[at * WARPS * 32] = most;
          const float wanted = fmaxf(fminf(wide > unit ? fminf(2.f * wide, 0x1p125f) : unit, 16.f * most), LEAST_UNIT);
          inv_unit[at] = one_over(__float_as_uint(wanted) & 0xff800000u);
          least_unit = fminf(least_unit, one_over(inv_unit[at]));
          l[at] = l[at] * a[i] * unit * inv_unit[at];  // (step by step: weights count whatever became of the unit)
          a[i] = a[i] * unit * inv_unit[at];           // the sums so far, in the new unit
          bs[at] *= a[i];
        }
#pragma unroll
        for (int j = 0; j < HD / 8; ++j) {
#pragma unroll
          for (int i = 0; i < 4; ++i) o[x][j][i] *= a[PRECISE ? 0 : i / 2];
        }
      }
    }
    uint32_t wf[PAGES][NM][4];  // the weights as A fragments
    float inverse[PAGES][4];
    if (!PRECISE) {
#pragma unroll
      for (int h = 0; h < PAGES; ++h) {
#pragma unroll
        for (int j = 0; j < 4; ++j) inverse[h][j] = __fdividef(1.f, step[h][j]);
      }
    }
#pragma unroll
    for (int h = 0; h < PAGES; ++h) {
#pragma unroll
      for (int x = 0; x < NM; ++x) {
#pragma unroll
        for (int i = 0; i < RM; ++i) {
          const int at = x * RM + i;
          float e[4], w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            e[j] = pow2(z[h][at][j] - m[at]);
            e[j] *= inv_unit[at];
            w[j] = e[j] * step[h][j];
          }
          if (PRECISE) {
            split_f16(w[0], w[1], wf[h][x][0], wf[h][x][1]);
            split_f16(w[2], w[3], wf[h][x][2], wf[h][x][3]);
          } else {
            wf[h][x][i] = pack_f16(w[0], w[1]);
            wf[h][x][2 + i] = pack_f16(w[2], w[3]);
            // The sums take the weights as they were rounded: the row stays an average of its values, and a key that
            // takes nearly all of it gives its value without the rounding.  (Not those below fp16's normal numbers,
            // which the products hardly notice: a key of much weight and small values counts in the sums all the same.)
            const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&wf[h][x][i]));
            const float2 c = __half22float2(*reinterpret_cast<const __half2*>(&wf[h][x][2 + i]));
            const float rounded[4] = {a.x, a.y, c.x, c.y};
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (w[j] >= 0x1p-14f) e[j] = rounded[j] * inverse[h][j];
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            l[at] += e[j];
            bs[at] = fmaf(e[j], base[h][j], bs[at]);
          }
        }
      }
    }
    // V: row pairs t and t + 4, channels [CHUNK r, CHUNK (r + 1))
    uint32_t v[PAGES][2][NW];
#pragma unroll
    for (int h = 0; h < PAGES; ++h) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const unsigned char* at = page[h] + P::V + (t + 4 * i) * 2 * P::ROW + P::place(t + 4 * i, r) * P::CHUNK;
        if (NW == 4)
          *reinterpret_cast<uint4*>(v[h][i]) = *reinterpret_cast<const uint4*>(at);
        else
          *reinterpret_cast<uint2*>(v[h][i]) = *reinterpret_cast<const uint2*>(at);
      }
    }
#pragma unroll
    for (int c = 0; c < NW; ++c) {
      uint32_t u[PAGES][2][4];
#pragma unroll
      for (int h = 0; h < PAGES; ++h) {
        kv4_codes(v[h][0][c], u[h][0]);
        kv4_codes(v[h][1][c], u[h][1]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int x = 0; x < NM; ++x) {
          float* sum = o[x][4 * c + i];
          if constexpr (PRECISE) {
            // the tensor cores round their sums toward zero: in a chain over all pages that would be a bias
            float d[4];
            mma_f16_first(d, wf[0][x][0], wf[0][x][1], wf[0][x][2], wf[0][x][3], u[0][0][i], u[0][1][i]);
            if (PAGES == 2)
              mma_f16(d, wf[PAGES - 1][x][0], wf[PAGES - 1][x][1], wf[PAGES - 1][x][2], wf[PAGES - 1][x][3], u[PAGES - 1][0][i], u[PAGES - 1][1][i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += d[j];
          } else {
#pragma unroll
            for (int h = 0; h < PAGES; ++h)
              mma_f16(o[x][4 * c + i], wf[h][x][0], wf[h][x][1], wf[h][x][2], wf[h][x][3], u[h][0][i], u[h][1][i]);
          }
        }
      }
    }
    __syncwarp();
    if (RTW > 1 && lane < PAGES) mbar_arrive(empty + stage + lane);
    stage += PAGES;
    if (stage == STAGES) {
      stage = 0;
      phase ^= 1;
    }
    // the next pages, into the places of the round before this one
    if (rt == 0) {
      for (int i = 0; i < PAGES && asked < mine; ++i) {
        if (RTW > 1 && asked >= STAGES && !mbar_wait_warp(empty + ask_stage, ask_phase, &sh_abort, WAIT_NS)) break;
        request();
      }
    }
  }

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
  for (int x = 0; x < NM; ++x) {
#pragma unroll
    for (int j = 0; j < HD / 8; ++j) {
#pragma unroll
      for (int i = 0; i < RM; ++i) {
        const float* d = o[x][j];
        *reinterpret_cast<float2*>(sums + ((PRECISE ? 8 : 16) * x + r + 8 * i) * S::PITCH + 8 * j + 2 * t) =
            make_float2(((PRECISE ? d[0] + d[2] : d[2 * i]) + bs[x * RM + i]) * one_over(inv_unit[x * RM + i]),
                        ((PRECISE ? d[1] + d[3] : d[2 * i + 1]) + bs[x * RM + i]) * one_over(inv_unit[x * RM + i]));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NR; ++i)
    if (t == 0) {  // rows r, r + 8, .. of the tile
      ml[(warp * TILE + r + 8 * i) * 2] = m[i];
      ml[(warp * TILE + r + 8 * i) * 2 + 1] = l[i] * one_over(inv_unit[i]);
    }
  __syncthreads();

  constexpr int LINE = HD + 4;
  float* ws = p.ws + (static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x) * S::ROWS * LINE;
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
    if (PARTS == CLUSTER) {  // stays here, in the place of its first slice
#pragma unroll
      for (int i = 0; i < W; ++i) mine[i] = acc[i];
      __syncwarp();
      if (lane == 0) *reinterpret_cast<float2*>(ml + (w0 * TILE + at) * 2) = make_float2(M, L);
      continue;
    }
    float* line = ws + my * LINE;
    if constexpr (W == 4)
      *reinterpret_cast<float4*>(line + W * lane) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    else
      *reinterpret_cast<float2*>(line + W * lane) = make_float2(acc[0], acc[1]);
    if (lane == 0) {
      line[HD] = M;
      line[HD + 1] = L;
    }
  }
  if constexpr (PARTS == CLUSTER) {
    static_assert(RTW == 1 && S::SLICES > 1, "a merged row is put in order in the place of its second slice");
    cluster_arrive();
    cluster_wait();
    for (int my = split + splits * warp; my < here; my += splits * WARPS) {
      constexpr int W = HD / 32;
      float* mine = reinterpret_cast<float*>(smem) + my * S::PITCH + W * lane;
      float v[CLUSTER_MOST][W], m_of = NONE, l_of = 0.f;  // lane c: of part c
#pragma unroll
      for (int c = 0; c < CLUSTER_MOST; ++c) {
        const uint32_t from = dsmem_addr(smem_u32(mine), min(c, splits - 1));
        if constexpr (W == 4)
          asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[c][0]), "=f"(v[c][1]), "=f"(v[c][2]), "=f"(v[c][3]) : "r"(from));
        else
          asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v[c][0]), "=f"(v[c][1]) : "r"(from));
      }
      if (lane < splits)
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m_of), "=f"(l_of) : "r"(dsmem_addr(smem_u32(ml + my * 2), lane)));
      float M = m_of;
#pragma unroll
      for (int o = 1; o < CLUSTER_MOST; o <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      M = __shfl_sync(0xffffffffu, M, 0);
      const float e = exp2f(m_of - M);
      float L = 0.f, acc[W] = {};
#pragma unroll
      for (int c = 0; c < CLUSTER_MOST; ++c) {
        const float f = __shfl_sync(0xffffffffu, e, c), l = __shfl_sync(0xffffffffu, l_of, c);
        if (c >= splits) break;
        L = fmaf(f, l, L);
#pragma unroll
        for (int i = 0; i < W; ++i) acc[i] = fmaf(f, v[c][i], acc[i]);
      }
      float* order = mine + RTW * TILE * S::PITCH;
#pragma unroll
      for (int i = 0; i < W; ++i) order[i] = acc[i];
      __syncwarp();
      store_row<HD>(p, bg, row0 + my, lane, M, L, order - W * lane);
    }
    cluster_arrive();  // the others have read what is here
    cluster_wait();
  }
}

// Merges the splits of a row: four warps take every fourth split, and their sums are added in the warps' order.  (By the
// last block of the tile to arrive, 64 rows of 15 splits took longer than the attention itself.)
template <int HD, bool DEAL>
__global__ void __launch_bounds__(128) join_kv4_kernel(const __grid_constant__ Kv4AttnParams p, int rows, int blocks) {
  constexpr int LINE = HD + 4, W = HD / 32;  // W: columns of a lane
  __shared__ float sh_acc[4][HD];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, n_rows = p.nq * (p.H / p.c.G);
  const int bg = static_cast<int>(blockIdx.x / n_rows), row = static_cast<int>(blockIdx.x % n_rows);
  int splits = p.splits;
  size_t part = static_cast<size_t>(bg * blocks + row / rows) * splits;  // the row's first
  if (DEAL) {
    const Deal d = deal_slots(p, lane);
    const int b = bg / p.c.G;
    splits = __shfl_sync(0xffffffffu, d.parts, b);
    if (splits == 1) return;  // written by its only part
    part = static_cast<size_t>(bg % p.c.G * blocks + row / rows) * p.slots + __shfl_sync(0xffffffffu, d.first, b);
  }
  const float* ws = p.ws + (part * rows + row % rows) * LINE;
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

// scores_j += sum over rows of weight p_j, p_j = 2^(z_j - lse): the first matrix product alone, on K's half of a page.
// The fragments of up to 64 rows are held in shared memory, a page's codes are unpacked once for all of them.
// Measured: 32 queries (24 that count) of 32 heads over 16384 rows (40 MB) 27.2 us, bound by the latency of products and
// exponentials (tensor pipe 38 %, issue 45 %); two pages a time and eight warps a block, which halves the
// fragments' way from shared memory, took 41 when one page took 33.
template <int HD, typename TQ, bool DEAL>
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

  const int group = p.H / p.c.G, g = blockIdx.y % p.c.G;
  int b = blockIdx.y / p.c.G, split = blockIdx.x, splits = gridDim.x;
  if (DEAL) {
    const Deal d = deal_slots(p, lane);
    b = sequence_of(d, split, splits);
    if (split >= splits) return;  // (the whole block; a slot that is left over)
  }
  const int bg = b * p.c.G + g;
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
  const int p0 = static_cast<int>(static_cast<long long>(pages) * split / splits);
  const int p1 = static_cast<int>(static_cast<long long>(pages) * (split + 1) / splits);
  const int mine = max(0, (p1 - p0 - warp + WARPS - 1) / WARPS);
  const int* table = p.c.table + static_cast<size_t>(b) * p.c.max_pages;
  float* scores = p.scores + static_cast<size_t>(bg) * p.ld_scores;
  int used = 0;  // stages taken since the start
  bool ok = true;
  for (int tile0 = 0; tile0 < tiles; tile0 += SCORE_TILES) {
    const int held = min(SCORE_TILES, tiles - tile0);
    // (table entries 32 at a time, one per lane, as in the attention)
    auto entries = [&](int k) { return k + lane < mine ? block_of(p, table, p0 + warp + (k + lane) * WARPS) : 0; };
    int blocks_now = entries(0), blocks_next = entries(32);
    auto request = [&](int k) {  // k counts up from 0
      const int block = __shfl_sync(0xffffffffu, blocks_now, k & 31);
      if (lane == 0) {
        uint64_t* bar = bars + (used + k) % STAGES;
        unsigned char* dst = ring + (used + k) % STAGES * S::PAGE;
        const unsigned char* src = p.c.pool + (static_cast<size_t>(block) * p.c.G + g) * P::BYTES;
        mbar_arrive_expect_tx(bar, S::PAGE);
        bulk_load(dst, src, P::V, bar);
        bulk_load(dst + P::V, src + P::KS, 4 * KV4_ROWS, bar);
      }
      if ((k & 31) == 31) {
        blocks_now = blocks_next;
        blocks_next = entries(k + 33);
      }
    };
    if (ok)
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
      auto tile = [&](int i, auto hidden) {  // hidden(row of the tile, j): is key j hidden from it?
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
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float z = fmaf(step[x] * rf.x, s[x / 2][x % 2] + s[x / 2][2 + x % 2], base[x] * rf.y);
          const float e = rf.w * pow2(z - rf.z);
          sum[x] += hidden(i * ROWS + r, x) ? 0.f : e;
        }
      };
      if (slot0 + KV4_ROWS <= all.n) {
        // every row sees these keys; rows past the last have weight 0 and logits of 0
#pragma unroll 2
        for (int i = 0; i < held; ++i) tile(i, [](int, int) { return false; });
      } else {
#pragma unroll 1
        for (int i = 0; i < held; ++i)
          tile(i, [&](int row, int x) {
            Seen seen = all;
            seen.local = reinterpret_cast<const unsigned long long*>(smem + S::LOCAL)[row];
            return !(seen(slot0 + 2 * t + (x & 1) + 8 * (x >> 1)) && reinterpret_cast<const float4*>(smem + S::ROWF)[row].w != 0.f);
          });
      }
      // over the rows: a lane hands on half of its sums at each step, and lanes r = 2 x, 2 x + 1 end with that of key x
      float half[2], whole;
#pragma unroll
      for (int x = 0; x < 2; ++x) half[x] = (r & 4 ? sum[2 + x] : sum[x]) + __shfl_xor_sync(0xffffffffu, r & 4 ? sum[x] : sum[2 + x], 16);
      whole = (r & 2 ? half[1] : half[0]) + __shfl_xor_sync(0xffffffffu, r & 2 ? half[0] : half[1], 8);
      whole += __shfl_xor_sync(0xffffffffu, whole, 4);
      const int slot = slot0 + 2 * t + (r >> 1 & 1) + 8 * (r >> 2);
      // (its only writer: a sum in memory, so that the warp waits for no old value)
      if (!(r & 1) && slot < all.total && slot < p.ld_scores) red_add_f32(scores + slot, whole);
      __syncwarp();
      if (k + STAGES < mine) request(k + STAGES);
    }
    used += mine;
  }
}

template <auto KERNEL>
cudaError_t launch_sized(size_t smem, dim3 grid, const Kv4AttnParams& p, cudaStream_t s) {
  const cudaError_t e = allow_smem<KERNEL>(smem);
  return e != cudaSuccess ? e : launch_pdl(KERNEL, grid, dim3(WARPS * 32), smem, s, p);
}

}  // namespace

// How a call's rows are cut: one term per weight where the result is rounded to bf16 alone and there are rows enough
// to fill a matrix with them (32 heads over 16384 rows, 64 queries 105 us, with two terms 153; 16 queries 40.8 and
// 45.2); two matrices per warp from there on, and warps that share pages for more rows (with one matrix and no
// sharing 143 and 287 us where these took 102 and 146, 16 queries 41.9 and 51.7 for 41.8 and 43.7).
namespace {
struct Cut {
  bool precise;
  int nm, rtw, rows;  // matrices of a warp, tiles at a time, rows of a block
};
Cut cut_of(const Kv4AttnParams& p) {
  const int rows = p.nq * (p.H / p.c.G);
  const bool precise = rows <= 8 || p.out_f32 || p.out_lo || p.lse;
  const int matrix = precise ? 8 : 16, nm = rows <= matrix ? 1 : 2;
  const int rtw = rows <= nm * matrix ? 1 : rows <= 2 * nm * matrix || !precise ? 2 : 4;
  return Cut{precise, nm, rtw, nm * matrix * rtw};
}
}  // namespace

long long kv4_attn_blocks(const Kv4AttnParams& p) {  // (any call's: more than 31 bits)
  const Cut c = cut_of(p);
  return static_cast<long long>((p.nq * (p.H / p.c.G) + c.rows - 1) / c.rows) * p.c.B * p.c.G;
}

namespace {
int blocks_of(const Kv4AttnParams& p) { return static_cast<int>(kv4_attn_blocks(p)); }  // of a call that was taken
// Blocks that are resident at once (launch bounds): three of one matrix in two terms (1 query over 16384 rows 30.6 us,
// with two blocks 32.0; 8 of 256 to 4096 rows 40 and 56), although their 168 registers spill up to 76 bytes; otherwise two,
// at 20 bytes at most (4 queries of groups of 4 heads, bf16 out, 16384 rows: 17.9 us, with three 20.5), and two in
// clusters (1 query over 512 rows: 6.7, 7.3).
int slots_of(const Cut& c) { return (c.nm == 1 && c.precise ? 3 : 2) * tc_num_sms(); }
size_t ws_floats(const Kv4AttnParams& p) {
  const size_t parts = p.slots ? static_cast<size_t>(blocks_of(p)) / p.c.B * p.slots : static_cast<size_t>(blocks_of(p)) * p.splits;
  return parts * cut_of(p).rows * (p.c.hd + 4);
}
}  // namespace

// The parts of the pages: `want` of every sequence, or (0) as many as are resident, none left for a second wave, dealt
// to the sequences of a batch by their lengths.  The host knows the table's length, not the context's: with a table of four
// times the context 1 query over 512 rows takes 7.6 us instead of 6.7 (no cluster), over 16384 rows 30.8 and 30.6.
void kv4_attn_split(Kv4AttnParams* p, int want, size_t most_floats) {
  const Cut c = cut_of(*p);
  const int blocks = blocks_of(*p), at_once = WARPS / c.rtw * (c.nm == 1 ? 2 : 1);
  const int most = std::min((p->c.max_pages + at_once - 1) / at_once, PARTS_MOST);
  p->slots = 0;
  p->splits = want ? want : std::max(1, std::min(slots_of(c) / blocks, most));
  if (!want) {  // no more than it takes for as few rounds
    const int rounds = (p->c.max_pages + p->splits * at_once - 1) / (p->splits * at_once);
    p->splits = (p->c.max_pages + rounds * at_once - 1) / (rounds * at_once);
  }
  while (p->splits > 1 && ws_floats(*p) > most_floats) --p->splits;
  if (want || p->c.B == 1 || p->c.B > DEAL_MOST || most == 1) return;
  p->least_pages = at_once;
  p->slots = slots_of(c) / (blocks / p->c.B);
  if (p->slots >= p->c.B * most) p->slots = 0;  // there are enough to cut every sequence as finely as it can be
  while (p->slots > p->c.B && ws_floats(*p) > most_floats) --p->slots;
  if (p->slots <= p->c.B) p->slots = 0;
}

namespace {
template <int HD, typename TQ, bool PRECISE, int NM, int RTW, Parts PARTS>
cudaError_t launch_parts(const Kv4AttnParams& p, cudaStream_t s) {
  using S = Shape<HD, PRECISE, NM, RTW>;
  const int blocks = blocks_of(p);
  const dim3 grid = PARTS == DEALT ? dim3(p.slots, blocks / p.c.B) : dim3(p.splits, blocks);
  constexpr auto kernel = attn_kv4_kernel<HD, TQ, PRECISE, NM, RTW, PARTS>;
  if (PARTS == CLUSTER) {
    const cudaError_t e = allow_smem<kernel>(S::BYTES);
    return e != cudaSuccess ? e : launch_pdl_cluster(kernel, grid, dim3(WARPS * 32), p.splits, S::BYTES, s, p);
  }
  const cudaError_t e = launch_sized<kernel>(S::BYTES, grid, p, s);
  if (e != cudaSuccess || (PARTS == EQUAL && p.splits == 1)) return e;
  const long long rows = static_cast<long long>(p.nq) * p.c.B * p.H;
  return launch_pdl(join_kv4_kernel<HD, PARTS == DEALT>, dim3(static_cast<unsigned>(rows)), dim3(128), 0, s, p, S::ROWS, blocks / (p.c.B * p.c.G));
}
template <int HD, typename TQ, bool PRECISE, int NM, int RTW>
cudaError_t launch_attn(const Kv4AttnParams& p, cudaStream_t s) {
  if (p.slots) return launch_parts<HD, TQ, PRECISE, NM, RTW, DEALT>(p, s);
  if constexpr (RTW == 1)
    if (p.splits > 1 && p.splits <= CLUSTER_MOST && blocks_of(p) * p.splits <= 2 * tc_num_sms()) return launch_parts<HD, TQ, PRECISE, NM, RTW, CLUSTER>(p, s);
  return launch_parts<HD, TQ, PRECISE, NM, RTW, EQUAL>(p, s);
}
template <int HD, typename TQ>
cudaError_t launch_cut(const Kv4AttnParams& p, cudaStream_t s) {
  const Cut c = cut_of(p);
  if (!c.precise)
    return c.nm == 1 ? launch_attn<HD, TQ, false, 1, 1>(p, s) : c.rtw == 1 ? launch_attn<HD, TQ, false, 2, 1>(p, s) : launch_attn<HD, TQ, false, 2, 2>(p, s);
  if (c.nm == 1) return launch_attn<HD, TQ, true, 1, 1>(p, s);
  return c.rtw == 1 ? launch_attn<HD, TQ, true, 2, 1>(p, s) : c.rtw == 2 ? launch_attn<HD, TQ, true, 2, 2>(p, s) : launch_attn<HD, TQ, true, 2, 4>(p, s);
}
}  // namespace

cudaError_t attention_kv4(const Kv4AttnParams& p, cudaStream_t s) {
  if (p.c.hd == 128) return p.q_f32 ? launch_cut<128, float>(p, s) : launch_cut<128, bf16>(p, s);
  return p.q_f32 ? launch_cut<64, float>(p, s) : launch_cut<64, bf16>(p, s);
}

namespace {
template <int HD, typename TQ>
cudaError_t launch_score(const Kv4AttnParams& p, const dim3& grid, cudaStream_t s) {
  return p.slots ? launch_sized<score_kv4_kernel<HD, TQ, true>>(ScoreSmem<HD>::BYTES, grid, p, s)
                 : launch_sized<score_kv4_kernel<HD, TQ, false>>(ScoreSmem<HD>::BYTES, grid, p, s);
}
}  // namespace

cudaError_t kv4_score(const Kv4AttnParams& call, cudaStream_t s) {
  Kv4AttnParams p = call;
  const int bg = p.c.B * p.c.G, resident = 4 * tc_num_sms();  // four blocks per SM
  const int most = (p.c.max_pages + WARPS - 1) / WARPS, slots = resident / p.c.G;
  p.least_pages = WARPS;
  p.slots = p.c.B > 1 && p.c.B <= DEAL_MOST && slots > p.c.B && slots < p.c.B * std::min(most, PARTS_MOST) ? slots : 0;
  const dim3 grid = p.slots ? dim3(p.slots, p.c.G) : dim3(std::max(1, std::min(resident / bg, most)), bg);
  if (p.c.hd == 128) return p.q_f32 ? launch_score<128, float>(p, grid, s) : launch_score<128, bf16>(p, grid, s);
  return p.q_f32 ? launch_score<64, float>(p, grid, s) : launch_score<64, bf16>(p, grid, s);
}

}  // namespace chimera
