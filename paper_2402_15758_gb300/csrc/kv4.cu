// The 4-bit KV cache's rows: written from fresh K and V rows, read back, and moved when the rows
// that drew little attention leave (layout and rounding rule in kv4.cuh).
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "kv4.cuh"
#include "launch.cuh"

namespace chimera {
namespace {

// Address of the page that holds `slot` of sequence b for head g; null, with the error
// flagged, when the slot or its block lies outside the table or the pool.
__device__ __forceinline__ unsigned char* page_of(const Kv4Pool& c, int b, int g, int slot) {
  if (slot < 0 || slot / KV4_ROWS >= c.max_pages) {
    atomicOr(c.err, ERR_CAPACITY);
    return nullptr;
  }
  const int block = c.table[static_cast<size_t>(b) * c.max_pages + slot / KV4_ROWS];
  if (block < 0 || block >= c.n_blocks) {
    atomicOr(c.err, ERR_BAD_INDEX);
    return nullptr;
  }
  return c.pool + (static_cast<size_t>(block) * c.G + g) * (KV4_ROWS * c.hd + 128);
}

struct RowArgs {
  Kv4Pool c;
  void* k;
  void* v;
  int ldk, ldv, rows;
  const int* slot0;
  const int* counts;
  int vec;  // rows and their heads start on 16 bytes
};

// Eight consecutive values of a row.
template <typename T>
__device__ __forceinline__ void store8(T* dst, bool vec, const float (&x)[8]) {
  if (!vec) {
#pragma unroll
    for (int j = 0; j < 8; ++j) dst[j] = from_f<T>(x[j]);
    return;
  }
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(dst) = make_uint4(u[0], u[1], u[2], u[3]);
  }
}

// What a thread of the row kernels does: eight channels of one head, K or V, for the two rows of a pair of slots
// (they share the words of V), as far as both belong to the call.
template <int HD>
struct Piece {
  static constexpr int LANES = HD / 8;  // threads of a row
  bool there[2];
  int which, slot, part, g;  // slot: of the pair's first row; part: which eight channels
  long long row[2];          // of k and v
  // Block: heads (K's, then V's) by pairs; grid: pairs, heads, sequences.  Nothing is divided.
  __device__ __forceinline__ Piece(const RowArgs& a, const Kv4Pool& c, int pairs, int at) {
    const int piece = blockIdx.y * blockDim.x + threadIdx.x, of_k = c.G * LANES, b = blockIdx.z;
    const bool any = piece < 2 * of_k && at < pairs;
    which = piece >= of_k;
    part = piece % LANES;
    g = any ? (which ? piece - of_k : piece) / LANES : 0;
    const int s0 = a.slot0[b], count = a.counts ? min(a.counts[b], a.rows) : a.rows;
    slot = (s0 & ~1) + 2 * at;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int k = slot + r - s0;
      there[r] = any && k >= 0 && k < count;
      row[r] = static_cast<long long>(b) * a.rows + max(k, 0);
    }
  }
  __device__ __forceinline__ unsigned char* page(const RowArgs& a) const {
    return there[0] || there[1] ? page_of(a.c, blockIdx.z, g, slot) : nullptr;
  }
};

// Rounds a row's eight values of this thread: the row's minimum and maximum over its LANES threads, then the codes,
// four bits each.  A code is rint of the correctly rounded quotient, which one step of Markstein's correction
// (q + (d - q step) / step, the remainder in one rounding) gives here: a step has 8 bits, so the remainder is
// exact, and no quotient of 24 bits by 8 lies within 2^-10 units of a point where its rounding turns.  (bf16 values
// meet ties too often for a branch around a division: 41 us for 4 x 1000 rows of 32 heads.)
__device__ __forceinline__ float reciprocal(float x) {  // to 2^-23, for normal numbers: the correction needs no more
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float ROUNDER = 12582912.f;  // 3 2^22: a sum with it is rounded to a whole number, in its last bits
constexpr uint32_t ROUNDER_BITS = 0x4b400000u;
template <int LANES>
__device__ __forceinline__ uint32_t round8(const float (&x)[8], uint32_t& scale) {
  float lo = x[0], hi = x[0], bad = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo = fminf(lo, x[j]);
    hi = fmaxf(hi, x[j]);
    bad = fmaf(x[j], 0.f, bad);  // NaN from a value that is not finite
  }
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const uint32_t spoilt = __ballot_sync(0xffffffffu, bad != 0.f) >> (threadIdx.y * blockDim.x + threadIdx.x) % 32 / LANES * LANES;
  const bf16 base16 = __float2bfloat16_rn(lo), step16 = __float2bfloat16_rn(__fmul_rn(hi - lo, 1.f / 15.f));
  const float base = __bfloat162float(base16), step = __bfloat162float(step16);
  const bool fine = (spoilt & ((1u << LANES) - 1u)) == 0 && isfinite(hi - lo) && isfinite(base);
  scale = fine ? __bfloat16_as_ushort(step16) | static_cast<uint32_t>(__bfloat16_as_ushort(base16)) << 16 : 0x7fc00000u;
  if (!fine || !(step > 0.f)) return 0;
  // (a power of two keeps the reciprocal and the remainder among the normal numbers)
  const float up = step < 0x1p-60f ? 0x1p100f : step > 0x1p60f ? 0x1p-100f : 1.f, unit = step * up, inv = reciprocal(unit);
  uint32_t codes = 0;
#pragma unroll
  for (int j = 7; j >= 0; --j) {
    const float d = (x[j] - base) * up, q = d * inv;
    const float exact = fmaf(fmaf(-q, unit, d), inv, q);
    codes = codes * 16 + (__float_as_uint(fminf(fmaxf(exact, 0.f), 15.f) + ROUNDER) - ROUNDER_BITS);
  }
  return codes;
}

// Eight values as they lie, converted when they are used.
template <typename T>
struct Raw {
  uint32_t u[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T* src, bool vec) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < sizeof(T) / 2; ++i) *reinterpret_cast<uint4*>(u + 4 * i) = reinterpret_cast<const uint4*>(src)[i];
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(src[j]);
    } else {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(src);
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = h[2 * i] | static_cast<uint32_t>(h[2 * i + 1]) << 16;
    }
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[j] = __uint_as_float(sizeof(T) == 4 ? u[j % (2 * sizeof(T))] : j & 1 ? u[j / 2] & 0xffff0000u : u[j / 2] << 16);
  }
};

// Two pairs of rows a thread, all their loads in flight.  Measured: 4 x 1000 bf16 rows of 32 heads of 128 (83 MB) 29.4 us,
// 2.8 TB/s; one pair a thread 30.9.  Every value takes a minimum, a maximum, a check and eight steps to its code: an
// instruction is issued in 85 % of the cycles, DRAM works at 26 %.
constexpr int APPEND_PAIRS = 2;

template <int HD, typename T>
__global__ void __launch_bounds__(256) kv4_append_kernel(RowArgs a, int pairs) {
  pdl_wait();
  pdl_trigger();
  using P = Kv4<HD>;
  const int first = blockIdx.x * blockDim.y * APPEND_PAIRS;
  Raw<T> raw[APPEND_PAIRS][2];
#pragma unroll
  for (int i = 0; i < APPEND_PAIRS; ++i) {
    const Piece<HD> w(a, a.c, pairs, first + i * blockDim.y + threadIdx.y);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      raw[i][r] = Raw<T>{};
      if (w.there[r])
        raw[i][r].load(static_cast<const T*>(w.which ? a.v : a.k) + w.row[r] * (w.which ? a.ldv : a.ldk) + w.g * HD + 8 * w.part, a.vec);
    }
  }
#pragma unroll
  for (int i = 0; i < APPEND_PAIRS; ++i) {
    if (first + i * static_cast<int>(blockDim.y) >= pairs) return;  // (the whole block)
    const Piece<HD> w(a, a.c, pairs, first + i * blockDim.y + threadIdx.y);
    unsigned char* page = w.page(a);
    uint32_t codes[2], scale[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float x[8];
      raw[i][r].values(x);
      codes[r] = round8<Piece<HD>::LANES>(x, scale[r]);
    }
    if (!page) continue;
    const int row = w.slot % KV4_ROWS;
    if (!w.which) {
#pragma unroll
      for (int r = 0; r < 2; ++r)
        if (w.there[r]) *reinterpret_cast<uint32_t*>(page + (row + r) * P::ROW + 4 * w.part) = codes[r];
    } else {
      unsigned char* at = page + P::v_half(row, 2 * w.part);  // words 2 part and 2 part + 1 are neighbours
      if (w.there[0] && w.there[1]) {
        *reinterpret_cast<uint2*>(at) = make_uint2(__byte_perm(codes[0], codes[1], 0x5410), __byte_perm(codes[0], codes[1], 0x7632));
      } else {
        const int r = w.there[0] ? 0 : 1;
        *reinterpret_cast<uint16_t*>(at + 2 * r) = static_cast<uint16_t>(codes[r]);
        *reinterpret_cast<uint16_t*>(at + 2 * r + 4) = static_cast<uint16_t>(codes[r] >> 16);
      }
    }
    if (w.part < 2 && (w.part ? w.there[1] : w.there[0]))
      *reinterpret_cast<uint32_t*>(page + (w.which ? P::VS : P::KS) + 4 * (row + w.part)) = w.part ? scale[1] : scale[0];
  }
}

// Measured: the rows above 17.4 us, 4.8 TB/s (issue 80 % busy); 2 x 8192 bf16 rows of 32 heads (340 MB) 64.6 us, 5.3 TB/s: memory.
template <int HD, typename T>
__global__ void __launch_bounds__(256) kv4_read_kernel(RowArgs a, int pairs) {
  pdl_wait();
  pdl_trigger();
  using P = Kv4<HD>;
  const Piece<HD> w(a, a.c, pairs, blockIdx.x * blockDim.y + threadIdx.y);
  const unsigned char* page = w.page(a);
  if (!page) return;
  const int row = w.slot % KV4_ROWS;
  uint2 c;  // codes of the pair's rows
  if (!w.which) {
    c.x = *reinterpret_cast<const uint32_t*>(page + row * P::ROW + 4 * w.part);
    c.y = *reinterpret_cast<const uint32_t*>(page + (row + 1) * P::ROW + 4 * w.part);
  } else {
    c = *reinterpret_cast<const uint2*>(page + P::v_half(row, 2 * w.part));
    c = make_uint2(__byte_perm(c.x, c.y, 0x5410), __byte_perm(c.x, c.y, 0x7632));
  }
  const uint2 scale = *reinterpret_cast<const uint2*>(page + (w.which ? P::VS : P::KS) + 4 * row);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (!w.there[r]) continue;
    const uint32_t codes = r ? c.y : c.x, s = r ? scale.y : scale.x;
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)  // (a code as the last bits of 2^23: a conversion takes four times as long)
      x[j] = fmaf(kv4_step(s), __uint_as_float(and_or(codes >> (4 * j), 15u, 0x4b000000u)) - 8388608.f, kv4_base(s));
    store8<T>(static_cast<T*>(w.which ? a.v : a.k) + w.row[r] * (w.which ? a.ldv : a.ldk) + w.g * HD + 8 * w.part, a.vec, x);
  }
}

// ---------------------------------------------------------------------------
// eviction
// ---------------------------------------------------------------------------
constexpr int SEL_THREADS = 1024;

// A sum as an unsigned number of the same order; sums that are no numbers come last, -0 is 0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (isnan(x)) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int DIGIT = 11, BINS = 1 << DIGIT;  // 32 bits in three digits (11, 11, 10)
constexpr int SEL_WARPS = SEL_THREADS / 32, HELD = 16;  // keys that a thread holds in registers

// Sum of v over the warps before this one (a warp's v in any lane), and over all.
__device__ __forceinline__ int warps_before(int v, int* sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  __syncthreads();
  if (lane == 0) sums[warp] = v;
  __syncthreads();
  const int x = sums[lane];
  total = __reduce_add_sync(0xffffffffu, x);
  return __reduce_add_sync(0xffffffffu, lane < warp ? x : 0);
}

// One block per (sequence, head): the kept slots.  The (budget - recent)-th largest key of the older slots is found
// digit by digit, three histograms of up to 2048 bins; then one ordered pass takes every slot above it and
// the first ones that equal it.  A warp owns a contiguous part of the slots, so the order of warps, rounds
// and lanes is the slots' and the loads are coalesced.  Measured: 64 heads of 6000 to 16384 slots 14 us, in one
// block per head: three passes of shared-memory atomics and their barriers.
__global__ void __launch_bounds__(SEL_THREADS) kv4_select_kernel(Kv4EvictParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ int hist[BINS];
  __shared__ int sums[SEL_WARPS];
  __shared__ uint32_t sh_digit;
  __shared__ int sh_need;
  const int bg = blockIdx.x, b = bg / p.c.G, tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  const int cap = min(p.ld_scores, p.c.max_pages * KV4_ROWS);
  int n = p.n_ctx[b];
  if (n < 0 || n > cap) {
    if (tid == 0) atomicOr(p.c.err, ERR_CAPACITY);
    n = min(max(n, 0), cap);
  }
  const float* x = p.scores + static_cast<size_t>(bg) * p.ld_scores;
  int* kept = p.kept + static_cast<size_t>(bg) * p.budget;
  float* out = p.scores_out + static_cast<size_t>(bg) * p.budget;
  if (bg % p.c.G == 0 && tid == 0) p.n_out[b] = min(n, p.budget);
  if (n <= p.budget) {
    for (int i = tid; i < p.budget; i += SEL_THREADS) {
      kept[i] = i < n ? i : -1;
      out[i] = i < n ? x[i] : 0.f;
    }
    return;
  }
  const int older = n - p.recent, want = p.budget - p.recent;
  for (int i = tid; i < p.recent; i += SEL_THREADS) {
    kept[want + i] = older + i;
    out[want + i] = x[older + i];
  }
  if (want == 0) return;
  const int rounds = (older + SEL_THREADS - 1) / SEL_THREADS;  // of a warp, 32 slots each
  const int begin = warp * rounds * 32 + lane;                 // this thread's first slot
  float held[HELD];
#pragma unroll
  for (int j = 0; j < HELD; ++j) held[j] = j < rounds && begin + 32 * j < older ? x[begin + 32 * j] : 0.f;
  // f(slot, value, whether there is one), over this warp's slots in order
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < HELD; ++j)
      if (j < rounds) f(begin + 32 * j, held[j], begin + 32 * j < older);
    for (int j = HELD; j < rounds; ++j) {
      const int i = begin + 32 * j;
      f(i, i < older ? x[i] : 0.f, i < older);
    }
  };
  uint32_t prefix = 0;  // of the key looked for: the digits found so far
  int need = want;      // keys with this prefix that stay
  int width = DIGIT;
  for (int shift = 32 - DIGIT; shift >= 0; shift -= width) {
    for (int i = tid; i < BINS; i += SEL_THREADS) hist[i] = 0;
    __syncthreads();
    each([&](int, float v, bool there) {
      const uint32_t key = order_key(v);
      if (there && (shift + width == 32 || key >> (shift + width) == prefix)) atomicAdd(&hist[key >> shift & ((1u << width) - 1)], 1);
    });
    __syncthreads();
    // thread t has the bins BINS - 1 - 2 t and the one below: counts from the largest digit down
    const int top = BINS - 1 - 2 * tid, h0 = hist[top], h1 = hist[top - 1];
    int before = h0 + h1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += y;
    }
    int total;
    before += warps_before(__shfl_sync(0xffffffffu, before, 31), sums, total) - h0 - h1;
    if (before < need && before + h0 + h1 >= need) {
      const bool first = before + h0 >= need;
      sh_digit = first ? top : top - 1;
      sh_need = need - before - (first ? 0 : h0);
    }
    __syncthreads();
    prefix = prefix << width | sh_digit;
    need = sh_need;
    if (shift == 32 - 2 * DIGIT) width = 32 - 2 * DIGIT;
  }
  // slots of this warp above the key, and equal to it
  int above = 0, equal = 0, total;
  each([&](int, float v, bool there) {
    const uint32_t key = order_key(v);
    above += there && key > prefix;
    equal += there && key == prefix;
  });
  above = __reduce_add_sync(0xffffffffu, above);
  equal = __reduce_add_sync(0xffffffffu, equal);
  const int equal_before = warps_before(equal, sums, total);
  int left = min(max(need - equal_before, 0), equal);  // equal ones that stay
  int at = warps_before(above + left, sums, total);
  const uint32_t below = (1u << lane) - 1;
  each([&](int i, float v, bool there) {
    const uint32_t key = order_key(v);
    const uint32_t same = __ballot_sync(0xffffffffu, there && key == prefix);
    const bool stays = there && (key > prefix || (key == prefix && __popc(same & below) < left));
    const uint32_t all = __ballot_sync(0xffffffffu, stays);
    if (stays) {
      kept[at + __popc(all & below)] = i;
      out[at + __popc(all & below)] = v;
    }
    at += __popc(all);
    left = max(left - __popc(same), 0);
  });
}

// 128 threads gather the 16 rows kept in a destination page, 16 bytes a time: a K row's codes as they are, a V chunk from
// the chunks of its two rows.  A block finds the rows of 8 pages at once, and a thread has its loads of two pages in
// flight: 2 x 8192 rows of 32 heads (142 MB; 205 MB with the sectors that hold them) 34 us, 6 TB/s of sectors.  One
// page a thread took 46 us, waiting for slot, table entry and codes in turn, four pages (58 registers) 44.
constexpr int MOVE_ONCE = 2, MOVE_PAGES = 4 * MOVE_ONCE;
template <int HD>
__global__ void __launch_bounds__(512, 4) kv4_move_kernel(Kv4EvictParams p) {
  pdl_wait();
  pdl_trigger();
  using P = Kv4<HD>;
  const int bg = blockIdx.y, b = bg / p.c.G, g = bg % p.c.G, tid = threadIdx.x % 128, which = threadIdx.x / 128;
  const int page0 = blockIdx.x * MOVE_PAGES;
  __shared__ const unsigned char* sh_src[MOVE_PAGES][KV4_ROWS];  // pages of the rows; null: not kept, or no such block
  __shared__ int sh_row[MOVE_PAGES][KV4_ROWS];
  __shared__ unsigned char* sh_dst[MOVE_PAGES];
  if (threadIdx.x < MOVE_PAGES * KV4_ROWS) {
    const int i = page0 * KV4_ROWS + threadIdx.x;
    const int slot = i < p.budget ? p.kept[static_cast<size_t>(bg) * p.budget + i] : -1;
    sh_src[threadIdx.x / KV4_ROWS][threadIdx.x % KV4_ROWS] = slot >= 0 ? page_of(p.c, b, g, slot) : nullptr;
    sh_row[threadIdx.x / KV4_ROWS][threadIdx.x % KV4_ROWS] = slot & (KV4_ROWS - 1);
  } else if (threadIdx.x < MOVE_PAGES * KV4_ROWS + MOVE_PAGES) {
    const int at = threadIdx.x - MOVE_PAGES * KV4_ROWS;
    Kv4Pool d = p.c;
    d.table = p.dst_table;
    d.max_pages = p.dst_pages;
    sh_dst[at] = (page0 + at) * KV4_ROWS < p.budget ? page_of(d, b, g, (page0 + at) * KV4_ROWS) : nullptr;
  }
  __syncthreads();
  const bool is_v = tid < 64;
  const int pair = tid / 8, chunk = tid % 8;                                             // V's
  const int k_row = (tid - 64) / (P::ROW / 16), k_at = (tid - 64) % (P::ROW / 16) * 16;  // K's
  const int first = is_v ? 2 * pair : k_row < KV4_ROWS ? k_row : -1;                      // row of the page
  using Chunk = typename std::conditional<HD == 128, uint4, uint2>::type;
  constexpr int WORDS = P::CHUNK / 4;
  uint4 x[MOVE_ONCE];  // K: 16 bytes; V: the first row's chunk
  Chunk y[MOVE_ONCE];  // V: the second row's
  uint32_t scale[MOVE_ONCE];
#pragma unroll
  for (int j = 0; j < MOVE_ONCE; ++j) {
    const int at = which * MOVE_ONCE + j;
    if (!sh_dst[at]) continue;
    const unsigned char* s0 = first >= 0 ? sh_src[at][first] : nullptr;
    if (s0 && !is_v) x[j] = *reinterpret_cast<const uint4*>(s0 + sh_row[at][first] * P::ROW + k_at);
    if (is_v) {
      const int r0 = sh_row[at][first], r1 = sh_row[at][first + 1];
      const unsigned char* s1 = sh_src[at][first + 1];
      *reinterpret_cast<Chunk*>(x + j) = y[j] = Chunk{};
      if (s0) *reinterpret_cast<Chunk*>(x + j) = *reinterpret_cast<const Chunk*>(s0 + P::V + r0 / 2 * 2 * P::ROW + P::place(r0 / 2, chunk) * P::CHUNK);
      if (s1) y[j] = *reinterpret_cast<const Chunk*>(s1 + P::V + r1 / 2 * 2 * P::ROW + P::place(r1 / 2, chunk) * P::CHUNK);
    }
    if (tid < 2 * KV4_ROWS) {
      const int row = tid % KV4_ROWS;
      if (sh_src[at][row]) scale[j] = *reinterpret_cast<const uint32_t*>(sh_src[at][row] + (tid < KV4_ROWS ? P::KS : P::VS) + 4 * sh_row[at][row]);
    }
  }
#pragma unroll
  for (int j = 0; j < MOVE_ONCE; ++j) {
    const int at = which * MOVE_ONCE + j;
    unsigned char* dst = sh_dst[at];
    if (!dst) continue;
    const bool there = first >= 0 && (sh_src[at][first] || (is_v && sh_src[at][first + 1]));
    if (there && !is_v) *reinterpret_cast<uint4*>(dst + k_row * P::ROW + k_at) = x[j];
    if (there && is_v) {
      // halves of the words: row 2 pair from the half of its parity, row 2 pair + 1 likewise
      const uint32_t pick = (sh_row[at][first] & 1 ? 0x32u : 0x10u) | (sh_row[at][first + 1] & 1 ? 0x7600u : 0x5400u);
      uint32_t* a = reinterpret_cast<uint32_t*>(x + j);
      const uint32_t* c = reinterpret_cast<const uint32_t*>(y + j);
#pragma unroll
      for (int i = 0; i < WORDS; ++i) a[i] = __byte_perm(a[i], c[i], pick);
      *reinterpret_cast<Chunk*>(dst + P::V + pair * 2 * P::ROW + P::place(pair, chunk) * P::CHUNK) = *reinterpret_cast<const Chunk*>(x + j);
    }
    if (tid < 2 * KV4_ROWS && sh_src[at][tid % KV4_ROWS])
      *reinterpret_cast<uint32_t*>(dst + (tid < KV4_ROWS ? P::KS : P::VS) + 4 * (tid % KV4_ROWS)) = scale[j];
  }
}

// The rows of a call lie in rows / 2 + 1 pairs of slots at most, wherever the first one starts.
template <typename K>
cudaError_t launch_rows(K kernel, const RowArgs& a, cudaStream_t s, int each = 1) {  // each: pairs of a thread
  const int pairs = a.rows / 2 + 1, pieces = 2 * a.c.G * (a.c.hd / 8);
  int x = std::min(pieces, 256);
  if (x > 128 && x % 32) x = 128;
  int y = 256 / x;
  y -= x * y % 32 ? y % 2 : 0;  // whole warps (pieces are a multiple of 16)
  return launch_pdl(kernel, dim3((pairs + y * each - 1) / (y * each), (pieces + x - 1) / x, a.c.B), dim3(x, y), 0, s, a, pairs);
}
RowArgs row_args(const Kv4Pool& c, void* k, void* v, int f32, int ldk, int ldv, int rows, const int* slot0, const int* counts) {
  const int wide = f32 ? 4 : 8;  // values in 16 bytes
  const bool vec = (reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % 16 == 0 && ldk % wide == 0 && ldv % wide == 0;
  return RowArgs{c, k, v, ldk, ldv, rows, slot0, counts, vec};
}

}  // namespace

cudaError_t kv4_append(const Kv4Pool& c, const void* k, const void* v, int f32, int ldk, int ldv, int rows,
                       const int* slot0, const int* counts, cudaStream_t s) {
  const RowArgs a = row_args(c, const_cast<void*>(k), const_cast<void*>(v), f32, ldk, ldv, rows, slot0, counts);
  if (c.hd == 128)
    return f32 ? launch_rows(kv4_append_kernel<128, float>, a, s, APPEND_PAIRS) : launch_rows(kv4_append_kernel<128, bf16>, a, s, APPEND_PAIRS);
  return f32 ? launch_rows(kv4_append_kernel<64, float>, a, s, APPEND_PAIRS) : launch_rows(kv4_append_kernel<64, bf16>, a, s, APPEND_PAIRS);
}

cudaError_t kv4_read(const Kv4Pool& c, void* k, void* v, int f32, int ldk, int ldv, int rows, const int* slot0,
                     const int* counts, cudaStream_t s) {
  const RowArgs a = row_args(c, k, v, f32, ldk, ldv, rows, slot0, counts);
  if (c.hd == 128)
    return f32 ? launch_rows(kv4_read_kernel<128, float>, a, s) : launch_rows(kv4_read_kernel<128, bf16>, a, s);
  return f32 ? launch_rows(kv4_read_kernel<64, float>, a, s) : launch_rows(kv4_read_kernel<64, bf16>, a, s);
}

cudaError_t kv4_evict(const Kv4EvictParams& p, cudaStream_t s) {
  const int bg = p.c.B * p.c.G;
  cudaError_t e = launch_pdl(kv4_select_kernel, dim3(bg), dim3(SEL_THREADS), 0, s, p);
  if (e != cudaSuccess) return e;
  const dim3 grid(((p.budget + KV4_ROWS - 1) / KV4_ROWS + MOVE_PAGES - 1) / MOVE_PAGES, bg);
  return p.c.hd == 128 ? launch_pdl(kv4_move_kernel<128>, grid, dim3(512), 0, s, p)
                       : launch_pdl(kv4_move_kernel<64>, grid, dim3(512), 0, s, p);
}

}  // namespace chimera
