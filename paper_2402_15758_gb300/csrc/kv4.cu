// The 4-bit KV cache's rows: written from fresh K and V rows, read back, and moved when the rows
// that drew little attention leave (layout and rounding rule in kv4.cuh).
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
};

// A warp rounds one row of one head, K or V: lane l has channels E l .. E l + E - 1 (E = HD / 32),
// a minimum and a maximum over the warp, and one store of E codes.
template <int HD, typename T>
__global__ void __launch_bounds__(256) kv4_append_kernel(RowArgs a) {
  pdl_wait();
  pdl_trigger();
  constexpr int E = HD / 32;
  const int lane = threadIdx.x & 31;
  const long long item = static_cast<long long>(blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32;
  const long long items = 2LL * a.c.B * a.rows * a.c.G;
  if (item >= items) return;
  const int g = static_cast<int>(item % a.c.G);
  const int which = static_cast<int>(item / a.c.G % 2);
  const long long r = item / (2 * a.c.G);
  const int b = static_cast<int>(r / a.rows), i = static_cast<int>(r % a.rows);
  if (a.counts && i >= a.counts[b]) return;
  const T* src = static_cast<const T*>(which ? a.v : a.k) + r * (which ? a.ldv : a.ldk) + g * HD + lane * E;
  float x[E];
#pragma unroll
  for (int j = 0; j < E; ++j) x[j] = to_f<T>(src[j]);
  const int slot = a.slot0[b] + i;
  unsigned char* page = page_of(a.c, b, g, slot);
  if (!page) return;
  float lo = x[0], hi = x[0];
  bool fine = true;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    lo = fminf(lo, x[j]);
    hi = fmaxf(hi, x[j]);
    fine = fine && isfinite(x[j]);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  fine = __all_sync(0xffffffffu, fine) && isfinite(hi - lo);
  const bf16 base16 = __float2bfloat16_rn(lo), step16 = __float2bfloat16_rn(__fmul_rn(hi - lo, 1.f / 15.f));
  const float base = __bfloat162float(base16), step = __bfloat162float(step16);
  fine = fine && isfinite(base);
  uint32_t codes = 0;
  if (fine && step > 0.f) {
#pragma unroll
    for (int j = 0; j < E; ++j)
      codes |= static_cast<uint32_t>(fminf(fmaxf(rintf(__fdiv_rn(x[j] - base, step)), 0.f), 15.f)) << (4 * j);
  }
  const int row = slot % KV4_ROWS;
  using P = Kv4<HD>;
  if (E == 4) {
    unsigned char* at = which ? page + P::v_half(row, lane) : page + row * P::ROW + 2 * lane;
    *reinterpret_cast<uint16_t*>(at) = static_cast<uint16_t>(codes);
  } else {
    unsigned char* at = which ? page + P::v_half(row, lane / 2) + (lane & 1) : page + row * P::ROW + lane;
    *at = static_cast<unsigned char>(codes);
  }
  if (lane == 0) {
    const uint32_t s16 = fine ? __bfloat16_as_ushort(step16) : 0u, b16 = fine ? __bfloat16_as_ushort(base16) : 0x7fc0u;
    *reinterpret_cast<uint32_t*>(page + (which ? P::VS : P::KS) + 4 * row) = s16 | b16 << 16;
  }
}

template <int HD, typename T>
__global__ void __launch_bounds__(256) kv4_read_kernel(RowArgs a) {
  pdl_wait();
  pdl_trigger();
  constexpr int E = HD / 32;
  const int lane = threadIdx.x & 31;
  const long long item = static_cast<long long>(blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32;
  const long long items = 2LL * a.c.B * a.rows * a.c.G;
  if (item >= items) return;
  const int g = static_cast<int>(item % a.c.G);
  const int which = static_cast<int>(item / a.c.G % 2);
  const long long r = item / (2 * a.c.G);
  const int b = static_cast<int>(r / a.rows), i = static_cast<int>(r % a.rows);
  if (a.counts && i >= a.counts[b]) return;
  const int slot = a.slot0[b] + i;
  const unsigned char* page = page_of(a.c, b, g, slot);
  if (!page) return;
  const int row = slot % KV4_ROWS;
  using P = Kv4<HD>;
  uint32_t codes;
  if (E == 4)
    codes = *reinterpret_cast<const uint16_t*>(which ? page + P::v_half(row, lane) : page + row * P::ROW + 2 * lane);
  else
    codes = *(which ? page + P::v_half(row, lane / 2) + (lane & 1) : page + row * P::ROW + lane);
  const uint32_t w = *reinterpret_cast<const uint32_t*>(page + (which ? P::VS : P::KS) + 4 * row);
  T* dst = static_cast<T*>(which ? a.v : a.k) + r * (which ? a.ldv : a.ldk) + g * HD + lane * E;
#pragma unroll
  for (int j = 0; j < E; ++j) dst[j] = from_f<T>(fmaf(kv4_step(w), static_cast<float>(codes >> (4 * j) & 15u), kv4_base(w)));
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

// Sum of v over the threads before this one, and the total, for the whole block.
__device__ __forceinline__ int block_before(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < SEL_THREADS / 32; ++w) {
    if (w < warp) before += warp_sums[w];
    total += warp_sums[w];
  }
  return before + x - v;
}

// One block per (sequence, head): the kept slots.  The (budget - recent)-th largest key of the
// older slots is found digit by digit (four passes of 8 bits), then one ordered pass takes
// every slot above it and the first ones that equal it.
__global__ void __launch_bounds__(SEL_THREADS) kv4_select_kernel(Kv4EvictParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ int hist[256];
  __shared__ int warp_sums[SEL_THREADS / 32];
  __shared__ uint32_t sh_prefix;
  __shared__ int sh_need;
  const int bg = blockIdx.x, b = bg / p.c.G, tid = threadIdx.x;
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
  uint32_t prefix = 0;
  int need = want;  // keys with this prefix that stay
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < older; i += SEL_THREADS) {
      const uint32_t key = order_key(x[i]);
      if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&hist[key >> shift & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int d = 255, left = need;
      while (d > 0 && hist[d] < left) left -= hist[d--];
      sh_prefix = prefix << 8 | d;
      sh_need = left;
    }
    __syncthreads();
    prefix = sh_prefix;
    need = sh_need;
    __syncthreads();
  }
  // thread t takes a contiguous part of the older slots, so that the order of threads is the slots'
  const int per = (older + SEL_THREADS - 1) / SEL_THREADS;
  const int i0 = min(tid * per, older), i1 = min(i0 + per, older);
  int above = 0, equal = 0, total;
  for (int i = i0; i < i1; ++i) {
    const uint32_t key = order_key(x[i]);
    above += key > prefix;
    equal += key == prefix;
  }
  int before_equal = block_before(equal, warp_sums, total);
  const int mine = min(max(need - before_equal, 0), equal);
  int at = block_before(above + mine, warp_sums, total);
  int left = mine;
  for (int i = i0; i < i1; ++i) {
    const uint32_t key = order_key(x[i]);
    if (key > prefix || (key == prefix && left-- > 0)) {
      kept[at] = i;
      out[at] = x[i];
      ++at;
    }
  }
}

// One block per (destination page, sequence and head): gathers the 16 rows kept there.
template <int HD>
__global__ void __launch_bounds__(128) kv4_move_kernel(Kv4EvictParams p) {
  pdl_wait();
  pdl_trigger();
  using P = Kv4<HD>;
  const int bg = blockIdx.y, b = bg / p.c.G, g = bg % p.c.G, page = blockIdx.x, tid = threadIdx.x;
  __shared__ const unsigned char* src[KV4_ROWS];
  __shared__ int row_of[KV4_ROWS];
  __shared__ unsigned char* dst;
  if (tid < KV4_ROWS) {
    const int i = page * KV4_ROWS + tid;
    const int slot = i < p.budget ? p.kept[static_cast<size_t>(bg) * p.budget + i] : -1;
    src[tid] = slot >= 0 ? page_of(p.c, b, g, slot) : nullptr;
    row_of[tid] = slot % KV4_ROWS;
  }
  if (tid == KV4_ROWS) {
    Kv4Pool d = p.c;
    d.table = p.dst_table;
    d.max_pages = p.dst_pages;
    dst = page_of(d, b, g, page * KV4_ROWS);
  }
  __syncthreads();
  if (!dst || !__syncthreads_or(tid < KV4_ROWS && src[tid])) return;
  for (int w = tid; w < KV4_ROWS * HD / 8; w += 128) {  // K words
    const int row = w / (HD / 8), c = w % (HD / 8);
    if (src[row])
      *reinterpret_cast<uint32_t*>(dst + row * P::ROW + 4 * c) =
          *reinterpret_cast<const uint32_t*>(src[row] + row_of[row] * P::ROW + 4 * c);
  }
  for (int w = tid; w < KV4_ROWS * HD / 4; w += 128) {  // V halfwords
    const int row = w / (HD / 4), c = w % (HD / 4);
    if (src[row])
      *reinterpret_cast<uint16_t*>(dst + P::v_half(row, c)) = *reinterpret_cast<const uint16_t*>(src[row] + P::v_half(row_of[row], c));
  }
  if (tid < 2 * KV4_ROWS) {
    const int row = tid % KV4_ROWS, at = tid < KV4_ROWS ? P::KS : P::VS;
    if (src[row])
      *reinterpret_cast<uint32_t*>(dst + at + 4 * row) = *reinterpret_cast<const uint32_t*>(src[row] + at + 4 * row_of[row]);
  }
}

template <typename K>
cudaError_t launch_rows(K kernel, const RowArgs& a, cudaStream_t s) {
  const long long warps = 2LL * a.c.B * a.rows * a.c.G;
  if (warps == 0) return cudaSuccess;
  return launch_pdl(kernel, dim3(static_cast<unsigned>((warps + 7) / 8)), dim3(256), 0, s, a);
}

}  // namespace

cudaError_t kv4_append(const Kv4Pool& c, const void* k, const void* v, int f32, int ldk, int ldv, int rows,
                       const int* slot0, const int* counts, cudaStream_t s) {
  const RowArgs a{c, const_cast<void*>(k), const_cast<void*>(v), ldk, ldv, rows, slot0, counts};
  if (c.hd == 128)
    return f32 ? launch_rows(kv4_append_kernel<128, float>, a, s) : launch_rows(kv4_append_kernel<128, bf16>, a, s);
  return f32 ? launch_rows(kv4_append_kernel<64, float>, a, s) : launch_rows(kv4_append_kernel<64, bf16>, a, s);
}

cudaError_t kv4_read(const Kv4Pool& c, void* k, void* v, int f32, int ldk, int ldv, int rows, const int* slot0,
                     const int* counts, cudaStream_t s) {
  const RowArgs a{c, k, v, ldk, ldv, rows, slot0, counts};
  if (c.hd == 128)
    return f32 ? launch_rows(kv4_read_kernel<128, float>, a, s) : launch_rows(kv4_read_kernel<128, bf16>, a, s);
  return f32 ? launch_rows(kv4_read_kernel<64, float>, a, s) : launch_rows(kv4_read_kernel<64, bf16>, a, s);
}

cudaError_t kv4_evict(const Kv4EvictParams& p, cudaStream_t s) {
  const int bg = p.c.B * p.c.G;
  cudaError_t e = launch_pdl(kv4_select_kernel, dim3(bg), dim3(SEL_THREADS), 0, s, p);
  if (e != cudaSuccess) return e;
  const dim3 grid((p.budget + KV4_ROWS - 1) / KV4_ROWS, bg);
  return p.c.hd == 128 ? launch_pdl(kv4_move_kernel<128>, grid, dim3(128), 0, s, p)
                       : launch_pdl(kv4_move_kernel<64>, grid, dim3(128), 0, s, p);
}

}  // namespace chimera
