// Eviction by accumulated weight: per sequence and key head the first, the recent and the heaviest tokens are
// found (a radix selection on the bits of the weights), and their rows copied to other pages.
//
// The order of the weights is that of their bits as unsigned numbers after the usual flip (a negative number has all
// bits flipped, another its sign bit); -0 counts as +0, a NaN as less than everything.  Protected tokens never enter
// the selection.  Ties go to the lower slot.
//
// Measured: eight sequences up to 16 385 tokens cut to 8192, 8 key heads of 128: 79 us, of which the rows take 52 (5.2 TB/s) and the
// selection 22 (its latencies and a block's instructions per token; two of the eight sequences are longer than 8192, which is 16
// blocks, and the copies wait for them); 1285 tokens of 16 heads cut to 1024: 9.7 us.
#include "xkv_paged_internal.cuh"

namespace xkv {

namespace {

constexpr int kSelThreads = 1024;
constexpr int kHeld = 49152;             // keys held in shared memory (longer sequences: the rest is read again)

__device__ __forceinline__ uint32_t order_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix over the block's threads of two counts packed into 64 bits; total in *sum.
__device__ __forceinline__ uint64_t block_prefix(uint64_t x, uint64_t* s_warp, uint64_t* sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = inc;
  __syncthreads();
  if (warp == 0) {
    uint64_t w = s_warp[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    s_warp[lane] = w;
  }
  __syncthreads();
  *sum = s_warp[31];
  return inc - x + (warp ? s_warp[warp - 1] : 0ull);
}

// One block per (key head, sequence): what it keeps, in order, to kept.
__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const __grid_constant__ EvictArgs a, int held) {
  extern __shared__ uint32_t s_key[];                 // [held] keys of the middle tokens
  __shared__ uint32_t s_hist[2048];
  __shared__ uint64_t s_warp[32];
  __shared__ uint32_t s_found[2];                     // digit, rank left
  grid_dependency_wait();
  const int h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x;
  int len = a.seqs.lens[s];
  if (!seq_len_ok(a.cache, a.seqs, len)) {
    if (tid == 0) paged_report(a.cache.status, (int)XKV_E_INVALID);
    len = 0;
  }
  int32_t* kept = a.kept + ((int64_t)s * a.cache.n_kv_heads + h) * a.keep;
  if (h == 0 && tid == 0) a.lens_out[s] = min(len, a.keep);
  if (len <= a.keep) {
    for (int i = tid; i < a.keep; i += kSelThreads) kept[i] = i < len ? i : -1;
    return;
  }
  const int lo = a.n_first, n = len - a.n_first - a.n_recent;       // the middle, n > want
  const int want = a.keep - a.n_first - a.n_recent;
  for (int i = tid; i < lo; i += kSelThreads) kept[i] = i;
  for (int i = tid; i < a.n_recent; i += kSelThreads) kept[lo + want + i] = len - a.n_recent + i;
  if (want == 0) return;
  const int32_t* table = a.seqs.table + (int64_t)s * a.seqs.table_width;
  const int shift = a.cache.page_shift;
  auto key_on = [&](int page, int j) {                // key of middle token j on that page
    if ((unsigned)page < (unsigned)a.cache.n_pages) return order_key(a.cache.weights[weight_offset(a.cache, page, h, lo + j)]);
    paged_report(a.cache.status, (int)XKV_E_INVALID);
    return order_key(0.f);                            // a page that does not exist reads as zero
  };
  const int in_smem = min(n, held);
  constexpr int kAhead = 8;                           // tokens of a thread whose pages, and then weights, are asked for at once
  for (int j0 = tid; j0 < in_smem; j0 += kAhead * kSelThreads) {
    int page[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u * kSelThreads;
      page[u] = j < in_smem ? table[(lo + j) >> shift] : 0;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u * kSelThreads;
      if (j < in_smem) s_key[j] = key_on(page[u], j);
    }
  }
  auto key = [&](int j) { return j < in_smem ? s_key[j] : key_on(table[(lo + j) >> shift], j); };
  // three digits of 11, 11 and 10 bits from the top: the want-th largest key
  uint32_t prefix = 0;
  int left = want;                                    // rank, from the top, among the keys that match the prefix
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const int digits = pass == 2 ? 1024 : 2048;
    const uint32_t above = pass == 0 ? 0u : pass == 1 ? 0xFFE00000u : 0xFFFFFC00u;
    for (int i = tid; i < 2048; i += kSelThreads) s_hist[i] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += kSelThreads) {
      const uint32_t k = key(j);
      if ((k & above) == prefix) atomicAdd(&s_hist[(k >> low) & (digits - 1)], 1u);
    }
    __syncthreads();
    // thread t owns digits 2t and 2t + 1 counted from the top
    const int d0 = digits - 1 - 2 * tid, d1 = d0 - 1;
    const uint32_t c0 = d0 >= 0 ? s_hist[d0] : 0u, c1 = d1 >= 0 ? s_hist[d1] : 0u;
    uint64_t sum;
    const uint32_t before = (uint32_t)block_prefix((uint64_t)c0 + c1, s_warp, &sum);
    if (before < (uint32_t)left && before + c0 + c1 >= (uint32_t)left) {
      const bool first = before + c0 >= (uint32_t)left;
      s_found[0] = (uint32_t)(first ? d0 : d1);
      s_found[1] = (uint32_t)left - before - (first ? 0u : c0);
    }
    __syncthreads();
    prefix |= s_found[0] << low;
    left = (int)s_found[1];
    __syncthreads();
  }
  // kept: every key above `prefix`, and the first `left` that equal it.  A thread owns a run of tokens
  // (an odd number of them: no two threads of a warp on one bank).
  const int run = ((n + kSelThreads - 1) / kSelThreads) | 1;
  const int j0 = min(n, tid * run), j1 = min(n, j0 + run);
  uint32_t more = 0, same = 0;
  for (int j = j0; j < j1; ++j) {
    const uint32_t k = key(j);
    more += k > prefix;
    same += k == prefix;
  }
  uint64_t sum;
  const uint64_t before = block_prefix(((uint64_t)same << 32) | more, s_warp, &sum);
  uint32_t at_more = (uint32_t)before, at_same = (uint32_t)(before >> 32);
  for (int j = j0; j < j1; ++j) {
    const uint32_t k = key(j);
    if (k > prefix || (k == prefix && at_same < (uint32_t)left))
      kept[lo + at_more + min(at_same, (uint32_t)left)] = lo + j;
    at_more += k > prefix;
    at_same += k == prefix;
  }
}

// Rows of the survivors to their new pages: a 16-byte piece of K and of V per thread and step, kU steps in flight.
constexpr int kMoveThreads = 256;
constexpr int kU = 2;                   // (8 sequences cut to 8192 tokens: 4 in flight 86 us, 8 104, 2 79)
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ EvictArgs a, int lanes_log2) {
  grid_dependency_wait();
  const int s = blockIdx.z, h = blockIdx.y;
  const int piece = threadIdx.x & ((1 << lanes_log2) - 1);
  const int rows = kMoveThreads >> lanes_log2;
  const int32_t* kept = a.kept + ((int64_t)s * a.cache.n_kv_heads + h) * a.keep;
  const int n = a.lens_out[s];
  const int i0 = blockIdx.x * rows * kU + (threadIdx.x >> lanes_log2);
  uint4 k[kU], v[kU];
  float w[kU];
  int64_t to[kU], to_w[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    const int i = i0 + u * rows;
    to[u] = -1;
    if (i >= n) continue;
    const int slot = kept[i];
    const int src = page_at(a.cache, a.seqs.table, a.seqs.table_width, s, slot);
    const int dst = page_at(a.cache, a.dst_table, a.dst_width, s, i);
    if (dst < 0) continue;
    if (src < 0) {                                       // a page that does not exist reads as zero
      const int64_t at = 2 * row_offset(a.cache, dst, h, i) + 16 * piece;
      *reinterpret_cast<uint4*>(a.cache.k + at) = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(a.cache.v + at) = make_uint4(0, 0, 0, 0);
      if (piece == 0) a.cache.weights[weight_offset(a.cache, dst, h, i)] = 0.f;
      continue;
    }
    const int64_t from = 2 * row_offset(a.cache, src, h, slot) + 16 * piece;
    k[u] = *reinterpret_cast<const uint4*>(a.cache.k + from);
    v[u] = *reinterpret_cast<const uint4*>(a.cache.v + from);
    w[u] = a.cache.weights[weight_offset(a.cache, src, h, slot)];
    to[u] = 2 * row_offset(a.cache, dst, h, i) + 16 * piece;
    to_w[u] = weight_offset(a.cache, dst, h, i);
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    if (to[u] < 0) continue;
    *reinterpret_cast<uint4*>(a.cache.k + to[u]) = k[u];
    *reinterpret_cast<uint4*>(a.cache.v + to[u]) = v[u];
    if (piece == 0) a.cache.weights[to_w[u]] = w[u];
  }
}

}  // namespace

cudaError_t evict_device_setup() {
  return cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeld * 4);
}

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t st) {
  // keys of the longest sequence the table can hold, up to what fits
  const int64_t longest = (int64_t)a.seqs.table_width << a.cache.page_shift;
  int held = (int)(longest < kHeld ? longest : kHeld);
  void* p0[2] = {(void*)&a, (void*)&held};
  cudaError_t e = launch_overlapped((const void*)evict_select_kernel, dim3(a.cache.n_kv_heads, a.seqs.n_seqs), dim3(kSelThreads), p0,
                                    (size_t)held * 4, st);
  if (e != cudaSuccess) return e;
  int lanes_log2 = a.head_dim == 64 ? 3 : 4;
  const int rows = (kMoveThreads >> lanes_log2) * kU;
  void* p1[2] = {(void*)&a, (void*)&lanes_log2};
  e = launch_overlapped((const void*)evict_move_kernel, dim3((a.keep + rows - 1) / rows, a.cache.n_kv_heads, a.seqs.n_seqs), dim3(kMoveThreads), p1, 0, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace xkv
