// The line of work of the paged attention kernels.  An item is a set of query rows of one sequence that share a key head;
// it meets the cached tokens it sees in units of 128.  All units of all items, sequence by sequence, are laid out on one
// line that is cut into equal pieces, one per block: lengths may differ as they like, every block has the same work.
// Where a piece ends inside an item its partial result goes to scratch and is merged with the others'.
#pragma once

#include "xkv_paged_internal.cuh"

namespace xkv {
namespace {

constexpr int kUnit = 128;

struct Cut {
  uint32_t piece, longer;          // the first `longer` pieces have piece + 1 units, the others `piece`
  __device__ __forceinline__ Cut(uint32_t total, uint32_t grid) { piece = total / grid; longer = total - piece * grid; }
  __device__ __forceinline__ uint32_t start(uint32_t b) const { return b * piece + min(b, longer); }
  __device__ __forceinline__ uint32_t owner(uint32_t unit) const {
    const uint32_t head = longer * (piece + 1);
    return unit < head ? unit / (piece + 1) : longer + (unit - head) / piece;
  }
};

// prefix[s] = units before sequence s, prefix[n_seqs] = all of them; `units` gives a sequence's.  All THREADS threads of the block
// (at least 32 * 32 / 8, a multiple of 32) call it; it ends with a barrier.
template <int THREADS, typename F>
__device__ __forceinline__ void line_prefix(int n_seqs, uint32_t* prefix, uint32_t* s_warp, F units) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (n_seqs + THREADS - 1) / THREADS;
  uint32_t sum = 0;
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    const uint32_t u = s < n_seqs ? units(s) : 0u;
    if (s < n_seqs) prefix[s] = sum;               // (of this thread's own so far)
    sum += u;
  }
  uint32_t inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) s_warp[warp] = inc;
  __syncthreads();
  uint32_t before = inc - sum;
  for (int w = 0; w < warp; ++w) before += s_warp[w];
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    if (s < n_seqs) prefix[s] += before;
  }
  if (tid == THREADS - 1) prefix[n_seqs] = before + sum;
  __syncthreads();
}

// The sequence that a unit belongs to: the last s with prefix[s] <= unit (sequences without units are skipped).
__device__ __forceinline__ int line_seq(const uint32_t* prefix, int n_seqs, uint32_t unit) {
  int lo = 0, hi = n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= unit) lo = mid; else hi = mid;
  }
  return lo;
}

}  // namespace
}  // namespace xkv
