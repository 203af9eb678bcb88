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

// What is done once per item (queries, first scores, merging, results) takes as long as some units.  Where a block's piece is long
// an item therefore has kItemCost more places on the line than it has units, so that blocks with many short items have fewer
// units; where pieces are a few units only, those count.
constexpr uint32_t kItemCost = 2, kLongPiece = 8;

// prefix[s] = places on the line before sequence s, prefix[n_seqs] = all of them; `work` gives a sequence's items and units.  All THREADS
// threads of the block (a multiple of 32) call it; it ends with a barrier.  Returns the places that an item has more than units.
struct Work { uint32_t items, units; };
template <int THREADS, typename F>
__device__ __forceinline__ uint32_t line_prefix(int n_seqs, uint32_t* prefix, uint2* s_warp, F work) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (n_seqs + THREADS - 1) / THREADS;
  uint2 sum = make_uint2(0, 0);
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    if (s >= n_seqs) break;
    const Work w = work(s);
    sum.x += w.items; sum.y += w.units;
  }
  uint2 inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, inc.x, o), y = __shfl_up_sync(0xffffffffu, inc.y, o);
    if (lane >= o) { inc.x += x; inc.y += y; }
  }
  if (lane == 31) s_warp[warp] = inc;
  __syncthreads();
  uint2 before = make_uint2(inc.x - sum.x, inc.y - sum.y), all = make_uint2(0, 0);
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) { before.x += s_warp[w].x; before.y += s_warp[w].y; }
    all.x += s_warp[w].x; all.y += s_warp[w].y;
  }
  const uint32_t cost = all.y >= kLongPiece * gridDim.x ? kItemCost : 0;
  for (int i = 0; i < per; ++i) {
    const int s = tid * per + i;
    if (s >= n_seqs) break;
    prefix[s] = before.y + cost * before.x;
    const Work w = work(s);
    before.x += w.items; before.y += w.units;
  }
  if (tid == 0) prefix[n_seqs] = all.y + cost * all.x;
  __syncthreads();
  return cost;
}

// The sequence that a place belongs to: the last s with prefix[s] <= place (sequences without work are skipped).
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
