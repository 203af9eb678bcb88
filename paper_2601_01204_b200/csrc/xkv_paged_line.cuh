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

// What is done once per item (queries, first scores, merging, results) takes as long as some units.  An item therefore has kItemCost
// more places on the line than units, so that blocks with many short items have fewer units.  (Chunks of four prompts 617 us
// without, 583 with 2, 585 with 4, at that time; 64 decoding sequences 154 -> 111 together with a shorter merge.  A unit of an item
// that has one tile alone takes as long as one of two: counted as half, a frame over 16384 tokens 136 -> 164 us.)
// Where pieces are a few units only, those count, and items cost nothing, unless ALWAYS: a constant, which the chunk attention has
// registers for (532 us instead of 538).
constexpr uint32_t kItemCost = 2, kLongPiece = 8;

// prefix[s] = places on the line before sequence s, prefix[n_seqs] = all of them; `work` gives a sequence's items and units.  All THREADS
// threads of the block (a multiple of 32) call it; it ends with a barrier.  Returns the places that an item has more than units.
struct Work { uint32_t items, units; };
template <int THREADS, bool ALWAYS, typename F>
__device__ __forceinline__ uint32_t line_prefix(int n_seqs, uint32_t* prefix, uint2* s_warp, F work) {
  constexpr int kPer = (kMaxSeqs + THREADS - 1) / THREADS;       // sequences of a thread
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Work w[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int s = i * THREADS + tid;                             // (in rounds of THREADS sequences)
    w[i] = s < n_seqs ? work(s) : Work{0u, 0u};
  }
  uint2 done = make_uint2(0, 0);                                 // of the rounds before
  uint2 before[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (i > 0 && i * THREADS >= n_seqs) break;
    uint2 inc = make_uint2(w[i].items, w[i].units);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, inc.x, o), y = __shfl_up_sync(0xffffffffu, inc.y, o);
      if (lane >= o) { inc.x += x; inc.y += y; }
    }
    if (i > 0) __syncthreads();
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    before[i] = make_uint2(done.x + inc.x - w[i].items, done.y + inc.y - w[i].units);
    for (int v = 0; v < THREADS / 32; ++v) {
      if (v < warp) { before[i].x += s_warp[v].x; before[i].y += s_warp[v].y; }
      done.x += s_warp[v].x; done.y += s_warp[v].y;
    }
  }
  const uint32_t cost = ALWAYS || done.y >= kLongPiece * gridDim.x ? kItemCost : 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int s = i * THREADS + tid;
    if (s < n_seqs) prefix[s] = before[i].y + cost * before[i].x;
  }
  if (tid == 0) prefix[n_seqs] = done.y + cost * done.x;
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
