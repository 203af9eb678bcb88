// Declarations shared by the translation units of the paged cache and the rotary positions.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "xkv_internal.cuh"
#include "xkv_paged.h"

namespace xkv {

constexpr int kMaxSeqs = 1024;
constexpr int kMaxPairs = 64;            // turned pairs of a token, all axes (head_dim / 2)

// ---- what a kernel knows of the cache and of a call's sequences ----------------

struct PagedView {
  uint8_t* k; uint8_t* v;                // pools
  float* weights;                        // [n_pages][n_kv_heads][page_tokens], or null
  int64_t page_stride, head_stride, slot_stride;     // elements (of 2 bytes)
  int n_heads, n_kv_heads, group;        // group = query heads of a key head
  int page_shift, n_pages;
  int* status;
};

struct SeqView {
  int n_seqs, n_tokens, max_new, table_width;
  const int32_t* q_start; const int32_t* lens; const int32_t* table;
};

// The tokens of one sequence: rows [row0, row0 + n_new) of the token tensors, len cached tokens with them.
struct Seq { int row0, n_new, len; };

#ifdef __CUDACC__
__device__ __forceinline__ void paged_report(int* status, int code) { atomicCAS(status, 0, code); }

__device__ __forceinline__ bool seq_len_ok(const PagedView& c, const SeqView& b, int len) {
  return len >= 0 && len <= (b.table_width << c.page_shift);
}
// Sequence s with its numbers checked; one that reaches outside its bounds is empty.
__device__ __forceinline__ Seq seq_at(const PagedView& c, const SeqView& b, int s) {
  const int lo = b.q_start[s], hi = b.q_start[s + 1], len = b.lens[s];
  const bool ok = lo >= 0 && hi >= lo && hi <= b.n_tokens && hi - lo <= b.max_new && seq_len_ok(c, b, len);
  if (!ok) paged_report(c.status, (int)XKV_E_INVALID);
  Seq q;
  q.row0 = ok ? lo : 0;
  q.n_new = ok ? hi - lo : 0;
  q.len = ok ? len : 0;
  return q;
}
// Page of a slot (0 <= slot < len), or -1 if the table names none.
__device__ __forceinline__ int page_at(const PagedView& c, const int32_t* table, int table_width, int s, int slot) {
  const int p = table[(int64_t)s * table_width + (slot >> c.page_shift)];
  if ((unsigned)p < (unsigned)c.n_pages) return p;
  paged_report(c.status, (int)XKV_E_INVALID);
  return -1;
}
__device__ __forceinline__ int64_t row_offset(const PagedView& c, int page, int head, int slot) {
  return (int64_t)page * c.page_stride + (int64_t)head * c.head_stride +
         (int64_t)(slot & ((1 << c.page_shift) - 1)) * c.slot_stride;
}
__device__ __forceinline__ int64_t weight_offset(const PagedView& c, int page, int head, int slot) {
  return (((int64_t)page * c.n_kv_heads + head) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));
}
#endif

// ---- tokens: rotary positions, append ------------------------------------------

struct RotaryPlan {
  int pairs, axes, rot, interleaved;     // pairs of one axis
  float magnitude;                       // negative angles for the inverse are in `turns`
  const int32_t* positions; int64_t pos_stride;
  double turns[kMaxPairs];               // turns per position of pair i (an angle over 2 pi)
};

struct TokenTensor {
  const uint8_t* in; uint8_t* out;       // out null: to the pages
  int64_t in_ts, in_hs, out_ts, out_hs;  // elements
  int heads;
};

struct TokenArgs {
  TokenTensor q, k, v;                   // heads = 0: absent
  RotaryPlan rot;                        // axes = 0: nothing is turned
  int n, head_dim;
  int append;                            // k, v and weights go to the pages
  PagedView cache; SeqView seqs;
};
cudaError_t launch_tokens(const TokenArgs& a, int dtype, int sm_count, cudaStream_t st);

// ---- eviction ------------------------------------------------------------------

struct EvictArgs {
  PagedView cache; SeqView seqs;
  const int32_t* dst_table; int dst_width;
  int keep, n_first, n_recent, head_dim;
  int32_t* kept; int32_t* lens_out;
};
cudaError_t launch_evict(const EvictArgs& a, cudaStream_t st);
cudaError_t evict_device_setup();

// ---- attention and weights -------------------------------------------------------

struct PagedAttnArgs {
  PagedView cache; SeqView seqs;
  const uint8_t* q; int64_t q_ts, q_hs;
  uint8_t* out; int64_t o_ts, o_hs;
  float* lse;
  float scale_log2;
  int full;                              // every token of the sequence is seen
};

// Tensor maps of the two pools for copies of `rows` token slots by 64 channels (16-byte pieces permuted within 128-byte
// rows as the matrix operands want them), and scratch: partial results of work that was cut between blocks.
struct PoolMaps { CUtensorMap k, v; };
struct PagedScratch {
  float* o;              // [2 * blocks][rows][head_dim] accumulators
  float2* ml;            // [2 * blocks][rows] running maximum (log2 units) and sum
  unsigned int* count;   // [blocks] arrivals at the item that starts in a block and goes on in the next one (0 between calls)
  unsigned int* again;   // [2 + max_seqs] the chunk kernel's: whether any, blocks done, sequences with rows to look at again (0 between calls)
};
constexpr int kFewRows = 16;       // rows of the kernel for few rows (a tile of a warp's matrix instruction)
constexpr int kChunkRows = 256;    // rows of the kernel for chunks (two tiles of tcgen05.mma)
cudaError_t make_pool_maps(const PagedView& c, int head_dim, int dtype, int rows, PoolMaps* maps);
cudaError_t attn_few_setup();
// group * max_new <= kFewRows
cudaError_t launch_attn_few(const PagedAttnArgs& a, const PoolMaps& maps, const PagedScratch& s, int head_dim, int dtype, int sm_count,
                            cudaStream_t st);
size_t attn_chunk_cut_bytes();
cudaError_t attn_chunk_setup();
// Any numbers of new tokens; maps: copies of min(page_tokens, 128) slots; cuts: attn_chunk_cut_bytes() per multiprocessor.
cudaError_t launch_attn_chunk(const PagedAttnArgs& a, const PoolMaps& maps, const PagedScratch& s, void* cuts, int head_dim, int dtype,
                              int sm_count, cudaStream_t st);
// Tensor map of a token tensor: boxes of 64 channels, `heads` heads and `toks` tokens.
cudaError_t make_token_map(const void* base, int64_t ts, int64_t hs, int n, int n_heads, int head_dim, int dtype, int heads, int toks,
                           CUtensorMap* map);
cudaError_t launch_paged_attn_simple(const PagedAttnArgs& a, int head_dim, int dtype, cudaStream_t st);

struct PagedWeightArgs {
  PagedView cache; SeqView seqs;
  const uint8_t* q; int64_t q_ts, q_hs;
  const float* lse;
  float scale_log2, decay;
  int full;
};
cudaError_t weights_setup();
// maps: as for launch_attn_chunk
cudaError_t launch_paged_weights(const PagedWeightArgs& a, const PoolMaps& maps, int head_dim, int dtype, int sm_count, cudaStream_t st);

}  // namespace xkv

struct xkv_paged {
  xkv_paged_params p;
  xkv::PagedView view;
  int sm_count, device;
  uint8_t* ws; size_t ws_bytes;
  xkv::PagedScratch scratch;
  xkv::PoolMaps maps16, maps_page;       // 16 slots at a time, min(page_tokens, 128) slots at a time
  void* cuts;
};
