// Attention over the paged cache without tensor cores: a warp per query row, fp32 throughout.  Kept as an
// independent cross-check of the other kernels (impl = 1); never the default.
#include "xkv_paged_row.cuh"

namespace xkv {

namespace {

template <typename T, int D>
__global__ void __launch_bounds__(128) paged_attn_simple_kernel(const __grid_constant__ PagedAttnArgs a) {
  __shared__ float s_q[4][D];
  grid_dependency_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.x * 4 + warp, g = blockIdx.y;
  // the sequence whose row this is; all are looked at, so that one with numbers out of bounds hides no other
  int lo = -1;
  for (int s0 = 0; s0 < a.seqs.n_seqs; s0 += 32) {
    bool mine = false;
    if (s0 + lane < a.seqs.n_seqs) {
      const Seq x = seq_at(a.cache, a.seqs, s0 + lane);
      mine = row >= x.row0 && row < x.row0 + x.n_new;
    }
    const uint32_t who = __ballot_sync(0xffffffffu, mine);
    if (who) lo = s0 + __ffs(who) - 1;
  }
  if (lo < 0) return;
  const Seq q = seq_at(a.cache, a.seqs, lo);
  const float lse = attend_row<T, D>(a, lo, q, row, g, s_q[warp]);
  if (a.lse && lane == 0) a.lse[(int64_t)g * a.seqs.n_tokens + row] = lse;
}

}  // namespace

cudaError_t launch_paged_attn_simple(const PagedAttnArgs& a, int head_dim, int dtype, cudaStream_t st) {
  const void* fn;
  if (dtype == XKV_BF16) fn = head_dim == 64 ? (const void*)paged_attn_simple_kernel<__nv_bfloat16, 64> : (const void*)paged_attn_simple_kernel<__nv_bfloat16, 128>;
  else fn = head_dim == 64 ? (const void*)paged_attn_simple_kernel<__half, 64> : (const void*)paged_attn_simple_kernel<__half, 128>;
  void* params[1] = {(void*)&a};
  const cudaError_t e = launch_overlapped(fn, dim3((a.seqs.n_tokens + 3) / 4, a.cache.n_heads), dim3(128), params, 0, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace xkv
