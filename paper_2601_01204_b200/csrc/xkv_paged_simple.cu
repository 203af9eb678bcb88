// Attention over the paged cache without tensor cores: a warp per query row, fp32 throughout.  Kept as an
// independent cross-check of the other kernels (impl = 1); never the default.
#include "xkv_paged_internal.cuh"

namespace xkv {

namespace {

__device__ __forceinline__ float2 two(uint32_t u, __nv_bfloat16) {
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
}
__device__ __forceinline__ float2 two(uint32_t u, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
__device__ __forceinline__ uint32_t pack(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack(float a, float b, __half) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

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
  const int seen = a.full ? q.len : max(0, q.len - q.n_new + (row - q.row0) + 1);
  const int h = g / a.cache.group;
  const uint8_t* qp = a.q + 2 * ((int64_t)g * a.q_hs + (int64_t)row * a.q_ts);
  for (int c = lane; c < D / 2; c += 32) {
    const float2 x = two(*reinterpret_cast<const uint32_t*>(qp + 4 * c), T());
    s_q[warp][2 * c] = x.x; s_q[warp][2 * c + 1] = x.y;
  }
  __syncwarp();
  float m = -INFINITY, l = 0.f, acc[D / 32];           // channels 2 lane + 64 i and the next
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = 0.f;
  for (int j0 = 0; j0 < seen; j0 += 32) {
    const int j = j0 + lane;
    float s = -INFINITY;
    int64_t off = -1;
    if (j < seen) {
      const int page = page_at(a.cache, a.seqs.table, a.seqs.table_width, lo, j);
      if (page >= 0) off = 2 * row_offset(a.cache, page, h, j);
      float d = 0.f;
      if (off >= 0)
        for (int c = 0; c < D / 2; ++c) {
          const float2 x = two(*reinterpret_cast<const uint32_t*>(a.cache.k + off + 4 * c), T());
          d = fmaf(s_q[warp][2 * c], x.x, d);
          d = fmaf(s_q[warp][2 * c + 1], x.y, d);
        }
      s = d * a.scale_log2;
    }
    float top = s;
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    top = fmaxf(m, top);
    const float ref = top == -INFINITY ? 0.f : top;
    const float p = exp2f(s - ref), fade = exp2f(m - ref);
    m = top;
    l = l * fade + p;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] *= fade;
    const int n = min(32, seen - j0);
    for (int i = 0; i < n; ++i) {
      const float pi = __shfl_sync(0xffffffffu, p, i);
      const int64_t oi = __shfl_sync(0xffffffffu, off, i);
      if (oi < 0) continue;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const float2 x = two(*reinterpret_cast<const uint32_t*>(a.cache.v + oi + 4 * (lane + 32 * c)), T());
        acc[2 * c] = fmaf(pi, x.x, acc[2 * c]);
        acc[2 * c + 1] = fmaf(pi, x.y, acc[2 * c + 1]);
      }
    }
  }
  for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);     // (a NaN stays one)
  uint8_t* op = a.out + 2 * ((int64_t)g * a.o_hs + (int64_t)row * a.o_ts);
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
    *reinterpret_cast<uint32_t*>(op + 4 * (lane + 32 * c)) = pack(acc[2 * c] * inv, acc[2 * c + 1] * inv, T());
  if (a.lse && lane == 0)
    a.lse[(int64_t)g * a.seqs.n_tokens + row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
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
