// Attention of one query row, computed by one warp without tensor cores, fp32 throughout: the cross-check of the other kernels, and
// what takes the few rows that the tensor cores cannot serve (xkv_paged_chunk.cu).
#pragma once

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

// Row `row` of the token tensors, which is of sequence `seq` with numbers `q`, for query head g; s_q: room for D floats of this warp's.
// Writes the output and returns the log sum exp (-infinity: the row sees nothing).
template <typename T, int D>
__device__ __forceinline__ float attend_row(const PagedAttnArgs& a, int seq, const Seq& q, int row, int g, float* s_q) {
  const int lane = threadIdx.x & 31;
  const int seen = a.full ? q.len : max(0, q.len - q.n_new + (row - q.row0) + 1);
  const int h = g / a.cache.group;
  __syncwarp();                                        // (the row before is done with s_q)
  const uint8_t* qp = a.q + 2 * ((int64_t)g * a.q_hs + (int64_t)row * a.q_ts);
  for (int c = lane; c < D / 2; c += 32) {
    const float2 x = two(*reinterpret_cast<const uint32_t*>(qp + 4 * c), T());
    s_q[2 * c] = x.x; s_q[2 * c + 1] = x.y;
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
      const int page = page_at(a.cache, a.seqs.table, a.seqs.table_width, seq, j);
      if (page >= 0) off = 2 * row_offset(a.cache, page, h, j);
      float d = 0.f;
      if (off >= 0)
        for (int c = 0; c < D / 2; ++c) {
          const float2 x = two(*reinterpret_cast<const uint32_t*>(a.cache.k + off + 4 * c), T());
          d = fmaf(s_q[2 * c], x.x, d);
          d = fmaf(s_q[2 * c + 1], x.y, d);
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
  return l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

}  // namespace
}  // namespace xkv
