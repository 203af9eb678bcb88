// Rotary positions and the append to the pages: one kernel that reads every token row once and writes it once.
//
// A block takes a few tokens.  Their sines and cosines are computed once, in shared memory, and serve all heads:
// the angle is formed as position * (turns per position) in 64 bits, its whole turns are dropped there, and what is
// left (at most half a turn) goes to sincospif in 32 bits.  64 positions of a full head cost 4 096 such angles, the rows
// that they turn (40 heads of 128 channels) 1.3 MB of traffic.  After that a thread moves 16 or 32 bytes of a row
// at a time: a pair of 16-byte pieces half an axis apart, or one piece of interleaved pairs.
//
// What bounds it is memory: 8192 tokens of 32 + 8 heads of 128 channels 33 us (5.1 TB/s), 4043 tokens of four prompts into their pages
// 23 us (4.3 TB/s); one token per sequence is a launch (4.4 us in a graph).
#include "xkv_paged_internal.cuh"

namespace xkv {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTok = 8;               // tokens of a block (16: too few blocks for even rounds, 8192 tokens of 40 heads 51 us, 8: 34)

template <typename T> struct Two;
template <> struct Two<__nv_bfloat16> {
  static __device__ __forceinline__ float2 get(uint32_t u) {
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint32_t put(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float one(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
};
template <> struct Two<__half> {
  static __device__ __forceinline__ float2 get(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
  static __device__ __forceinline__ uint32_t put(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float one(uint16_t u) { return __half2float(*reinterpret_cast<const __half*>(&u)); }
};

// How the channels of a row are dealt to the threads that share it.
//   kHalves  a pair of 16-byte pieces half an axis apart (rotary_dim a multiple of 16), or one piece behind the turned ones
//   kPairs   one 16-byte piece of interleaved pairs, or of channels that stay (turned channels a multiple of 8)
//   kSingle  a pair of channels, or one that stays (any rotary_dim)
enum Layout { kHalves, kPairs, kSingle };

// The rows of a block in the order in which the threads take them: heads of a token beside each other, or tokens of a head, as
// they lie in memory.
struct Deal {
  int per;                 // tokens of a block, a power of two
  int per_log2, items_log2;
  int tokens_first;        // tokens of a head beside each other
  uint32_t magic;          // 2^32 / heads of a block, rounded up (rows of a block * heads < 2^32 / heads)
  int share;               // heads of a block
};

template <typename T, Layout L, bool APPEND>
__global__ void __launch_bounds__(kThreads, 4) tokens_kernel(const __grid_constant__ TokenArgs a, const __grid_constant__ Deal d) {
  __shared__ __align__(16) float2 s_cs[kMaxTok][kMaxPairs];        // (read two pairs at a time)
  __shared__ int64_t s_page[kMaxTok];         // row offset of the token's slot at head 0, -1: not written, -2: nobody's row
  __shared__ int64_t s_weight[kMaxTok];
  __shared__ int s_seq[kMaxTok], s_slot[kMaxTok];      // sequence of a token, -1: nobody's; its slot there, may be negative
  const int tid = threadIdx.x;
  if (APPEND) {
    if (tid < kMaxTok) s_seq[tid] = -1;
    __syncthreads();
  }
  grid_dependency_wait();
  const int tok0 = blockIdx.x * d.per;
  const int toks = min(d.per, a.n - tok0);
  const int all_pairs = a.rot.axes * a.rot.pairs;
  if (APPEND) {
    // Every sequence looks for its rows in the block, so that one with numbers out of bounds hides no other (and its loads are one
    // behind another at most: a search through q_start would take one for every halving).
    for (int s = tid; s < a.seqs.n_seqs; s += kThreads) {
      const Seq q = seq_at(a.cache, a.seqs, s);
      for (int t = max(0, q.row0 - tok0); t < min(toks, q.row0 + q.n_new - tok0); ++t) {
        s_seq[t] = s;
        s_slot[t] = q.len - q.n_new + (tok0 + t - q.row0);
      }
    }
  }
  for (int e = tid; e < toks * all_pairs; e += kThreads) {
    const int t = e / all_pairs, p = e - t * all_pairs;
    const int axis = p / a.rot.pairs, i = p - axis * a.rot.pairs;
    const double x = (double)a.rot.positions[axis * a.rot.pos_stride + tok0 + t] * a.rot.turns[i];
    const double part = x - rint(x);                   // in [-1/2, 1/2] turns
    float s, c;
    sincospif(2.f * (float)part, &s, &c);
    s_cs[t][p] = make_float2(c * a.rot.magnitude, s * a.rot.magnitude);
  }
  if (APPEND) {
    __syncthreads();
    if (tid < toks) {
      const int seq = s_seq[tid], slot = s_slot[tid];
      const int page = seq >= 0 && slot >= 0 ? page_at(a.cache, a.seqs.table, a.seqs.table_width, seq, slot) : -1;
      s_page[tid] = seq < 0 ? -2 : page < 0 ? -1 : row_offset(a.cache, page, 0, slot);
      if (page >= 0) s_weight[tid] = weight_offset(a.cache, page, 0, slot);
    }
  }
  __syncthreads();
  const int lanes = 1 << d.items_log2;                   // threads that share a row
  const int item = tid & (lanes - 1);
  const int heads = a.q.heads + a.k.heads + a.v.heads;
  const int half = a.rot.rot >> 1;
  const int turned = a.rot.axes * a.rot.rot;             // channels
  // what this thread does in a row: a pair of places to turn, or a place to copy
  constexpr int kW = L == kSingle ? 1 : 8;               // channels of a place
  int c0 = 0, c1 = -1, pair = -1;
  bool active;
  if (L == kPairs) {
    active = item < a.head_dim / 8;
    c0 = item * 8;
    if (c0 < turned) pair = c0 >> 1;
  } else {
    // items [0, turned / 2 / kW): (axis, place in its first half); then the places behind
    const int pairs = turned / 2 / kW;
    active = item < pairs + (a.head_dim - turned) / kW;
    if (item < pairs) {
      if (L == kSingle && a.rot.interleaved) { pair = item; c0 = 2 * item; c1 = c0 + 1; }
      else {
        const int each = half / kW;
        const int axis = item / each, i = item - axis * each;
        c0 = axis * a.rot.rot + i * kW;
        c1 = c0 + half;
        pair = axis * a.rot.pairs + i * kW;
      }
    } else {
      c0 = turned + (item - pairs) * kW;
    }
  }
  if (!active) return;
  const int step = kThreads >> d.items_log2;
  constexpr int kU = L == kPairs ? 8 : 4;                // rows in flight per thread
  const int h_lo = blockIdx.y * d.share;                 // blockIdx.y: a share of the heads
  const int total = d.share << d.per_log2;               // (of the last share some may be none: `heads` ends it)
  for (int base = tid >> d.items_log2; base < total; base += kU * step) {
    uint4 x0[kU], x1[L == kPairs ? 1 : kU];
    uint8_t* dst[kU];
    uint32_t tk = 0, plain = 0;                          // token of row u (4 bits each); rows that are not turned
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int c = base + u * step;
      dst[u] = nullptr;
      int t, h;
      if (d.tokens_first) { t = c & (d.per - 1); h = c >> d.per_log2; }
      else { t = (int)__umulhi((uint32_t)c, d.magic); h = c - t * d.share; }
      h += h_lo;
      if (c >= total || t >= toks || h >= heads) continue;
      const int row = tok0 + t;
      tk |= (uint32_t)t << (4 * u);
      const int64_t page = APPEND ? s_page[t] : 0;
      if (page == -2) continue;                          // nobody's row
      const uint8_t* src;
      if (h < a.q.heads) {
        src = a.q.in + 2 * ((int64_t)h * a.q.in_hs + (int64_t)row * a.q.in_ts);
        dst[u] = a.q.out + 2 * ((int64_t)h * a.q.out_hs + (int64_t)row * a.q.out_ts);
      } else if ((h -= a.q.heads) < a.k.heads) {
        if (page < 0) continue;
        src = a.k.in + 2 * ((int64_t)h * a.k.in_hs + (int64_t)row * a.k.in_ts);
        if (APPEND) {
          dst[u] = a.cache.k + 2 * (page + (int64_t)h * a.cache.head_stride);
          if (item == 0 && a.cache.weights) a.cache.weights[s_weight[t] + ((int64_t)h << a.cache.page_shift)] = 0.f;
        } else {
          dst[u] = a.k.out + 2 * ((int64_t)h * a.k.out_hs + (int64_t)row * a.k.out_ts);
        }
      } else if (APPEND) {
        h -= a.k.heads;
        if (page < 0) continue;
        src = a.v.in + 2 * ((int64_t)h * a.v.in_hs + (int64_t)row * a.v.in_ts);
        dst[u] = a.cache.v + 2 * (page + (int64_t)h * a.cache.head_stride);
        plain |= 1u << u;
      } else {
        continue;
      }
      if (L != kSingle) {
        x0[u] = *reinterpret_cast<const uint4*>(src + 2 * c0);
        if (L == kHalves && c1 >= 0) x1[u] = *reinterpret_cast<const uint4*>(src + 2 * c1);
      } else {
        x0[u].x = *reinterpret_cast<const uint16_t*>(src + 2 * c0);
        if (c1 >= 0) x1[u].x = *reinterpret_cast<const uint16_t*>(src + 2 * c1);
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (!dst[u]) continue;
      if (pair >= 0 && !((plain >> u) & 1)) {
        const float2* cs = &s_cs[(tk >> (4 * u)) & 7][pair];
        if (L == kPairs) {                               // four pairs of one piece
          uint32_t* w = &x0[u].x;
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const float4 r = *reinterpret_cast<const float4*>(cs + i);
            const float2 x = Two<T>::get(w[i]), y = Two<T>::get(w[i + 1]);
            w[i] = Two<T>::put(x.x * r.x - x.y * r.y, x.y * r.x + x.x * r.y);
            w[i + 1] = Two<T>::put(y.x * r.z - y.y * r.w, y.y * r.z + y.x * r.w);
          }
        } else if (L == kHalves) {
          uint32_t* w0 = &x0[u].x;
          uint32_t* w1 = &x1[u].x;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 r = *reinterpret_cast<const float4*>(cs + 2 * i);
            const float2 x = Two<T>::get(w0[i]), y = Two<T>::get(w1[i]);
            w0[i] = Two<T>::put(x.x * r.x - y.x * r.y, x.y * r.z - y.y * r.w);
            w1[i] = Two<T>::put(y.x * r.x + x.x * r.y, y.y * r.z + x.y * r.w);
          }
        } else {
          const float x = Two<T>::one((uint16_t)x0[u].x), y = Two<T>::one((uint16_t)x1[u].x);
          x0[u].x = Two<T>::put(x * cs->x - y * cs->y, 0.f) & 0xFFFFu;
          x1[u].x = Two<T>::put(y * cs->x + x * cs->y, 0.f) & 0xFFFFu;
        }
      }
      if (L != kSingle) {
        // (rows that go to the pages will be read soon; those of xkv_rotary make way for others first: 34 -> 33 us)
        if (APPEND) *reinterpret_cast<uint4*>(dst[u] + 2 * c0) = x0[u]; else __stcs(reinterpret_cast<uint4*>(dst[u] + 2 * c0), x0[u]);
        if (L == kHalves && c1 >= 0) {
          if (APPEND) *reinterpret_cast<uint4*>(dst[u] + 2 * c1) = x1[u]; else __stcs(reinterpret_cast<uint4*>(dst[u] + 2 * c1), x1[u]);
        }
      } else {
        *reinterpret_cast<uint16_t*>(dst[u] + 2 * c0) = (uint16_t)x0[u].x;
        if (c1 >= 0) *reinterpret_cast<uint16_t*>(dst[u] + 2 * c1) = (uint16_t)x1[u].x;
      }
    }
  }
}

template <typename T, bool APPEND>
const void* kernel_of(Layout l) {
  return l == kHalves ? (const void*)tokens_kernel<T, kHalves, APPEND> : l == kPairs ? (const void*)tokens_kernel<T, kPairs, APPEND>
                                                                                     : (const void*)tokens_kernel<T, kSingle, APPEND>;
}
template <typename T>
const void* kernel_of(Layout l, bool append) { return append ? kernel_of<T, true>(l) : kernel_of<T, false>(l); }

}  // namespace

cudaError_t launch_tokens(const TokenArgs& a, int dtype, int sm_count, cudaStream_t st) {
  const int turned = a.rot.axes * a.rot.rot;
  Layout l = kSingle;
  if (a.rot.interleaved) { if (turned % 8 == 0) l = kPairs; }
  else if (turned == 0 || a.rot.rot % 16 == 0) l = kHalves;
  const int items = l == kPairs ? a.head_dim / 8 : l == kHalves ? turned / 16 + (a.head_dim - turned) / 8 : turned / 2 + (a.head_dim - turned);
  Deal d;
  d.items_log2 = 0;
  while ((1 << d.items_log2) < items) ++d.items_log2;
  const int heads = a.q.heads + a.k.heads + a.v.heads;
  // Blocks of at most kMaxTok tokens; with few tokens the heads are shared out too, until every multiprocessor has two blocks.
  d.per_log2 = 3;
  while (d.per_log2 > 0 && (int64_t)((a.n + (1 << d.per_log2) - 1) >> d.per_log2) < 2 * sm_count) --d.per_log2;
  d.per = 1 << d.per_log2;
  const int blocks = (a.n + d.per - 1) >> d.per_log2;
  int shares = 1;
  while (blocks * shares < 2 * sm_count && shares * 2 <= heads && ((int64_t)d.per * heads << d.items_log2) / (2 * shares) >= kThreads) shares <<= 1;
  d.share = (heads + shares - 1) / shares;
  d.magic = d.share == 1 ? 0 : (uint32_t)((0x100000000ull + d.share - 1) / d.share);
  const TokenTensor& most = a.k.heads > a.q.heads ? a.k : a.q;
  d.tokens_first = d.share == 1 || most.in_hs > most.in_ts;
  void* params[2] = {(void*)&a, (void*)&d};
  const void* fn = dtype == XKV_BF16 ? kernel_of<__nv_bfloat16>(l, a.append) : kernel_of<__half>(l, a.append);
  const cudaError_t e = launch_overlapped(fn, dim3(blocks, shares), dim3(kThreads), params, 0, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace xkv
