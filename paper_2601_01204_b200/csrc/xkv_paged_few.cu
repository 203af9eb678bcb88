// Attention of few query rows (at most 16 per sequence and key head: single tokens, and a few tokens of small groups) over
// the paged cache.  What bounds it is reading K and V once, so everything serves to keep copies in flight.
//
// A warp works alone: 16 cached tokens at a time, whose K and V rows its own bulk copies (TMA) bring to its own ring of
// stages in shared memory.  Scores by mma.sync m16n8k16 (rows of the group x 8 tokens), running maximum and sum
// per row in registers, P straight from the scores' registers into the product with V.  16 of tcgen05.mma's 128 rows would be
// used here, and its accumulators would take a trip through tensor memory; a warp's own instruction needs no
// exchange with other warps until its share is done.  Per 16 tokens of 128 channels a warp issues 32 of
// them, 16 ldmatrix and 8 exponentials a lane for 8 KB of copies.
//
// P is rounded to the type of V for its product (the instruction takes both operands in 16 bits): an error of half a step per weight, 2^-8
// for bf16 and 2^-11 for fp16, beside which those of the fp32 sums do not count.  The sum of the weights is that of the unrounded ones.
//
// Measured: 64 sequences, 164 834 tokens, 32 / 8 heads of 128: 113 us, 6.0 TB/s; one token over 1024, 16 heads of 64: 7.6 us; the
// first with four new tokens each, causal, 128 us.
//
// The copies run ahead over the ends of items, so that a block with many short sequences never waits for memory at
// their seams.  At the end of its part of an item the eight warps merge through shared memory.
// Blocks that share an item leave partial results; the last one to arrive merges them in the order of the pieces, so
// results do not depend on who came last.
#include "xkv_paged_line.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kStep = 16;                                  // tokens of a warp's step
constexpr int kSeqsHeld = 64;                              // sequences whose numbers stay in shared memory (the others' are read again)
constexpr int kMergeFloats = kWarps * kFewRows * 40;       // 16 rows of 32 channels and 8 of padding (no bank conflicts) per warp

template <int D> struct Few {
  static constexpr int kHalf = kStep * D * 2;              // bytes of K (or V) of a step
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kStages = 192 * 1024 / (kWarps * kStage);      // 3 (d = 128), 6 (d = 64)
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr size_t kBytes = 1024 + kRing;
};

struct FewArgs {
  PagedAttnArgs a;
  PagedScratch s;
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool BF16>
__device__ __forceinline__ float number(uint32_t u) {      // of 16 bits
  return BF16 ? __uint_as_float(u << 16) : __half2float(__ushort_as_half((unsigned short)u));
}
// Whether some value of the first `tokens` of a step (at `v` in shared memory) is not finite; the same in the whole warp.  Adding the
// exponent's lowest bit to an exponent of ones carries into the place of the sign.
template <int D, bool BF16>
__device__ __forceinline__ bool strange_values(uint32_t v, int tokens) {
  constexpr uint32_t kExp = BF16 ? 0x7F807F80u : 0x7C007C00u, kOne = BF16 ? 0x00800080u : 0x04000400u;
  const int lane = threadIdx.x & 31;
  uint32_t strange = 0;
#pragma unroll
  for (int i = 0; i < Few<D>::kHalf / 512; ++i) {          // 4 rows of 128 bytes at a time, 16 rows a slab
    uint32_t w[4];
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(v + 512 * i + 16 * lane) : "memory");
    uint32_t x = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) x |= (w[j] & kExp) + kOne;
    if (4 * (i & 3) + (lane >> 3) < tokens) strange |= x;
  }
  return __any_sync(0xffffffffu, (strange & 0x80008000u) != 0);
}

// The parts of items in a block's piece, one after the other.
struct FewWalk {
  uint32_t pos, end, cost;               // on the line, which has cost + units places per item
  int seq, head, len, row0, n_new;       // of the current part
  uint32_t per;                          // places of an item of the sequence
  uint32_t item_lo;                      // the item's place on the line
  int key0, key1;                        // tokens of the part
  bool whole;                            // it is all of its item
  __device__ __forceinline__ bool next(const FewArgs& f, const uint32_t* prefix, const Seq* held) {
    int units;
    do {
      if (pos >= end) return false;
      uint32_t rel = 0;
      if (seq < 0 || pos >= prefix[seq + 1]) {
        seq = line_seq(prefix, f.a.seqs.n_seqs, pos);
        const Seq q = seq < kSeqsHeld ? held[seq] : seq_at(f.a.cache, f.a.seqs, seq);
        len = q.len; row0 = q.row0; n_new = q.n_new;
        per = cost + (uint32_t)max(1, (len + kUnit - 1) / kUnit);
        rel = pos - prefix[seq];
        head = (int)(rel / per);
        rel -= (uint32_t)head * per;
      } else {                           // the sequence's next item begins
        ++head;
      }
      item_lo = pos - rel;
      const uint32_t stop = min(per - rel, end - pos);
      const int lo = (int)(max(rel, cost) - cost);
      units = (int)(max(rel + stop, cost) - cost) - lo;
      key0 = lo * kUnit;
      key1 = min((lo + units) * kUnit, len);
      whole = units == (int)(per - cost);
      pos += stop;
    } while (units == 0);                // (no more than the cost of an item that begins here)
    return true;
  }
};

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) attn_few_kernel(const __grid_constant__ FewArgs f, const __grid_constant__ PoolMaps maps) {
  using C = Few<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_bar[kWarps * C::kStages];
  __shared__ __align__(16) float s_merge[kMergeFloats];
  __shared__ float2 s_ml[kWarps][kFewRows];
  __shared__ uint32_t s_prefix[kMaxSeqs + 1];
  __shared__ Seq s_seq[kSeqsHeld];
  __shared__ uint2 s_warp[kWarps];
  __shared__ uint32_t s_abort, s_last;
  const PagedAttnArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t ring = ((smem_u32(smem_raw) + 1023u) & ~1023u) + (uint32_t)warp * C::kStages * C::kStage;
  const uint32_t bar = smem_u32(s_bar) + 8 * warp * C::kStages;
  const WaitCtx wc{smem_u32(&s_abort)};
  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < kWarps * C::kStages; ++i) mbar_init(smem_u32(s_bar) + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  grid_dependency_wait();
  const uint32_t cost = line_prefix<kThreads, false>(a.seqs.n_seqs, s_prefix, s_warp, [&](int s) {
    const Seq q = seq_at(a.cache, a.seqs, s);
    if (s < kSeqsHeld) s_seq[s] = q;
    // (a sequence with new tokens but without cached ones has a unit too: its rows become zero)
    const uint32_t items = q.n_new == 0 ? 0u : (uint32_t)a.cache.n_kv_heads;
    return Work{items, items * (uint32_t)max(1, (q.len + kUnit - 1) / kUnit)};
  });
  const uint32_t total = s_prefix[a.seqs.n_seqs];
  if (total == 0) return;
  const Cut cut(total, gridDim.x);
  FewWalk walk;
  walk.pos = cut.start(blockIdx.x);
  walk.end = cut.start(blockIdx.x + 1);
  walk.cost = cost;
  walk.seq = -1;

  // ---- copies: this warp's steps of all parts, kStages of them ahead ----
  FewWalk ahead = walk;
  int a_key = 0;                          // next step's first token
  bool a_more = ahead.next(f, s_prefix, s_seq);
  if (a_more) a_key = ahead.key0 + kStep * warp;
  int ids = 0, id_key = -1;               // pages of this lane's step among the next 32 (lane l: l * kWarps steps on)
  uint32_t put = 0;                       // steps asked for
  auto ask = [&]() {                      // the next step's copies, if there is one
    while (a_more && a_key >= ahead.key1) {
      a_more = ahead.next(f, s_prefix, s_seq);
      if (a_more) a_key = ahead.key0 + kStep * warp;
      id_key = -1;
    }
    if (!a_more) return;
    constexpr int kSpan = kStep * kWarps;
    int i = id_key < 0 ? 32 : (a_key - id_key) / kSpan;
    if (i >= 32) {
      id_key = a_key;
      const int key = a_key + lane * kSpan;
      ids = key < ahead.key1 ? page_at(a.cache, a.seqs.table, a.seqs.table_width, ahead.seq, key) : -1;
      i = 0;
    }
    int page = __shfl_sync(0xffffffffu, ids, i);
    if (page < 0) page = a.cache.n_pages;            // outside the map: zeros
    if (lane == 0) {
      const uint32_t st = put % C::kStages, dst = ring + st * C::kStage, b = bar + 8 * st;
      const int slot = a_key & ((1 << a.cache.page_shift) - 1);
      mbar_expect_tx(b, C::kStage);
#pragma unroll
      for (int c = 0; c < D / 64; ++c) tma_4d(dst + c * kStep * 128, &maps.k, 64 * c, slot, ahead.head, page, b);
#pragma unroll
      for (int c = 0; c < D / 64; ++c) tma_4d(dst + C::kHalf + c * kStep * 128, &maps.v, 64 * c, slot, ahead.head, page, b);
    }
    ++put;
    a_key += kSpan;
  };
  for (int i = 0; i < C::kStages; ++i) ask();

  const int g = lane >> 2, t = lane & 3;
  uint32_t got = 0;                       // steps consumed
  int part = 0;
  for (; walk.next(f, s_prefix, s_seq); ++part) {
    const int rows = walk.n_new * a.cache.group;
    // ---- queries: rows g and g + 8 of the item, row r = (new token r / group, head r mod group) ----
    uint32_t qf[D / 16][4];
    int limit[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = g + 8 * e;
      const int i = r / a.cache.group, hq = walk.head * a.cache.group + (r - i * a.cache.group);
      limit[e] = a.full || r >= rows ? walk.len : walk.len - walk.n_new + i + 1;
      const uint8_t* qp = a.q + 2 * ((int64_t)hq * a.q_hs + (int64_t)(walk.row0 + i) * a.q_ts) + 4 * t;
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        qf[k][e] = r < rows ? *reinterpret_cast<const uint32_t*>(qp + 32 * k) : 0u;
        qf[k][e + 2] = r < rows ? *reinterpret_cast<const uint32_t*>(qp + 32 * k + 16) : 0u;
      }
    }
    const int least = a.full ? walk.len : walk.len - walk.n_new + 1;     // tokens below it are seen by every row
    const bool several = least < walk.len;                               // some token is seen by some rows only
    float o[D / 8][4];
#pragma unroll
    for (int j = 0; j < D / 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    for (int key = walk.key0 + kStep * warp; key < walk.key1; key += kStep * kWarps) {
      const uint32_t st = got % C::kStages, base = ring + st * C::kStage;
      mbar_wait(bar + 8 * st, (got / C::kStages) & 1, wc);
      __syncwarp();
      // ---- scores of 16 rows x 16 tokens ----
      float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
      {
        const int row = ((lane >> 4) << 3) + (lane & 7);
        const uint32_t at = base + row * 128;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const int chunk = (2 * k & 7) + ((lane >> 3) & 1);
          uint32_t b[4];
          ldsm4(at + (k >> 2) * (kStep * 128) + ((chunk ^ (row & 7)) << 4), b);
          mma16816<BF16>(s0, qf[k], b[0], b[1]);
          mma16816<BF16>(s1, qf[k], b[2], b[3]);
        }
      }
      if (key + kStep > least) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k0 = key + 2 * t + (i & 1);
          if (k0 >= limit[i >> 1]) s0[i] = -INFINITY;
          if (k0 + 8 >= limit[i >> 1]) s1[i] = -INFINITY;
        }
      }
      // ---- softmax: running maximum per row over the quad that holds it ----
      uint32_t p[4];
      float fade[2];
      bool grew = false;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float top = fmaxf(fmaxf(s0[2 * e], s0[2 * e + 1]), fmaxf(s1[2 * e], s1[2 * e + 1]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)) * a.scale_log2;
        fade[e] = 1.f;
        if (top > m[e]) {
          fade[e] = exp2f(m[e] - top);           // 0 at first
          m[e] = top;
          l[e] *= fade[e];
          grew = true;
        }
        const float ref = m[e] == -INFINITY ? 0.f : m[e];
        const float p0 = fast_exp2(fmaf(s0[2 * e], a.scale_log2, -ref)), p1 = fast_exp2(fmaf(s0[2 * e + 1], a.scale_log2, -ref));
        const float p2 = fast_exp2(fmaf(s1[2 * e], a.scale_log2, -ref)), p3 = fast_exp2(fmaf(s1[2 * e + 1], a.scale_log2, -ref));
        l[e] += (p0 + p1) + (p2 + p3);
        p[e] = BF16 ? pack_bf2(p0, p1) : pack_h2(p0, p1);
        p[e + 2] = BF16 ? pack_bf2(p2, p3) : pack_h2(p2, p3);
      }
      if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
        for (int j = 0; j < D / 8; ++j) { o[j][0] *= fade[0]; o[j][1] *= fade[0]; o[j][2] *= fade[1]; o[j][3] *= fade[1]; }
      }
      // ---- P V ----
      {
        const int row = (((lane >> 3) & 1) << 3) + (lane & 7);
        const uint32_t at0 = base + C::kHalf, at = at0 + row * 128;
        // tokens behind the end may hold anything, NaN included, which a weight of 0 would not silence: their rows count as zero
        const bool tail = key + kStep > walk.len, hides = several && key + kStep > least;
        uint32_t mask0 = 0xffffffffu, mask1 = 0xffffffffu;
        if (tail) {
          const int k0 = key + 2 * t;
          mask0 = (k0 < walk.len ? 0xffffu : 0u) | (k0 + 1 < walk.len ? 0xffff0000u : 0u);
          mask1 = (k0 + 8 < walk.len ? 0xffffu : 0u) | (k0 + 9 < walk.len ? 0xffff0000u : 0u);
        }
        if (hides && strange_values<D, BF16>(at0, walk.len - key)) {
          // Values that are not finite, of which some rows do not see all: 0 times such a value is a NaN.  Token by token, then, with those
          // rows alone that see it (and the same weights, sums in fp32 as there).
          for (int k = 0; k < kStep && key + k < walk.len; ++k) {
            const int src = (lane & ~3) | ((k & 7) >> 1);
            float w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t u = __shfl_sync(0xffffffffu, k < 8 ? p[e] : p[e + 2], src);
              w[e] = number<BF16>((k & 1) ? u >> 16 : u & 0xffffu);
            }
#pragma unroll
            for (int j = 0; j < D / 8; ++j) {
              const uint32_t u = ld_shared_u32(at0 + (j >> 3) * (kStep * 128) + k * 128 + (((j & 7) ^ (k & 7)) << 4) + 4 * t);
              const float v0 = number<BF16>(u & 0xffffu), v1 = number<BF16>(u >> 16);
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (key + k < limit[e]) { o[j][2 * e] = fmaf(w[e], v0, o[j][2 * e]); o[j][2 * e + 1] = fmaf(w[e], v1, o[j][2 * e + 1]); }
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            const int chunk = (2 * j & 7) + (lane >> 4);
            uint32_t b[4];
            ldsm4t(at + (j >> 2) * (kStep * 128) + ((chunk ^ (row & 7)) << 4), b);
            if (tail) { b[0] &= mask0; b[1] &= mask1; b[2] &= mask0; b[3] &= mask1; }
            mma16816<BF16>(o[2 * j], p, b[0], b[1]);
            mma16816<BF16>(o[2 * j + 1], p, b[2], b[3]);
          }
        }
      }
      __syncwarp();                       // every lane has read the stage
      ++got;
      ask();                              // into the stage just read
    }
    // ---- the warps' parts of the part ----
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
      l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
      if (t == 0) s_ml[warp][g + 8 * e] = make_float2(m[e], l[e]);
    }
    const bool whole = walk.whole;
    const uint32_t slot = 2 * blockIdx.x + (part ? 1 : 0);
    // As many channels at a time as the rows leave room for (all 128 with 4 rows): row r, channel c of warp w at [(w * R + r) * pad + c].
    // (32 at a time whatever the rows, and items without a cost in the cut: 154 us for 64 decoding sequences instead of 111.)
    const int log_r = rows <= 4 ? 2 : rows <= 8 ? 3 : 4;
    const int span = min(D, 512 >> log_r), pad = span + 8;
    for (int c0 = 0; c0 < D; c0 += span) {
#pragma unroll
      for (int j = 0; j < D / 8; ++j)
        if (8 * j >= c0 && 8 * j < c0 + span)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (g + 8 * e < rows)
              *reinterpret_cast<float2*>(&s_merge[((warp << log_r) + g + 8 * e) * pad + 8 * j - c0 + 2 * t]) = make_float2(o[j][2 * e], o[j][2 * e + 1]);
      __syncthreads();
      for (int i = tid; i < rows * (span / 4); i += kThreads) {         // (row, 4 channels)
        const int r = i / (span / 4), c = (i - r * (span / 4)) * 4;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_ml[w][r].x);
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float2 ml = s_ml[w][r];
          const float wgt = exp2f(ml.x - ref);
          const float4 y = *reinterpret_cast<const float4*>(&s_merge[((w << log_r) + r) * pad + c]);
          sum += wgt * ml.y;
          x.x += wgt * y.x; x.y += wgt * y.y; x.z += wgt * y.z; x.w += wgt * y.w;
        }
        if (whole) {
          if (sum == 0.f) x = make_float4(0.f, 0.f, 0.f, 0.f);       // (a row that sees nothing, whatever a weight of 0 met)
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          const int n = r / a.cache.group, hq = walk.head * a.cache.group + (r - n * a.cache.group);
          uint2 out;
          out.x = BF16 ? pack_bf2(x.x * inv, x.y * inv) : pack_h2(x.x * inv, x.y * inv);
          out.y = BF16 ? pack_bf2(x.z * inv, x.w * inv) : pack_h2(x.z * inv, x.w * inv);
          *reinterpret_cast<uint2*>(a.out + 2 * ((int64_t)hq * a.o_hs + (int64_t)(walk.row0 + n) * a.o_ts + c0 + c)) = out;
          if (c0 == 0 && c == 0 && a.lse)
            a.lse[(int64_t)hq * a.seqs.n_tokens + walk.row0 + n] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
        } else {
          *reinterpret_cast<float4*>(&f.s.o[((int64_t)slot * kFewRows + r) * D + c0 + c]) = x;
          if (c0 == 0 && c == 0) f.s.ml[slot * kFewRows + r] = make_float2(top, sum);
        }
      }
      __syncthreads();
    }
    if (whole) continue;
    // ---- an item that several blocks share: the last to arrive merges the pieces in their order ----
    const uint32_t first = cut.owner(walk.item_lo + cost), parts = cut.owner(walk.item_lo + walk.per - 1) - first + 1;
    // (the barrier before orders this block's partial results before the addition, the one behind it the others' after it)
    if (tid == 0) {
      uint32_t before;
      asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(f.s.count + first) : "memory");
      s_last = before == parts - 1;
    }
    __syncthreads();
    if (!s_last) continue;
    // (in the block where it starts the item may follow another one)
    const uint32_t slot0 = 2 * first + (cut.start(first) < walk.item_lo ? 1 : 0);
    // Threads take (row, 4 channels); where there are fewer of those than threads, groups of threads share out the pieces
    // and join through shared memory.
    const int work = rows * (D / 4);
    int groups = 1;
    while (groups * 2 * work <= kThreads && groups < 8) groups *= 2;
    float4* s_x = reinterpret_cast<float4*>(s_merge);            // [groups * work]
    for (int i0 = 0; i0 < work * groups; i0 += kThreads) {
      const int i = i0 + tid;
      const int grp = i / work, at = i - grp * work, r = at / (D / 4), c = (at - r * (D / 4)) * 4;
      float top = -INFINITY, sum = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < work * groups) {
        for (uint32_t p0 = grp; p0 < parts; p0 += 4 * groups) {
          float2 ml[4];
          float4 y[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint32_t p = p0 + u * groups;
            ml[u] = make_float2(-INFINITY, 0.f);
            y[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (p < parts) {
              const uint32_t sl = p == 0 ? slot0 : 2 * (first + p);
              ml[u] = __ldcg(&f.s.ml[sl * kFewRows + r]);
              y[u] = __ldcg(reinterpret_cast<const float4*>(&f.s.o[((int64_t)sl * kFewRows + r) * D + c]));
            }
          }
          const float nt = fmaxf(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), top);
          const float ref = nt == -INFINITY ? 0.f : nt;
          const float fade = exp2f(top - ref);
          top = nt;
          sum *= fade; x.x *= fade; x.y *= fade; x.z *= fade; x.w *= fade;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const float wgt = exp2f(ml[u].x - ref);
            sum += wgt * ml[u].y;
            x.x += wgt * y[u].x; x.y += wgt * y[u].y; x.z += wgt * y[u].z; x.w += wgt * y[u].w;
          }
        }
      }
      if (groups > 1) {                    // (then one pass does it: work * groups <= kThreads)
        __shared__ float2 s_g[kThreads];
        __syncthreads();
        s_x[tid] = x;
        s_g[tid] = make_float2(top, sum);
        __syncthreads();
        if (grp == 0 && i < work) {
          for (int q = 1; q < groups; ++q) {
            const float2 ml = s_g[q * work + at];
            const float4 y = s_x[q * work + at];
            const float nt = fmaxf(top, ml.x), ref = nt == -INFINITY ? 0.f : nt;
            const float f0 = exp2f(top - ref), f1 = exp2f(ml.x - ref);
            top = nt;
            sum = sum * f0 + ml.y * f1;
            x.x = x.x * f0 + y.x * f1; x.y = x.y * f0 + y.y * f1; x.z = x.z * f0 + y.z * f1; x.w = x.w * f0 + y.w * f1;
          }
        }
        __syncthreads();
      }
      if (grp == 0 && i < work) {
        if (sum == 0.f) x = make_float4(0.f, 0.f, 0.f, 0.f);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int n = r / a.cache.group, hq = walk.head * a.cache.group + (r - n * a.cache.group);
        uint2 out;
        out.x = BF16 ? pack_bf2(x.x * inv, x.y * inv) : pack_h2(x.x * inv, x.y * inv);
        out.y = BF16 ? pack_bf2(x.z * inv, x.w * inv) : pack_h2(x.z * inv, x.w * inv);
        *reinterpret_cast<uint2*>(a.out + 2 * ((int64_t)hq * a.o_hs + (int64_t)(walk.row0 + n) * a.o_ts + c)) = out;
        if (c == 0 && a.lse)
          a.lse[(int64_t)hq * a.seqs.n_tokens + walk.row0 + n] =
              sum == 0.f ? -INFINITY : ((top == -INFINITY ? 0.f : top) + log2f(sum)) * 0.69314718055994531f;
      }
    }
    if (tid == 0) f.s.count[first] = 0;
    __syncthreads();
  }
  if (ld_shared_u32(wc.abort_flag)) {     // a wait ran out: nothing may be in flight when the block ends
    for (uint32_t i = 0; i < (uint32_t)C::kStages && i < put; ++i) {
      const uint32_t n = put - 1 - i;
      for (uint32_t it = 0; it < (1u << 22) && !mbar_try(bar + 8 * (n % C::kStages), (n / C::kStages) & 1); ++it) {}
    }
  }
  __syncthreads();
  if (tid == 0 && s_abort) atomicExch(a.cache.status, (int)XKV_E_TIMEOUT);
}

}  // namespace

template <int D, bool BF16>
static cudaError_t setup_one() {
  return cudaFuncSetAttribute(attn_few_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Few<D>::kBytes);
}
cudaError_t attn_few_setup() {
  cudaError_t e = setup_one<64, true>();
  if (e == cudaSuccess) e = setup_one<64, false>();
  if (e == cudaSuccess) e = setup_one<128, true>();
  if (e == cudaSuccess) e = setup_one<128, false>();
  return e;
}

cudaError_t launch_attn_few(const PagedAttnArgs& a, const PoolMaps& maps, const PagedScratch& s, int head_dim, int dtype, int sm_count,
                            cudaStream_t st) {
  FewArgs f;
  f.a = a;
  f.s = s;
  // no more blocks than units can be (the lengths are the device's)
  const int64_t most = (int64_t)a.seqs.n_seqs * a.cache.n_kv_heads * ((((int64_t)a.seqs.table_width << a.cache.page_shift) + kUnit - 1) / kUnit + 1);
  const unsigned grid = (unsigned)(most < sm_count ? most : sm_count);
  void* params[2] = {(void*)&f, (void*)&maps};
  const void* fn;
  size_t smem;
  if (head_dim == 64) { fn = dtype == XKV_BF16 ? (const void*)attn_few_kernel<64, true> : (const void*)attn_few_kernel<64, false>; smem = Few<64>::kBytes; }
  else { fn = dtype == XKV_BF16 ? (const void*)attn_few_kernel<128, true> : (const void*)attn_few_kernel<128, false>; smem = Few<128>::kBytes; }
  const cudaError_t e = launch_overlapped(fn, dim3(grid), dim3(kThreads), params, smem, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace xkv
