// Attention of chunks of new tokens over the paged cache for sm_100a: tcgen05.mma with accumulators in tensor memory,
// operands staged by TMA straight from the pages.
//
// Rows.  The query heads of a key head are rows beside each other: with G of them a tile of 128 rows takes 128 / G tokens, row
// r = (token r / G, head r mod G), so that one pass over K and V serves the whole group.  (Of a group that does not divide
// 128 the last rows stay unused.)  An item is two such tiles; see xkv_paged_line.cuh for how the work is cut.
//
// One block, 20 warps:
//   16 warps    softmax: a warp takes 16 rows of a tile; a quad of lanes holds 128 scores each of two rows, and writes P (16
//               bits) back to tensor memory.  The accumulator is rescaled only when a row's maximum has grown by more than
//               2^14 over the reference, which keeps P inside fp16's range.
//   2 warps     issue the MMAs of tile 0 resp. 1 (a converged warp, one elected lane).
//   1 warp      copies: Q tiles of the next part, K and V of the next units, page by page.
//   1 warp      clears, in the unit where a sequence ends, the rows of V behind its end that share a K-step of 16 with its
//               last token: what the memory holds there may be NaN, which a weight of 0 would not silence.  (Steps behind that
//               one are not multiplied at all, and scores behind the end are replaced before they are used.)
//
// Tensor memory, head_dim 64: as in the packed attention a tile has three blocks of 64 columns that scores and P take in turn, so
// that the next scores are computed during the softmax.  head_dim 128: the accumulators take half of the 512 columns and a
// tile has 128 for its scores, whose first half P overwrites; the other tile's MMAs fill the time.
//
// P is rounded to the type of V for its product, as in the kernel for few rows; sums, maxima, accumulators and parts are fp32.
//
// Measured: a frame of 1374 queries over 16384 tokens, 16 heads of 64, 137 us (673 TFLOP/s; the exponentials alone need 80); chunks of
// four prompts, 32 / 8 heads of 128, 522 us (1.02 PFLOP/s, at 1.53 GHz and 980 W).  What bounds it is the chain scores -> exponentials -> P -> accumulator.
//
// Values that are not finite.  P is 0 where a row does not see a token, and 0 times a NaN or an infinity of V is a NaN: a new token's
// value that is not finite would reach the tokens before it.  A softmax warp that writes a NaN behind a finite sum
// marks the sequence, and the merge looks at the rows of marked sequences again, and at rows that it merged to a NaN: those whose NaN can be
// the work of tokens that they do not see are computed once more, a warp per row, from the tokens that they see.  (That is slow,
// some microseconds a row; without a mark it costs a maximum per word that is written, and the merge one look at a word.)
//
// Every wait is bounded (see mbar_wait); when one runs out the block carries on without waiting and reports XKV_E_TIMEOUT.
#include <type_traits>

#include "xkv_paged_line.cuh"
#include "xkv_paged_row.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace {

constexpr int kThreads = 640;
constexpr int kSW = 16;                       // softmax warps; 16, 17: MMA of tile 0, 1; 18: copies; 19: tails
constexpr uint32_t kRowThreads = 256;         // threads that work on one tile
constexpr float kGrow = 14.f;                 // see the packed attention
constexpr uint32_t kSpinLimit = 1u << 22;

template <int D> struct Chunk {
  static constexpr int kSlabs = D / 64;                       // 128 rows x 64 channels (128 bytes), 16 KB
  static constexpr int kTile = kSlabs * 16384;
  static constexpr int kNK = D == 64 ? 4 : 2, kNV = D == 64 ? 4 : 2;
  static constexpr int kOffK = 2 * kTile, kOffV = kOffK + kNK * kTile, kOffBar = kOffV + kNV * kTile;
  static constexpr int kBars = 2 * kNK + 3 * kNV + 2 + 2 + 2 + 2 + 4 + 4 + 2 + 4 + 2;
  static constexpr int kOffPrefix = kOffBar + 512;
  static constexpr size_t kBytes = kOffPrefix + (kMaxSeqs + 1) * 4 + 1024;
  // tensor memory columns
  static constexpr int kColTile = D == 64 ? 192 : 128;        // * t
  static constexpr int kColO = D == 64 ? 384 : 256;           // + D t
};

// What is needed to merge an item whose units several blocks share; written by the block it starts in.
struct CutItem { int row0, n_new, head, pair, parts, slot0, seq, pad; };

struct ChunkArgs {
  PagedAttnArgs a;
  PagedScratch s;
  CutItem* cuts;          // [blocks]
  int tpt;                // tokens of a tile
  int box_rows;           // slots of a copy: min(page_tokens, 128)
  int q_toks;             // tokens of a copy of queries: those of a tile, or fewer if no sequence has that many new ones
};

__device__ __forceinline__ int units_of(int vis) { return max(1, (vis + kUnit - 1) / kUnit); }
// Tokens that the first `toks` new tokens of a sequence see, the last of them at least.
__device__ __forceinline__ int seen_by(const PagedAttnArgs& a, const Seq& q, int toks) {
  return a.full ? q.len : max(0, q.len - q.n_new + min(q.n_new, toks));
}

// The parts of items in a block's piece, one after the other.
struct ChunkWalk {
  uint32_t pos, end;                         // on the line, which has kItemCost + units places per item
  Seq q;
  int seq, head, pair, pairs;
  int tile_lo, nt;                           // units [tile_lo, tile_lo + nt) of the item
  int units;                                 // of the item
  int nt0, nt1;                              // of them those of tile 0 and 1
  uint32_t item_lo;                          // the item's place on the line
  __device__ __forceinline__ void start(uint32_t from, uint32_t to) { pos = from; end = to; seq = -1; }
  __device__ __forceinline__ void open(const ChunkArgs& f) {
    q = seq_at(f.a.cache, f.a.seqs, seq);
    pairs = (q.n_new + 2 * f.tpt - 1) / (2 * f.tpt);
  }
  __device__ __forceinline__ bool next(const ChunkArgs& f, const uint32_t* prefix) {
    uint32_t rel = 0;                        // place within the item
    do {
      if (pos >= end) return false;
      if (seq < 0) {                         // where the piece begins
        seq = line_seq(prefix, f.a.seqs.n_seqs, pos);
        open(f);
        const uint32_t per = (prefix[seq + 1] - prefix[seq]) / (uint32_t)f.a.cache.n_kv_heads;
        rel = pos - prefix[seq];
        head = (int)(rel / per);
        rel -= (uint32_t)head * per;
        for (pair = 0;; ++pair) {
          units = units_of(seen_by(f.a, q, (pair + 1) * 2 * f.tpt));
          if (rel < (uint32_t)units + kItemCost) break;
          rel -= (uint32_t)units + kItemCost;
        }
      } else {                               // the next item begins
        rel = 0;
        if (++pair == pairs) {
          pair = 0;
          if (++head == f.a.cache.n_kv_heads) {
            head = 0;
            do ++seq; while (prefix[seq + 1] == pos);
            open(f);
          }
        }
        units = units_of(seen_by(f.a, q, (pair + 1) * 2 * f.tpt));
      }
      item_lo = pos - rel;
      const uint32_t stop = min((uint32_t)units + kItemCost - rel, end - pos);
      tile_lo = (int)(max(rel, kItemCost) - kItemCost);
      nt = (int)(max(rel + stop, kItemCost) - kItemCost) - tile_lo;
      pos += stop;
    } while (nt == 0);                       // (no more than the cost of an item that begins here)
    nt0 = part_of(f, 2 * pair);
    nt1 = part_of(f, 2 * pair + 1);
    return true;
  }
  __device__ __forceinline__ int part_of(const ChunkArgs& f, int tile) const {
    const int ut = tile * f.tpt < q.n_new ? units_of(seen_by(f.a, q, (tile + 1) * f.tpt)) : 0;
    return max(0, min(nt, ut - tile_lo));
  }
};

__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr, uint32_t lbo) {        // make_desc with a leading byte offset
  return make_desc(saddr) - ((uint64_t)1 << 16) + ((uint64_t)(lbo >> 4) << 16);
}
// Maxima of two pairs of 16-bit numbers, NaN where either is.
template <bool BF16>
__device__ __forceinline__ uint32_t max_nan_pair(uint32_t a, uint32_t b) {
  uint32_t r;
  if (BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <bool BF16>
__device__ __forceinline__ bool any_nan(uint32_t x) {
  constexpr uint32_t kInf = BF16 ? 0x7F80u : 0x7C00u;
  return (x & 0x7FFFu) > kInf || ((x >> 16) & 0x7FFFu) > kInf;
}

// O *= alpha for the calling warp's 16 rows (two per thread); a real call, to keep its registers out of the softmax loop.
template <int D>
__device__ __noinline__ void rescale_chunk_rows(uint32_t col_o, float alpha0, float alpha1) {
#pragma unroll 1
  for (int c = 0; c < D; c += 64) {
    uint32_t ro[32];
    XKV_TMEM_LD_64(col_o + c, ro, 0);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 32; ++i) ro[i] = __float_as_uint(__uint_as_float(ro[i]) * ((i & 2) ? alpha1 : alpha0));
    XKV_TMEM_ST_64(col_o + c, ro);
  }
  tc_wait_st();
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1)
attn_chunk_kernel(const __grid_constant__ ChunkArgs f, const __grid_constant__ PoolMaps maps, const __grid_constant__ CUtensorMap q_map) {
  using C = Chunk<D>;
  constexpr int kNK = C::kNK, kNV = C::kNV, kTile = C::kTile, kSlabs = C::kSlabs;
  extern __shared__ uint8_t smem_raw[];
  const PagedAttnArgs& a = f.a;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* sgen = smem_raw + (sbase - smem_u32(smem_raw));
  const uint32_t sQ = sbase, sK = sbase + C::kOffK, sV = sbase + C::kOffV;
  const uint32_t b_kfull = sbase + C::kOffBar, b_kfree = b_kfull + 8 * kNK, b_vfull = b_kfree + 8 * kNK, b_vfree = b_vfull + 8 * kNV;
  const uint32_t b_qfull = b_vfree + 8 * kNV, b_qfree = b_qfull + 16, b_sfull = b_qfree + 16, b_sfree = b_sfull + 16;
  // [2 tiles][2], even and odd steps: P V done, P written (the warps of a tile may be almost a step apart)
  const uint32_t b_pvdone = b_sfree + 16, b_pfull = b_pvdone + 32, b_ofree = b_pfull + 32;
  const uint32_t b_vfix = b_ofree + 16;       // [kNV], one per stage: a stage is not filled again before both tiles have passed it
  const uint32_t b_phalf = b_vfix + 8 * kNV;  // [2 tiles][2] head_dim 128: P of the unit's first 64 tokens written
  const uint32_t b_turn = b_phalf + 32;       // [2] head_dim 128: it is this tile's turn at the exponentials
  static_assert(8 * C::kBars <= 512 - 16, "barriers");
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sgen + C::kOffBar + 496);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sgen + C::kOffBar + 500);
  const WaitCtx wc{sbase + C::kOffBar + 500};
  uint32_t* prefix = reinterpret_cast<uint32_t*>(sgen + C::kOffPrefix);
  __shared__ uint2 s_warp[kThreads / 32];

  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) {
    *abort_flag = 0;
    for (int i = 0; i < kNK; ++i) { mbar_init(b_kfull + 8 * i, 1); mbar_init(b_kfree + 8 * i, 2); }
    for (int i = 0; i < kNV; ++i) { mbar_init(b_vfull + 8 * i, 1); mbar_init(b_vfree + 8 * i, 3); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(b_qfull + 8 * t, 1); mbar_init(b_qfree + 8 * t, 1); mbar_init(b_sfull + 8 * t, 1);
      mbar_init(b_sfree + 8 * t, kRowThreads); mbar_init(b_ofree + 8 * t, kRowThreads);
      mbar_init(b_pvdone + 16 * t, 1); mbar_init(b_pvdone + 16 * t + 8, 1);
      mbar_init(b_pfull + 16 * t, kRowThreads); mbar_init(b_pfull + 16 * t + 8, kRowThreads);
      mbar_init(b_phalf + 16 * t, kRowThreads); mbar_init(b_phalf + 16 * t + 8, kRowThreads);
    }
    for (int i = 0; i < kNV; ++i) mbar_init(b_vfix + 8 * i, 32);
    for (int t = 0; t < 2; ++t) mbar_init(b_turn + 8 * t, 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kSW) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_dependency_wait();
  line_prefix<kThreads, true>(a.seqs.n_seqs, prefix, s_warp, [&](int s) {
    const Seq q = seq_at(a.cache, a.seqs, s);
    const int pairs = (q.n_new + 2 * f.tpt - 1) / (2 * f.tpt);
    Work w = {(uint32_t)pairs, 0u};
    if (a.full) w.units = (uint32_t)pairs * (uint32_t)units_of(q.len);
    else for (int p = 0; p < pairs; ++p) w.units += (uint32_t)units_of(seen_by(a, q, (p + 1) * 2 * f.tpt));
    w.items *= (uint32_t)a.cache.n_kv_heads;
    w.units *= (uint32_t)a.cache.n_kv_heads;
    return w;
  });
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  const Cut cut(prefix[a.seqs.n_seqs], gridDim.x);
  ChunkWalk walk;
  walk.start(cut.start(blockIdx.x), cut.start(blockIdx.x + 1));

  if (warp < kSW) {
    // ============== softmax warps, 16 rows of a tile each ==============
    const int t = (warp >> 2) & 1;
    const int r = (warp & 3) * 32 + 16 * (warp >> 3) + (lane >> 2);         // rows r and r + 8 of the tile
    const int cq2 = 2 * (lane & 3);          // this thread's columns: cq2 and the next of every 8
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32 + 16 * (warp >> 3)) << 16);
    const uint32_t col_t = lane_addr + C::kColTile * t;
    const uint32_t colO = lane_addr + C::kColO + D * t;
    const uint32_t sfull = b_sfull + 8 * t, pfull = b_pfull + 16 * t, phalf = b_phalf + 16 * t, pvdone = b_pvdone + 16 * t;
    const uint64_t sc2 = pack_f2(a.scale_log2, a.scale_log2);
    const int G = a.cache.group, used = f.tpt * G;
    uint32_t turns = 0;                      // steps at which the tiles took turns so far
    uint32_t cnt = 0;                        // steps this tile has been through (barrier phases)
    for (int part = 0; walk.next(f, prefix); ++part) {
      const int nt = t ? walk.nt1 : walk.nt0;
      const int tok0 = (2 * walk.pair + t) * f.tpt;
      if (tok0 >= walk.q.n_new) continue;       // the pair has no second tile
      const int tok_a = tok0 + r / G, tok_b = tok0 + (r + 8) / G;
      const bool has_a = r < used && tok_a < walk.q.n_new, has_b = r + 8 < used && tok_b < walk.q.n_new;
      const int base = a.full ? walk.q.len : walk.q.len - walk.q.n_new + 1;
      // slots below these are seen by row r and row r + 8 (rows of nobody: as many as the tile sees at least)
      const int lim_a = a.full || !has_a ? base : base + tok_a, lim_b = a.full || !has_b ? base : base + tok_b;
      const int least = a.full ? base : base + tok0;
      float m0 = -INFINITY, m1 = -INFINITY;     // reference maxima of the two rows (scaled, log2 units; the same in the quad)
      uint64_t l0 = 0ull, l1 = 0ull;            // partial sums of this thread's columns (packed fp32 pairs)
      for (int jj = 0; jj < nt; ++jj, ++cnt) {
        const int first = (walk.tile_lo + jj) * kUnit;
        mbar_wait(sfull, cnt & 1, wc);
        __syncwarp();            // the waits may leave the warp diverged; tcgen05.ld/st are warp-collective
        tc_fence_after();
        // Half of the columns at a time: 32 scores a thread (all 64 in registers spill, and with the shared memory that this kernel takes
        // there is no L1 to spill to: chunks of four prompts 674 us instead of 646, at that time).
        const uint32_t col_s = D == 64 ? col_t + 64 * (cnt & 1) : col_t;
        uint32_t sc[32];
        auto load = [&](int half) {
          XKV_TMEM_LD_64(col_s + 64 * half, sc, 0);
          tc_wait_ld();
          if (first + kUnit > least) {
            const int la = lim_a - first - 64 * half - cq2, lb = lim_b - first - 64 * half - cq2;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (8 * (i >> 2) + (i & 1) >= ((i & 2) ? lb : la)) sc[i] = 0xff800000u;           // -inf: exponential 0
          }
        };
        auto tops = [&](float& top0, float& top1) {
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            top0 = max3(top0, __uint_as_float(sc[4 * g]), __uint_as_float(sc[4 * g + 1]));
            top1 = max3(top1, __uint_as_float(sc[4 * g + 2]), __uint_as_float(sc[4 * g + 3]));
          }
        };
        auto over_quad = [&](float& top0, float& top1) {       // (and scaled)
#pragma unroll
          for (int o = 1; o < 4; o <<= 1) {
            top0 = fmaxf(top0, __shfl_xor_sync(0xffffffffu, top0, o));
            top1 = fmaxf(top1, __shfl_xor_sync(0xffffffffu, top1, o));
          }
          top0 *= a.scale_log2;
          top1 *= a.scale_log2;
        };
        auto columns = [&](uint32_t* pk) {
          const float ref0 = m0 == -INFINITY ? 0.f : -m0, ref1 = m1 == -INFINITY ? 0.f : -m1;      // (a row that sees nothing)
          const uint64_t nm0 = pack_f2(ref0, ref0), nm1 = pack_f2(ref1, ref1);
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            const uint32_t* x = sc + 4 * g;
            const uint64_t x0 = fma_f2(pack_f2(__uint_as_float(x[0]), __uint_as_float(x[1])), sc2, nm0);
            const uint64_t x1 = fma_f2(pack_f2(__uint_as_float(x[2]), __uint_as_float(x[3])), sc2, nm1);
            const float e0 = fast_exp2(f2_lo(x0)), e1 = fast_exp2(f2_hi(x0)), e2 = fast_exp2(f2_lo(x1)), e3 = fast_exp2(f2_hi(x1));
            l0 = add_f2(l0, pack_f2(e0, e1));
            l1 = add_f2(l1, pack_f2(e2, e3));
            pk[2 * g] = BF16 ? pack_bf2(e0, e1) : pack_h2(e0, e1);
            pk[2 * g + 1] = BF16 ? pack_bf2(e2, e3) : pack_h2(e2, e3);
          }
        };
        // The reference maximum of a row is its maximum over the part's first unit, and moves only when the row's maximum has grown by more
        // than 2^kGrow over it.  So the exponentials of a later unit need not wait for its maxima: they are computed against the
        // reference as it is, the maxima beside them, and in the rare case that a row has outgrown its reference, once more.
        if (jj == 0) {
          load(0);
          tops(m0, m1);
          load(1);
          tops(m0, m1);
          over_quad(m0, m1);
        }
        const uint32_t colP = D == 64 ? col_t + 128 * (cnt & 1) : col_t;       // (over scores of these rows only)
        uint32_t pk[16];
        float top0 = -INFINITY, top1 = -INFINITY;
        const uint64_t l0_before = l0, l1_before = l1;
        // head_dim 128: the tiles take turns at the exponentials: while one has the special-function units to itself, the MMAs of the
        // other run.  (Left alone they fall into step, both at their exponentials and then both at their MMAs: 583 us for the
        // chunks of four prompts instead of 525.  head_dim 64 has its scores a step ahead and loses 10 % by turns.)
        const bool both = D == 128 && jj < min(walk.nt0, walk.nt1);
        load(0);
        tops(top0, top1);
        if (both) {
          if (t) mbar_wait(b_turn + 8, turns & 1, wc);
          else if (turns > 0) mbar_wait(b_turn, (turns - 1) & 1, wc);
          __syncwarp();
        }
        columns(pk);
        load(1);
        if (jj > 0) {
          tops(top0, top1);
          over_quad(top0, top1);
          if (__any_sync(0xffffffffu, top0 > m0 + kGrow || top1 > m1 + kGrow)) {
            float alpha0 = 1.f, alpha1 = 1.f;
            if (top0 > m0 + kGrow) { alpha0 = exp2f(m0 - top0); m0 = top0; }
            if (top1 > m1 + kGrow) { alpha1 = exp2f(m1 - top1); m1 = top1; }
            l0 = mul_f2(l0_before, pack_f2(alpha0, alpha0));
            l1 = mul_f2(l1_before, pack_f2(alpha1, alpha1));
            load(0);
            columns(pk);
            // the accumulator is quiescent once the previous step's PV has completed
            mbar_wait(pvdone + 8 * ((cnt - 1) & 1), ((cnt - 1) >> 1) & 1, wc);
            __syncwarp();
            tc_fence_after();
            rescale_chunk_rows<D>(colO, alpha0, alpha1);
            load(1);
          }
        }
        if (D == 64) {
          tc_fence_before();
          mbar_arrive(b_sfree + 8 * t);
        }
        XKV_TMEM_ST_P32(colP, pk);
        if (D == 128) {          // the first half of P V may begin
          tc_wait_st();
          tc_fence_before();
          mbar_arrive(phalf + 8 * (cnt & 1));
        }
        columns(pk);
        if (both) {
          __syncwarp();
          if (lane == 0) mbar_arrive(b_turn + 8 * (t ^ 1));
          ++turns;
        }
        XKV_TMEM_ST_P32(colP + 32, pk);
        tc_wait_st();
        tc_fence_before();
        mbar_arrive(pfull + 8 * (cnt & 1));
      }
      // ---- end of the part ----
      const bool whole = walk.nt == walk.units;
      const size_t slot = (size_t)2 * blockIdx.x + (part == 0 ? 0 : 1);
      const size_t prow = (slot * 2 + t) * 128 + r;
      if (nt == 0) {               // (an item whose first tile ended in an earlier piece)
        if ((lane & 3) == 0) { f.s.ml[prow] = make_float2(-INFINITY, 0.f); f.s.ml[prow + 8] = make_float2(-INFINITY, 0.f); }
        continue;
      }
      mbar_wait(pvdone + 8 * ((cnt - 1) & 1), ((cnt - 1) >> 1) & 1, wc);    // the last PV (they complete in order)
      __syncwarp();
      tc_fence_after();
      float s0 = f2_lo(l0) + f2_hi(l0), s1 = f2_lo(l1) + f2_hi(l1);
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        s0 += __shfl_xor_sync(0xffffffffu, s0, o);
        s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      }
      const int head_a = walk.head * G + r % G, head_b = walk.head * G + (r + 8) % G;
      const int64_t row_a = walk.q.row0 + tok_a, row_b = walk.q.row0 + tok_b;
      uint32_t nan_a = 0u, nan_b = 0u;              // NaN if an output of the row is
#pragma unroll 1
      for (int c = 0; c < D; c += 64) {
        uint32_t ro[32];
        XKV_TMEM_LD_64(colO + c, ro, 0);
        tc_wait_ld();
        if (c + 64 == D) {
          tc_fence_before();
          mbar_arrive(b_ofree + 8 * t);
        }
        if (whole) {
          const float inv0 = s0 == 0.f ? 0.f : 1.f / s0, inv1 = s1 == 0.f ? 0.f : 1.f / s1;
          uint8_t* oa = a.out + 2 * (head_a * a.o_hs + row_a * a.o_ts + c + cq2);
          uint8_t* ob = a.out + 2 * (head_b * a.o_hs + row_b * a.o_ts + c + cq2);
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            const float x0 = __uint_as_float(ro[4 * g]) * inv0, x1 = __uint_as_float(ro[4 * g + 1]) * inv0;
            const float x2 = __uint_as_float(ro[4 * g + 2]) * inv1, x3 = __uint_as_float(ro[4 * g + 3]) * inv1;
            const uint32_t wa = BF16 ? pack_bf2(x0, x1) : pack_h2(x0, x1), wb = BF16 ? pack_bf2(x2, x3) : pack_h2(x2, x3);
            // (a row that sees nothing is zero, whatever a weight of 0 met)
            if (has_a) *reinterpret_cast<uint32_t*>(oa + 16 * g) = s0 == 0.f ? 0u : wa;
            if (has_b) *reinterpret_cast<uint32_t*>(ob + 16 * g) = s1 == 0.f ? 0u : wb;
            nan_a = max_nan_pair<BF16>(nan_a, wa);
            nan_b = max_nan_pair<BF16>(nan_b, wb);
          }
        } else {
          float* dst = f.s.o + prow * D + c + cq2;
#pragma unroll
          for (int g = 0; g < 8; ++g) {
            *reinterpret_cast<float2*>(dst + 8 * g) = make_float2(__uint_as_float(ro[4 * g]), __uint_as_float(ro[4 * g + 1]));
            *reinterpret_cast<float2*>(dst + 8 * D + 8 * g) = make_float2(__uint_as_float(ro[4 * g + 2]), __uint_as_float(ro[4 * g + 3]));
          }
        }
      }
      // (not of the last new token, which sees all, nor where the sum says as much, or nothing was seen; of a frame all tokens see all)
      if (whole && !a.full && ((any_nan<BF16>(nan_a) && s0 > 0.f && has_a && tok_a + 1 < walk.q.n_new) ||
                               (any_nan<BF16>(nan_b) && s1 > 0.f && has_b && tok_b + 1 < walk.q.n_new)))
        f.s.again[0] = f.s.again[2 + walk.seq] = 1u;
      if ((lane & 3) == 0) {
        if (!whole) { f.s.ml[prow] = make_float2(m0, s0); f.s.ml[prow + 8] = make_float2(m1, s1); }
        else if (a.lse) {
          if (has_a) a.lse[(int64_t)head_a * a.seqs.n_tokens + row_a] = s0 == 0.f ? -INFINITY : (m0 + log2f(s0)) * 0.69314718055994531f;
          if (has_b) a.lse[(int64_t)head_b * a.seqs.n_tokens + row_b] = s1 == 0.f ? -INFINITY : (m1 + log2f(s1)) * 0.69314718055994531f;
        }
      }
    }
    tc_fence_before();
  } else if (warp < kSW + 2) {
    // =========================== MMA issuers ==================================
    const uint32_t t = warp - kSW;
    const uint32_t idesc_qk = make_idesc(128, BF16, false), idesc_pv = make_idesc(D, BF16, true);
    const uint64_t dq = make_desc(sQ + t * kTile), dk0 = make_desc(sK), dv0 = desc_mn(sV, 16384);
    const uint32_t d_tile = tmem + C::kColTile * t, d_o = tmem + C::kColO + D * t;
    uint32_t kb = 0, kph = 0, vb = 0, vph = 0;      // ring positions and their parities
    uint32_t cs = 0, cq = 0;                        // scores and parts with this tile so far
    uint32_t fix = 0;                               // parities of the stages' ends of sequences, one bit each
    auto scores = [&](int jj, int nt) {             // S of step cs, if the tile has it
      mbar_wait(b_kfull + 8 * kb, kph, wc);
      const bool active = jj < nt;
      if (active) {
        if (jj == 0) mbar_wait(b_qfull + 8 * t, cq & 1, wc);
        // the columns: scores of the step before are in registers, P of the one before that (head_dim 128: of the step
        // before) is consumed
        if (D == 64) {
          if (cs > 0) mbar_wait(b_sfree + 8 * t, (cs - 1) & 1, wc);
          if (cs > 1) mbar_wait(b_pvdone + 16 * t + 8 * (cs & 1), ((cs >> 1) - 1) & 1, wc);
        } else if (cs > 0) {
          mbar_wait(b_pvdone + 16 * t + 8 * ((cs - 1) & 1), ((cs - 1) >> 1) & 1, wc);
        }
      }
      __syncwarp();
      tc_fence_after();
      if (elect_one()) {
        if (active) {
          const uint64_t dk = dk0 + (uint64_t)(kb * (kTile >> 4));
          const uint32_t d_s = D == 64 ? d_tile + 64 * (cs & 1) : d_tile;
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {   // 16 channels per step: 32 B inside the swizzle span
            const uint64_t at = (uint64_t)((ks >> 2) * (16384 >> 4) + (ks & 3) * 2);
            mma_ss(d_s, dq + at, dk + at, idesc_qk, ks > 0 ? 1u : 0u);
          }
          tc_commit(b_sfull + 8 * t);
          if (jj == nt - 1) tc_commit(b_qfree + 8 * t);
        }
        tc_commit(b_kfree + 8 * kb);
      }
      __syncwarp();
      if (active) ++cs;
      if (++kb == (uint32_t)kNK) { kb = 0; kph ^= 1; }
    };
    auto values = [&](int jj, int nt, uint32_t c) {     // P V of step c
      const bool active = jj < nt;
      const int valid = walk.q.len - (walk.tile_lo + jj) * kUnit;
      const int steps = valid >= kUnit ? 8 : max(1, (valid + 15) / 16);
      mbar_wait(b_vfull + 8 * vb, vph, wc);
      if (valid < kUnit && (valid & 15) && valid > 0) { mbar_wait(b_vfix + 8 * vb, (fix >> vb) & 1, wc); fix ^= 1u << vb; }
      const uint64_t dv = dv0 + (uint64_t)(vb * (kTile >> 4));
      const uint32_t d_p = D == 64 ? d_tile + 128 * (c & 1) : d_tile;
      auto multiply = [&](int from, int to) {
        __syncwarp();
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int ks = from; ks < to; ++ks)   // 16 tokens per step: 2048 B of every slab of V, 8 columns of P
            if (ks < steps) mma_ts(d_o, d_p + 8 * ks, dv + (uint64_t)((ks * 2048) >> 4), idesc_pv, (jj > 0 || ks > 0) ? 1u : 0u);
          if (to == 8) tc_commit(b_pvdone + 16 * t + 8 * (c & 1));
        }
        __syncwarp();
      };
      if (active) {
        if (D == 128) mbar_wait(b_phalf + 16 * t + 8 * (c & 1), (c >> 1) & 1, wc);
        else mbar_wait(b_pfull + 16 * t + 8 * (c & 1), (c >> 1) & 1, wc);
        if (jj == 0 && cq > 0) mbar_wait(b_ofree + 8 * t, (cq - 1) & 1, wc);
        if (D == 128) {
          multiply(0, 4);
          mbar_wait(b_pfull + 16 * t + 8 * (c & 1), (c >> 1) & 1, wc);
          multiply(4, 8);
        } else {
          multiply(0, 8);
        }
      }
      if (elect_one()) tc_commit(b_vfree + 8 * vb);
      __syncwarp();
      if (++vb == (uint32_t)kNV) { vb = 0; vph ^= 1; }
    };
    while (walk.next(f, prefix)) {
      const int nt = t ? walk.nt1 : walk.nt0;
      if (D == 64) {
        // the scores are a whole step ahead of P V
#pragma unroll 1
        for (int jj = 0; jj <= walk.nt; ++jj) {
          if (jj < walk.nt) scores(jj, nt);
          if (jj > 0) values(jj - 1, nt, cs - (jj < nt ? 2u : 1u));
        }
      } else {
#pragma unroll 1
        for (int jj = 0; jj < walk.nt; ++jj) {
          scores(jj, nt);
          values(jj, nt, cs - 1);
        }
      }
      if (nt > 0) ++cq;
    }
    tc_fence_before();
  } else if (warp == kSW + 2) {
    // =========================== copies =======================================
    uint32_t g = 0, cq[2] = {0, 0};
    const int page_mask = (1 << a.cache.page_shift) - 1;
    const int per_unit = kUnit / f.box_rows;              // copies of a unit, 1..8
    while (walk.next(f, prefix)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if ((t ? walk.nt1 : walk.nt0) == 0) continue;
        if (cq[t] > 0) mbar_wait<1000>(b_qfree + 8 * t, (cq[t] - 1) & 1, wc);
        __syncwarp();
        if (lane == 0) {
          mbar_expect_tx(b_qfull + 8 * t, (uint32_t)(kSlabs * 128 * f.q_toks * a.cache.group));
#pragma unroll
          for (int c = 0; c < kSlabs; ++c)
            tma_3d(sQ + t * kTile + c * 16384, &q_map, 64 * c, walk.head * a.cache.group, walk.q.row0 + (2 * walk.pair + t) * f.tpt, b_qfull + 8 * t);
        }
        ++cq[t];
      }
      int ids = 0, ids_at = -1;                           // pages of the next 32 copies, one per lane
      for (int jj = 0; jj < walk.nt; ++jj, ++g) {
        const int first = (walk.tile_lo + jj) * kUnit;
        const int boxes = min(per_unit, max(1, (walk.q.len - first + f.box_rows - 1) / f.box_rows));
        if (ids_at < 0 || jj - ids_at >= 32 / per_unit) {
          ids_at = jj;
          const int slot = first + lane * f.box_rows;
          // (slots behind the end have no page; nor have those behind the part, which are not looked up)
          ids = slot < walk.q.len && slot < (walk.tile_lo + walk.nt) * kUnit ? page_at(a.cache, a.seqs.table, a.seqs.table_width, walk.seq, slot) : -1;
          if (ids < 0) ids = a.cache.n_pages;             // outside the map: zeros
        }
        const uint32_t ks = g % kNK, vs = g % kNV;
        const int id0 = (jj - ids_at) * per_unit;
        mbar_wait<1000>(b_kfree + 8 * ks, ((g / kNK) & 1) ^ 1, wc);
        __syncwarp();
        if (lane == 0) mbar_expect_tx(b_kfull + 8 * ks, (uint32_t)(boxes * f.box_rows * 128 * kSlabs));
        for (int i = 0; i < boxes; ++i) {
          const int page = __shfl_sync(0xffffffffu, ids, id0 + i);
          if (lane == 0)
#pragma unroll
            for (int c = 0; c < kSlabs; ++c)
              tma_4d(sK + ks * kTile + c * 16384 + i * f.box_rows * 128, &maps.k, 64 * c, (first + i * f.box_rows) & page_mask, walk.head, page, b_kfull + 8 * ks);
        }
        mbar_wait<1000>(b_vfree + 8 * vs, ((g / kNV) & 1) ^ 1, wc);
        __syncwarp();
        if (lane == 0) mbar_expect_tx(b_vfull + 8 * vs, (uint32_t)(boxes * f.box_rows * 128 * kSlabs));
        for (int i = 0; i < boxes; ++i) {
          const int page = __shfl_sync(0xffffffffu, ids, id0 + i);
          if (lane == 0)
#pragma unroll
            for (int c = 0; c < kSlabs; ++c)
              tma_4d(sV + vs * kTile + c * 16384 + i * f.box_rows * 128, &maps.v, 64 * c, (first + i * f.box_rows) & page_mask, walk.head, page, b_vfull + 8 * vs);
        }
        __syncwarp();
      }
    }
    // Drain (bounded, and not cut short by the abort flag): nothing may be in flight at exit.
    if (lane == 0) {
      auto drain = [&](uint32_t full, uint32_t stages, uint32_t issued) {
        for (uint32_t i = 0; i < stages && i < issued; ++i) {
          const uint32_t gi = issued - 1 - i;
          for (uint32_t it = 0; it < kSpinLimit; ++it)
            if (mbar_try(full + 8 * (gi % stages), (gi / stages) & 1)) break;
        }
      };
      drain(b_kfull, kNK, g);
      drain(b_vfull, kNV, g);
      drain(b_qfull, 1, cq[0]);
      drain(b_qfull + 8, 1, cq[1]);
    }
    __syncwarp();
  } else {
    // =========================== ends of sequences ============================
    uint32_t g = 0;
    while (walk.next(f, prefix)) {
      for (int jj = 0; jj < walk.nt; ++jj, ++g) {
        const int valid = walk.q.len - (walk.tile_lo + jj) * kUnit;
        const uint32_t vs = g % kNV;
        // (every unit is waited for, and released, by this warp too: a wait by parity has to follow its barrier phase by phase)
        mbar_wait<1000>(b_vfull + 8 * vs, (g / kNV) & 1, wc);
        __syncwarp();
        if (lane == 0) mbar_arrive(b_vfree + 8 * vs);
        if (valid >= kUnit || valid <= 0 || !(valid & 15)) continue;
        const int rows = 16 - (valid & 15);
        for (int i = lane; i < rows * 8 * kSlabs; i += 32) {
          const int row = valid + (i >> 3) % rows, c = (i >> 3) / rows;
          *reinterpret_cast<uint4*>(sgen + C::kOffV + vs * kTile + c * 16384 + row * 128 + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async();
        mbar_arrive(b_vfix + 8 * vs);
      }
    }
    // the item that starts in this block's piece and goes on in the next one, for the merge
    if (lane == 0) {
      CutItem ci;
      ci.parts = 0;
      ChunkWalk w;
      w.start(cut.start(blockIdx.x), cut.start(blockIdx.x + 1));
      for (int part = 0; w.next(f, prefix); ++part) {
        if (w.tile_lo == 0 && w.nt < w.units) {
          ci.row0 = w.q.row0; ci.n_new = w.q.n_new; ci.head = w.head; ci.pair = w.pair; ci.seq = w.seq;
          ci.parts = (int)cut.owner(w.item_lo + kItemCost + (uint32_t)w.units - 1) - (int)blockIdx.x + 1;
          ci.slot0 = 2 * blockIdx.x + (part == 0 ? 0 : 1);
        }
      }
      f.cuts[blockIdx.x] = ci;
    }
    __syncwarp();
  }
  __syncthreads();
  if (tid == 0 && *abort_flag) atomicExch(a.cache.status, (int)XKV_E_TIMEOUT);
  if (warp == kSW) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// Rows of a marked sequence again, a warp per row.  What the row's output holds as NaN may come from values that the row does not see: if new
// tokens behind it have values there that are not finite, and no token up to it has a NaN there, which the output would have to show.
template <typename T, int D>
__device__ __noinline__ void look_again(const ChunkArgs& f, int seq, int tok, int g, float* s_q) {
  const PagedAttnArgs& a = f.a;
  const Seq q = seq_at(a.cache, a.seqs, seq);
  const int lane = threadIdx.x & 31, row = q.row0 + tok, h = g / a.cache.group;
  const int seen = q.len - q.n_new + tok + 1;
  if (seen <= 0) return;                               // zero, as it should be
  constexpr int kWords = D / 64;                       // channels 2 lane + 64 i and the next
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  constexpr uint32_t kExp = kBf16 ? 0x7F807F80u : 0x7C007C00u;
  auto special = [&](uint32_t w, bool nan) {           // of the two numbers of a word, bits 0 and 16: not finite, or NaN
    const uint32_t e = w & kExp, f2 = w & ~kExp & 0x7FFF7FFFu;
    const bool lo = (e & 0xFFFFu) == (kExp & 0xFFFFu) && (!nan || (f2 & 0xFFFFu)), hi = (e >> 16) == (kExp >> 16) && (!nan || (f2 >> 16));
    return (lo ? 1u : 0u) | (hi ? 0x10000u : 0u);
  };
  const uint8_t* op = a.out + 2 * ((int64_t)g * a.o_hs + (int64_t)row * a.o_ts);
  auto words = [&](int slot, uint32_t (&w)[kWords]) {  // of a value
    const int page = page_at(a.cache, a.seqs.table, a.seqs.table_width, seq, slot);
#pragma unroll
    for (int i = 0; i < kWords; ++i)
      w[i] = page < 0 ? 0u : *reinterpret_cast<const uint32_t*>(a.cache.v + 2 * row_offset(a.cache, page, h, slot) + 4 * (lane + 32 * i));
  };
  uint32_t open = 0;                                   // of this lane's channels those in question, word i's at bits i and 16 + i
#pragma unroll
  for (int i = 0; i < kWords; ++i) open |= special(*reinterpret_cast<const uint32_t*>(op + 4 * (lane + 32 * i)), true) << i;
  if (!__any_sync(0xffffffffu, open != 0)) return;
  uint32_t from = 0;
#pragma unroll 4
  for (int j = seen; j < q.len; ++j) {
    uint32_t w[kWords];
    words(j, w);
#pragma unroll
    for (int i = 0; i < kWords; ++i) from |= special(w[i], false) << i;
  }
  open &= from;
  for (int j = seen - 1; j >= max(0, q.len - q.n_new); --j) {
    if (!__any_sync(0xffffffffu, open != 0)) return;
    uint32_t w[kWords];
    words(j, w);
#pragma unroll
    for (int i = 0; i < kWords; ++i) open &= ~(special(w[i], true) << i);
  }
  if (__any_sync(0xffffffffu, open != 0)) attend_row<T, D>(a, seq, q, row, g, s_q);
}

// Merge of the items that were cut between blocks, in the order of the pieces: 32 rows per block, (row, 8 channels) per thread.
constexpr int kMergeRows = 32;
// Answers whether the row is to be looked at again, as above.
template <int D, bool BF16>
__device__ __forceinline__ bool merge_rows(const ChunkArgs& f, const CutItem& ci) {
  const PagedAttnArgs& a = f.a;
  const int G = a.cache.group;
  const int t = (int)blockIdx.x / (128 / kMergeRows);
  const int r = ((int)blockIdx.x % (128 / kMergeRows)) * kMergeRows + (int)threadIdx.x / (D / 8), c = ((int)threadIdx.x % (D / 8)) * 8;
  const int tok = (2 * ci.pair + t) * f.tpt + r / G;
  if (r >= f.tpt * G || tok >= ci.n_new) return false;
  float m = -INFINITY, l = 0.f;
  float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int p0 = 0; p0 < ci.parts; p0 += 4) {
    float2 ml[4];
    float4 x[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      ml[j] = make_float2(-INFINITY, 0.f);
      x[j] = y[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p0 + j < ci.parts) {
        const size_t slot = p0 + j == 0 ? (size_t)ci.slot0 : (size_t)2 * (blockIdx.y + p0 + j);
        const size_t prow = (slot * 2 + t) * 128 + r;
        ml[j] = f.s.ml[prow];
        const float4* po = reinterpret_cast<const float4*>(f.s.o + prow * D + c);
        x[j] = po[0];
        y[j] = po[1];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)             // (a part without this tile has no accumulators: whatever was there before)
      if (ml[j].x == -INFINITY) x[j] = y[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    const float mc = fmaxf(fmaxf(m, fmaxf(ml[0].x, ml[1].x)), fmaxf(ml[2].x, ml[3].x));
    const float ref = mc == -INFINITY ? 0.f : mc;
    const float sc = exp2f(m - ref);
    m = mc;
    l *= sc;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] *= sc;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float w = exp2f(ml[j].x - ref);        // 0 for an absent piece
      l += w * ml[j].y;
      acc[0] += w * x[j].x; acc[1] += w * x[j].y; acc[2] += w * x[j].z; acc[3] += w * x[j].w;
      acc[4] += w * y[j].x; acc[5] += w * y[j].y; acc[6] += w * y[j].z; acc[7] += w * y[j].w;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int64_t head = ci.head * G + r % G, row = ci.row0 + tok;
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = BF16 ? pack_bf2(acc[2 * i] * inv, acc[2 * i + 1] * inv) : pack_h2(acc[2 * i] * inv, acc[2 * i + 1] * inv);
  *reinterpret_cast<uint4*>(a.out + 2 * (head * a.o_hs + row * a.o_ts + c)) = make_uint4(o[0], o[1], o[2], o[3]);
  if (c == 0 && a.lse) a.lse[head * a.seqs.n_tokens + row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  bool strange = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) strange |= any_nan<BF16>(o[i]);
  return strange && !a.full && l > 0.f && tok + 1 < ci.n_new;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kMergeRows * D / 8) chunk_merge_kernel(const __grid_constant__ ChunkArgs f) {
  grid_dependency_wait();
  using T = typename std::conditional<BF16, __nv_bfloat16, __half>::type;
  constexpr int kWarps = kMergeRows * D / 8 / 32;
  __shared__ float s_q[kWarps][D];
  __shared__ bool s_last;
  const CutItem ci = f.cuts[blockIdx.y];
  const bool again = f.s.again[0] != 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, G = f.a.cache.group;
  // (the barrier makes the merged rows visible to the warps that look at them again)
  if (ci.parts != 0 && __syncthreads_or(merge_rows<D, BF16>(f, ci))) {
    const int t = (int)blockIdx.x / (128 / kMergeRows), r0 = ((int)blockIdx.x % (128 / kMergeRows)) * kMergeRows;
    for (int r = r0 + warp; r < r0 + kMergeRows; r += kWarps) {
      const int tok = (2 * ci.pair + t) * f.tpt + r / G;
      if (r < f.tpt * G && tok < ci.n_new) look_again<T, D>(f, ci.seq, tok, ci.head * G + r % G, s_q[warp]);
    }
  }
  if (!again) return;
  // ---- marked sequences: a share of the rows that no block merged ----
  const uint32_t warps = gridDim.x * gridDim.y * kWarps, me = (blockIdx.y * gridDim.x + blockIdx.x) * kWarps + warp;
  for (int s = 0; s < f.a.seqs.n_seqs; ++s) {
    if (!f.s.again[2 + s]) continue;
    const int n_new = seq_at(f.a.cache, f.a.seqs, s).n_new;
    for (int64_t i = me; i < (int64_t)n_new * f.a.cache.n_heads; i += warps) {
      const int tok = (int)(i / f.a.cache.n_heads), g = (int)(i - (int64_t)tok * f.a.cache.n_heads);
      bool merged = false;
      for (uint32_t y = lane; y < gridDim.y; y += 32) {
        const CutItem c = f.cuts[y];
        merged |= c.parts != 0 && c.seq == s && c.head == g / G && c.pair == tok / (2 * f.tpt);
      }
      if (!__any_sync(0xffffffffu, merged)) look_again<T, D>(f, s, tok, g, s_q[warp]);
    }
  }
  // the last block to come clears the marks
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = atomicAdd(f.s.again + 1, 1u) == gridDim.x * gridDim.y - 1;
  }
  __syncthreads();
  if (!s_last) return;
  for (int s = threadIdx.x; s < f.a.seqs.n_seqs; s += blockDim.x) f.s.again[2 + s] = 0;
  if (threadIdx.x == 0) f.s.again[0] = f.s.again[1] = 0;
}

}  // namespace

size_t attn_chunk_cut_bytes() { return sizeof(CutItem); }

template <int D, bool BF16>
static cudaError_t setup_one() {
  return cudaFuncSetAttribute(attn_chunk_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Chunk<D>::kBytes);
}
cudaError_t attn_chunk_setup() {
  cudaError_t e = setup_one<64, true>();
  if (e == cudaSuccess) e = setup_one<64, false>();
  if (e == cudaSuccess) e = setup_one<128, true>();
  if (e == cudaSuccess) e = setup_one<128, false>();
  return e;
}

cudaError_t launch_attn_chunk(const PagedAttnArgs& a, const PoolMaps& maps, const PagedScratch& s, void* cuts, int head_dim, int dtype,
                              int sm_count, cudaStream_t st) {
  ChunkArgs f;
  f.a = a;
  f.s = s;
  f.cuts = reinterpret_cast<CutItem*>(cuts);
  f.tpt = 128 / a.cache.group;
  f.box_rows = min(1 << a.cache.page_shift, 128);
  f.q_toks = min(f.tpt, a.seqs.max_new);
  CUtensorMap q_map;
  cudaError_t e = make_token_map(a.q, a.q_ts, a.q_hs, a.seqs.n_tokens, a.cache.n_heads, head_dim, dtype, a.cache.group, f.q_toks, &q_map);
  if (e != cudaSuccess) return e;
  const int grid = sm_count;
  void* p0[3] = {(void*)&f, (void*)&maps, (void*)&q_map};
  void* p1[1] = {(void*)&f};
  const bool bf16 = dtype == XKV_BF16;
  const void *k0, *k1;
  size_t smem;
  if (head_dim == 64) {
    k0 = bf16 ? (const void*)attn_chunk_kernel<64, true> : (const void*)attn_chunk_kernel<64, false>;
    k1 = bf16 ? (const void*)chunk_merge_kernel<64, true> : (const void*)chunk_merge_kernel<64, false>;
    smem = Chunk<64>::kBytes;
  } else {
    k0 = bf16 ? (const void*)attn_chunk_kernel<128, true> : (const void*)attn_chunk_kernel<128, false>;
    k1 = bf16 ? (const void*)chunk_merge_kernel<128, true> : (const void*)chunk_merge_kernel<128, false>;
    smem = Chunk<128>::kBytes;
  }
  e = launch_overlapped(k0, dim3(grid), dim3(kThreads), p0, smem, st);
  if (e != cudaSuccess) return e;
  e = launch_overlapped(k1, dim3(256 / kMergeRows, grid), dim3(kMergeRows * head_dim / 8), p1, 0, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace xkv
