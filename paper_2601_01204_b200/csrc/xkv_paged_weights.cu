// Softmax weights that every cached token got from the new tokens: sum over rows of exp(q.k scale - lse), with the lse of the
// attention, so that no row needs a maximum or a second pass.
//
// The scores are computed transposed, S^T = K Q^T: tcgen05.mma with the 128 tokens of a unit as its rows, in tensor memory one
// token per lane, and the query rows (128 / G tokens of G heads, as in the chunk attention) as its columns.  A thread
// then owns a token and adds its weights up in registers; nothing is exchanged between lanes, and the sums have a fixed order.
// K is read once, stays in shared memory for all query tiles; the query tiles come from the L2 again for every unit.
//
// One block, 20 warps: 16 exponential warps in four groups (a group is four warps, one per quarter of the lanes), one MMA issuer,
// one for copies, one that stages -lse per column, one idle.  Of a tile of 128 columns each group takes 32, and at the
// end of a unit the groups' sums meet in shared memory.  FEW: at most 32 rows per sequence and key head (single tokens): a
// group takes a whole unit, four units are in flight, and nothing has to meet.
//
// What bounds it: with many rows the exponentials (16 per clock and multiprocessor; the MMAs need a quarter to a half of that time),
// with few rows reading K.
#include "xkv_paged_line.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace {

constexpr int kThreads = 640;
constexpr int kEW = 16;                       // exponential warps; 16: MMA, 17: copies, 18: lse
constexpr uint32_t kSpinLimit = 1u << 22;

template <int D> struct Weigh {
  static constexpr int kSlabs = D / 64;
  static constexpr int kTile = kSlabs * 16384;
  static constexpr int kNK = D == 64 ? 6 : 3, kNQ = D == 64 ? 4 : 3;
  static constexpr int kOffQ = kNK * kTile, kOffBar = kOffQ + kNQ * kTile;
  static constexpr int kOffLse = kOffBar + 512, kOffSum = kOffLse + 4 * 512, kOffSeq = kOffSum + 2 * 4 * 512;
  static constexpr int kOffPrefix = kOffSeq + kMaxSeqs * 12;
  static constexpr size_t kBytes = kOffPrefix + (kMaxSeqs + 1) * 4 + 1024;
};

struct WeighArgs {
  PagedWeightArgs a;
  int tpt, box_rows;
};

// Units of the block: every gridDim.x-th of the line.
struct UnitWalk {
  uint32_t pos, total, step;
  int seq, head, first;                  // first token of the unit
  int row0, n_new, len;
  int tile0, tiles;                      // query tiles that see a token of the unit
  __device__ __forceinline__ bool next(const WeighArgs& f, const uint32_t* prefix, const Seq* seqs) {
    if (pos >= total) return false;
    seq = line_seq(prefix, f.a.seqs.n_seqs, pos);
    const Seq q = seqs[seq];
    row0 = q.row0; n_new = q.n_new; len = q.len;
    const uint32_t per = (uint32_t)((q.len + kUnit - 1) / kUnit), rel = pos - prefix[seq];
    head = (int)(rel / per);
    first = (int)(rel - (uint32_t)head * per) * kUnit;
    // new token i sees slot j iff i >= j - (len - n_new)
    tile0 = f.a.full ? 0 : max(0, first - (len - n_new)) / f.tpt;
    tiles = (n_new + f.tpt - 1) / f.tpt - tile0;
    pos += step;
    return true;
  }
};

__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* map, int c, int slot, int head, int page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(c), "r"(slot), "r"(head), "r"(page), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int c, int head, int tok, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(c), "r"(head), "r"(tok), "r"(bar) : "memory");
}
#define XKV_TMEM_LD_32(taddr, r)                                                                    \
  asm volatile(                                                                                     \
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"                                                    \
      "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"                                      \
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"                    \
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),             \
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),       \
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),     \
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])      \
      : "r"(taddr) : "memory")

template <int D, bool BF16, bool FEW>
__global__ void __launch_bounds__(kThreads, 1)
weights_kernel(const __grid_constant__ WeighArgs f, const __grid_constant__ PoolMaps maps, const __grid_constant__ CUtensorMap q_map) {
  using C = Weigh<D>;
  constexpr int kNK = C::kNK, kNQ = C::kNQ, kTile = C::kTile, kSlabs = C::kSlabs;
  extern __shared__ uint8_t smem_raw[];
  const PagedWeightArgs& a = f.a;
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* sgen = smem_raw + (sbase - smem_u32(smem_raw));
  const uint32_t sK = sbase, sQ = sbase + C::kOffQ;
  const uint32_t b_kfull = sbase + C::kOffBar, b_kfree = b_kfull + 8 * kNK, b_qfull = b_kfree + 8 * kNK, b_qfree = b_qfull + 8 * kNQ;
  const uint32_t b_sfull = b_qfree + 8 * kNQ, b_sfree = b_sfull + 32, b_lfull = b_sfree + 32;      // [4] buffers of scores
  static_assert(8 * (2 * kNK + 2 * kNQ + 12) <= 512 - 16, "barriers");
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sgen + C::kOffBar + 496);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sgen + C::kOffBar + 500);
  const WaitCtx wc{sbase + C::kOffBar + 500};
  float* s_lse = reinterpret_cast<float*>(sgen + C::kOffLse);        // [4][128] -lse in log2 units
  float* s_sum = reinterpret_cast<float*>(sgen + C::kOffSum);        // [2][4][128]
  Seq* seqs = reinterpret_cast<Seq*>(sgen + C::kOffSeq);
  uint32_t* prefix = reinterpret_cast<uint32_t*>(sgen + C::kOffPrefix);
  __shared__ uint32_t s_warp[kThreads / 32];

  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) {
    *abort_flag = 0;
    for (int i = 0; i < kNK; ++i) { mbar_init(b_kfull + 8 * i, 1); mbar_init(b_kfree + 8 * i, 1); }
    for (int i = 0; i < kNQ; ++i) { mbar_init(b_qfull + 8 * i, 1); mbar_init(b_qfree + 8 * i, 1); }
    for (int i = 0; i < 4; ++i) { mbar_init(b_sfull + 8 * i, 1); mbar_init(b_sfree + 8 * i, FEW ? 4 : kEW); mbar_init(b_lfull + 8 * i, 32); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kEW) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_dependency_wait();
  line_prefix<kThreads>(a.seqs.n_seqs, prefix, s_warp, [&](int s) {
    const Seq q = seq_at(a.cache, a.seqs, s);
    seqs[s] = q;
    return q.n_new == 0 ? 0u : (uint32_t)a.cache.n_kv_heads * (uint32_t)((q.len + kUnit - 1) / kUnit);
  });
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  UnitWalk walk;
  walk.pos = blockIdx.x;
  walk.step = gridDim.x;
  walk.total = prefix[a.seqs.n_seqs];
  const int G = a.cache.group;

  if (warp < kEW) {
    // ============== exponentials: thread = token of the unit ==============
    const int group = warp >> 2;
    const int key = (warp & 3) * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint64_t sc2 = pack_f2(a.scale_log2, a.scale_log2);
    uint32_t cnt = 0;                       // tiles so far, of all groups
    for (uint32_t unit = 0; walk.next(f, prefix, seqs); ++unit) {
      // the unit's old weights and their places, for the group that will write them
      const bool mine = (unit & 3) == (uint32_t)group;
      float* place = nullptr;
      float old = 0.f;
      if (mine && walk.first + key < walk.len) {
        const int page = page_at(a.cache, a.seqs.table, a.seqs.table_width, walk.seq, walk.first + key);
        if (page >= 0) {
          place = a.cache.weights + weight_offset(a.cache, page, walk.head, walk.first + key);
          if (a.decay != 0.f) old = *place;
        }
      }
      float total = 0.f;
      const int base = walk.len - walk.n_new;                 // token i sees slots <= base + i
      for (int j = 0; j < walk.tiles; ++j, ++cnt) {
        if (FEW && !mine) continue;
        const uint32_t buf = cnt & 3, ph = (cnt >> 2) & 1;
        const int tok0 = (walk.tile0 + j) * f.tpt;
        const int cols = min(f.tpt, walk.n_new - tok0) * G;
        const int c0 = FEW ? 0 : 32 * group;
        mbar_wait(b_sfull + 8 * buf, ph, wc);
        mbar_wait(b_lfull + 8 * buf, ph, wc);
        __syncwarp();
        tc_fence_after();
        if (c0 < cols) {
          uint32_t s[32];
          XKV_TMEM_LD_32(lane_addr + 128 * buf + c0, s);
          tc_wait_ld();
          const float4* nl = reinterpret_cast<const float4*>(s_lse + 128 * buf + c0);
          // columns that see the token: tokens i >= slot - base; columns behind the tile's rows belong to nobody
          const int lo = a.full ? 0 : (walk.first + key - base - tok0) * G - c0, hi = cols - c0;
          uint64_t sum = 0ull;
          const bool plain = hi >= 32 && (a.full || walk.first + kUnit - 1 <= base + tok0);      // (the same in all threads)
          if (plain) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float4 n = nl[i];
              const uint64_t x0 = fma_f2(pack_f2(__uint_as_float(s[4 * i]), __uint_as_float(s[4 * i + 1])), sc2, pack_f2(n.x, n.y));
              const uint64_t x1 = fma_f2(pack_f2(__uint_as_float(s[4 * i + 2]), __uint_as_float(s[4 * i + 3])), sc2, pack_f2(n.z, n.w));
              sum = add_f2(sum, pack_f2(fast_exp2(f2_lo(x0)), fast_exp2(f2_hi(x0))));
              sum = add_f2(sum, pack_f2(fast_exp2(f2_lo(x1)), fast_exp2(f2_hi(x1))));
            }
          } else {
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float2 n = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(nl) + i);
              const float p0 = fast_exp2(fmaf(__uint_as_float(s[i]), a.scale_log2, n.x)), p1 = fast_exp2(fmaf(__uint_as_float(s[i + 1]), a.scale_log2, n.y));
              sum = add_f2(sum, pack_f2(i >= lo && i < hi ? p0 : 0.f, i + 1 >= lo && i + 1 < hi ? p1 : 0.f));
            }
          }
          total += f2_lo(sum) + f2_hi(sum);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(b_sfree + 8 * buf);
      }
      if (!FEW) {
        float* sums = s_sum + (unit & 1) * 512;
        sums[group * 128 + key] = total;
        asm volatile("bar.sync 1, 512;" ::: "memory");
        if (mine) total = (sums[key] + sums[128 + key]) + (sums[256 + key] + sums[384 + key]);
      }
      if (place) *place = a.decay * old + total;
    }
    tc_fence_before();
  } else if (warp == kEW) {
    // =========================== MMA issuer ===================================
    const uint64_t dk0 = make_desc(sK), dq0 = make_desc(sQ);
    uint32_t kb = 0, kph = 0, qb = 0, qph = 0, cnt = 0;
    while (walk.next(f, prefix, seqs)) {
      mbar_wait(b_kfull + 8 * kb, kph, wc);
      for (int j = 0; j < walk.tiles; ++j, ++cnt) {
        const uint32_t buf = cnt & 3;
        const int cols = min(f.tpt, walk.n_new - (walk.tile0 + j) * f.tpt) * G;
        mbar_wait(b_qfull + 8 * qb, qph, wc);
        if (cnt >= 4) mbar_wait(b_sfree + 8 * buf, ((cnt >> 2) - 1) & 1, wc);
        __syncwarp();
        tc_fence_after();
        if (elect_one()) {
          const uint32_t idesc = make_idesc((cols + 15) & ~15, BF16, false);
          const uint64_t dk = dk0 + (uint64_t)(kb * (kTile >> 4)), dq = dq0 + (uint64_t)(qb * (kTile >> 4));
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint64_t at = (uint64_t)((ks >> 2) * (16384 >> 4) + (ks & 3) * 2);
            mma_ss(tmem + 128 * buf, dk + at, dq + at, idesc, ks > 0 ? 1u : 0u);
          }
          tc_commit(b_sfull + 8 * buf);
          tc_commit(b_qfree + 8 * qb);
          if (j == walk.tiles - 1) tc_commit(b_kfree + 8 * kb);
        }
        __syncwarp();
        if (++qb == (uint32_t)kNQ) { qb = 0; qph ^= 1; }
      }
      if (++kb == (uint32_t)kNK) { kb = 0; kph ^= 1; }
    }
    tc_fence_before();
  } else if (warp == kEW + 1) {
    // =========================== copies =======================================
    const int page_mask = (1 << a.cache.page_shift) - 1;
    const int per_unit = kUnit / f.box_rows;
    uint32_t g = 0, gq = 0;
    auto pages = [&](const UnitWalk& w) {                 // of a unit's copies, one per lane; none: outside the map
      const int slot = w.first + lane * f.box_rows;
      const int p = lane < per_unit && slot < w.len ? page_at(a.cache, a.seqs.table, a.seqs.table_width, w.seq, slot) : -1;
      return p < 0 ? a.cache.n_pages : p;
    };
    UnitWalk ahead = walk;
    bool more = ahead.next(f, prefix, seqs);
    int ids = more ? pages(ahead) : 0;
    while (more) {
      const UnitWalk w = ahead;
      const int now = ids;
      more = ahead.next(f, prefix, seqs);
      if (more) ids = pages(ahead);                       // (the next unit's look-ups run beside this one's copies)
      const uint32_t ks = g % kNK;
      const int boxes = min(per_unit, (w.len - w.first + f.box_rows - 1) / f.box_rows);
      mbar_wait<500>(b_kfree + 8 * ks, ((g / kNK) & 1) ^ 1, wc);
      __syncwarp();
      if (lane == 0) mbar_expect_tx(b_kfull + 8 * ks, (uint32_t)(boxes * f.box_rows * 128 * kSlabs));
      for (int i = 0; i < boxes; ++i) {
        const int page = __shfl_sync(0xffffffffu, now, i);
        if (lane == 0)
#pragma unroll
          for (int c = 0; c < kSlabs; ++c)
            tma_4d(sK + ks * kTile + c * 16384 + i * f.box_rows * 128, &maps.k, 64 * c, (w.first + i * f.box_rows) & page_mask, w.head, page, b_kfull + 8 * ks);
      }
      ++g;
      for (int j = 0; j < w.tiles; ++j, ++gq) {
        const uint32_t qs = gq % kNQ;
        mbar_wait<200>(b_qfree + 8 * qs, ((gq / kNQ) & 1) ^ 1, wc);
        __syncwarp();
        if (lane == 0) {
          mbar_expect_tx(b_qfull + 8 * qs, (uint32_t)(kSlabs * 128 * f.tpt * G));
#pragma unroll
          for (int c = 0; c < kSlabs; ++c)
            tma_3d(sQ + qs * kTile + c * 16384, &q_map, 64 * c, w.head * G, w.row0 + (w.tile0 + j) * f.tpt, b_qfull + 8 * qs);
        }
        __syncwarp();
      }
    }
    if (lane == 0) {
      auto drain = [&](uint32_t full, uint32_t stages, uint32_t issued) {
        for (uint32_t i = 0; i < stages && i < issued; ++i) {
          const uint32_t gi = issued - 1 - i;
          for (uint32_t it = 0; it < kSpinLimit; ++it)
            if (mbar_try(full + 8 * (gi % stages), (gi / stages) & 1)) break;
        }
      };
      drain(b_kfull, kNK, g);
      drain(b_qfull, kNQ, gq);
    }
    __syncwarp();
  } else if (warp == kEW + 2) {
    // =========================== -lse of a tile's columns =====================
    uint32_t cnt = 0;
    while (walk.next(f, prefix, seqs)) {
      for (int j = 0; j < walk.tiles; ++j, ++cnt) {
        const uint32_t buf = cnt & 3;
        const int tok0 = (walk.tile0 + j) * f.tpt;
        const int cols = min(f.tpt, walk.n_new - tok0) * G;
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = lane + 32 * i;
          x[i] = -INFINITY;
          if (c < cols) {
            const int tok = c / G;
            const float v = a.lse[(int64_t)(walk.head * G + (c - tok * G)) * a.seqs.n_tokens + walk.row0 + tok0 + tok];
            x[i] = v == -INFINITY ? v : -v * 1.4426950408889634f;        // (a row that saw nothing gives nothing)
          }
        }
        if (cnt >= 4) mbar_wait<100>(b_sfree + 8 * buf, ((cnt >> 2) - 1) & 1, wc);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) s_lse[128 * buf + lane + 32 * i] = x[i];
        mbar_arrive(b_lfull + 8 * buf);
      }
    }
  }
  __syncthreads();
  if (tid == 0 && *abort_flag) atomicExch(a.cache.status, (int)XKV_E_TIMEOUT);
  if (warp == kEW) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

template <int D, bool BF16>
cudaError_t setup_one() {
  const cudaError_t e = cudaFuncSetAttribute(weights_kernel<D, BF16, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Weigh<D>::kBytes);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(weights_kernel<D, BF16, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Weigh<D>::kBytes);
}

template <int D, bool BF16>
const void* kernel_of(bool few) {
  return few ? (const void*)weights_kernel<D, BF16, true> : (const void*)weights_kernel<D, BF16, false>;
}

}  // namespace

cudaError_t weights_setup() {
  cudaError_t e = setup_one<64, true>();
  if (e == cudaSuccess) e = setup_one<64, false>();
  if (e == cudaSuccess) e = setup_one<128, true>();
  if (e == cudaSuccess) e = setup_one<128, false>();
  return e;
}

cudaError_t launch_paged_weights(const PagedWeightArgs& a, const PoolMaps& maps, int head_dim, int dtype, int sm_count, cudaStream_t st) {
  WeighArgs f;
  f.a = a;
  f.tpt = 128 / a.cache.group;
  f.box_rows = min(1 << a.cache.page_shift, 128);
  CUtensorMap q_map;
  cudaError_t e = make_token_map(a.q, a.q_ts, a.q_hs, a.seqs.n_tokens, a.cache.n_heads, head_dim, dtype, a.cache.group, f.tpt, &q_map);
  if (e != cudaSuccess) return e;
  const bool few = (int64_t)a.seqs.max_new * a.cache.group <= 32, bf16 = dtype == XKV_BF16;
  const int64_t most = (int64_t)a.seqs.n_seqs * a.cache.n_kv_heads * ((((int64_t)a.seqs.table_width << a.cache.page_shift) + kUnit - 1) / kUnit);
  const unsigned grid = (unsigned)(most < sm_count ? most : sm_count);
  const void* fn;
  if (head_dim == 64) fn = bf16 ? kernel_of<64, true>(few) : kernel_of<64, false>(few);
  else fn = bf16 ? kernel_of<128, true>(few) : kernel_of<128, false>(few);
  void* p[3] = {(void*)&f, (void*)&maps, (void*)&q_map};
  e = launch_overlapped(fn, dim3(grid), dim3(kThreads), p, head_dim == 64 ? Weigh<64>::kBytes : Weigh<128>::kBytes, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace xkv
