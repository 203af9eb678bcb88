// Softmax weights that every cached token got from the new tokens: sum over rows of exp(q.k scale - lse), with the lse of the
// attention, so that no row needs a maximum or a second pass.
//
// The scores are computed transposed, S^T = K Q^T: tcgen05.mma with the 128 tokens of a unit as its rows, in tensor memory one
// token per lane, and the query rows (128 / G tokens of G heads, as in the chunk attention) as its columns.  A thread
// then owns a token and adds its weights up in registers; nothing is exchanged between lanes, and the sums have a fixed order.
// K is read once, stays in shared memory for all query tiles; the query tiles come from the L2 again for every unit.
//
// An item is two units (256 tokens) of a head.  Each query tile that is fetched meets both: with one unit the tiles came from
// the L2 at 7.4 TB/s, and nothing else mattered (a frame over 16384 tokens 102 us, 65 without the exponentials).
//
// One block, 20 warps: 16 exponential warps in four groups (a group is four warps, one per quarter of the lanes), one MMA issuer,
// one for copies, two that stage -lse per column.  A group has a unit of the item and every second tile, with a buffer of
// scores of its own (2 units x 2 parities x 128 columns are all of tensor memory); at the item's end the two parities meet in shared
// memory.  (Half of the columns of every tile instead: 113 us for the frame; what a warp does per tile besides its exponentials counts.)
//
// What bounds it: with many rows the exponentials (16 per clock and multiprocessor; a quarter of them are polynomials on the FMA
// pipes; the MMAs need a quarter to a half of that time), with few rows reading K.  Measured: a frame of 1374 queries over 16384
// tokens, 16 heads of 64, 96 us (107 without the polynomials; the exponentials alone 80 on the special-function unit); 16 single
// tokens over 38 880, 8 key heads of 128, 22.8 us.
#include "xkv_paged_line.cuh"
#include "xkv_ptx.cuh"

namespace xkv {

namespace {

constexpr int kThreads = 640;
constexpr int kEW = 16;                       // exponential warps; 16: MMA, 17: copies, 18, 19: lse
constexpr uint32_t kSpinLimit = 1u << 22;
constexpr int kLse = 4;                       // staged tiles of -lse
// Places where the parities of an item meet.  The group that adds them up does so before it leaves the item's last tile L, whose -lse is
// replaced only then.  So its neighbour of the same parity stays before L + 4, the MMAs, which come in order, before L + 6, the
// groups of the other parity that have scores to read before L + 7, and those that have none (causal) before L + 11, by their own
// -lse.  Items that meet have two tiles at least: the eighth of them after this one begins at L + 15.
constexpr int kSums = 8;

template <int D> struct Weigh {
  static constexpr int kSlabs = D / 64;
  static constexpr int kTile = kSlabs * 16384;               // 128 rows
  static constexpr int kNK = D == 64 ? 3 : 2, kNQ = D == 64 ? 4 : 2;
  static constexpr int kOffQ = kNK * 2 * kTile, kOffBar = kOffQ + kNQ * kTile;
  static constexpr int kOffLse = kOffBar + 512, kOffSum = kOffLse + kLse * 512, kOffSeq = kOffSum + kSums * 2 * 512;
  static constexpr int kOffPrefix = kOffSeq + kMaxSeqs * 12;
  static constexpr size_t kBytes = kOffPrefix + (kMaxSeqs + 1) * 4 + 1024;
};

struct WeighArgs {
  PagedWeightArgs a;
  int tpt, box_rows;
  int q_toks;              // tokens of a copy of queries: those of a tile, or fewer if no sequence has that many new ones
};

// Items of the block: every gridDim.x-th of the line.
struct ItemWalk {
  uint32_t pos, total, step;
  uint32_t rel, per, seq_end;            // item of the head, items of a head, where the sequence ends on the line
  int seq, head, first;                  // first token of the item
  int row0, n_new, len, all_tiles;
  int tile0, tiles;                      // query tiles that see a token of the item
  int skip;                              // of them those that see none of its second unit
  __device__ __forceinline__ bool next(const WeighArgs& f, const uint32_t* prefix, const Seq* seqs) {
    if (pos >= total) return false;
    if (pos >= seq_end) {
      seq = line_seq(prefix, f.a.seqs.n_seqs, pos);
      const Seq q = seqs[seq];
      row0 = q.row0; n_new = q.n_new; len = q.len;
      seq_end = prefix[seq + 1];
      per = (uint32_t)((q.len + 2 * kUnit - 1) / (2 * kUnit));
      rel = pos - prefix[seq];
      head = (int)(rel / per);
      rel -= (uint32_t)head * per;
      all_tiles = (n_new + f.tpt - 1) / f.tpt;
    } else {                             // (without a division per item and warp)
      rel += step;
      if (rel >= 4 * per) { const uint32_t h = rel / per; head += (int)h; rel -= h * per; }
      while (rel >= per) { rel -= per; ++head; }
    }
    first = (int)rel * 2 * kUnit;
    tile0 = first_tile(f, first);
    tiles = all_tiles - tile0;
    skip = first + kUnit < len ? first_tile(f, first + kUnit) - tile0 : tiles;
    pos += step;
    return true;
  }
  // new token i sees slot j iff i >= j - (len - n_new)
  __device__ __forceinline__ int first_tile(const WeighArgs& f, int slot) const {
    return f.a.full || slot <= len - n_new ? 0 : (slot - (len - n_new)) / f.tpt;
  }
};

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

template <int D, bool BF16>
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
  const uint32_t b_sfull = b_qfree + 8 * kNQ, b_sfree = b_sfull + 32;       // [4]: unit + 2 * parity of the tile
  const uint32_t b_lfull = b_sfree + 32, b_lfree = b_lfull + 8 * kLse, b_sums = b_lfree + 8 * kLse;      // [kLse], [kLse], [kSums][2 units]
  static_assert(8 * (2 * kNK + 2 * kNQ + 8 + 2 * kLse + 2 * kSums) <= 512 - 16, "barriers");
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sgen + C::kOffBar + 496);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sgen + C::kOffBar + 500);
  const WaitCtx wc{sbase + C::kOffBar + 500};
  float* s_lse = reinterpret_cast<float*>(sgen + C::kOffLse);        // [kLse][128] -lse in log2 units
  float* s_sum = reinterpret_cast<float*>(sgen + C::kOffSum);        // [kSums][2][128]
  Seq* seqs = reinterpret_cast<Seq*>(sgen + C::kOffSeq);
  uint32_t* prefix = reinterpret_cast<uint32_t*>(sgen + C::kOffPrefix);
  __shared__ uint2 s_warp[kThreads / 32];

  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) {
    *abort_flag = 0;
    for (int i = 0; i < kNK; ++i) { mbar_init(b_kfull + 8 * i, 1); mbar_init(b_kfree + 8 * i, 1); }
    for (int i = 0; i < kNQ; ++i) { mbar_init(b_qfull + 8 * i, 1); mbar_init(b_qfree + 8 * i, 1); }
    for (int i = 0; i < 4; ++i) { mbar_init(b_sfull + 8 * i, 1); mbar_init(b_sfree + 8 * i, 4); }
    for (int i = 0; i < kLse; ++i) { mbar_init(b_lfull + 8 * i, 32); mbar_init(b_lfree + 8 * i, 8); }
    for (int i = 0; i < 2 * kSums; ++i) mbar_init(b_sums + 8 * i, 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kEW) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_dependency_wait();
  line_prefix<kThreads, false>(a.seqs.n_seqs, prefix, s_warp, [&](int s) {       // (items alone count here: none is cut)
    const Seq q = seq_at(a.cache, a.seqs, s);
    seqs[s] = q;
    return Work{0u, q.n_new == 0 ? 0u : (uint32_t)a.cache.n_kv_heads * (uint32_t)((q.len + 2 * kUnit - 1) / (2 * kUnit))};
  });
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
  ItemWalk walk;
  walk.pos = blockIdx.x;
  walk.step = gridDim.x;
  walk.total = prefix[a.seqs.n_seqs];
  walk.seq_end = 0;
  const int G = a.cache.group;

  if (warp < kEW) {
    // ============== exponentials: thread = token of a unit ==============
    const uint32_t u = warp >> 3;                          // unit of the item
    const uint32_t odd = (warp >> 2) & 1;                  // parity of the tiles
    const int key = (warp & 3) * 32 + lane;
    const uint32_t buf = u + 2 * odd, scores = tmem + ((uint32_t)((warp & 3) * 32) << 16) + 128 * buf;
    const uint64_t sc2 = pack_f2(a.scale_log2, a.scale_log2);
    uint32_t cnt = 0, ph = 0;                // tiles of the block so far; phase of this group's buffer
    const bool adds = a.decay == 1.f, fades = a.decay != 0.f && !adds;
    uint32_t sum_at = 0, sum_ph = 0;         // place where the next item's parities meet, and its phase
    for (; walk.next(f, prefix, seqs); cnt += (uint32_t)walk.tiles) {
      const int token = walk.first + kUnit * (int)u + key;
      const int from = u ? walk.skip : 0;                    // the unit's first tile
      const bool writes = ((cnt + (uint32_t)walk.tiles - 1) & 1) == odd;       // the item's last tile is this group's
      // the old weight and its place, asked for here and looked at after the group's first tile
      const bool in = writes && token < walk.len;
      int page = -1;
      if (in) page = a.seqs.table[(int64_t)walk.seq * a.seqs.table_width + (token >> a.cache.page_shift)];
      float* place = nullptr;
      float old = 0.f, total = 0.f;
      const int base = walk.len - walk.n_new;                // token i sees slots <= base + i
      const int j0 = (int)((odd - cnt) & 1);
      for (int j = j0; j < walk.tiles; j += 2) {
        const uint32_t at = (cnt + (uint32_t)j) % kLse;
        const int tok0 = (walk.tile0 + j) * f.tpt;
        const int cols = min(f.tpt, walk.n_new - tok0) * G;
        mbar_wait(b_lfull + 8 * at, ((cnt + (uint32_t)j) / kLse) & 1, wc);
        if (j >= from) {
          mbar_wait(b_sfull + 8 * buf, ph, wc);
          ph ^= 1;
          __syncwarp();
          tc_fence_after();
          // columns [lo, cols) see the token: tokens i >= token - base; columns behind the tile's rows belong to nobody
          const bool all = a.full || walk.first + kUnit * (int)u + kUnit - 1 <= base + tok0;      // (the same in all threads)
          const int lo = all ? 0 : (token - base - tok0) * G;      // (of a unit far behind the new tokens the product could pass 32 bits)
          uint64_t sum = 0ull, sum1 = 0ull;
#pragma unroll 1
          for (int c0 = 0; c0 < cols; c0 += 32) {
            uint32_t s[32];
            XKV_TMEM_LD_32(scores + c0, s);
            tc_wait_ld();
            const float4* nl = reinterpret_cast<const float4*>(s_lse + 128 * at + c0);
            if (all && c0 + 32 <= cols) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float4 n = nl[i];
                const uint64_t x0 = fma_f2(pack_f2(__uint_as_float(s[4 * i]), __uint_as_float(s[4 * i + 1])), sc2, pack_f2(n.x, n.y));
                const uint64_t x1 = fma_f2(pack_f2(__uint_as_float(s[4 * i + 2]), __uint_as_float(s[4 * i + 3])), sc2, pack_f2(n.z, n.w));
                sum = add_f2(sum, pack_f2(fast_exp2(f2_lo(x0)), fast_exp2(f2_hi(x0))));
                sum1 = add_f2(sum1, (i & 1) ? exp2_pair<5>(x1) : pack_f2(fast_exp2(f2_lo(x1)), fast_exp2(f2_hi(x1))));
              }
            } else {
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float2 n = *reinterpret_cast<const float2*>(reinterpret_cast<const float*>(nl) + i);
                const float p0 = fast_exp2(fmaf(__uint_as_float(s[i]), a.scale_log2, n.x)), p1 = fast_exp2(fmaf(__uint_as_float(s[i + 1]), a.scale_log2, n.y));
                sum = add_f2(sum, pack_f2(c0 + i >= lo && c0 + i < cols ? p0 : 0.f, c0 + i + 1 >= lo && c0 + i + 1 < cols ? p1 : 0.f));
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(b_sfree + 8 * buf);
          total += (f2_lo(sum) + f2_hi(sum)) + (f2_lo(sum1) + f2_hi(sum1));
        }
        if (in && !place) {
          if ((unsigned)page < (unsigned)a.cache.n_pages) {
            place = a.cache.weights + weight_offset(a.cache, page, walk.head, token);
            if (fades) old = *place;
          } else {
            paged_report(a.cache.status, (int)XKV_E_INVALID);
          }
        }
        if (j == walk.tiles - 1) {
          if (walk.tiles > 1) {
            mbar_wait(b_sums + 8 * (2 * sum_at + u), sum_ph, wc);
            __syncwarp();
            total += s_sum[(2 * sum_at + u) * 128 + key];
          }
          if (place) {
            // (added where nothing fades, so that sequences that share the slot lose no update)
            if (adds) atomicAdd(place, total); else *place = a.decay * old + total;
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(b_lfree + 8 * at);
      }
      if (walk.tiles > 1) {
        if (!writes) {
          s_sum[(2 * sum_at + u) * 128 + key] = total;
          __syncwarp();
          if (lane == 0) mbar_arrive(b_sums + 8 * (2 * sum_at + u));
        }
        if (++sum_at == kSums) { sum_at = 0; sum_ph ^= 1; }
      }
    }
    tc_fence_before();
  } else if (warp == kEW) {
    // =========================== MMA issuer ===================================
    const uint64_t dk0 = make_desc(sK), dq0 = make_desc(sQ);
    uint32_t kb = 0, kph = 0, qb = 0, qph = 0, cnt = 0;
    uint32_t par = 0, used = 0;              // of the four buffers: phases, and whether they have held scores
    while (walk.next(f, prefix, seqs)) {
      mbar_wait(b_kfull + 8 * kb, kph, wc);
      for (int j = 0; j < walk.tiles; ++j, ++cnt) {
        const int cols = min(f.tpt, walk.n_new - (walk.tile0 + j) * f.tpt) * G;
        const uint32_t idesc = make_idesc((cols + 15) & ~15, BF16, false);
        const uint64_t dq = dq0 + (uint64_t)(qb * (kTile >> 4));
        mbar_wait(b_qfull + 8 * qb, qph, wc);
#pragma unroll
        for (uint32_t u = 0; u < 2; ++u) {
          if (u && j < walk.skip) break;
          const uint32_t buf = u + 2 * (cnt & 1);
          if ((used >> buf) & 1) mbar_wait(b_sfree + 8 * buf, ((par >> buf) & 1) ^ 1, wc);
          used |= 1u << buf;
          par ^= 1u << buf;
          __syncwarp();
          tc_fence_after();
          if (elect_one()) {
            const uint64_t dk = dk0 + (uint64_t)((2 * kb + u) * (kTile >> 4));
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const uint64_t at = (uint64_t)((ks >> 2) * (16384 >> 4) + (ks & 3) * 2);
              mma_ss(tmem + 128 * buf, dk + at, dq + at, idesc, ks > 0 ? 1u : 0u);
            }
            tc_commit(b_sfull + 8 * buf);
          }
          __syncwarp();
        }
        if (elect_one()) {
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
    const int per_item = 2 * kUnit / f.box_rows;          // copies, 2..16
    uint32_t g = 0, gq = 0;
    auto pages = [&](const ItemWalk& w) {                 // of an item's copies, one per lane; none: outside the map
      const int slot = w.first + lane * f.box_rows;
      const int p = lane < per_item && slot < w.len ? page_at(a.cache, a.seqs.table, a.seqs.table_width, w.seq, slot) : -1;
      return p < 0 ? a.cache.n_pages : p;
    };
    ItemWalk ahead = walk;
    bool more = ahead.next(f, prefix, seqs);
    int ids = more ? pages(ahead) : 0;
    while (more) {
      const ItemWalk w = ahead;
      const int now = ids;
      more = ahead.next(f, prefix, seqs);
      if (more) ids = pages(ahead);                       // (the next item's look-ups run beside this one's copies)
      const uint32_t ks = g % kNK;
      const int boxes = min(per_item, (w.len - w.first + f.box_rows - 1) / f.box_rows);
      mbar_wait<500>(b_kfree + 8 * ks, ((g / kNK) & 1) ^ 1, wc);
      __syncwarp();
      if (lane == 0) mbar_expect_tx(b_kfull + 8 * ks, (uint32_t)(boxes * f.box_rows * 128 * kSlabs));
      {
        const int i = lane / kSlabs, c = lane % kSlabs;         // (a copy per lane)
        const int page = __shfl_sync(0xffffffffu, now, i);
        if (i < boxes)
          tma_4d(sK + (2 * ks + (i * f.box_rows) / kUnit) * kTile + c * 16384 + ((i * f.box_rows) & (kUnit - 1)) * 128, &maps.k, 64 * c,
                 (w.first + i * f.box_rows) & page_mask, w.head, page, b_kfull + 8 * ks);
      }
      ++g;
      for (int j = 0; j < w.tiles; ++j, ++gq) {
        const uint32_t qs = gq % kNQ;
        mbar_wait(b_qfree + 8 * qs, ((gq / kNQ) & 1) ^ 1, wc);
        __syncwarp();
        if (lane == 0) {
          mbar_expect_tx(b_qfull + 8 * qs, (uint32_t)(kSlabs * 128 * f.q_toks * G));
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
  } else {
    // =========================== -lse of a tile's columns =====================
    // Two warps take turns; each asks for the values of its next tile before it hands over those of this one, so that their way
    // from memory is never waited for (one warp, one tile at a time: 246 us for a frame over 16384 tokens instead of 109).
    int64_t off[4];                         // of this lane's columns: place after the tile's first value
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = lane + 32 * i, tok = c / G;
      off[i] = (int64_t)(c - tok * G) * a.seqs.n_tokens + tok;
    }
    int j = -1;
    bool live = walk.next(f, prefix, seqs);
    uint32_t cnt = 0xffffffffu;             // the tile at hand
    auto advance = [&]() {                  // to the next tile of the block
      if (!live) return;
      ++cnt;
      if (++j == walk.tiles) { j = 0; live = walk.next(f, prefix, seqs); }
    };
    auto fetch = [&](float (&x)[4]) {
      const int tok0 = (walk.tile0 + j) * f.tpt;
      const int cols = min(f.tpt, walk.n_new - tok0) * G;
      const float* src = a.lse + (int64_t)walk.head * G * a.seqs.n_tokens + walk.row0 + tok0;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = lane + 32 * i < cols ? src[off[i]] : -INFINITY;
    };
    auto put = [&](uint32_t now, const float (&x)[4]) {
      const uint32_t at = now % kLse;
      if (now >= (uint32_t)kLse) mbar_wait(b_lfree + 8 * at, ((now / kLse) - 1) & 1, wc);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i)           // (a row that saw nothing, lse -inf, gives nothing)
        s_lse[128 * at + lane + 32 * i] = x[i] == -INFINITY ? x[i] : -x[i] * 1.4426950408889634f;
      mbar_arrive(b_lfull + 8 * at);
    };
    float x[4], y[4];
    for (int i = 0; i <= warp - (kEW + 2); ++i) advance();
    if (live) fetch(x);
    while (live) {
      uint32_t now = cnt;
      advance();
      advance();
      if (live) fetch(y);
      put(now, x);
      if (!live) break;
      now = cnt;
      advance();
      advance();
      if (live) fetch(x);
      put(now, y);
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
  return cudaFuncSetAttribute(weights_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Weigh<D>::kBytes);
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
  f.q_toks = min(f.tpt, a.seqs.max_new);
  CUtensorMap q_map;
  cudaError_t e = make_token_map(a.q, a.q_ts, a.q_hs, a.seqs.n_tokens, a.cache.n_heads, head_dim, dtype, a.cache.group, f.q_toks, &q_map);
  if (e != cudaSuccess) return e;
  const bool bf16 = dtype == XKV_BF16;
  const int64_t most = (int64_t)a.seqs.n_seqs * a.cache.n_kv_heads * ((((int64_t)a.seqs.table_width << a.cache.page_shift) + 2 * kUnit - 1) / (2 * kUnit));
  const unsigned grid = (unsigned)(most < sm_count ? most : sm_count);
  const void* fn;
  if (head_dim == 64) fn = bf16 ? (const void*)weights_kernel<64, true> : (const void*)weights_kernel<64, false>;
  else fn = bf16 ? (const void*)weights_kernel<128, true> : (const void*)weights_kernel<128, false>;
  void* p[3] = {(void*)&f, (void*)&maps, (void*)&q_map};
  e = launch_overlapped(fn, dim3(grid), dim3(kThreads), p, head_dim == 64 ? Weigh<64>::kBytes : Weigh<128>::kBytes, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace xkv
