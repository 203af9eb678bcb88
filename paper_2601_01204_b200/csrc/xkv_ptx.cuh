// PTX wrappers shared by the tensor-core kernels: mbarriers with bounded waits, tensor memory, tcgen05.mma and its
// descriptors, packed arithmetic.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace xkv {
namespace {

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
constexpr uint32_t kSuspendNs = 2000;
// The same with a time the hardware may keep the thread suspended before it answers "not yet"
// (it answers at once when the phase completes).
__device__ __forceinline__ bool mbar_try_suspend(uint32_t bar, uint32_t parity, uint32_t ns) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity), "r"(ns) : "memory");
  return ok != 0;
}
// Up to 64 suspended tries in a loop of three instructions (try, branch out, count and branch back).
__device__ __forceinline__ bool mbar_try_many(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .pred q;\n\t.reg .u32 n;\n\t"
      "mov.u32 n, 64;\n\t"
      "XKV_TRY_%=:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "@p bra XKV_DONE_%=;\n\t"
      "sub.u32 n, n, 1;\n\t"
      "setp.ne.u32 q, n, 0;\n\t"
      "@q bra XKV_TRY_%=;\n\t"
      "XKV_DONE_%=:\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity), "r"(kSuspendNs) : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint64_t global_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
// Bounded wait.  On exhaustion a per-CTA flag goes up, and every later wait of the CTA gives up at
// once; at its end the CTA records the failure in the status words of the caches that it worked on.
struct WaitCtx { uint32_t abort_flag; };      // address in shared memory
__device__ __forceinline__ uint32_t ld_shared_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared_u32(uint32_t addr, uint32_t v) {
  asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// Threads on the critical chain (softmax warps, MMA issuers: SLEEP_NS below 128) retry at once, each
// try suspended by the hardware for a short while: their wake-up latency is part of every step.
// Threads that wait long and have slack (operand producers, the copy thread) sleep SLEEP_NS between
// tries, so that their polls (shared-memory instructions) do not take issue slots and queue space
// from the softmax warps.  The wait gives up after one second AND kWaitMinRounds rounds of tries
// (32 or 64 each): the rounds only count while the thread runs, so that a kernel that was
// descheduled for a while (a GPU shared between processes) does not time out on the clock alone.
constexpr uint64_t kWaitLimitNs = 1000000000ull;      // one second ...
constexpr uint32_t kWaitMinRounds = 1u << 12;         // ... and this many rounds, then XKV_E_TIMEOUT
constexpr int kSlack = 1000;     // sleep of the producers and the copy thread (256: 16-bit at 32768 tokens 6440 instead of 6290 us)
template <int SLEEP_NS = 32>
__device__ __forceinline__ void mbar_wait(uint32_t bar, uint32_t parity, const WaitCtx& wc) {
  if (mbar_try(bar, parity)) return;          // the common case costs one instruction
  if (ld_shared_u32(wc.abort_flag)) return;
  const uint64_t t0 = global_ns();
  uint32_t rounds = 0;
  do {
    if (SLEEP_NS >= 128) {
#pragma unroll 1
      for (int it = 0; it < 32; ++it) {
        if (mbar_try_suspend(bar, parity, kSuspendNs)) return;
        __nanosleep(SLEEP_NS);
      }
    } else if (mbar_try_many(bar, parity)) {
      return;
    }
  } while (++rounds < kWaitMinRounds || global_ns() - t0 < kWaitLimitNs);
  st_shared_u32(wc.abort_flag, 1u);
}
__device__ __forceinline__ float fast_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// packed fp32 pairs (two floats in one 64-bit register)
__device__ __forceinline__ uint64_t pack_f2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float f2_lo(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float f2_hi(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ uint64_t fma_f2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add_f2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul_f2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {         // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// 2^x of two numbers on the FMA pipes, for a share of the exponentials where the special-function unit is what bounds a kernel: x = n + r
// with n the nearest whole number, a polynomial in r whose relative error on [-1/2, 1/2] is minimax (coefficients by the
// Remez exchange), times 2^n.  Relative error 2.1e-7 (degree 5), 2.7e-6 (4), 7.5e-5 (3) in fp32.
// Outside its range it answers as fast_exp2 does, so that it makes no difference which of them a number meets: a NaN stays one,
// results below 2^-126 are 0 (n is -127 at least, whose scale is 0), from 127.5 on they are infinite (n counts as 128 at most; that is
// done on its bits, one instruction with the sum: on x it costs the weights of a frame 2 %).  +infinity itself gives a NaN.
template <int DEGREE>
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
  constexpr float kMagic = 12582912.f;       // 1.5 * 2^23: adding it rounds to a whole number, in the low bits of the sum
  constexpr float c[3][6] = {{0.9999280571937561f, 0.6932609677314758f, 0.2426111251115799f, 0.0551716685295105f, 0.f, 0.f},
                             {0.9999992847442627f, 0.6931217908859253f, 0.240247443318367f, 0.05591785907745361f, 0.009570102207362652f, 0.f},
                             {1.0000001192092896f, 0.6931469440460205f, 0.24022120237350464f, 0.05550713092088699f, 0.009675540961325169f,
                              0.0013276472454890609f}};
  x = pack_f2(max_nan(f2_lo(x), -127.f), max_nan(f2_hi(x), -127.f));
  const uint64_t t = add_f2(x, pack_f2(kMagic, kMagic));
  const uint64_t n = add_f2(t, pack_f2(-kMagic, -kMagic));
  const uint64_t r = fma_f2(n, pack_f2(-1.f, -1.f), x);
  uint64_t p = pack_f2(c[DEGREE - 3][DEGREE], c[DEGREE - 3][DEGREE]);
#pragma unroll
  for (int i = DEGREE - 1; i >= 0; --i) p = fma_f2(p, r, pack_f2(c[DEGREE - 3][i], c[DEGREE - 3][i]));
  auto scale = [](uint32_t bits) { return __uint_as_float((uint32_t)__viaddmin_s32((int)bits, 127 - 0x4B400000, 255) << 23); };
  uint64_t y;
  asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(y) : "l"(p), "l"(pack_f2(scale((uint32_t)t), scale((uint32_t)(t >> 32)))));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// One lane of a converged warp.  The issuing warps run converged and let one elected lane issue, so
// that descriptors and addresses stay warp-uniform and live in uniform registers: inside a branch
// that only one lane takes, every tcgen05.mma is preceded by moves of its operands into them.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// D[tmem] (+)= A[smem] * B[smem]
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}

// Tensor memory <-> registers, 16 lanes (rows) of the calling warp's quarter.  Of every 8 columns lane l holds, as in
// the accumulators of a warp-level MMA, columns 2 (l mod 4) and the next of row l / 4 (registers 4g, 4g + 1) and of row
// l / 4 + 8 (4g + 2, 4g + 3).  A pair of neighbours makes one 32-bit word of 16-bit P, and of every 4 words lane l
// holds word l mod 4 of the same two rows (2g, 2g + 1).  LD_64, ST_64: 64 columns; ST_P32: 32 words.
#define XKV_TMEM_LD_64(taddr, r, o)                                                                 \
  asm volatile(                                                                                     \
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 {"                                                    \
      "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"                                      \
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"                    \
      : "=r"(r[(o) + 0]), "=r"(r[(o) + 1]), "=r"(r[(o) + 2]), "=r"(r[(o) + 3]),                     \
        "=r"(r[(o) + 4]), "=r"(r[(o) + 5]), "=r"(r[(o) + 6]), "=r"(r[(o) + 7]),                     \
        "=r"(r[(o) + 8]), "=r"(r[(o) + 9]), "=r"(r[(o) + 10]), "=r"(r[(o) + 11]),                   \
        "=r"(r[(o) + 12]), "=r"(r[(o) + 13]), "=r"(r[(o) + 14]), "=r"(r[(o) + 15]),                 \
        "=r"(r[(o) + 16]), "=r"(r[(o) + 17]), "=r"(r[(o) + 18]), "=r"(r[(o) + 19]),                 \
        "=r"(r[(o) + 20]), "=r"(r[(o) + 21]), "=r"(r[(o) + 22]), "=r"(r[(o) + 23]),                 \
        "=r"(r[(o) + 24]), "=r"(r[(o) + 25]), "=r"(r[(o) + 26]), "=r"(r[(o) + 27]),                 \
        "=r"(r[(o) + 28]), "=r"(r[(o) + 29]), "=r"(r[(o) + 30]), "=r"(r[(o) + 31])                  \
      : "r"(taddr) : "memory")

#define XKV_TMEM_ST_64(taddr, r)                                                                    \
  asm volatile(                                                                                     \
      "tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], {"                                              \
      "%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"                                     \
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"                           \
      ::"r"(taddr),                                                                                 \
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),                                                 \
        "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),                                                 \
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),                                               \
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),                                             \
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),                                             \
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),                                             \
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),                                             \
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory")

#define XKV_TMEM_ST_P32(taddr, r)                                                                   \
  asm volatile(                                                                                     \
      "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {"                                              \
      "%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"                                    \
      ::"r"(taddr),                                                                                 \
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),                                                 \
        "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),                                                 \
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),                                               \
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory")

// Shared-memory matrix descriptor, 128-byte swizzle, 8-row groups 1024 B apart.
__device__ __forceinline__ uint64_t make_desc(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr >> 4) & 0x3FFF);        // start address
  d |= (uint64_t)1 << 16;                        // leading byte offset (unused with one swizzle span)
  d |= (uint64_t)(1024 >> 4) << 32;              // stride byte offset between 8-row groups
  d |= (uint64_t)1 << 46;                        // descriptor version of this architecture
  d |= (uint64_t)2 << 61;                        // SWIZZLE_128B
  return d;
}

// Instruction descriptor for kind::f16: fp32 accumulate, M = 128.
__device__ __forceinline__ uint32_t make_idesc(int n_dim, bool bf16, bool b_mn_major) {
  uint32_t d = 0;
  d |= 1u << 4;                                  // D format fp32
  d |= (bf16 ? 1u : 0u) << 7;                    // A format
  d |= (bf16 ? 1u : 0u) << 10;                   // B format
  d |= (b_mn_major ? 1u : 0u) << 16;             // B major
  d |= (uint32_t)(n_dim >> 3) << 17;
  d |= (uint32_t)(128 >> 4) << 24;
  return d;
}

// Copies by tensor map: a box of a pool (64 channels from `c`, slots from `slot` of a head and page; a page outside the map reads as zero) and
// of a token tensor.
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* map, int c, int slot, int head, int page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(c), "r"(slot), "r"(head), "r"(page), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int c, int head, int tok, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(c), "r"(head), "r"(tok), "r"(bar) : "memory");
}

__device__ __forceinline__ uint32_t swz_off(int row, int chunk) {
  return (uint32_t)((row >> 3) * 1024 + (row & 7) * 128 + ((chunk ^ (row & 7)) << 4));
}

__device__ __forceinline__ uint32_t pack_h2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_bf2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace
}  // namespace xkv
