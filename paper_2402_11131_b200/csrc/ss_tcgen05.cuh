// What the kernels on tcgen05 share: barriers, waits with a bound, TMA, tcgen05 and TMEM instructions, descriptors.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include "ss_common.cuh"

namespace ss {

constexpr long long kWaitCycles = 2000000000ll;   // bound of every mbarrier wait (~1 s)

// PTX wrappers
__device__ __forceinline__ uint32_t smem_u32(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ float4 ld_shared_v4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait: gives up when another thread of the CTA already gave up, or after kWaitCycles.
static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort, int* status) {
    const long long t0 = clock64();
    for (;;) {
        for (int i = 0; i < 256; ++i) {
            if (mbar_try(bar, parity)) return true;
            if (*abort) return false;
        }
        if (clock64() - t0 > kWaitCycles) {
            *abort = 1;
            set_status(status, SS_ERR_DEVICE_TIMEOUT);
            return false;
        }
    }
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort, int* status) {
    if (mbar_try(bar, parity)) return true;
    return mbar_wait_slow(bar, parity, abort, status);
}
// the same for a whole warp: either every lane saw the phase complete or every lane gives up
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int* abort, int* status) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort, status));
}
// Waits whose bound is in the kernel's control block (abort; wait_limit, in units of 1024 cycles): the caller may shorten it
// through the workspace header.
__device__ __forceinline__ long long limit_cycles(const int& wait_limit) {
    return static_cast<long long>(*const_cast<const volatile int*>(&wait_limit)) << 10;
}
static __device__ __noinline__ bool mbar_wait_limit_slow(uint32_t bar, uint32_t parity, volatile int* abort, const int* wait_limit, int* status) {
    const long long t0 = clock64(), limit = limit_cycles(*wait_limit);
    for (;;) {
        for (int i = 0; i < 256; ++i) {
            if (mbar_try(bar, parity)) return true;
            if (*abort) return false;
        }
        if (clock64() - t0 > limit) {
            *abort = 1;
            set_status(status, SS_ERR_DEVICE_TIMEOUT);
            return false;
        }
    }
}
template <typename Control>
__device__ __forceinline__ bool mbar_wait_limit(uint32_t bar, uint32_t parity, Control* c, int* status) {
    if (mbar_try(bar, parity)) return true;
    return mbar_wait_limit_slow(bar, parity, &c->abort, &c->wait_limit, status);
}
template <typename Control>
__device__ __forceinline__ bool mbar_wait_limit_warp(uint32_t bar, uint32_t parity, Control* c, int* status) {
    return __all_sync(0xffffffffu, mbar_wait_limit(bar, parity, c, status));
}
// the whole warp, without a branch that its lanes could take differently
template <typename Control>
__device__ __forceinline__ bool mbar_wait_uniform(uint32_t bar, uint32_t parity, Control* c, int* status) {
    if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
    volatile int* const abort = &c->abort;
    const long long t0 = clock64();
    while (!__all_sync(0xffffffffu, mbar_try(bar, parity))) {
        const bool late = clock64() - t0 > limit_cycles(c->wait_limit);
        if (__any_sync(0xffffffffu, late || *abort != 0)) {
            if (late && *abort == 0) {
                *abort = 1;
                set_status(status, SS_ERR_DEVICE_TIMEOUT);
            }
            return false;
        }
    }
    return true;
}
// after giving up: a short bounded wait that lets a copy already in flight land
static __device__ __noinline__ void mbar_drain(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    while (!mbar_try(bar, parity) && clock64() - t0 < kWaitCycles / 16) {}
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
__device__ __forceinline__ void named_barrier(int id, int threads) {
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void st_shared_v2(uint32_t addr, uint32_t x, uint32_t y) {
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ float2 ld_shared_v2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void tma_prefetch_desc(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// lane 0's value, which the compiler knows to be the same in all lanes
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }
// D[tmem] (+)= A * B, bf16 inputs, fp32 accumulate, issued by one elected lane of a warp that comes here in step (a commit stands
// for the products of its own thread; the election is deterministic).  STEPS (1 or 4) steps of 16 elements of the contraction
// inside one 64-element box go in one block; a step is an addition to the low word of an operand's descriptor (or to its TMEM
// column).  The first one accumulates if `acc` is not zero.  With the warp's index and the loop bounds known to be uniform (see
// uniform()) the operands are kept in uniform registers; where a single thread issues in a branch of its own, or a lane's
// predicate comes from a register, every MMA takes an instruction chain that competes with the softmax warps for issue slots:
// 8 + 4 MMAs of a 64-key tile beside them then take some 1.1 k cycles instead of the 512 to 736 that they execute in.
#define SS_MMA_STEP(A, B, P) "@e tcgen05.mma.cta_group::1.kind::f16 [%0], " A ", " B ", %5, " P ";\n\t"
#define SS_MMA_NEXT(SA, SB) "add.u32 x, %1, " SA ";\n\tmov.b64 a, {x, %2};\n\tadd.u32 x, %3, " SB ";\n\tmov.b64 b, {x, %4};\n\t" SS_MMA_STEP("a", "b", "t")
#define SS_MMA_NEXT_TS(SA, SB) "add.u32 y, %1, " SA ";\n\tadd.u32 x, %2, " SB ";\n\tmov.b64 b, {x, %3};\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [y], b, %4, t;\n\t"
template <int STEPS>
__device__ __forceinline__ void tc_mma_steps(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    const uint32_t alo = static_cast<uint32_t>(a), ahi = static_cast<uint32_t>(a >> 32), blo = static_cast<uint32_t>(b), bhi = static_cast<uint32_t>(b >> 32);
    if constexpr (STEPS == 1)
        asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 a, b;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
                     SS_MMA_STEP("a", "b", "p") "}" ::"r"(d), "r"(alo), "r"(ahi), "r"(blo), "r"(bhi), "r"(idesc), "r"(acc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, e, t;\n\t.reg .b32 x;\n\t.reg .b64 a, b;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %6, 0;\n\tsetp.eq.u32 t, 0, 0;\n\t"
                     "mov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\t"
                     SS_MMA_STEP("a", "b", "p") SS_MMA_NEXT("2", "2") SS_MMA_NEXT("4", "4") SS_MMA_NEXT("6", "6") "}"
                     ::"r"(d), "r"(alo), "r"(ahi), "r"(blo), "r"(bhi), "r"(idesc), "r"(acc) : "memory");
    static_assert(STEPS == 1 || STEPS == 4, "of a box of 64 elements");
}
// four steps with A in TMEM (8 columns a step) and B MN-major (2048 bytes a step)
__device__ __forceinline__ void tc_mma_ts_steps(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    const uint32_t blo = static_cast<uint32_t>(b), bhi = static_cast<uint32_t>(b >> 32);
    asm volatile("{\n\t.reg .pred p, e, t;\n\t.reg .b32 x, y;\n\t.reg .b64 b;\n\telect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %5, 0;\n\tsetp.eq.u32 t, 0, 0;\n\t"
                 "mov.b64 b, {%2, %3};\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t"
                 SS_MMA_NEXT_TS("8", "128") SS_MMA_NEXT_TS("16", "256") SS_MMA_NEXT_TS("24", "384") "}"
                 ::"r"(d), "r"(a), "r"(blo), "r"(bhi), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void tc_commit_e(uint32_t bar) {
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                 ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define SS_R16(r, o) "=r"(r[o + 0]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), \
                     "=r"(r[o + 6]), "=r"(r[o + 7]), "=r"(r[o + 8]), "=r"(r[o + 9]), "=r"(r[o + 10]), "=r"(r[o + 11]), \
                     "=r"(r[o + 12]), "=r"(r[o + 13]), "=r"(r[o + 14]), "=r"(r[o + 15])
#define SS_W16(r, o) "r"(r[o + 0]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), \
                     "r"(r[o + 6]), "r"(r[o + 7]), "r"(r[o + 8]), "r"(r[o + 9]), "r"(r[o + 10]), "r"(r[o + 11]), \
                     "r"(r[o + 12]), "r"(r[o + 13]), "r"(r[o + 14]), "r"(r[o + 15])
// N consecutive fp32 columns of this thread's TMEM lane <-> registers r[O .. O+N-1]
template <int O, int N>
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[N]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : SS_R16(r, O) : "r"(taddr) : "memory");
}
template <int O, int N>
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[N]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : SS_R16(r, O), SS_R16(r, O + 16) : "r"(taddr) : "memory");
}
template <int O, int N>
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[N]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
        ::SS_W16(r, O), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::SS_W16(r, 0), SS_W16(r, 16), "r"(taddr) : "memory");
}
// 64 columns starting at taddr
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, uint32_t (&r)[64]) {
    tmem_ld32<0>(taddr, r);
    tmem_ld32<32>(taddr + 32, r);
}

// packed pairs of fp32 (one instruction for two values)
__device__ __forceinline__ unsigned long long pack_f32x2(float lo, float hi) {
    unsigned long long v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
    return v;
}
__device__ __forceinline__ void unpack_f32x2(unsigned long long v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ unsigned long long fma_f32x2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long add_f32x2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}

// Shared-memory matrix descriptors (swizzle-128B canonical layouts, 8-row groups 1024 B apart).
//   K-major  (Q, K, P): rows of 128 B, the contraction index contiguous; a 16-element step is +32 B.
//   MN-major (V): rows of 128 B are keys (contraction), the 64 contiguous elements are head_dim;
//                 the next 64 elements of head_dim start `lbo` bytes further; a 16-key step is +2048 B.
__device__ __forceinline__ uint64_t desc_k_major(uint32_t addr) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (1ull << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_mn_major(uint32_t addr, uint32_t lbo) {
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(lbo >> 4) << 16) |
           (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: fp32 accumulator, bf16 A and B, M = 128
__host__ __device__ constexpr uint32_t idesc_bf16(int n, bool a_mn_major, bool b_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (a_mn_major ? (1u << 15) : 0u) | (b_mn_major ? (1u << 16) : 0u) |
           (static_cast<uint32_t>(n >> 3) << 17) |
           (static_cast<uint32_t>(128 >> 4) << 24);
}

}  // namespace ss
