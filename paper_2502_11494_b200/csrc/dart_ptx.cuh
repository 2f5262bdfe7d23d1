// PTX of sm_100a that several kernels use: barriers in shared memory, bulk and tensor copies, tcgen05, bounded waits.
#pragma once
#include <cuda.h>

#include "dart_common.cuh"

namespace dart {
namespace sweep {

constexpr int kStatusTimeout = -7;

// ---- PTX wrappers -------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void *ptr) { return (uint32_t)__cvta_generic_to_shared(ptr); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) // (does not wait, unlike try_wait)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return ok != 0;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *tm, int x, int y, uint32_t bar,
                                            unsigned long long policy)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
                 " [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(dst),
                 "l"(tm), "r"(x), "r"(y), "r"(bar), "l"(policy)
                 : "memory");
}
// Plain bulk copy of `bytes` contiguous bytes (16-byte aligned, a multiple of 16) into shared memory.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, unsigned long long policy)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar), "l"(policy)
                 : "memory");
}
// Four rows (given by index) x one box width of columns -> four consecutive 128-byte rows at dst.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap *tm, int x, int r0, int r1, int r2, int r3,
                                            uint32_t bar, unsigned long long policy)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes.L2::cache_hint"
                 " [%0], [%1, {%2, %3, %4, %5, %6}], [%7], %8;" ::"r"(dst),
                 "l"(tm), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ int ld_acquire(const int *ptr)
{
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(ptr) : "memory");
    return v;
}
__device__ __forceinline__ void st_release(int *ptr, int v)
{
    asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(ptr), "r"(v) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
// OR of a predicate over a 128-thread warp group; doubles as the group's barrier
template <int kBarrierId, int kCount>
__device__ __forceinline__ bool group_any(bool pred)
{
    uint32_t r;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbar.red.or.pred p, %2, %3, q;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(r)
                 : "r"((uint32_t)pred), "n"(kBarrierId), "n"(kCount)
                 : "memory");
    return r != 0;
}
// Shared-memory matrix descriptor of a K-major, 128B-swizzled bf16 tile (rows at a 128-byte pitch,
// groups of 8 rows 1024 bytes apart).
__device__ __forceinline__ unsigned long long umma_desc(uint32_t saddr)
{
    unsigned long long d = 0;
    d |= (unsigned long long)((saddr & 0x3ffffu) >> 4);  // start address
    d |= (unsigned long long)1 << 16;                    // leading byte offset (unused for this layout)
    d |= (unsigned long long)(1024 >> 4) << 32;          // stride byte offset: 8 rows x 128 bytes
    d |= (unsigned long long)1 << 46;                    // descriptor version of sm_100
    d |= (unsigned long long)2 << 61;                    // 128-byte swizzle
    return d;
}
__device__ __forceinline__ void umma_bf16(uint32_t tmem_d, unsigned long long da, unsigned long long db, uint32_t idesc,
                                          uint32_t accumulate)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(tmem_d),
                 "l"(da), "l"(db), "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void umma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float *v)
{
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}

// ---- bounded waits --------------------------------------------------------------------------------
struct Ctl {
    volatile int *abort_flag; // shared memory
    int *status;              // global status word
    unsigned long long limit_cycles; // SM clock cycles (the clock runs at <= 2.1 GHz)
    __device__ __forceinline__ bool aborted() const { return *abort_flag != 0; }
    // records the first wait that expired: status[1] = where (kWait*), status[2] = task index, status[3] = CTA
    __device__ void give_up(int where, long long task) const
    {
        *abort_flag = 1;
        if (atomicCAS(status, 0, kStatusTimeout) == 0) {
            status[1] = where;
            status[2] = (int)task;
            status[3] = (int)blockIdx.x;
        }
    }
    // Waits poll without any bookkeeping first; only a wait that lasts starts reading the SM's cycle
    // counter (cheap, unlike the global nanosecond timer) and compares it with the limit.
    __device__ bool wait_bar(uint32_t bar, uint32_t parity, int where, long long task) const
    {
        for (int it = 0; it < 64; ++it)
            if (mbar_try_wait(bar, parity)) return true;
        const long long t0 = clock64();
        for (uint32_t it = 0;; ++it) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((it & 31u) == 31u) {
                if (aborted()) return false;
                if ((unsigned long long)(clock64() - t0) > limit_cycles) {
                    give_up(where, task);
                    return false;
                }
            }
        }
    }
    // After a failure: waits for work that is already in flight (a copy into shared memory, an MMA), whatever the
    // abort flag says: a CTA must not exit, nor free TMEM, while such work is pending.  Bounded by the time limit only.
    __device__ void wait_landed(uint32_t bar, uint32_t parity) const
    {
        const long long t0 = clock64();
        while (!mbar_try_wait(bar, parity))
            if ((unsigned long long)(clock64() - t0) > limit_cycles) return;
    }
    // waits until *flag >= target
    __device__ bool wait_flag(const int *flag, int where, long long task, int target = 1) const
    {
        for (int it = 0; it < 16; ++it) {
            if (ld_acquire(flag) >= target) return true;
            __nanosleep(32);
        }
        const long long t0 = clock64();
        for (uint32_t it = 0;; ++it) {
            if (ld_acquire(flag) >= target) return true;
            __nanosleep(64);
            if ((it & 15u) == 15u) {
                if (aborted()) return false;
                if ((unsigned long long)(clock64() - t0) > limit_cycles) {
                    give_up(where, task);
                    return false;
                }
            }
        }
    }
};

struct Ring {
    int depth;
    int stage = 0;
    uint32_t phase = 0;
    __device__ explicit Ring(int d) : depth(d) {}
    __device__ __forceinline__ void advance()
    {
        if (++stage == depth) {
            stage = 0;
            phase ^= 1u;
        }
    }
};

} // namespace sweep
} // namespace dart
