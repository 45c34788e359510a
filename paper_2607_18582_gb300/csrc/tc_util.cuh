// What the tensor-core kernels share: bounded mbarrier waits, operand descriptors, the election of an
// issuing lane, and the tensor-map encoder.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace mure {

constexpr long long kSpin = 2000000000LL;    // default wait limit: about a second at the SM clock

// The CTA's abort state: set by the role whose wait ran out (after `limit` cycles), seen
// by every other role's waits.
struct WaitCtl {
    int abort;
    long long limit;
};

__device__ __forceinline__ uint32_t smem_u32(const void *p)
{
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// Shared-memory matrix descriptor: K-major operand, 128-byte swizzle, 8-row groups
// 1024 bytes apart.
__device__ __forceinline__ uint64_t sw128_desc(uint32_t saddr)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFF);          // start address
    d |= (uint64_t)1 << 16;                          // leading byte offset (unused for swizzled K-major)
    d |= (uint64_t)(1024 >> 4) << 32;                // stride byte offset: next 8-row group
    d |= (uint64_t)1 << 46;                          // descriptor version
    d |= (uint64_t)2 << 61;                          // 128-byte swizzle
    return d;
}

// Byte offset of 16-byte chunk `chunk` of row r in a 128-byte-swizzled K-major tile.
__host__ __device__ __forceinline__ uint32_t sw128_off(int r, int chunk)
{
    return (uint32_t)(r * 128 + ((chunk ^ (r & 7)) << 4));
}

__device__ __forceinline__ void mbar_init(uint32_t a, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(a), "r"(count));
}

__device__ __forceinline__ void mbar_arrive(uint32_t a)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(a) : "memory");
}

__device__ __forceinline__ void mbar_expect_tx(uint32_t a, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(a), "r"(bytes) : "memory");
}

__device__ __forceinline__ bool mbar_try(uint32_t a, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(a), "r"(parity)
        : "memory");
    return ok != 0;
}

// Wait for the phase of parity `parity`, polling every ~NS nanoseconds (a sleeping
// warp leaves the issue slots of its SM sub-partition to the producers); false when
// another role has aborted or the wait limit has passed (then this role aborts the
// CTA).
template <int NS = 0>
__device__ __forceinline__ bool wait_phase(uint32_t a, uint32_t parity, volatile WaitCtl *abort_flag)
{
    if (mbar_try(a, parity)) return true;
    const long long t0 = clock64();
    for (;;) {
        if (NS > 0) __nanosleep(NS);
        if (mbar_try(a, parity)) return true;
        if (abort_flag->abort) return false;
        if (clock64() - t0 > abort_flag->limit) { abort_flag->abort = 1; return false; }
    }
}

// The same for a whole warp: every lane polls, the verdict is the warp's AND, so the
// .sync.aligned tensor-memory instructions that follow see a converged warp.
template <int NS = 0>
__device__ __forceinline__ bool warp_wait_phase(uint32_t a, uint32_t parity, volatile WaitCtl *abort_flag)
{
    const bool ok = wait_phase<NS>(a, parity, abort_flag);
    return __all_sync(0xffffffffu, ok);
}

// Teardown wait: bounded by the default limit whatever the CTA's limit, ignores the
// abort flag, so that copies and MMAs in flight land before shared and tensor memory
// are released.
__device__ __forceinline__ void wait_phase_drain(uint32_t a, uint32_t parity)
{
    const long long t0 = clock64();
    while (!mbar_try(a, parity))
        if (clock64() - t0 > kSpin) return;
}

// One lane of a converged warp (the same one every time).  The tensor-core and bulk-copy
// instructions take their operands from uniform registers; in a branch on the lane number the
// compiler cannot know that a single lane runs it.  So the issuing warps run their loops whole,
// with warp-uniform operands, and elect a lane around the instructions themselves, and the copying
// warps elect the lane that copies.  Measured (lane-number branches before, kernel times): the window
// GEMM of LeNet's second convolution 8.93 -> 8.32 ms (1,000 mutants x 10,000 inputs), ResNet-20's
// staged convolutions 19.2 -> 18.5 ms (60 x 600).
__device__ __forceinline__ bool elect_one()
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok));
    return ok != 0;
}

__device__ __forceinline__ void mma_commit(uint32_t mbar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(mbar)
                 : "memory");
}

// cuTensorMapEncodeTiled through the runtime's driver entry point (no link to libcuda); looked up once, a second
// thread's first call waits for the first one's.
inline PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder()
{
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool there = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
                           q == cudaDriverEntryPointSuccess;
        return there ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f) : nullptr;
    }();
    return fn;
}

}  // namespace mure
