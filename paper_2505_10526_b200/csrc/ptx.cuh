// mbarrier and TMA wrappers shared by the kernels (inline PTX, sm_100a).
#pragma once

#include <cuda.h>
#include <stdint.h>

namespace massv {

#ifndef MASSV_SPIN_LIMIT
#define MASSV_SPIN_LIMIT (1u << 24)
#endif
constexpr uint32_t kSpinLimit = MASSV_SPIN_LIMIT;   // polls before a device-side wait gives up (a test build shortens it)

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded wait: gives up after kSpinLimit polls (or when another role already
// gave up), raising the CTA's abort flag instead of spinning forever.
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    for (uint32_t i = 0; i < kSpinLimit; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 255u) == 255u && *abort_flag) return false;
    }
    *abort_flag = 1;
    return false;
}

// The same for a whole warp: every lane polls and the warp takes one decision, so that
// warp-collective instructions after the wait are never reached by part of a warp.
__device__ __forceinline__ bool mbar_wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    const bool ok = mbar_wait(bar, parity, abort_flag);
    return __all_sync(0xffffffffu, ok);
}

// For three barriers at once: the polls' latencies overlap (shared memory that matrix products keep busy answers one in 200 cycles).
__device__ __forceinline__ bool mbar_wait_warp3(uint64_t* bar0, uint32_t parity0, uint64_t* bar1, uint32_t parity1, uint64_t* bar2, uint32_t parity2,
                                                volatile int* abort_flag) {
    bool ok = false;
    for (uint32_t i = 0; i < kSpinLimit; ++i) {
        uint32_t all;
        asm volatile(
            "{\n\t.reg .pred p, q, r;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 r, [%5], %6;\n\t"
            "and.pred p, p, q;\n\tand.pred p, p, r;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(all)
            : "r"(smem_u32(bar0)), "r"(parity0), "r"(smem_u32(bar1)), "r"(parity1), "r"(smem_u32(bar2)), "r"(parity2)
            : "memory");
        if (all) { ok = true; break; }
        if ((i & 255u) == 255u && *abort_flag) break;
    }
    if (!ok) *abort_flag = 1;
    return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar)), "l"(policy)
        : "memory");
}

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)), "l"(policy)
        : "memory");
}

// Plain 1-D copies into shared memory, without an eviction hint: by the bulk engine (16-byte multiples, signalled on an mbarrier)
// and by the calling thread.
__device__ __forceinline__ void bulk_load_1d(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src),
                 "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void cp_async_16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// ---- a row held by the CTAs of one cluster (1 .. 16): barrier of all their threads, loads from a peer's shared memory
__device__ __forceinline__ void row_barrier(int n_ctas) {        // all threads of the row's CTAs
    if (n_ctas == 1) { __syncthreads(); return; }
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_smem(const void* local, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(local)), "r"((uint32_t)rank));
    return r;
}
__device__ __forceinline__ unsigned long long peer_load_u64(const void* local, int rank) {
    unsigned long long v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer_smem(local, rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t peer_load_u32(const void* local, int rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(peer_smem(local, rank)) : "memory");
    return v;
}

// Host: 2-D bf16 tensor map over [rows, cols] (cols contiguous) with a box of
// [box_rows, 64 cols] and the 128-byte swizzle.  Returns false if the driver
// entry point is unavailable or rejects the shape.
bool make_tensor_map_bf16_2d(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint32_t box_rows);
// The same matrix as a 3-D map [cols / 64, rows, 64], box [blocks, box_rows, 64]: one copy brings several groups of 64
// columns (cols a multiple of 64; groups past the end are filled with zeros).
bool make_tensor_map_bf16_blocks(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint32_t box_rows, uint32_t blocks);
// [rows, heads, d] with boxes of box_heads heads of box_rows consecutive rows (64 elements of d); rows past the end come as zeros.
bool make_tensor_map_bf16_heads(CUtensorMap* map, const void* base, uint64_t rows, uint64_t heads, uint64_t d, uint32_t box_rows, uint32_t box_heads);

}  // namespace massv
