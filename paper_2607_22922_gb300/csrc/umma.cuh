// Matrix products on the tensor cores: tiles that TMA brings into shared
// memory in the 128-byte swizzle, tcgen05.mma into TMEM, and bounded waits.
//
// Operand tiles.  An operand is a matrix of 16-bit elements; "K-major" rows run
// along the summed index, "MN-major" rows along the other.  A TMA box is 64
// elements (128 bytes) of a row by some rows; in shared memory a row takes 128
// bytes, its eight 16-byte chunks permuted by chunk ^ (row mod 8).  K-major:
// box rows are the tile's rows; 64 of the sum per stage.  MN-major: box rows
// are 64 steps of the sum, and a tile of 64 n columns is n boxes of 8 KB.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "layers.cuh"
#include "scan_common.cuh"

namespace ifvs {

constexpr int kStepK = 64;                     // summed elements per stage
constexpr uint32_t kBoxBytes = 64 * 128;       // an MN-major box

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- descriptors (PTX ISA, tcgen05 matrix and instruction descriptors) -------
// layout type 2: 128-byte swizzle; groups of 8 rows 1024 bytes apart; MN-major:
// 64-element blocks kBoxBytes apart
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, bool mn_major) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(mn_major ? kBoxBytes >> 4 : 1u) << 16) |
           ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// what to add to a descriptor for the next 16 of the sum
__host__ __device__ constexpr uint64_t desc_step(bool mn_major) { return (mn_major ? 16u * 128u : 32u) >> 4; }

// D float32 = A B, A and B both bfloat16 (or float16)
__host__ __device__ constexpr uint32_t mma_desc(int m, int n, bool f16, bool a_mn, bool b_mn) {
    return (1u << 4) | ((f16 ? 0u : 1u) << 7) | ((f16 ? 0u : 1u) << 10) | ((a_mn ? 1u : 0u) << 15) |
           ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// CG CTAs (1, or a pair) work on one MMA.  In a pair each CTA holds its 128 rows
// of A and of the accumulator and half of B's columns; the pair's first CTA
// issues for both, with addresses that hold in both.
template <int CG>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
            : "memory");
}
// arrives on `bar` (of both CTAs of a pair) when the MMAs issued so far are done
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
}
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns) {
    if constexpr (CG == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}

// ---- pairs of CTAs --------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a shared-memory address of this CTA as the pair's first CTA has it
__device__ __forceinline__ uint32_t in_first(uint32_t addr) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(addr));
    return at;
}

__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&v)[32]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
// loads are complete when the wait is; the registers pass through it so that
// no use of them can be moved above it
__device__ __forceinline__ void tmem_wait(float (&v)[32]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                   "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]),
                   "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]),
                   "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}

// ---- TMA -----------------------------------------------------------------------
// to this CTA's memory; the bytes count on `bar`, in a pair on its first CTA's
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
            "[%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, "
            "%3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(in_first(bar))
            : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, int x, int y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x),
                 "r"(y), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void tma_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// at most N of this thread's stores still read shared memory
template <int N>
__device__ __forceinline__ void tma_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void tma_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// on `bar`, in a pair on its first CTA's
template <int CG>
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    if constexpr (CG == 1) {
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
    } else {
        asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_first(bar)) : "memory");
    }
}

// ---- bounded waits ----------------------------------------------------------------
// A wait that runs out marks the CTA dead (every other wait then returns at
// once) and the handle's error words; the roles leave their loops, and the
// kernel waits, bounded again, for its copies and MMAs before it returns.
struct Watch {
    volatile int* dead;     // shared memory
    Waits by;
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) const {
        if (mbar_try_wait(bar, parity)) return true;
        const long long t0 = clock64();
        for (;;) {
            if (mbar_try_wait(bar, parity)) return true;
            if (*dead) return false;
            if (clock64() - t0 > by.cycles) {
                *dead = 1;
                by.err[kErrWait] = 1;
                return false;
            }
        }
    }
};

// The place in a ring of S stages: fills and drains alternate parities
template <int S>
struct Ring {
    uint32_t at = 0, parity = 0;
    __device__ __forceinline__ void next() {
        if (++at == S) {
            at = 0;
            parity ^= 1u;
        }
    }
};

// two floats -> two 16-bit elements, the first in the low half
__device__ __forceinline__ uint32_t pack16(float a, float b, bool f16) {
    uint32_t d;
    if (f16)
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    else
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    return d;
}

// ---- tensor maps (host) ---------------------------------------------------------
// rows x cols matrix of 16-bit elements, rows `stride` elements apart; box of 64
// columns by box_rows rows.  Anything outside reads as zeros and is not written.
// box_cols 32: boxes of 32 columns in the 64-byte swizzle (chunk ^ (row / 2 mod 4)).
cudaError_t make_map(CUtensorMap* map, int type, const void* p, int64_t rows, int64_t cols, int64_t stride,
                     int box_rows, int box_cols = 64);

// Tile t of a grid of tiles: bands of kBand row tiles, columns outermost
// inside a band, so that tiles that run together share operand tiles in L2.
__device__ __forceinline__ int2 tile_of(int t, int m_tiles, int n_tiles) {
    constexpr int kBand = 16;
    const int band = t / (kBand * n_tiles), first = band * kBand;
    const int rows = min(kBand, m_tiles - first), r = t - first * n_tiles;
    return make_int2(first + r % rows, r / rows);
}

}  // namespace ifvs
