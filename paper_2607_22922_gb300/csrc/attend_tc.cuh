// Attention on the tensor cores' tiles: what the forward pass and the gradient share.
#pragma once

#include "attend.cuh"
#include "tiles.cuh"

namespace ifvs {

constexpr uint32_t kHalfBytes = 128 * 128;      // 128 rows of 64 elements, swizzled

// Rows [T][heads][dh], `ld` elements apart, of 16-bit elements; a box is 64 elements of
// box_heads heads of box_rows rows: box_heads x box_rows rows of 128 bytes in shared
// memory, heads innermost.  Elements beyond dh and rows beyond T read as zeros.
// box_dims 32: boxes of 32 elements in the 64-byte swizzle (chunk ^ (row / 2 mod 4)).
cudaError_t make_head_map(CUtensorMap* map, int type, const void* p, int64_t T, int heads, int dh, int64_t ld, int box_heads,
                          int box_rows, int box_dims = 64);

__device__ __forceinline__ void tma_load_heads(uint32_t dst, const CUtensorMap* map, int d, int head, int row, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
        "[%5];" ::"r"(dst),
        "l"(map), "r"(d), "r"(head), "r"(row), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tma_store_heads(const CUtensorMap* map, int d, int head, int row, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(d), "r"(head),
                 "r"(row), "r"(src)
                 : "memory");
}

// Operand B of a sum over the tile's rows (MN-major), 64-element blocks of 128 rows
__device__ __forceinline__ uint64_t rows_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(kHalfBytes >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}

// A from TMEM: rows are lanes, two 16-bit elements of the sum per column
__device__ __forceinline__ void mma_f16_tmem_a(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
}

// 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The waits of a kernel whose units may be of any size, so that one may last as long as another
// unit's tiles: it has run out when the CTA has got no further for its bound.  A poll is one load of
// both words: the gradient of 1000 short sequences takes 104 us so, 112 with a bound of the wait's
// own before the second word is looked at.
struct Pulse {
    alignas(8) int dead;             // as Watch's
    uint32_t last;                   // clock() when the CTA last got further
};
struct UnitWatch {
    Pulse* pulse;                    // shared memory
    Waits by;
    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) const {
        while (!mbar_try_wait(bar, parity)) {
            uint32_t dead, last;
            asm volatile("ld.volatile.shared.v2.u32 {%0, %1}, [%2];" : "=r"(dead), "=r"(last) : "r"(smem_addr(pulse)) : "memory");
            if (dead) return false;
            // (2^32 cycles are four bounds and two seconds: polls are more frequent)
            if ((uint32_t)clock() - last > (uint32_t)by.cycles) {
                *(volatile int*)&pulse->dead = 1;
                by.err[kErrWait] = 1;
                return false;
            }
        }
        return true;
    }
    // by the warp that finds units, for every batch, and by one thread of those that weigh, for
    // every 64th tile of a unit: far more often than a bound, and never in a short unit
    __device__ __forceinline__ void further() const { *(volatile uint32_t*)&pulse->last = (uint32_t)clock(); }
};

// Heads of a group that share a tile of 128 rows: all, where they divide it, else one
inline int tc_pack(const AttendArgs& a) { return (a.group & (a.group - 1)) == 0 && a.group <= 128 ? a.group : 1; }

cudaError_t launch_attend_tc(const AttendArgs& a, const AttendOut& o, int pack, int splits, float* part_out, float* part_lse,
                             cudaStream_t s);
// wide: 128 keys at a time instead of 64
cudaError_t launch_attend_short(const AttendArgs& a, const AttendOut& o, int pack, bool wide, cudaStream_t s);
// dk and dv, and dq of sequences of up to 64 keys; groups of a power of two up to 128 heads
cudaError_t launch_attend_grad_short(const AttendArgs& a, const AttendGrads& g, cudaStream_t s);
// delta: [Tq][heads] floats of workspace
cudaError_t launch_attend_grad_tc(const AttendArgs& a, const AttendGrads& g, int pack, int splits, float* delta, float* part_dk,
                                  float* part_dv, cudaStream_t s);

}  // namespace ifvs
