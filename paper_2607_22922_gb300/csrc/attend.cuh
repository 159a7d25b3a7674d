// Attention of packed sequences: what its kernels share.
//
// Queries and keys lie packed, sequence b in rows [offsets[b], offsets[b + 1]) of
// each.  The heads that share a key head are one group; kernels take its queries as
// rows of one matrix, row i = (token i / group, head i mod group), so that keys and
// values are read once for the group.
#pragma once

#include "layers.cuh"

namespace ifvs {

struct AttendArgs {
    int64_t Tq, Tk, B;
    int heads, kv_heads, group, dh, type;
    const int64_t *q_offsets, *kv_offsets;      // or null: B = 1
    const int32_t* kv_ids;                      // or null: no padding
    float scale;
    const void *q, *k, *v;
    int64_t ld_q, ld_k, ld_v;                   // elements between rows
    Waits waits;
    int num_sms;
};

struct AttendOut {
    void* out;
    int64_t ld;
    float* lse;             // [Tq][heads] or null
};

struct AttendGrads {
    const void *out, *d_out;
    const float* lse;
    int64_t ld_out, ld_d_out;
    void *dq, *dk, *dv;
    int64_t ld_dq, ld_dk, ld_dv;
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Tokens [at, at + len) of a sequence, inside 0..T whatever the offsets hold
struct Span {
    int64_t at, len;
};
__device__ __forceinline__ int64_t place(const int64_t* __restrict__ offsets, int64_t b, int64_t B, int64_t T) {
    if (offsets == nullptr) return b == 0 ? 0 : T;
    const int64_t v = __ldg(offsets + b);
    return v < 0 ? 0 : (v > T ? T : v);
}
__device__ __forceinline__ Span span_of(const int64_t* __restrict__ offsets, int64_t b, int64_t B, int64_t T) {
    const int64_t lo = place(offsets, b, B, T), hi = place(offsets, b + 1, B, T);
    return {lo, hi > lo ? hi - lo : 0};
}

// Tiles of 2^log rows (`group` a token) of all sequences, without their lengths on the
// host: sequence b has the slots from tokens-before(b) group / 2^log + b on, one more at
// least than its full tiles, so that slots(T, ...) of them hold every tile and one per
// sequence.  A warp finds a slot's sequence by 32 probes at a time.
struct Slot {
    int64_t b, tile;
};
__device__ __forceinline__ int64_t first_slot(const int64_t* offsets, int64_t b, int64_t B, int64_t T, int group, int log) {
    return ((place(offsets, b, B, T) * group) >> log) + b;
}
__device__ __forceinline__ Slot slot_of(const int64_t* __restrict__ offsets, int64_t B, int64_t T, int group, int log, int64_t slot) {
    const int lane = threadIdx.x & 31;
    uint32_t lo = 0, n = (uint32_t)B;       // the sequence is in lo .. lo + n - 1
    while (n > 1) {
        const uint32_t step = (n + 31) / 32, i = lane * step;
        const bool before = i < n && (lane == 0 || first_slot(offsets, lo + i, B, T, group, log) <= slot);
        const uint32_t last = (31 - __clz((int)__ballot_sync(0xFFFFFFFFu, before))) * step;
        lo += last;
        n = n - last < step ? n - last : step;
    }
    return {lo, slot - first_slot(offsets, lo, B, T, group, log)};
}
inline int64_t slots(int64_t T, int64_t B, int group, int log) { return ((T * group) >> log) + B; }

// Rows of a group's matrix from row `first` on: row i is token `token` + at(i).x, head
// at(i).y of the group.  Division by the group's size is a product with its inverse: exact
// below 2^22, and rows here are counted within a tile.
struct RowOf {
    int64_t token;
    uint32_t sub, group, inverse;
    __device__ __forceinline__ RowOf(int64_t first, int group_)
        : group((uint32_t)group_), inverse(0xFFFFFFFFu / (uint32_t)group_ + 1u) {
        // a division of 64 bits takes a hundred instructions
        token = first >> 32 ? first / group_ : (int64_t)((uint32_t)first / group);
        sub = (uint32_t)(first - token * group_);
    }
    __device__ __forceinline__ int2 at(int i) const {
        const uint32_t x = sub + (uint32_t)i, t = group == 1 ? x : __umulhi(x, inverse);
        return make_int2((int)t, (int)(x - t * group));
    }
};
// Where such rows lie: `ld` elements from token to token, dh from head to head
template <class T>
struct RowsAt {
    T* first;        // of the tile's first token, the group's first head
    int ld, dh;
    __device__ __forceinline__ RowsAt(T* p, int64_t token, int64_t ld_, int dh_) : first(p + token * ld_), ld((int)ld_), dh(dh_) {}
    __device__ __forceinline__ T* operator()(int2 at) const { return first + (int64_t)at.x * ld + at.y * dh; }
};

// The last CTA of a kernel that needs nothing of the one before it and may run beside it
// waits for that one, so that what comes after them waits for both.
__device__ __forceinline__ bool last_cta() {
    return blockIdx.x == gridDim.x - 1 && blockIdx.y == gridDim.y - 1 && blockIdx.z == gridDim.z - 1;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- tiles of warps: 16 x 8 x 16 products in registers ---------------------------------
__device__ __forceinline__ uint32_t smem32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

template <class T>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same_v<T, __half>)
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool TRANS>
__device__ __forceinline__ void ldmatrix(uint32_t (&r)[4], uint32_t addr) {
    if constexpr (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr)
                     : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr)
                     : "memory");
}
// 16 bytes to shared memory, zeros where !in
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// A tile of rows in shared memory: COLS 16-bit elements a row and 8 more, so that the
// eight rows that an ldmatrix reads at once begin in different banks.
template <int COLS>
struct Rows {
    static constexpr int kLd = COLS + 8;
    uint32_t at;
    __device__ __forceinline__ uint32_t addr(int row, int col) const { return at + (uint32_t)(row * kLd + col) * 2u; }
    // operand A: rows row0 .. + 15, elements col0 .. + 15
    __device__ __forceinline__ void a(uint32_t (&r)[4], int row0, int col0) const {
        const int l = threadIdx.x & 31;
        ldmatrix<false>(r, addr(row0 + (l & 15), col0 + (l >> 4) * 8));
    }
    // operand A of the transposed tile: its rows are columns col0 .. + 15 here
    __device__ __forceinline__ void a_t(uint32_t (&r)[4], int row0, int col0) const {
        const int l = threadIdx.x & 31;
        ldmatrix<true>(r, addr(row0 + (l & 7) + (l >> 4) * 8, col0 + ((l >> 3) & 1) * 8));
    }
    // operand B whose columns are rows here (a product with the transposed tile): 16 rows
    // from row0 (two n of 8: r[0], r[1] and r[2], r[3]), elements col0 .. + 15 of the sum
    __device__ __forceinline__ void b_t(uint32_t (&r)[4], int row0, int col0) const {
        const int l = threadIdx.x & 31;
        ldmatrix<false>(r, addr(row0 + (l & 7) + (l >> 4) * 8, col0 + ((l >> 3) & 1) * 8));
    }
    // operand B: rows row0 .. + 15 of the sum, 16 columns from col0 (two n of 8)
    __device__ __forceinline__ void b(uint32_t (&r)[4], int row0, int col0) const {
        const int l = threadIdx.x & 31;
        ldmatrix<true>(r, addr(row0 + (l & 15), col0 + (l >> 4) * 8));
    }
};

constexpr int kTileRows = 64, kTileKeys = 64, kTileLog = 6;

// Copies rows of a tile into shared memory: row(i) is row i's address, or null for zeros;
// dims dh .. DH - 1 are zeros.  any: an address of global memory, not read.
template <int DH, class T, class Row>
__device__ __forceinline__ void load_rows(const Rows<DH>& to, int rows, int dh, const void* any, const Row& row) {
    constexpr int C = DH / 8;
    for (int i = threadIdx.x; i < rows * C; i += blockDim.x) {
        const int r = i / C, c = i % C;
        const T* p = row(r);
        const bool in = p != nullptr && c * 8 < dh;
        copy16(to.addr(r, c * 8), in ? (const void*)(p + c * 8) : any, in);
    }
}

// ---- launchers --------------------------------------------------------------------------
size_t attend_bytes(const AttendArgs& a);
cudaError_t launch_attend(const AttendArgs& a, const AttendOut& o, uint8_t* work, cudaStream_t s);
size_t attend_grad_bytes(const AttendArgs& a);
cudaError_t launch_attend_grad(const AttendArgs& a, const AttendGrads& g, uint8_t* work, cudaStream_t s);

}  // namespace ifvs
