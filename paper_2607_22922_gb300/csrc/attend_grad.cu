// The gradient of attention (ifvs_attend_grad).
//
//   p = exp(s - lse), dp = do v, delta = sum over the keys of p dp = out do
//   ds = p (dp - delta), dq = scale ds k, dk = scale ds^T q, dv = p^T do
//
// p and ds are computed again tile by tile and rounded to the arrays' type, because the
// tensor cores multiply 16-bit operands; sums are float32, in a fixed order.  Where a
// sequence's keys are one tile, lse and delta come from the tile itself, else from the
// forward call's lse and (rounded) output.
#include "attend_tc.cuh"

namespace ifvs {

namespace {

using Scores = float2[kTileKeys / 8][2];       // of rows lane / 4 and + 8, keys 8 j + lane % 4 * 2 and the next
using Operands = uint32_t[kTileKeys / 16][4];    // 16 rows x 64 keys as operand A

// A warp's 16 rows from `row` on times the tile's keys, over DH; `blocks` of 16 keys.  bias:
// where a key's sums begin, or null: 0
template <class T, int DH>
__device__ __forceinline__ void scores(Scores& s, const Rows<DH>& q, int row, const Rows<DH>& k, int blocks, const float* bias) {
#pragma unroll
    for (int j = 0; j < kTileKeys / 8; ++j)
        s[j][0] = s[j][1] = bias ? *reinterpret_cast<const float2*>(bias + j * 8 + (threadIdx.x & 3) * 2) : make_float2(0.f, 0.f);
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) {
        uint32_t f[4];
        q.a(f, row, d * 16);
#pragma unroll
        for (int j = 0; j < kTileKeys / 16; ++j)
            if (j < blocks) {
                uint32_t b[4];
                k.b_t(b, j * 16, d * 16);
                mma16816<T>(reinterpret_cast<float(&)[4]>(s[2 * j]), f, b[0], b[1]);
                mma16816<T>(reinterpret_cast<float(&)[4]>(s[2 * j + 1]), f, b[2], b[3]);
            }
    }
}

__device__ __forceinline__ float2 both2(float v) { return make_float2(v, v); }

// p and ds of a warp's rows from the scores s and dp, in their places.  lse2: base 2,
// infinite for a row without keys.
__device__ __forceinline__ void slopes(Scores& s, Scores& dp, const float (&lse2)[2], const float (&delta)[2], float c, int blocks) {
#pragma unroll
    for (int j = 0; j < kTileKeys / 8; ++j)
        if (j / 2 < blocks)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float2 e = fma_(s[j][r], both2(c), both2(-lse2[r]));
                e.x = ex2(e.x);
                e.y = ex2(e.y);
                s[j][r] = e;
                dp[j][r] = mul_(e, add_(dp[j][r], both2(-delta[r])));
            }
}
// The same where the tile has all of the rows' keys
__device__ __forceinline__ void slopes_alone(Scores& s, Scores& dp, float c, int blocks) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float top = fmaxf(s[0][r].x, s[0][r].y);
#pragma unroll
        for (int j = 1; j < kTileKeys / 8; ++j) top = fmaxf(top, fmaxf(s[j][r].x, s[j][r].y));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2)) * c;
        const float base = top == -INFINITY ? 0.f : top;
        float2 l2 = both2(0.f), sum2 = l2;
#pragma unroll
        for (int j = 0; j < kTileKeys / 8; ++j)
            if (j / 2 < blocks) {
                float2 e = fma_(s[j][r], both2(c), both2(-base));
                e.x = ex2(e.x);
                e.y = ex2(e.y);
                s[j][r] = e;
                l2 = add_(l2, e);
                sum2 = fma_(e, dp[j][r], sum2);
            }
        float l = total(l2), sum = total(sum2);
#pragma unroll
        for (int x = 1; x <= 2; x <<= 1) {
            l += __shfl_xor_sync(0xFFFFFFFFu, l, x);
            sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l, delta = sum * inv;
#pragma unroll
        for (int j = 0; j < kTileKeys / 8; ++j)
            if (j / 2 < blocks) {
                s[j][r] = mul_(s[j][r], both2(inv));
                dp[j][r] = mul_(s[j][r], add_(dp[j][r], both2(-delta)));
            }
    }
}

template <class T>
__device__ __forceinline__ void to_operands(Operands& f, const Scores& x) {
#pragma unroll
    for (int j = 0; j < kTileKeys / 16; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[j][i] = pack2(x[2 * j + (i >> 1)][i & 1], T());
}

// acc += x y: y the keys' rows
template <class T, int DH>
__device__ __forceinline__ void times_keys(float (&acc)[DH / 8][4], const Operands& x, const Rows<DH>& y, int blocks) {
#pragma unroll
    for (int j = 0; j < kTileKeys / 16; ++j)
        if (j < blocks)
#pragma unroll
            for (int d = 0; d < DH / 16; ++d) {
                uint32_t b[4];
                y.b(b, j * 16, d * 16);
                mma16816<T>(acc[2 * d], x[j], b[0], b[1]);
                mma16816<T>(acc[2 * d + 1], x[j], b[2], b[3]);
            }
}

// acc += x^T y, its columns 16 d0 .. 16 d1 - 1: 16 of x's columns (keys) from `key`, x [64
// rows][64 keys] and y [64 rows] in shared memory
template <class T, int DH>
__device__ __forceinline__ void transposed_times(float (&acc)[DH / 8][4], const Rows<kTileKeys>& x, int key, const Rows<DH>& y, int d0,
                                                 int d1) {
#pragma unroll
    for (int r = 0; r < kTileRows / 16; ++r) {
        uint32_t f[4];
        x.a_t(f, r * 16, key);
#pragma unroll
        for (int d = 0; d < DH / 16; ++d)
            if (d >= d0 && d < d1) {
                uint32_t b[4];
                y.b(b, r * 16, d * 16);
                mma16816<T>(acc[2 * d], f, b[0], b[1]);
                mma16816<T>(acc[2 * d + 1], f, b[2], b[3]);
            }
    }
}

__device__ __forceinline__ void put_scores(const Rows<kTileKeys>& to, int row, const Operands& x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < kTileKeys / 16; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(to.addr(row + (lane >> 2) + 8 * (i & 1), j * 16 + (i >> 1) * 8 + (lane & 3) * 2)),
                         "r"(x[j][i])
                         : "memory");
}

// delta of a warp's 16 rows: two lanes a row, from shared memory's do and memory's out
template <class T, int DH, class Row>
__device__ __forceinline__ float delta_of(const Rows<DH>& d_out, int row, int dh, const Row& out) {
    const int lane = threadIdx.x & 31, r = row + (lane >> 1);
    const T* p = out(r);
    float2 sum = make_float2(0.f, 0.f);
    if (p)
        for (int c = lane & 1; c * 8 < dh; c += 2) {
            Pack<T, 8> x, y;
            x.load(p + c * 8);
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(y.w.x), "=r"(y.w.y), "=r"(y.w.z), "=r"(y.w.w)
                         : "r"(d_out.addr(r, c * 8))
                         : "memory");
#pragma unroll
            for (int j = 0; j < 4; ++j) sum = fma_(x.get(j), y.get(j), sum);
        }
    const float v = total(sum);
    return v + __shfl_xor_sync(0xFFFFFFFFu, v, 1);
}

// The rows' lse (base 2) and delta for the layout of the scores: rows lane / 4 and + 8
template <class T, int DH, class Out, class Lse>
__device__ __forceinline__ void row_terms(float (&lse2)[2], float (&delta)[2], const Rows<DH>& d_out, int row, int rows, int dh,
                                          const Out& out, const Lse& lse) {
    const int lane = threadIdx.x & 31;
    const float v = delta_of<T>(d_out, row, dh, out);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = (lane >> 2) + 8 * r;
        delta[r] = __shfl_sync(0xFFFFFFFFu, v, i * 2);
        const float l = row + i < rows ? lse(row + i) : -INFINITY;
        lse2[r] = l == -INFINITY ? INFINITY : l * kLog2e;
    }
}

// Stores a warp's 16 rows from registers, scaled; columns 16 d0 .. 16 d1 - 1.  to(i): row i
// of them.  counts(i): false for a row of zeros.
template <class T, int DH, class Row, class Counts>
__device__ __forceinline__ void put_rows(const float (&acc)[DH / 8][4], float scale, int rows, int dh, int d0, int d1, const Row& to,
                                         const Counts& counts) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = (lane >> 2) + 8 * r;
        if (i >= rows) continue;
        T* p = to(i) + (lane & 3) * 2;
        const bool in = counts(i);
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
            if (j * 8 < dh && j / 2 >= d0 && j / 2 < d1)
                *reinterpret_cast<uint32_t*>(p + j * 8) =
                    in ? pack2(make_float2(acc[j][2 * r] * scale, acc[j][2 * r + 1] * scale), T()) : 0u;
    }
}

// What a CTA of either kernel works on
template <class T>
struct Arrays {
    const T *q, *k, *v, *out, *d_out;
    T *dq, *dk, *dv;
    __device__ __forceinline__ Arrays(const AttendArgs& a, const AttendGrads& g, int hk) {
        const int64_t hq = (int64_t)hk * a.group * a.dh, h = (int64_t)hk * a.dh;
        q = (const T*)a.q + hq;
        k = (const T*)a.k + h;
        v = (const T*)a.v + h;
        out = (const T*)g.out + hq;
        d_out = (const T*)g.d_out + hq;
        dq = (T*)g.dq + hq;
        dk = (T*)g.dk + h;
        dv = (T*)g.dv + h;
    }
};

// ---- dk and dv, and dq of sequences whose keys are one tile ---------------------------------
// A CTA takes 64 keys and one part of the rows of their group, 64 at a time with the next
// on their way: each of its 4 warps makes p and ds of 16 rows, then adds 16 keys' sums over
// the 64 rows (a share of the columns for fewer keys).  Blocks of 16 keys behind the last are
// left out.  40 sequences of 40 queries and 16 keys, 8 heads of 64, take 11 us: one round of
// CTAs, bound by the chain of a CTA's loads, products and stores.
template <class T, int DH>
struct KeyTiles {
    Rows<DH> k, v, q[2], d_out[2];
    Rows<kTileKeys> p, ds;
    static constexpr uint32_t kBytes = Rows<DH>::kLd * 2 * 64;
    static constexpr size_t kSmem = 6 * kBytes + 2 * kTileRows * Rows<kTileKeys>::kLd * 2;
};

template <class T, int DH>
__global__ void __launch_bounds__(128, DH == 128 ? 2 : 3) k_attend_keys(AttendArgs a, AttendGrads g, int splits, float* part_dk, float* part_dv) {
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ __align__(8) float bias[kTileKeys];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y, split = blockIdx.z;
    start_dependents();
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const Slot slot = slot_of(a.kv_offsets, a.B, a.Tk, 1, kTileLog, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t key0 = slot.tile * kTileKeys;
    // without keys the first tile still writes dq
    if (slot.tile < 0 || (key0 >= ks.len && slot.tile > 0)) return;
    const bool alone = ks.len <= kTileKeys;
    const int keys = ks.len - key0 < kTileKeys ? (int)(ks.len - key0) : kTileKeys, blocks = (keys + 15) / 16;
    const Arrays<T> at(a, g, hk);
    const int64_t n_rows = qs.len * a.group, tiles = (n_rows + kTileRows - 1) / kTileRows;
    const int64_t t0 = tiles * split / splits, t1 = tiles * (split + 1) / splits;

    KeyTiles<T, DH> sm;
    const uint32_t base = smem32(raw);
    sm.k.at = base;
    sm.v.at = base + sm.kBytes;
    auto q_of = [&](int stage) { return Rows<DH>{base + (2 + 2 * stage) * sm.kBytes}; };
    auto do_of = [&](int stage) { return Rows<DH>{base + (3 + 2 * stage) * sm.kBytes}; };
    sm.p.at = base + 6 * sm.kBytes;
    sm.ds.at = sm.p.at + kTileRows * Rows<kTileKeys>::kLd * 2;
    auto load_queries = [&](int64_t t, int stage) {
        const int64_t row0 = t * kTileRows;
        const int rows = n_rows - row0 < kTileRows ? (int)(n_rows - row0) : kTileRows;
        const RowOf ro(row0, a.group);
        const RowsAt<const T> q(at.q, qs.at + ro.token, a.ld_q, a.dh), d_out(at.d_out, qs.at + ro.token, g.ld_d_out, a.dh);
        load_rows<DH, T>(q_of(stage), kTileRows, a.dh, a.q, [&](int i) { return i < rows ? q(ro.at(i)) : nullptr; });
        load_rows<DH, T>(do_of(stage), kTileRows, a.dh, a.q, [&](int i) { return i < rows ? d_out(ro.at(i)) : nullptr; });
    };
    auto key_in = [&](int i) { return i < keys && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key0 + i) >= 0); };
    if (t0 < t1) load_queries(t0, 0);
    load_rows<DH, T>(sm.k, blocks * 16, a.dh, a.q, [&](int i) { return key_in(i) ? at.k + (ks.at + key0 + i) * a.ld_k : nullptr; });
    load_rows<DH, T>(sm.v, blocks * 16, a.dh, a.q, [&](int i) { return key_in(i) ? at.v + (ks.at + key0 + i) * a.ld_v : nullptr; });
    copies_done();
    const bool seen = threadIdx.x < kTileKeys && key_in(threadIdx.x);
    if (threadIdx.x < kTileKeys) bias[threadIdx.x] = seen ? 0.f : -INFINITY;
    // where no key counts dq is zero, though what is not finite has NaN as its scores
    const bool some = __syncthreads_or(seen);
    const float c = a.scale * kLog2e;
    // this warp's share of dk and dv: 16 keys, columns 16 d0 .. 16 d1 - 1
    const int shares = blocks == 1 ? 4 : blocks == 2 ? 2 : 1, block = warp / shares, d0 = warp % shares * (DH / 16) / shares,
              d1 = (warp % shares + 1) * (DH / 16) / shares;

    float dk[DH / 8][4], dv[DH / 8][4];
#pragma unroll
    for (int j = 0; j < DH / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) dk[j][i] = dv[j][i] = 0.f;
    for (int64_t t = t0; t < t1; ++t) {
        const int stage = (int)(t - t0) & 1;
        const int64_t row0 = t * kTileRows;
        const int rows = n_rows - row0 < kTileRows ? (int)(n_rows - row0) : kTileRows;
        const RowOf ro(row0, a.group);
        const Rows<DH> sq = q_of(stage), sdo = do_of(stage);
        if (t + 1 < t1) load_queries(t + 1, stage ^ 1);
        copies_done();
        wait_copies<1>();
        __syncthreads();
        if (warp * 16 < rows) {
            Operands f;
            {
                Scores s, dp;
                scores<T>(s, sq, warp * 16, sm.k, blocks, bias);
                scores<T>(dp, sdo, warp * 16, sm.v, blocks, nullptr);
                if (alone) {
                    slopes_alone(s, dp, c, blocks);
                } else {
                    float lse2[2], delta[2];
                    const RowsAt<const T> out(at.out, qs.at + ro.token, g.ld_out, a.dh);
                    row_terms<T>(lse2, delta, sdo, warp * 16, rows, a.dh, [&](int i) { return i < rows ? out(ro.at(i)) : nullptr; },
                                 [&](int i) {
                                     const int2 r = ro.at(i);
                                     return __ldg(g.lse + (qs.at + ro.token + r.x) * a.heads + hk * a.group + r.y);
                                 });
                    slopes(s, dp, lse2, delta, c, blocks);
                }
                to_operands<T>(f, s);
                put_scores(sm.p, warp * 16, f);
                to_operands<T>(f, dp);
                put_scores(sm.ds, warp * 16, f);
            }
            if (alone) {
                float dq[DH / 8][4];
#pragma unroll
                for (int j = 0; j < DH / 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) dq[j][i] = 0.f;
                times_keys<T, DH>(dq, f, sm.k, blocks);
                const RowsAt<T> to(at.dq, qs.at + ro.token, g.ld_dq, a.dh);
                put_rows<T, DH>(dq, a.scale, rows - warp * 16, a.dh, 0, DH / 16, [&](int i) { return to(ro.at(warp * 16 + i)); },
                                [&](int) { return some; });
            }
        } else {                 // rows of zeros
            const Operands f = {};
            put_scores(sm.p, warp * 16, f);
            put_scores(sm.ds, warp * 16, f);
        }
        __syncthreads();
        if (block < blocks) {
            transposed_times<T, DH>(dv, sm.p, block * 16, sdo, d0, d1);
            transposed_times<T, DH>(dk, sm.ds, block * 16, sq, d0, d1);
        }
        __syncthreads();
    }
    wait_copies<0>();
    const int mine = keys - block * 16;
    if (splits == 1) {
        auto counts = [&](int i) { return bias[block * 16 + i] == 0.f; };
        put_rows<T, DH>(dk, a.scale, mine, a.dh, d0, d1, [&](int i) { return at.dk + (ks.at + key0 + block * 16 + i) * g.ld_dk; }, counts);
        put_rows<T, DH>(dv, 1.f, mine, a.dh, d0, d1, [&](int i) { return at.dv + (ks.at + key0 + block * 16 + i) * g.ld_dv; }, counts);
        return;
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = (lane >> 2) + 8 * r;
        if (i >= mine) continue;
        const int64_t to = (((int64_t)split * a.Tk + ks.at + key0 + block * 16 + i) * a.kv_heads + hk) * a.dh + (lane & 3) * 2;
        const bool in = bias[block * 16 + i] == 0.f;
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
            if (j * 8 < a.dh && j / 2 >= d0 && j / 2 < d1) {
                *reinterpret_cast<float2*>(part_dk + to + j * 8) =
                    in ? make_float2(dk[j][2 * r] * a.scale, dk[j][2 * r + 1] * a.scale) : both2(0.f);
                *reinterpret_cast<float2*>(part_dv + to + j * 8) = in ? make_float2(dv[j][2 * r], dv[j][2 * r + 1]) : both2(0.f);
            }
    }
}

// dk and dv from their parts, in order
template <class T>
__global__ void __launch_bounds__(256) k_attend_keys_join(AttendArgs a, AttendGrads g, int splits, const float* part_dk, const float* part_dv) {
    wait_before();
    const int64_t width = (int64_t)a.kv_heads * a.dh, n = a.Tk * width, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    const float* parts = blockIdx.y ? part_dv : part_dk;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float4 p = __ldcg(reinterpret_cast<const float4*>(parts + s * n + i));
        v.x += p.x;
        v.y += p.y;
        v.z += p.z;
        v.w += p.w;
    }
    const int64_t key = i / width, col = i - key * width;
    T* to = blockIdx.y ? (T*)g.dv + key * g.ld_dv : (T*)g.dk + key * g.ld_dk;
    *reinterpret_cast<uint2*>(to + col) = make_uint2(pack2(make_float2(v.x, v.y), T()), pack2(make_float2(v.z, v.w), T()));
}

// ---- dq of sequences with more keys than a tile ----------------------------------------------
// A CTA takes slots of 64 rows by turns, since most may have nothing to do.  It needs nothing
// of the kernel of the keys, whose last CTAs it runs beside.
template <class T, int DH>
struct RowTiles {
    static constexpr uint32_t kBytes = Rows<DH>::kLd * 2 * 64;
    static constexpr size_t kSmem = 6 * kBytes;
};

template <class T, int DH>
__global__ void __launch_bounds__(128, DH == 128 ? 2 : 3) k_attend_rows(AttendArgs a, AttendGrads g, int64_t n_slots) {
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ __align__(8) float bias[2][kTileKeys];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y;
    const uint32_t base = smem32(raw);
    constexpr uint32_t kBytes = RowTiles<T, DH>::kBytes;
    const Rows<DH> sq{base}, sdo{base + kBytes};
    auto k_of = [&](int stage) { return Rows<DH>{base + (2 + 2 * stage) * kBytes}; };
    auto v_of = [&](int stage) { return Rows<DH>{base + (3 + 2 * stage) * kBytes}; };
    const Arrays<T> at(a, g, hk);
    const float c = a.scale * kLog2e;
    // slots are looked at 32 at a time, one a lane
    Slot mine{};
    uint32_t todo = 0;
    for (int64_t n0 = blockIdx.x; todo || n0 < n_slots;) {
        if (!todo) {
            const int64_t n = n0 + lane * (int64_t)gridDim.x;
            n0 += 32 * (int64_t)gridDim.x;
            bool some = n < n_slots;
            if (some) {
                uint32_t lo = 0, count = (uint32_t)a.B;
                while (count > 1) {
                    const uint32_t half = count / 2;
                    if (first_slot(a.q_offsets, lo + half, a.B, a.Tq, a.group, kTileLog) <= n) {
                        lo += half;
                        count -= half;
                    } else {
                        count = half;
                    }
                }
                mine = Slot{lo, n - first_slot(a.q_offsets, lo, a.B, a.Tq, a.group, kTileLog)};
                some = mine.tile >= 0 && span_of(a.q_offsets, lo, a.B, a.Tq).len * a.group > mine.tile * kTileRows &&
                       span_of(a.kv_offsets, lo, a.B, a.Tk).len > kTileKeys;
            }
            todo = __ballot_sync(0xFFFFFFFFu, some);
            continue;
        }
        const int from = __ffs((int)todo) - 1;
        todo &= todo - 1;
        const Slot slot{__shfl_sync(0xFFFFFFFFu, mine.b, from), __shfl_sync(0xFFFFFFFFu, mine.tile, from)};
        const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
        const int64_t row0 = slot.tile * kTileRows, left = qs.len * a.group - row0;
        const int rows = left < kTileRows ? (int)left : kTileRows;
        const RowOf ro(row0, a.group);
        const RowsAt<const T> q(at.q, qs.at + ro.token, a.ld_q, a.dh), d_out(at.d_out, qs.at + ro.token, g.ld_d_out, a.dh),
            out(at.out, qs.at + ro.token, g.ld_out, a.dh);
        load_rows<DH, T>(sq, kTileRows, a.dh, a.q, [&](int i) { return i < rows ? q(ro.at(i)) : nullptr; });
        load_rows<DH, T>(sdo, kTileRows, a.dh, a.q, [&](int i) { return i < rows ? d_out(ro.at(i)) : nullptr; });
        auto key_in = [&](int64_t key) { return key < ks.len && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key) >= 0); };
        auto load_keys = [&](int64_t tile, int stage) {
            const int64_t key0 = tile * kTileKeys;
            load_rows<DH, T>(k_of(stage), kTileKeys, a.dh, a.q,
                             [&](int i) { return key_in(key0 + i) ? at.k + (ks.at + key0 + i) * a.ld_k : nullptr; });
            load_rows<DH, T>(v_of(stage), kTileKeys, a.dh, a.q,
                             [&](int i) { return key_in(key0 + i) ? at.v + (ks.at + key0 + i) * a.ld_v : nullptr; });
            if (threadIdx.x < kTileKeys) bias[stage][threadIdx.x] = key_in(key0 + threadIdx.x) ? 0.f : -INFINITY;
        };
        const int64_t tiles = (ks.len + kTileKeys - 1) / kTileKeys;
        load_keys(0, 0);
        copies_done();
        float dq[DH / 8][4], lse2[2] = {}, delta[2] = {};
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) dq[j][i] = 0.f;
        for (int64_t t = 0; t < tiles; ++t) {
            const int stage = (int)t & 1;
            if (t + 1 < tiles) load_keys(t + 1, stage ^ 1);
            copies_done();
            const int blocks = ks.len - t * kTileKeys < kTileKeys ? (int)(ks.len - t * kTileKeys + 15) / 16 : 4;
            wait_copies<1>();
            __syncthreads();
            if (t == 0)
                row_terms<T>(lse2, delta, sdo, warp * 16, rows, a.dh, [&](int i) { return i < rows ? out(ro.at(i)) : nullptr; },
                             [&](int i) {
                                 const int2 r = ro.at(i);
                                 return __ldg(g.lse + (qs.at + ro.token + r.x) * a.heads + hk * a.group + r.y);
                             });
            if (warp * 16 < rows) {
                Operands f;
                Scores s, dp;
                scores<T>(s, sq, warp * 16, k_of(stage), blocks, bias[stage]);
                scores<T>(dp, sdo, warp * 16, v_of(stage), blocks, nullptr);
                slopes(s, dp, lse2, delta, c, blocks);
                to_operands<T>(f, dp);
                times_keys<T, DH>(dq, f, k_of(stage), blocks);
            }
            __syncthreads();
        }
        const RowsAt<T> to(at.dq, qs.at + ro.token, g.ld_dq, a.dh);
        put_rows<T, DH>(dq, a.scale, rows - warp * 16, a.dh, 0, DH / 16, [&](int i) { return to(ro.at(warp * 16 + i)); },
                        [&](int i) { return (i < 8 ? lse2[0] : lse2[1]) != INFINITY; });         // no key counts
    }
    if (last_cta()) wait_before();
}

// How a call runs
struct Plan {
    bool tc;             // tiles of the tensor cores
    bool brief;          // the same for many short sequences
    int pack, splits;
    size_t delta_bytes;
};
Plan plan_of(const AttendArgs& a) {
    Plan p;
    p.pack = tc_pack(a);
    // Both sides in us, 8 heads with keys of their own, bfloat16, one call after the other: 1
    // sequence of 128 queries x 256 keys, heads of 64 (of 128), 9.7 against k_attend_keys and _rows'
    // 17.8 (12.9 and 24.5), 64 of them 76 and 179 (112 and 446), 4 of 1024 x 1024 53 and 253.
    // (The bound on the rows is not moved for many keys, where it costs: of 16 000 keys 127 queries take
    // 859 in k_attend_rows, whose CTAs walk all of the keys, 128 here 108 (1255 and 259).)
    p.tc = a.Tq * p.pack / a.B >= 128 && a.Tk / a.B >= 256;
    p.delta_bytes = p.tc ? padded((size_t)a.Tq * a.heads * 4) : 0;
    // Sequences whose keys mostly are one chunk: 200 of 32 x 40, heads of 64, 35 against
    // k_attend_keys' 47, of 120 x 60 47 and 92; 40 of 40 x 16 14.0 and 11.1, of 64 x 64 15.9 and
    // 15.4; heads of 128 64 and 249, 14.9 and 31.  (It counts rows in 32 bits, and its tensor
    // maps need a key.)
    p.brief = !p.tc && a.Tk > 0 && p.pack == a.group && a.Tq * a.group / a.B >= 32 && a.Tk / a.B <= kTileKeys && a.Tq * a.group <= 0x7FFFFF00 &&
              a.B * a.kv_heads >= (a.dh > 64 ? 2 : 4) * a.num_sms;
    if (p.brief) {
        p.splits = 1;
        return p;
    }
    // Parts of the rows, where the tiles of keys leave SMs without a CTA
    const int keys = p.tc ? 128 : kTileKeys, rows = p.tc ? 128 : kTileRows;
    const int64_t tiles = a.Tk / keys > a.B ? a.Tk / keys : a.B, ctas = tiles * a.kv_heads;
    const int64_t row_tiles = a.Tq * a.group / a.B / rows;
    int64_t n = (p.tc ? 1 : 3) * a.num_sms / ctas;
    if (n > row_tiles / 2) n = row_tiles / 2;
    if (n > 64) n = 64;
    p.splits = (int)(n < 1 ? 1 : n);
    return p;
}

template <class T, int DH>
cudaError_t run(const AttendArgs& a, const AttendGrads& g, bool brief, int splits, float* part_dk, float* part_dv, cudaStream_t s) {
    cudaError_t e = allow_smem(k_attend_keys<T, DH>, KeyTiles<T, DH>::kSmem);
    if (e == cudaSuccess) e = allow_smem(k_attend_rows<T, DH>, RowTiles<T, DH>::kSmem);
    if (e != cudaSuccess) return e;
    if (brief)
        e = launch_attend_grad_short(a, g, s);
    else
        e = launch_next(k_attend_keys<T, DH>, dim3((unsigned)slots(a.Tk, a.B, 1, kTileLog), (unsigned)a.kv_heads, (unsigned)splits), dim3(128),
                    KeyTiles<T, DH>::kSmem, false, s, a, g, splits, part_dk, part_dv);
    if (e != cudaSuccess || a.Tk <= kTileKeys || a.Tq == 0) return e;
    const int64_t n = slots(a.Tq, a.B, a.group, kTileLog), most = (3 * a.num_sms + a.kv_heads - 1) / a.kv_heads;
    return launch_next(k_attend_rows<T, DH>, dim3((unsigned)(n < most ? n : most), (unsigned)a.kv_heads), dim3(128),
                       RowTiles<T, DH>::kSmem, true, s, a, g, n);
}

}  // namespace

size_t attend_grad_bytes(const AttendArgs& a) {
    const Plan p = plan_of(a);
    return p.delta_bytes + (p.splits == 1 ? 0 : (size_t)p.splits * a.Tk * a.kv_heads * a.dh * 8);
}

cudaError_t launch_attend_grad(const AttendArgs& a, const AttendGrads& g, uint8_t* work, cudaStream_t s) {
    const Plan p = plan_of(a);
    float* delta = (float*)work;
    float* part_dk = p.splits > 1 ? (float*)(work + p.delta_bytes) : nullptr;
    float* part_dv = p.splits > 1 ? part_dk + (size_t)p.splits * a.Tk * a.kv_heads * a.dh : nullptr;
    auto go = [&](auto t) {
        using T = decltype(t);
        const cudaError_t e = p.tc           ? launch_attend_grad_tc(a, g, p.pack, p.splits, delta, part_dk, part_dv, s)
                              : a.dh <= 32 ? run<T, 32>(a, g, p.brief, p.splits, part_dk, part_dv, s)
                              : a.dh <= 64 ? run<T, 64>(a, g, p.brief, p.splits, part_dk, part_dv, s)
                                           : run<T, 128>(a, g, p.brief, p.splits, part_dk, part_dv, s);
        if (e != cudaSuccess || p.splits == 1 || a.Tk == 0) return e;
        return launch_next(k_attend_keys_join<T>, dim3((unsigned)((a.Tk * a.kv_heads * a.dh + 1023) / 1024), 2u), dim3(256), 0, false, s,
                           a, g, p.splits, (const float*)part_dk, (const float*)part_dv);
    };
    return a.type == IFVS_T_F16 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ifvs
