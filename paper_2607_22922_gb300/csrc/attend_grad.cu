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

// The two scores of a warp's 16 rows and the tile's keys: a = rows of `qa` times keys
// `kb`, accumulated over DH.
template <class T, int DH>
__device__ __forceinline__ void scores(float (&s)[kTileKeys / 8][4], const Rows<DH>& q, int row, const Rows<DH>& k) {
#pragma unroll
    for (int j = 0; j < kTileKeys / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[j][i] = 0.f;
#pragma unroll
    for (int d = 0; d < DH / 16; ++d) {
        uint32_t f[4];
        q.a(f, row, d * 16);
#pragma unroll
        for (int j = 0; j < kTileKeys / 16; ++j) {
            uint32_t b[4];
            k.b_t(b, j * 16, d * 16);
            mma16816<T>(s[2 * j], f, b[0], b[1]);
            mma16816<T>(s[2 * j + 1], f, b[2], b[3]);
        }
    }
}

__device__ __forceinline__ bool bit(uint32_t lo, uint32_t hi, int key) { return ((key < 32 ? lo : hi) >> (key & 31)) & 1u; }

// p and ds of a warp's rows from the scores s and dp, in their places.  lse2: base-2
// log-sum-exp, -infinity for a row that does not count.
template <class T>
__device__ __forceinline__ void slopes(float (&s)[kTileKeys / 8][4], float (&dp)[kTileKeys / 8][4], const float (&lse2)[2],
                                       const float (&delta)[2], float c, uint32_t lo, uint32_t hi) {
    const int two = (threadIdx.x & 3) * 2;
#pragma unroll
    for (int j = 0; j < kTileKeys / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = bit(lo, hi, j * 8 + two + (i & 1)) && lse2[i >> 1] != -INFINITY;
            const float p = in ? ex2(fmaf(s[j][i], c, -lse2[i >> 1])) : 0.f;
            dp[j][i] = in ? p * (dp[j][i] - delta[i >> 1]) : 0.f;
            s[j][i] = p;
        }
}

// acc += x y: x [16 rows][64 keys] in registers, y the keys' rows
template <class T, int DH>
__device__ __forceinline__ void times_keys(float (&acc)[DH / 8][4], const float (&x)[kTileKeys / 8][4], const Rows<DH>& y) {
#pragma unroll
    for (int j = 0; j < kTileKeys / 16; ++j) {
        uint32_t f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            f[i] = pack2(make_float2(x[2 * j + (i >> 1)][(i & 1) * 2], x[2 * j + (i >> 1)][(i & 1) * 2 + 1]), T());
#pragma unroll
        for (int d = 0; d < DH / 16; ++d) {
            uint32_t b[4];
            y.b(b, j * 16, d * 16);
            mma16816<T>(acc[2 * d], f, b[0], b[1]);
            mma16816<T>(acc[2 * d + 1], f, b[2], b[3]);
        }
    }
}

// acc += x^T y: 16 of x's columns (keys) from `key`, x [64 rows][64 keys] and y [64 rows] in
// shared memory
template <class T, int DH>
__device__ __forceinline__ void transposed_times(float (&acc)[DH / 8][4], const Rows<kTileKeys>& x, int key, const Rows<DH>& y) {
#pragma unroll
    for (int r = 0; r < kTileRows / 16; ++r) {
        uint32_t f[4];
        x.a_t(f, r * 16, key);
#pragma unroll
        for (int d = 0; d < DH / 16; ++d) {
            uint32_t b[4];
            y.b(b, r * 16, d * 16);
            mma16816<T>(acc[2 * d], f, b[0], b[1]);
            mma16816<T>(acc[2 * d + 1], f, b[2], b[3]);
        }
    }
}

template <class T>
__device__ __forceinline__ void put_scores(const Rows<kTileKeys>& to, int row, const float (&x)[kTileKeys / 8][4]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int j = 0; j < kTileKeys / 8; ++j)
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(to.addr(row + (lane >> 2) + 8 * r, j * 8 + (lane & 3) * 2)),
                         "r"(pack2(make_float2(x[j][2 * r], x[j][2 * r + 1]), T()))
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
        lse2[r] = row + i < rows ? lse(row + i) * kLog2e : -INFINITY;
    }
}

// Stores a warp's 16 rows from registers, scaled
template <class T, int DH, class Row>
__device__ __forceinline__ void put_rows(const float (&acc)[DH / 8][4], float scale, int rows, int dh, const Row& to) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = (lane >> 2) + 8 * r;
        if (i >= rows) continue;
        T* p = to(i);
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
            if (j * 8 < dh)
                *reinterpret_cast<uint32_t*>(p + j * 8 + (lane & 3) * 2) =
                    pack2(make_float2(acc[j][2 * r] * scale, acc[j][2 * r + 1] * scale), T());
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
// A CTA takes 64 keys and one part of the rows of their group, 64 at a time: each of its 4
// warps makes p and ds of 16 rows, then adds 16 keys' sums over the 64 rows.
template <class T, int DH>
struct KeyTiles {
    Rows<DH> k, v, q, d_out;
    Rows<kTileKeys> p, ds;
    static constexpr uint32_t kBytes = Rows<DH>::kLd * 2 * 64;
    static constexpr size_t kSmem = 4 * kBytes + 2 * kTileRows * Rows<kTileKeys>::kLd * 2;
};

template <class T, int DH>
__global__ void __launch_bounds__(128) k_attend_keys(AttendArgs a, AttendGrads g, int splits, float* part_dk, float* part_dv) {
    extern __shared__ __align__(16) uint8_t raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y, split = blockIdx.z;
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const Slot slot = slot_of(a.kv_offsets, a.B, a.Tk, 1, kTileKeys, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t key0 = slot.tile * kTileKeys;
    // without keys the first tile still writes dq
    if (slot.tile < 0 || (key0 >= ks.len && slot.tile > 0)) return;
    const bool alone = ks.len <= kTileKeys;
    const int keys = ks.len - key0 < kTileKeys ? (int)(ks.len - key0) : kTileKeys;
    const Arrays<T> at(a, g, hk);

    KeyTiles<T, DH> sm;
    sm.k.at = smem32(raw);
    sm.v.at = sm.k.at + sm.kBytes;
    sm.q.at = sm.v.at + sm.kBytes;
    sm.d_out.at = sm.q.at + sm.kBytes;
    sm.p.at = sm.d_out.at + sm.kBytes;
    sm.ds.at = sm.p.at + kTileRows * Rows<kTileKeys>::kLd * 2;
    auto key_in = [&](int i) { return i < keys && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key0 + i) >= 0); };
    load_rows<DH, T>(sm.k, kTileKeys, a.dh, a.q, [&](int i) { return key_in(i) ? at.k + (ks.at + key0 + i) * a.ld_k : nullptr; });
    load_rows<DH, T>(sm.v, kTileKeys, a.dh, a.q, [&](int i) { return key_in(i) ? at.v + (ks.at + key0 + i) * a.ld_v : nullptr; });
    const uint32_t lo = __ballot_sync(0xFFFFFFFFu, key_in(lane)), hi = __ballot_sync(0xFFFFFFFFu, key_in(32 + lane));
    const float c = a.scale * kLog2e;

    float dk[DH / 8][4], dv[DH / 8][4];
#pragma unroll
    for (int j = 0; j < DH / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) dk[j][i] = dv[j][i] = 0.f;
    const int64_t n_rows = qs.len * a.group, tiles = (n_rows + kTileRows - 1) / kTileRows;
    const int64_t t0 = tiles * split / splits, t1 = tiles * (split + 1) / splits;
    for (int64_t t = t0; t < t1; ++t) {
        const int64_t row0 = t * kTileRows;
        const int rows = n_rows - row0 < kTileRows ? (int)(n_rows - row0) : kTileRows;
        const RowOf ro(row0, a.group);
        auto token = [&](int i) { return qs.at + ro.token_of(i); };
        auto head = [&](int i) { return (int64_t)ro.head_of(i) * a.dh; };
        load_rows<DH, T>(sm.q, kTileRows, a.dh, a.q, [&](int i) { return i < rows ? at.q + token(i) * a.ld_q + head(i) : nullptr; });
        load_rows<DH, T>(sm.d_out, kTileRows, a.dh, a.q,
                         [&](int i) { return i < rows ? at.d_out + token(i) * g.ld_d_out + head(i) : nullptr; });
        copies_done();
        wait_copies<0>();
        __syncthreads();
        {
            float s[kTileKeys / 8][4], dp[kTileKeys / 8][4];
            scores<T>(s, sm.q, warp * 16, sm.k);
            scores<T>(dp, sm.d_out, warp * 16, sm.v);
            float lse2[2], delta[2];
            if (alone) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float top = -INFINITY;
#pragma unroll
                    for (int j = 0; j < kTileKeys / 8; ++j)
#pragma unroll
                        for (int i = 2 * r; i < 2 * r + 2; ++i)
                            if (bit(lo, hi, j * 8 + (lane & 3) * 2 + (i & 1))) top = fmaxf(top, s[j][i]);
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2)) * c;
                    const float base = top == -INFINITY ? 0.f : top;
                    float l = 0.f, sum = 0.f;
#pragma unroll
                    for (int j = 0; j < kTileKeys / 8; ++j)
#pragma unroll
                        for (int i = 2 * r; i < 2 * r + 2; ++i)
                            if (bit(lo, hi, j * 8 + (lane & 3) * 2 + (i & 1))) {
                                const float e = ex2(fmaf(s[j][i], c, -base));
                                l += e;
                                sum = fmaf(e, dp[j][i], sum);
                            }
#pragma unroll
                    for (int x = 1; x <= 2; x <<= 1) {
                        l += __shfl_xor_sync(0xFFFFFFFFu, l, x);
                        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
                    }
                    const bool in = warp * 16 + (lane >> 2) + 8 * r < rows && l != 0.f;
                    lse2[r] = in ? base + log2f(l) : -INFINITY;
                    delta[r] = in ? sum / l : 0.f;
                }
            } else {
                row_terms<T>(lse2, delta, sm.d_out, warp * 16, rows, a.dh,
                             [&](int i) { return i < rows ? at.out + token(i) * g.ld_out + head(i) : nullptr; },
                             [&](int i) { return __ldg(g.lse + token(i) * a.heads + hk * a.group + ro.head_of(i)); });
            }
            slopes<T>(s, dp, lse2, delta, c, lo, hi);
            put_scores<T>(sm.p, warp * 16, s);
            put_scores<T>(sm.ds, warp * 16, dp);
            if (alone) {
                float dq[DH / 8][4];
#pragma unroll
                for (int j = 0; j < DH / 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) dq[j][i] = 0.f;
                times_keys<T, DH>(dq, dp, sm.k);
                put_rows<T, DH>(dq, a.scale, rows - warp * 16, a.dh,
                                [&](int i) { return at.dq + token(warp * 16 + i) * g.ld_dq + head(warp * 16 + i); });
            }
        }
        __syncthreads();
        transposed_times<T, DH>(dv, sm.p, warp * 16, sm.d_out);
        transposed_times<T, DH>(dk, sm.ds, warp * 16, sm.q);
        __syncthreads();
    }
    copies_done();
    wait_copies<0>();
    const int mine = keys - warp * 16;
    if (splits == 1) {
        put_rows<T, DH>(dk, a.scale, mine, a.dh, [&](int i) { return at.dk + (ks.at + key0 + warp * 16 + i) * g.ld_dk; });
        put_rows<T, DH>(dv, 1.f, mine, a.dh, [&](int i) { return at.dv + (ks.at + key0 + warp * 16 + i) * g.ld_dv; });
        return;
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int i = (lane >> 2) + 8 * r;
        if (i >= mine) continue;
        const int64_t to = (((int64_t)split * a.Tk + ks.at + key0 + warp * 16 + i) * a.kv_heads + hk) * a.dh + (lane & 3) * 2;
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
            if (j * 8 < a.dh) {
                *reinterpret_cast<float2*>(part_dk + to + j * 8) = make_float2(dk[j][2 * r] * a.scale, dk[j][2 * r + 1] * a.scale);
                *reinterpret_cast<float2*>(part_dv + to + j * 8) = make_float2(dv[j][2 * r], dv[j][2 * r + 1]);
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
template <class T, int DH>
struct RowTiles {
    Rows<DH> q, d_out, k[2], v[2];
    static constexpr uint32_t kBytes = Rows<DH>::kLd * 2 * 64;
    static constexpr size_t kSmem = 6 * kBytes;
};

template <class T, int DH>
__global__ void __launch_bounds__(128) k_attend_rows(AttendArgs a, AttendGrads g) {
    extern __shared__ __align__(16) uint8_t raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y;
    const Slot slot = slot_of(a.q_offsets, a.B, a.Tq, a.group, kTileRows, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t row0 = slot.tile * kTileRows, left = qs.len * a.group - row0;
    if (slot.tile < 0 || left <= 0 || ks.len <= kTileKeys) return;
    const int rows = left < kTileRows ? (int)left : kTileRows;
    const RowOf ro(row0, a.group);
    const Arrays<T> at(a, g, hk);
    auto token = [&](int i) { return qs.at + ro.token_of(i); };
    auto head = [&](int i) { return (int64_t)ro.head_of(i) * a.dh; };
    RowTiles<T, DH> sm;
    sm.q.at = smem32(raw);
    sm.d_out.at = sm.q.at + sm.kBytes;
    for (int i = 0; i < 2; ++i) {
        sm.k[i].at = sm.q.at + (2 + 2 * i) * sm.kBytes;
        sm.v[i].at = sm.k[i].at + sm.kBytes;
    }
    load_rows<DH, T>(sm.q, kTileRows, a.dh, a.q, [&](int i) { return i < rows ? at.q + token(i) * a.ld_q + head(i) : nullptr; });
    load_rows<DH, T>(sm.d_out, kTileRows, a.dh, a.q,
                     [&](int i) { return i < rows ? at.d_out + token(i) * g.ld_d_out + head(i) : nullptr; });
    auto key_in = [&](int64_t key) { return key < ks.len && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key) >= 0); };
    auto load_keys = [&](int64_t tile, int stage) {
        const int64_t key0 = tile * kTileKeys;
        load_rows<DH, T>(sm.k[stage], kTileKeys, a.dh, a.q, [&](int i) { return key_in(key0 + i) ? at.k + (ks.at + key0 + i) * a.ld_k : nullptr; });
        load_rows<DH, T>(sm.v[stage], kTileKeys, a.dh, a.q, [&](int i) { return key_in(key0 + i) ? at.v + (ks.at + key0 + i) * a.ld_v : nullptr; });
    };
    const int64_t tiles = (ks.len + kTileKeys - 1) / kTileKeys;
    load_keys(0, 0);
    copies_done();
    float dq[DH / 8][4], lse2[2] = {}, delta[2] = {};
#pragma unroll
    for (int j = 0; j < DH / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) dq[j][i] = 0.f;
    const float c = a.scale * kLog2e;
    for (int64_t t = 0; t < tiles; ++t) {
        const int stage = (int)t & 1;
        if (t + 1 < tiles) load_keys(t + 1, stage ^ 1);
        copies_done();
        wait_copies<1>();
        __syncthreads();
        if (t == 0)
            row_terms<T>(lse2, delta, sm.d_out, warp * 16, rows, a.dh,
                         [&](int i) { return i < rows ? at.out + token(i) * g.ld_out + head(i) : nullptr; },
                         [&](int i) { return __ldg(g.lse + token(i) * a.heads + hk * a.group + ro.head_of(i)); });
        const uint32_t lo = __ballot_sync(0xFFFFFFFFu, key_in(t * kTileKeys + lane)),
                       hi = __ballot_sync(0xFFFFFFFFu, key_in(t * kTileKeys + 32 + lane));
        float s[kTileKeys / 8][4], dp[kTileKeys / 8][4];
        scores<T>(s, sm.q, warp * 16, sm.k[stage]);
        scores<T>(dp, sm.d_out, warp * 16, sm.v[stage]);
        slopes<T>(s, dp, lse2, delta, c, lo, hi);
        times_keys<T, DH>(dq, dp, sm.k[stage]);
        __syncthreads();
    }
    put_rows<T, DH>(dq, a.scale, rows - warp * 16, a.dh,
                    [&](int i) { return at.dq + token(warp * 16 + i) * g.ld_dq + head(warp * 16 + i); });
}

// How a call runs
struct Plan {
    bool tc;             // tiles of the tensor cores
    int pack, splits;
    size_t delta_bytes;
};
Plan plan_of(const AttendArgs& a) {
    Plan p;
    p.pack = tc_pack(a);
    p.tc = a.Tq * p.pack / a.B >= 128 && a.Tk / a.B >= 256;
    p.delta_bytes = p.tc ? padded((size_t)a.Tq * a.heads * 4) : 0;
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
cudaError_t run(const AttendArgs& a, const AttendGrads& g, int splits, float* part_dk, float* part_dv, cudaStream_t s) {
    cudaError_t e = allow_smem(k_attend_keys<T, DH>, KeyTiles<T, DH>::kSmem);
    if (e == cudaSuccess) e = allow_smem(k_attend_rows<T, DH>, RowTiles<T, DH>::kSmem);
    if (e != cudaSuccess) return e;
    e = launch_next(k_attend_keys<T, DH>, dim3((unsigned)slots(a.Tk, a.B, 1, kTileKeys), (unsigned)a.kv_heads, (unsigned)splits), dim3(128),
                    KeyTiles<T, DH>::kSmem, false, s, a, g, splits, part_dk, part_dv);
    if (e != cudaSuccess || a.Tk <= kTileKeys || a.Tq == 0) return e;
    return launch_next(k_attend_rows<T, DH>, dim3((unsigned)slots(a.Tq, a.B, a.group, kTileRows), (unsigned)a.kv_heads), dim3(128),
                       RowTiles<T, DH>::kSmem, false, s, a, g);
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
                              : a.dh <= 32 ? run<T, 32>(a, g, p.splits, part_dk, part_dv, s)
                              : a.dh <= 64 ? run<T, 64>(a, g, p.splits, part_dk, part_dv, s)
                                           : run<T, 128>(a, g, p.splits, part_dk, part_dv, s);
        if (e != cudaSuccess || p.splits == 1 || a.Tk == 0) return e;
        return launch_next(k_attend_keys_join<T>, dim3((unsigned)((a.Tk * a.kv_heads * a.dh + 1023) / 1024), 2u), dim3(256), 0, false, s,
                           a, g, p.splits, (const float*)part_dk, (const float*)part_dv);
    };
    return a.type == IFVS_T_F16 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ifvs
