// Attention of packed sequences (ifvs_attend).
//
//   s = scale q k, p = softmax(s) over the sequence's keys that are no padding,
//   out = p v, lse = log sum exp s
//
// One pass over the keys: a running maximum m and sum l of exp(s - m) in float32, the
// output rescaled where m grows.  exp(s - m), at most 1, is rounded to the arrays' type
// because the tensor cores multiply 16-bit operands; l sums the unrounded values.
#include "attend_tc.cuh"

namespace ifvs {

namespace {

// ---- tiles of warps: any lengths ---------------------------------------------------------
// A CTA takes 64 rows of one group and the keys of one split, 64 at a time; each of its 4
// warps holds 16 rows' output in registers.
template <class T, int DH>
struct WarpTiles {
    Rows<DH> q, k[2], v[2];
    static constexpr uint32_t kRowsBytes = Rows<DH>::kLd * 2;
    static constexpr size_t kSmem = (kTileRows + 4 * kTileKeys) * kRowsBytes;
};

template <class T, int DH>
__global__ void __launch_bounds__(128) k_attend(AttendArgs a, AttendOut o, int splits, float* part_out, float* part_lse) {
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ uint32_t valid_bits[2][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y, split = blockIdx.z;
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const Slot slot = slot_of(a.q_offsets, a.B, a.Tq, a.group, kTileRows, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t row0 = slot.tile * kTileRows, left = qs.len * a.group - row0;
    if (slot.tile < 0 || left <= 0) return;
    const int rows = left < kTileRows ? (int)left : kTileRows;
    const RowOf at(row0, a.group);
    // this split's keys, whole tiles
    const int64_t tiles = (ks.len + kTileKeys - 1) / kTileKeys;
    const int64_t t0 = tiles * split / splits, t1 = tiles * (split + 1) / splits;

    WarpTiles<T, DH> sm;
    sm.q.at = smem32(raw);
    for (int i = 0; i < 2; ++i) {
        sm.k[i].at = sm.q.at + (kTileRows + 2 * i * kTileKeys) * sm.kRowsBytes;
        sm.v[i].at = sm.k[i].at + kTileKeys * sm.kRowsBytes;
    }
    const T *q = (const T*)a.q + (int64_t)hk * a.group * a.dh, *k = (const T*)a.k + (int64_t)hk * a.dh,
            *v = (const T*)a.v + (int64_t)hk * a.dh;
    load_rows<DH, T>(sm.q, kTileRows, a.dh, a.q, [&](int i) {
        return i < rows ? q + (qs.at + at.token_of(i)) * a.ld_q + (int64_t)at.head_of(i) * a.dh : nullptr;
    });
    auto key_in = [&](int64_t key) { return key < ks.len && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key) >= 0); };
    auto load_keys = [&](int64_t tile, int stage) {
        const int64_t key0 = tile * kTileKeys;
        load_rows<DH, T>(sm.k[stage], kTileKeys, a.dh, a.q, [&](int i) { return key_in(key0 + i) ? k + (ks.at + key0 + i) * a.ld_k : nullptr; });
        load_rows<DH, T>(sm.v[stage], kTileKeys, a.dh, a.q, [&](int i) { return key_in(key0 + i) ? v + (ks.at + key0 + i) * a.ld_v : nullptr; });
        if (warp < 2) {
            const uint32_t bits = __ballot_sync(0xFFFFFFFFu, key_in(key0 + warp * 32 + lane));
            if (lane == 0) valid_bits[stage][warp] = bits;
        }
    };
    if (t0 < t1) load_keys(t0, 0);
    copies_done();

    float acc[DH / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < DH / 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    uint32_t qf[DH / 16][4];
    const float c = a.scale * kLog2e;
    const bool active = warp * 16 < rows;
    for (int64_t t = t0; t < t1; ++t) {
        const int stage = (int)(t - t0) & 1;
        if (t + 1 < t1) load_keys(t + 1, stage ^ 1);
        copies_done();
        wait_copies<1>();
        __syncthreads();
        if (active) {
            if (t == t0)
#pragma unroll
                for (int d = 0; d < DH / 16; ++d) sm.q.a(qf[d], warp * 16, d * 16);
            float s[kTileKeys / 8][4];
#pragma unroll
            for (int j = 0; j < kTileKeys / 8; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[j][i] = 0.f;
#pragma unroll
            for (int d = 0; d < DH / 16; ++d)
#pragma unroll
                for (int j = 0; j < kTileKeys / 16; ++j) {
                    uint32_t b[4];
                    sm.k[stage].b_t(b, j * 16, d * 16);
                    mma16816<T>(s[2 * j], qf[d], b[0], b[1]);
                    mma16816<T>(s[2 * j + 1], qf[d], b[2], b[3]);
                }
            const uint32_t lo = valid_bits[stage][0], hi = valid_bits[stage][1];
            if ((lo & hi) != 0xFFFFFFFFu)
#pragma unroll
                for (int j = 0; j < kTileKeys / 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = j * 8 + (lane & 3) * 2 + (i & 1);
                        if (!(((key < 32 ? lo : hi) >> (key & 31)) & 1u)) s[j][i] = -INFINITY;
                    }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < kTileKeys / 8; ++j) top = fmaxf(top, fmaxf(s[j][2 * r], s[j][2 * r + 1]));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                top = fmaxf(m[r], top * c);
                const float base = top == -INFINITY ? 0.f : top, shrink = ex2(m[r] - base);
                m[r] = top;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < kTileKeys / 8; ++j)
#pragma unroll
                    for (int i = 2 * r; i < 2 * r + 2; ++i) {
                        s[j][i] = ex2(fmaf(s[j][i], c, -base));
                        sum += s[j][i];
                    }
                l[r] = l[r] * shrink + sum;
#pragma unroll
                for (int j = 0; j < DH / 8; ++j) {
                    acc[j][2 * r] *= shrink;
                    acc[j][2 * r + 1] *= shrink;
                }
            }
#pragma unroll
            for (int j = 0; j < kTileKeys / 16; ++j) {
                uint32_t p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    p[i] = pack2(make_float2(s[2 * j + (i >> 1)][(i & 1) * 2], s[2 * j + (i >> 1)][(i & 1) * 2 + 1]), T());
#pragma unroll
                for (int d = 0; d < DH / 16; ++d) {
                    uint32_t b[4];
                    sm.v[stage].b(b, j * 16, d * 16);
                    mma16816<T>(acc[2 * d], p, b[0], b[1]);
                    mma16816<T>(acc[2 * d + 1], p, b[2], b[3]);
                }
            }
        }
        __syncthreads();
    }
    wait_copies<0>();
    __syncthreads();
    if (!active) return;
    float inv[2], ln[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], 1);
        l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], 2);
        inv[r] = l[r] == 0.f ? 0.f : 1.f / l[r];          // 0: no key
        ln[r] = l[r] == 0.f ? -INFINITY : m[r] + log2f(l[r]);
    }
    const int g = lane >> 2, two = (lane & 3) * 2;
    if (splits > 1) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int i = warp * 16 + g + 8 * r;
            if (i >= rows) continue;
            const int64_t to = ((int64_t)split * a.Tq + qs.at + at.token_of(i)) * a.heads + hk * a.group + at.head_of(i);
#pragma unroll
            for (int j = 0; j < DH / 8; ++j)
                if (j * 8 < a.dh)
                    *reinterpret_cast<float2*>(part_out + to * a.dh + j * 8 + two) =
                        make_float2(acc[j][2 * r] * inv[r], acc[j][2 * r + 1] * inv[r]);
            if ((lane & 3) == 0) part_lse[to] = ln[r];
        }
        return;
    }
    // through this warp's rows of the query tile, so that rows are written 16 bytes a lane
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(sm.q.addr(warp * 16 + g + 8 * r, j * 8 + two)),
                         "r"(pack2(make_float2(acc[j][2 * r] * inv[r], acc[j][2 * r + 1] * inv[r]), T()))
                         : "memory");
    __syncwarp();
    T* out = (T*)o.out + (int64_t)hk * a.group * a.dh;
    for (int i = lane; i < 16 * (DH / 8); i += 32) {
        const int r = warp * 16 + i / (DH / 8), d = i % (DH / 8) * 8;
        if (r >= rows || d >= a.dh) continue;
        uint4 w;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(sm.q.addr(r, d)) : "memory");
        *reinterpret_cast<uint4*>(out + (qs.at + at.token_of(r)) * o.ld + (int64_t)at.head_of(r) * a.dh + d) = w;
    }
    if (o.lse && (lane & 3) == 0)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int i = warp * 16 + g + 8 * r;
            if (i < rows) o.lse[(qs.at + at.token_of(i)) * a.heads + hk * a.group + at.head_of(i)] = ln[r] * kLn2;
        }
}

// Joins the splits of every row, in order: a warp per (token, head).
template <class T>
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs a, AttendOut o, int splits, const float* part_out, const float* part_lse) {
    wait_before();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), n = a.Tq * a.heads;
    if (row >= n) return;
    float top = -INFINITY;
    for (int s = 0; s < splits; ++s) top = fmaxf(top, __ldcg(part_lse + s * n + row));
    const float base = top == -INFINITY ? 0.f : top;
    const int64_t token = row / a.heads;
    T* out = (T*)o.out + token * o.ld + (row - token * a.heads) * a.dh;
    float l = 0.f;
    for (int s = 0; s < splits; ++s) l += ex2(__ldcg(part_lse + s * n + row) - base);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    for (int d = lane * 4; d < a.dh; d += 128) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
            const float w = ex2(__ldcg(part_lse + s * n + row) - base) * inv;
            const float4 p = __ldcg(reinterpret_cast<const float4*>(part_out + (s * n + row) * a.dh + d));
            sum.x = fmaf(w, p.x, sum.x);
            sum.y = fmaf(w, p.y, sum.y);
            sum.z = fmaf(w, p.z, sum.z);
            sum.w = fmaf(w, p.w, sum.w);
        }
        *reinterpret_cast<uint2*>(out + d) = make_uint2(pack2(make_float2(sum.x, sum.y), T()), pack2(make_float2(sum.z, sum.w), T()));
    }
    if (o.lse && lane == 0) o.lse[row] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
}

// How a call runs
struct Plan {
    bool tc;             // tiles of the tensor cores
    int pack, splits;
};
Plan plan_of(const AttendArgs& a) {
    Plan p;
    p.pack = tc_pack(a);
    p.tc = a.Tq * p.pack / a.B >= 128 && a.Tk / a.B >= 256;
    // Parts of the keys, where the rows leave SMs without a CTA: at least two tiles of the
    // average sequence each.
    const int group = p.tc ? p.pack : a.group, rows = p.tc ? 256 : kTileRows, keys = p.tc ? 128 : kTileKeys;
    const int64_t row_tiles = (a.Tq * group + rows - 1) / rows;
    const int64_t ctas = (row_tiles > a.B ? row_tiles : a.B) * (a.heads / group), tiles = a.Tk / a.B / keys;
    int64_t n = (p.tc ? 1 : 3) * a.num_sms / ctas;
    if (n > tiles / 2) n = tiles / 2;
    if (n > 64) n = 64;
    p.splits = (int)(n < 1 ? 1 : n);
    return p;
}

template <class T, int DH>
cudaError_t run(const AttendArgs& a, const AttendOut& o, int splits, float* part_out, float* part_lse, cudaStream_t s) {
    constexpr size_t smem = WarpTiles<T, DH>::kSmem;
    const cudaError_t e = allow_smem(k_attend<T, DH>, smem);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)slots(a.Tq, a.B, a.group, kTileRows), (unsigned)a.kv_heads, (unsigned)splits);
    return launch_next(k_attend<T, DH>, grid, dim3(128), smem, false, s, a, o, splits, part_out, part_lse);
}

}  // namespace

size_t attend_bytes(const AttendArgs& a) {
    const int splits = plan_of(a).splits;
    return splits == 1 ? 0 : padded((size_t)splits * a.Tq * a.heads * a.dh * 4) + padded((size_t)splits * a.Tq * a.heads * 4);
}

cudaError_t launch_attend(const AttendArgs& a, const AttendOut& o, uint8_t* work, cudaStream_t s) {
    const Plan p = plan_of(a);
    float *part_out = nullptr, *part_lse = nullptr;
    if (p.splits > 1) {
        part_out = (float*)work;
        part_lse = (float*)(work + padded((size_t)p.splits * a.Tq * a.heads * a.dh * 4));
    }
    auto go = [&](auto t) {
        using T = decltype(t);
        const cudaError_t e = p.tc           ? launch_attend_tc(a, o, p.pack, p.splits, part_out, part_lse, s)
                              : a.dh <= 32 ? run<T, 32>(a, o, p.splits, part_out, part_lse, s)
                              : a.dh <= 64 ? run<T, 64>(a, o, p.splits, part_out, part_lse, s)
                                           : run<T, 128>(a, o, p.splits, part_out, part_lse, s);
        if (e != cudaSuccess || p.splits == 1 || a.Tq == 0) return e;
        return launch_next(k_attend_join<T>, dim3((unsigned)((a.Tq * a.heads + 7) / 8)), dim3(256), 0, true, s, a, o, p.splits,
                           (const float*)part_out, (const float*)part_lse);
    };
    return a.type == IFVS_T_F16 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ifvs
