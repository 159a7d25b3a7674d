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
// A CTA of 4 warps takes up to 2^log_rows rows of one group and the keys of one split.  Up to 128
// keys stay in shared memory, and the warps go through tiles of 16 rows by themselves, the
// next tile's queries on their way; more keys pass 64 at a time, for 64 rows at a time.  200
// sequences of 32 queries and 40 keys, 8 heads of 64, take 18 us (1.6 TB/s): the chain of a
// CTA's loads, products and stores, of which an SM has four at a time.
constexpr int kWarps = 4, kResident = 128;

template <class T, int DH>
struct WarpTiles {
    static constexpr uint32_t kRowBytes = Rows<DH>::kLd * 2;
    static constexpr size_t kSmem = (2 * kResident + kWarps * 32) * kRowBytes;
    Rows<DH> k, v, q;        // kResident rows of keys and values; this warp's two tiles of queries
    __device__ __forceinline__ explicit WarpTiles(const void* smem) {
        k.at = smem32(smem);
        v.at = k.at + kResident * kRowBytes;
        q.at = v.at + (kResident + (threadIdx.x >> 5) * 32) * kRowBytes;
    }
};

// A warp's 16 rows on their way through the keys
template <class T, int DH>
struct Running {
    float acc[DH / 8][4], m[2], l[2];
    uint32_t q[DH / 16][4];
    __device__ __forceinline__ void begin(const Rows<DH>& from, int row) {
#pragma unroll
        for (int d = 0; d < DH / 16; ++d) from.a(q[d], row, d * 16);
        clear();
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
    }
    // up to 16 B keys from row `at` of k and v, `blocks` of 16; bias: 0, or -infinity for a key
    // that does not count, where its score's sum begins.  first: nothing came before.
    template <int B = kTileKeys / 16>
    __device__ __forceinline__ void step(const Rows<DH>& k, const Rows<DH>& v, int at, int blocks, const float* bias, float c, bool first) {
        const int lane = threadIdx.x & 31;
        float2 s[2 * B][2];
#pragma unroll
        for (int j = 0; j < B; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                s[2 * j + i][0] = s[2 * j + i][1] = *reinterpret_cast<const float2*>(bias + at + (2 * j + i) * 8 + (lane & 3) * 2);
            if (j < blocks)
#pragma unroll
                for (int d = 0; d < DH / 16; ++d) {
                    uint32_t b[4];
                    k.b_t(b, at + j * 16, d * 16);
                    mma16816<T>(reinterpret_cast<float(&)[4]>(s[2 * j]), q[d], b[0], b[1]);
                    mma16816<T>(reinterpret_cast<float(&)[4]>(s[2 * j + 1]), q[d], b[2], b[3]);
                }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float top = fmaxf(s[0][r].x, s[0][r].y);
#pragma unroll
            for (int j = 1; j < 2 * B; ++j) top = fmaxf(top, fmaxf(s[j][r].x, s[j][r].y));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            top = fmaxf(m[r], top * c);
            const float base = top == -INFINITY ? 0.f : top;
            const float2 c2 = make_float2(c, c), b2 = make_float2(-base, -base);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < 2 * B; ++j)
                if (j / 2 < blocks) {
                    float2 e = fma_(s[j][r], c2, b2);
                    e.x = ex2(e.x);
                    e.y = ex2(e.y);
                    s[j][r] = e;
                    sum = add_(sum, e);
                }
            if (first) {
                l[r] = total(sum);
            } else {
                const float shrink = ex2(m[r] - base);
                l[r] = l[r] * shrink + total(sum);
#pragma unroll
                for (int j = 0; j < DH / 8; ++j) {
                    acc[j][2 * r] *= shrink;
                    acc[j][2 * r + 1] *= shrink;
                }
            }
            m[r] = top;
        }
#pragma unroll
        for (int j = 0; j < B; ++j)
            if (j < blocks) {
                uint32_t p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = pack2(s[2 * j + (i >> 1)][i & 1], T());
#pragma unroll
                for (int d = 0; d < DH / 16; ++d) {
                    uint32_t b[4];
                    v.b(b, at + j * 16, d * 16);
                    mma16816<T>(acc[2 * d], p, b[0], b[1]);
                    mma16816<T>(acc[2 * d + 1], p, b[2], b[3]);
                }
            }
    }
    // 1 / l and the base-2 logarithm of the sum, of rows lane / 4 and + 8
    __device__ __forceinline__ void close(float (&inv)[2], float (&ln)[2]) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], 1);
            l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], 2);
            inv[r] = l[r] == 0.f ? 0.f : 1.f / l[r];          // 0: no key
            ln[r] = l[r] == 0.f ? -INFINITY : m[r] + log2f(l[r]);
        }
    }
};

template <class T, int DH>
__global__ void __launch_bounds__(kWarps * 32, DH == 128 ? 2 : 4)
k_attend(AttendArgs a, AttendOut o, int log_rows, int splits, float* part_out, float* part_lse) {
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ __align__(8) float bias[kResident];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y, split = blockIdx.z;
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const Slot slot = slot_of(a.q_offsets, a.B, a.Tq, a.group, log_rows, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t row0 = slot.tile << log_rows, left = qs.len * a.group - row0;
    if (slot.tile < 0 || left <= 0) return;
    const int rows = left < 1 << log_rows ? (int)left : 1 << log_rows;
    const RowOf ro(row0, a.group);
    // this split's keys, whole tiles
    const int64_t tiles = (ks.len + kTileKeys - 1) / kTileKeys;
    const int64_t t0 = tiles * split / splits, t1 = tiles * (split + 1) / splits;
    const WarpTiles<T, DH> sm(raw);
    const T *k = (const T*)a.k + (int64_t)hk * a.dh, *v = (const T*)a.v + (int64_t)hk * a.dh;
    const RowsAt<const T> q((const T*)a.q + (int64_t)hk * a.group * a.dh, qs.at + ro.token, a.ld_q, a.dh);
    const RowsAt<T> out((T*)o.out + (int64_t)hk * a.group * a.dh, qs.at + ro.token, o.ld, a.dh);
    // a row's place in arrays [Tq][heads]
    auto head_row = [&](int i) {
        const int2 r = ro.at(i);
        return (qs.at + ro.token + r.x) * a.heads + hk * a.group + r.y;
    };
    auto key_in = [&](int64_t key) { return key < ks.len && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key) >= 0); };
    // n keys from key0 on to row `to`, and the bias of up to 64 or all.  Whether one counts that
    // this thread has seen.
    auto load_keys = [&](int64_t key0, int n, int to) {
        bool some = false;
        const Rows<DH> dk{sm.k.addr(to, 0)}, dv{sm.v.addr(to, 0)};
        load_rows<DH, T>(dk, n, a.dh, a.q, [&](int i) { return key_in(key0 + i) ? k + (ks.at + key0 + i) * a.ld_k : nullptr; });
        load_rows<DH, T>(dv, n, a.dh, a.q, [&](int i) { return key_in(key0 + i) ? v + (ks.at + key0 + i) * a.ld_v : nullptr; });
        for (int i = threadIdx.x; i < (n + 63) / 64 * 64; i += kWarps * 32) {
            const bool in = i < n && key_in(key0 + i);
            bias[to + i] = in ? 0.f : -INFINITY;
            some = some || in;
        }
        return some;
    };
    // this warp's 16 rows from `row` on, to its buffer `to`
    auto load_queries = [&](int row, int to) {
        constexpr int C = DH / 8;
#pragma unroll 4
        for (int i = lane; i < 16 * C; i += 32) {
            const int r = row + i / C, d = i % C * 8;
            const bool in = r < rows && d < a.dh;
            copy16(sm.q.addr(to * 16 + i / C, d), in ? (const void*)(q(ro.at(r)) + d) : a.q, in);
        }
    };
    const float c = a.scale * kLog2e;
    const int g = lane >> 2, two = (lane & 3) * 2;
    Running<T, DH> run;
    // writes the 16 rows from `row` on, through this warp's buffer `by`; some: whether a key counts
    // (queries that are not finite have NaN as their scores, whatever the bias)
    auto put = [&](int row, int by, bool some) {
        float inv[2], ln[2];
        if (!some) run.clear();
        run.close(inv, ln);
        if (splits > 1) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = row + g + 8 * r;
                if (i >= rows) continue;
                const int64_t to = (int64_t)split * a.Tq * a.heads + head_row(i);
#pragma unroll
                for (int j = 0; j < DH / 8; ++j)
                    if (j * 8 < a.dh)
                        *reinterpret_cast<float2*>(part_out + to * a.dh + j * 8 + two) =
                            make_float2(run.acc[j][2 * r] * inv[r], run.acc[j][2 * r + 1] * inv[r]);
                if ((lane & 3) == 0) part_lse[to] = ln[r];
            }
            return;
        }
        __syncwarp();
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int j = 0; j < DH / 8; ++j)
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(sm.q.addr(by * 16 + g + 8 * r, j * 8 + two)),
                             "r"(pack2(make_float2(run.acc[j][2 * r] * inv[r], run.acc[j][2 * r + 1] * inv[r]), T()))
                             : "memory");
        __syncwarp();
        constexpr int C = DH / 8;
#pragma unroll 4
        for (int i = lane; i < 16 * C; i += 32) {
            const int r = row + i / C, d = i % C * 8;
            if (r >= rows || d >= a.dh) continue;
            uint4 w;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                         : "r"(sm.q.addr(by * 16 + i / C, d))
                         : "memory");
            __stcs(reinterpret_cast<uint4*>(out(ro.at(r)) + d), w);
        }
        if (o.lse && (lane & 3) == 0)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = row + g + 8 * r;
                if (i < rows) o.lse[head_row(i)] = ln[r] * kLn2;
            }
        __syncwarp();
    };

    const int64_t key0 = t0 * kTileKeys, key1 = t1 * kTileKeys < ks.len ? t1 * kTileKeys : ks.len;
    if (key1 - key0 <= kResident) {
        const int n = key1 > key0 ? (int)(key1 - key0) : 0, blocks = (n + 15) / 16;
        const bool seen = load_keys(key0, blocks * 16, 0);
        load_queries(warp * 16, 0);
        copies_done();
        wait_copies<0>();
        const bool some = __syncthreads_or(seen);
        int by = 0;
        for (int row = warp * 16; row < rows; row += kWarps * 16, by ^= 1) {
            if (row + kWarps * 16 < rows) load_queries(row + kWarps * 16, by ^ 1);
            copies_done();
            wait_copies<1>();
            __syncwarp();
            run.begin(sm.q, by * 16);
            for (int at = 0; at < blocks; at += 4) run.step(sm.k, sm.v, at * 16, min(blocks - at, 4), bias, c, at == 0);
            put(row, by, some);
        }
        return;
    }
    for (int row0 = 0; row0 < rows; row0 += kWarps * 16) {
        const int row = row0 + warp * 16;
        load_queries(row, 0);
        bool seen = load_keys(key0, kTileKeys, 0);
        copies_done();
        for (int64_t t = t0; t < t1; ++t) {
            const int stage = (int)(t - t0) & 1;
            if (t + 1 < t1) seen |= load_keys((t + 1) * kTileKeys, kTileKeys, (stage ^ 1) * kTileKeys);
            copies_done();
            wait_copies<1>();
            __syncthreads();
            if (t == t0) run.begin(sm.q, 0);
            if (row < rows) run.step(sm.k, sm.v, stage * kTileKeys, 4, bias, c, t == t0);
            __syncthreads();
        }
        const bool some = __syncthreads_or(seen);
        if (row < rows) put(row, 0, some);
    }
}

// ---- a few rows and many keys ---------------------------------------------------------------
// The call reads its keys and values once and is bound by that.  A CTA takes up to 16 rows of a
// group, which one tile of the products holds, and the keys of one split; each of its 4 warps
// takes every fourth chunk of 32 keys through a ring of its own, two chunks ahead, so that no
// warp waits for another before the end, where their sums are joined in shared memory.
// 8 sequences of one query and about 16 400 keys, 8 heads of 64 in float16: 55 us with the
// join, where 64 keys at a time for the whole CTA take 82.
constexpr int kFewRows = 16, kFewLog = 4, kFewKeys = 32, kFewStages = 3;

template <class T, int DH>
struct FewTiles {
    static constexpr uint32_t kRowBytes = Rows<DH>::kLd * 2, kStage = 2 * kFewKeys * kRowBytes;
    static constexpr uint32_t kQ = kFewRows * kRowBytes, kWarp = kFewStages * kStage;
    static constexpr size_t kSmem = kQ + kWarps * kWarp;
    static constexpr int kCtas = DH == 128 ? 1 : DH == 64 ? 2 : 3;       // of an SM
};

template <class T, int DH>
__global__ void __launch_bounds__(kWarps * 32, FewTiles<T, DH>::kCtas)
k_attend_few(AttendArgs a, AttendOut o, int splits, float* part_out, float* part_lse) {
    using Sh = FewTiles<T, DH>;
    constexpr int C = DH / 8;
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ __align__(8) float bias[kWarps][kFewStages][kFewKeys];
    __shared__ float top[kWarps][kFewRows], sum[kWarps][kFewRows];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y, split = blockIdx.z;
    if (splits > 1) start_dependents();
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const Slot slot = slot_of(a.q_offsets, a.B, a.Tq, a.group, kFewLog, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t row0 = slot.tile << kFewLog, left = qs.len * a.group - row0;
    if (slot.tile < 0 || left <= 0) return;
    const int rows = left < kFewRows ? (int)left : kFewRows;
    const RowOf ro(row0, a.group);
    const int64_t chunks = (ks.len + kFewKeys - 1) / kFewKeys;
    const int64_t t0 = chunks * split / splits + warp, t1 = chunks * (split + 1) / splits;
    const T *k = (const T*)a.k + (int64_t)hk * a.dh, *v = (const T*)a.v + (int64_t)hk * a.dh;
    const Rows<DH> sq{smem32(raw)};
    uint8_t* const ring = raw + Sh::kQ;
    const uint32_t mine = sq.at + Sh::kQ + warp * Sh::kWarp;
    auto keys_at = [&](int stage) { return Rows<DH>{mine + stage * Sh::kStage}; };
    auto values_at = [&](int stage) { return Rows<DH>{mine + stage * Sh::kStage + Sh::kStage / 2}; };
    // whether this lane's key of a chunk counts, asked for one chunk before it is copied
    auto counts = [&](int64_t t) {
        const int64_t key = t * kFewKeys + lane;
        return t < t1 && key < ks.len && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key) >= 0);
    };
    bool next = counts(t0), some = false;
    auto load = [&](int64_t t, int stage) {
        if (t < t1) {
            const uint32_t in = __ballot_sync(0xFFFFFFFFu, next);
            bias[warp][stage][lane] = next ? 0.f : -INFINITY;
            some = some || in != 0;
            const Rows<DH> dk = keys_at(stage), dv = values_at(stage);
            const T *ck = k + (ks.at + t * kFewKeys) * a.ld_k, *cv = v + (ks.at + t * kFewKeys) * a.ld_v;
#pragma unroll
            for (int i = 0; i < kFewKeys * C / 32; ++i) {
                const int r = (i * 32 + lane) / C, d = (i * 32 + lane) % C * 8;
                const bool there = ((in >> r) & 1u) && d < a.dh;
                copy16(dk.addr(r, d), there ? (const void*)(ck + r * a.ld_k + d) : a.q, there);
                copy16(dv.addr(r, d), there ? (const void*)(cv + r * a.ld_v + d) : a.q, there);
            }
            next = counts(t + kWarps);
        }
        copies_done();
    };
    {
        const RowsAt<const T> q((const T*)a.q + (int64_t)hk * a.group * a.dh, qs.at + ro.token, a.ld_q, a.dh);
#pragma unroll
        for (int i = threadIdx.x; i < kFewRows * C; i += kWarps * 32) {
            const int r = i / C, d = i % C * 8;
            const bool in = r < rows && d < a.dh;
            copy16(sq.addr(r, d), in ? (const void*)(q(ro.at(r)) + d) : a.q, in);
        }
        copies_done();
    }
    load(t0, 0);
    load(t0 + kWarps, 1);
    wait_copies<2>();
    __syncthreads();
    Running<T, DH> run;
    run.begin(sq, 0);
    const float c = a.scale * kLog2e;
    int stage = 0;
    for (int64_t t = t0; t < t1; t += kWarps) {
        load(t + 2 * kWarps, stage == 0 ? 2 : stage - 1);
        wait_copies<2>();
        __syncwarp();
        run.template step<kFewKeys / 16>(keys_at(stage), values_at(stage), 0, kFewKeys / 16, bias[warp][stage], c, t == t0);
        __syncwarp();
        stage = stage == 2 ? 0 : stage + 1;
    }
    wait_copies<0>();
    if (!some) run.clear();          // queries that are not finite have NaN as their scores, whatever the bias
    __syncthreads();
    // this warp's sums over its place in shared memory: [16 rows][DH] float32
    float* const sums = reinterpret_cast<float*>(ring + warp * Sh::kWarp);
    const int g = lane >> 2, two = (lane & 3) * 2;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float l = run.l[r];
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
#pragma unroll
        for (int j = 0; j < DH / 8; ++j)
            *reinterpret_cast<float2*>(sums + (g + 8 * r) * DH + j * 8 + two) = make_float2(run.acc[j][2 * r], run.acc[j][2 * r + 1]);
        if ((lane & 3) == 0) {
            top[warp][g + 8 * r] = run.m[r];
            sum[warp][g + 8 * r] = l;
        }
    }
    __syncthreads();
    // eight threads a row
    const int row = threadIdx.x >> 3;
    if (row >= rows) return;
    float m = -INFINITY, l = 0.f, weight[kWarps];
#pragma unroll
    for (int i = 0; i < kWarps; ++i) m = fmaxf(m, top[i][row]);
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        weight[i] = ex2(top[i][row] - base);
        l = fmaf(sum[i][row], weight[i], l);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l, ln = l == 0.f ? -INFINITY : m + log2f(l);
    const int2 at = ro.at(row);
    const int64_t token = qs.at + ro.token + at.x;
    const int head = hk * a.group + at.y;
    const int64_t to = ((int64_t)split * a.Tq + token) * a.heads + head;
    for (int d = (threadIdx.x & 7) * 8; d < a.dh; d += 64) {
        float x[8] = {};
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
            const float4* p = reinterpret_cast<const float4*>(ring + i * Sh::kWarp + (row * DH + d) * 4);
            const float4 lo = p[0], hi = p[1];
            x[0] = fmaf(lo.x, weight[i], x[0]);
            x[1] = fmaf(lo.y, weight[i], x[1]);
            x[2] = fmaf(lo.z, weight[i], x[2]);
            x[3] = fmaf(lo.w, weight[i], x[3]);
            x[4] = fmaf(hi.x, weight[i], x[4]);
            x[5] = fmaf(hi.y, weight[i], x[5]);
            x[6] = fmaf(hi.z, weight[i], x[6]);
            x[7] = fmaf(hi.w, weight[i], x[7]);
        }
        if (splits > 1) {
            float4* p = reinterpret_cast<float4*>(part_out + to * a.dh + d);
            p[0] = make_float4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
            p[1] = make_float4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
        } else {
            Pack<T, 8> q;
#pragma unroll
            for (int z = 0; z < 4; ++z) q.set(z, make_float2(x[2 * z] * inv, x[2 * z + 1] * inv));
            q.store((T*)o.out + token * o.ld + (int64_t)head * a.dh + d);
        }
    }
    if ((threadIdx.x & 7) == 0) {
        if (splits > 1)
            part_lse[to] = ln;
        else if (o.lse)
            o.lse[to] = ln * kLn2;
    }
}

// Joins the splits of every row, in order: a warp per (token, head), a split's weight (two
// beyond 32) in a lane.
constexpr int kMaxSplits = 64;
template <class T>
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs a, AttendOut o, int splits, const float* part_out, const float* part_lse) {
    wait_before();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), n = a.Tq * a.heads;
    if (row >= n) return;
    float ln[2], top = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        ln[i] = i * 32 + lane < splits ? __ldcg(part_lse + (i * 32 + lane) * n + row) : -INFINITY;
        top = fmaxf(top, ln[i]);
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
    const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        ln[i] = ex2(ln[i] - base);
        l += ln[i];
    }
    l = warp_sum(l);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t token = row / a.heads;
    T* out = (T*)o.out + token * o.ld + (row - token * a.heads) * a.dh;
    const int d = lane * 4;      // a head has at most 128 elements
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = 0; s < splits; ++s) {
        const float w = __shfl_sync(0xFFFFFFFFu, s < 32 ? ln[0] : ln[1], s & 31) * inv;
        if (d >= a.dh) continue;
        const float4 p = __ldcg(reinterpret_cast<const float4*>(part_out + (s * n + row) * a.dh + d));
        sum.x = fmaf(w, p.x, sum.x);
        sum.y = fmaf(w, p.y, sum.y);
        sum.z = fmaf(w, p.z, sum.z);
        sum.w = fmaf(w, p.w, sum.w);
    }
    if (d < a.dh)
        *reinterpret_cast<uint2*>(out + d) = make_uint2(pack2(make_float2(sum.x, sum.y), T()), pack2(make_float2(sum.z, sum.w), T()));
    if (o.lse && lane == 0) o.lse[row] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
}

// How a call runs
struct Plan {
    bool tc;             // tiles of the tensor cores
    bool brief;          // the same for many short sequences
    bool few;            // a few rows and many keys
    int pack, log_rows, splits;
};
Plan plan_of(const AttendArgs& a) {
    Plan p{};
    p.pack = tc_pack(a);
    // Both sides in us, 8 heads with keys of their own, bfloat16, one call after the other:
    // 128 queries x 256 keys, heads of 64 (of 128): 1 sequence 8.0 against k_attend's 10.1 (9.3
    // and 12.1), 8 sequences 8.4 against 14.4 (9.5 and 16.2); 4 of 1024 x 1024 18.9 against 50.8.
    // (The bound on the rows is not moved for many keys, where it costs: of 16 000 keys 127 queries take
    // 39 in k_attend, 128 here 25 (78 and 27).)
    p.tc = a.Tq * p.pack / a.B >= 128 && a.Tk / a.B >= 256;
    // Many sequences, each with a good part of a tile of 128 rows, whose keys mostly are one
    // chunk.  200 sequences of 120 x 60, heads of 64: 24.2 against k_attend's 34.8; of 32 x 40
    // 18.7 and 18.4; 40 of 64 x 64 10.5 and 9.1: below about three tiles' worth of rows an SM it
    // is the longer.  Heads of 128: 40.4 and 66.1, 23.6 and 36.8, 12.5 and 14.9.  (It counts keys and
    // the places behind them in 32 bits.  Its copies need a key: a tensor map has no empty side.)
    p.brief = !p.tc && a.Tk > 0 && a.Tk <= 0x7FFFFF00 && a.Tq * p.pack / a.B >= 32 &&
              (a.dh > 64 ? slots(a.Tq, a.B, p.pack, 7) * (a.heads / p.pack) >= 2 * a.num_sms
                         : a.Tq * a.heads / 128 >= 3 * a.num_sms);
    if (p.brief) {
        p.log_rows = 7;
        p.splits = 1;
        return p;
    }
    // One tile of rows and more keys than k_attend holds; a few more keys only where there are few
    // CTAs.  One query, 8 heads of 64 (of 128), 300 sequences: 130 keys 40.7 against k_attend's 38.9
    // (103 and 88), 512 keys 64.4 and 84.7 (146 and 206), 4096 keys 376 and 547 (748 and 1476);
    // 1 sequence of 130 keys, heads of 128, 7.2 and 11.1; 8 heads sharing 4096 keys of 300, 55
    // and 128.
    const int64_t few_tiles = (a.Tq * a.group >> kFewLog) + 1, few_ctas = (few_tiles > a.B ? few_tiles : a.B) * a.kv_heads;
    p.few = !p.tc && a.Tq * a.group / a.B <= kFewRows && a.Tk / a.B > (few_ctas <= a.num_sms ? kResident : 2 * kResident);
    if (p.few) {
        // Parts of the keys: as many CTAs as the SMs hold at once, of two chunks a warp at least
        const int64_t ctas = few_ctas;
        int64_t n = (int64_t)(a.dh <= 32 ? 3 : a.dh <= 64 ? 2 : 1) * a.num_sms / ctas;
        const int64_t most = a.Tk / a.B / (2 * kWarps * kFewKeys);
        if (n > most) n = most;
        if (n > kMaxSplits) n = kMaxSplits;
        p.splits = (int)(n < 1 ? 1 : n);
        return p;
    }
    const int group = p.tc ? p.pack : a.group, keys = p.tc ? 128 : kTileKeys;
    auto ctas = [&](int log) {
        const int64_t tiles = (a.Tq * group >> log) + 1;
        return (tiles > a.B ? tiles : a.B) * (a.heads / group);
    };
    // Rows of a CTA: more use the keys in shared memory again, as long as the SMs have work
    p.log_rows = p.tc ? 8 : 9;
    while (!p.tc && p.log_rows > 6 && ctas(p.log_rows) < 4 * a.num_sms) --p.log_rows;
    // Parts of the keys, where the rows leave SMs without a CTA: at least two tiles of the
    // average sequence each.  (4099 queries x 17 403 keys, 8 heads of 128, are 128 CTAs and 8 of
    // 3 rows.  Cut 1 : 0.19 they leave SMs idle at the end instead, and take 3 us more, and the
    // join.)
    const int64_t tiles = a.Tk / a.B / keys;
    int64_t n = (p.tc ? 1 : 3) * a.num_sms / ctas(p.log_rows);
    if (n > tiles / 2) n = tiles / 2;
    if (n > kMaxSplits) n = kMaxSplits;
    p.splits = (int)(n < 1 ? 1 : n);
    return p;
}

template <class T, int DH>
cudaError_t run(const AttendArgs& a, const AttendOut& o, const Plan& p, float* part_out, float* part_lse, cudaStream_t s) {
    if (p.few) {
        const cudaError_t e = allow_smem(k_attend_few<T, DH>, FewTiles<T, DH>::kSmem);
        if (e != cudaSuccess) return e;
        const dim3 grid((unsigned)slots(a.Tq, a.B, a.group, kFewLog), (unsigned)a.kv_heads, (unsigned)p.splits);
        return launch_next(k_attend_few<T, DH>, grid, dim3(kWarps * 32), FewTiles<T, DH>::kSmem, false, s, a, o, p.splits, part_out, part_lse);
    }
    constexpr size_t smem = WarpTiles<T, DH>::kSmem;
    const cudaError_t e = allow_smem(k_attend<T, DH>, smem);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)slots(a.Tq, a.B, a.group, p.log_rows), (unsigned)a.kv_heads, (unsigned)p.splits);
    return launch_next(k_attend<T, DH>, grid, dim3(kWarps * 32), smem, false, s, a, o, p.log_rows, p.splits, part_out, part_lse);
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
        if (p.brief) return launch_attend_short(a, o, p.pack, a.Tk / a.B > 48, s);
        const cudaError_t e = p.tc           ? launch_attend_tc(a, o, p.pack, p.splits, part_out, part_lse, s)
                              : a.dh <= 32 ? run<T, 32>(a, o, p, part_out, part_lse, s)
                              : a.dh <= 64 ? run<T, 64>(a, o, p, part_out, part_lse, s)
                                           : run<T, 128>(a, o, p, part_out, part_lse, s);
        if (e != cudaSuccess || p.splits == 1 || a.Tq == 0) return e;
        return launch_next(k_attend_join<T>, dim3((unsigned)((a.Tq * a.heads + 7) / 8)), dim3(256), 0, true, s, a, o, p.splits,
                           (const float*)part_out, (const float*)part_lse);
    };
    return a.type == IFVS_T_F16 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ifvs
