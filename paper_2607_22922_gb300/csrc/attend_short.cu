// Attention of many short sequences on the tensor cores (ifvs_attend).
//
// Persistent CTAs take units, a tile of 128 rows of one group each, whose keys are mostly one
// chunk of KEYS.  A warp finds units by 32 at a time and loads their queries, keys and values
// by TMA; a warp issues the MMAs; two groups of four warps take units by turns, so that one
// group's exponentials and output run beside the other's MMAs:
//   tensor pipe:  s_0  s_1 | o_0 s_2 | o_1 s_3 | ...
// A thread holds a row's scores.  Sequences with more keys go on chunk by chunk as in
// attend_tc.cu.  Rows leave through shared memory by TMA, 32 at a time.
#include "attend_tc.cuh"

namespace ifvs {

namespace {

constexpr int kSoftWarps = 8, kLoader = 8, kIssuer = 9, kFixer = 10, kThreads = 352;
constexpr int kInfos = 8;

template <int DH, int KEYS>
struct ShortShape {
    static constexpr int kHalves = DH / 64;
    static constexpr uint32_t kQ = kHalves * kHalfBytes;                 // 128 rows
    static constexpr uint32_t kKeyHalf = KEYS * 128, kK = kHalves * kKeyHalf, kKv = 2 * kK;
    static constexpr int kQs = DH == 128 ? 2 : (KEYS == 64 ? 5 : 4);
    static constexpr int kKvs = DH == 128 ? (KEYS == 64 ? 4 : 2) : (KEYS == 64 ? 6 : 4);
    static constexpr uint32_t kOut = kSoftWarps * 32 * 128;              // 32 rows of 64 elements a warp
    static constexpr size_t kSmem = 1024 + kQs * kQ + kKvs * kKv + kOut;
};

// A unit; rows = 0: there are no more
struct Unit {
    int64_t token, key;      // of the first row and key
    int rows, keys, head, kv_head;
};

template <int QS, int KS, int KEYS>
struct ShortBars {
    uint64_t unit_full[kInfos], unit_empty[kInfos], q_full[QS], q_empty[QS], kv_full[KS], kv_empty[KS], fixed[KS], s_full[2], p_full[2],
        o_full[2], drain;
    Unit units[kInfos];
    uint32_t mask[KS][KEYS / 32];
    uint32_t tmem;
    int dead;
};

__device__ __forceinline__ uint64_t keys_rows_desc(uint32_t addr, uint32_t half_bytes) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(half_bytes >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}

// A place in a ring and the parity of its next fill
template <int N>
struct Place {
    uint32_t at = 0, parity = 0;
    __device__ __forceinline__ void next() {
        if (++at == N) {
            at = 0;
            parity ^= 1u;
        }
    }
};

template <class T, int DH, int KEYS>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_short(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
               const __grid_constant__ CUtensorMap mo, AttendArgs a, AttendOut o, int pack, int64_t n_units) {
    using Sh = ShortShape<DH, KEYS>;
    constexpr int QS = Sh::kQs, KS = Sh::kKvs, W = KEYS / 32;
    constexpr bool kF16 = std::is_same_v<T, __half>;
    __shared__ __align__(16) ShortBars<QS, KS, KEYS> bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const uint32_t q_at = dynamic_smem(), kv_at = q_at + QS * Sh::kQ, out_at = kv_at + KS * Sh::kKv;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kInfos; ++i) {
            mbar_init(smem_addr(&bars.unit_full[i]), 1);
            mbar_init(smem_addr(&bars.unit_empty[i]), kSoftWarps + 2);
        }
        for (int i = 0; i < QS; ++i) {
            mbar_init(smem_addr(&bars.q_full[i]), 1);
            mbar_init(smem_addr(&bars.q_empty[i]), 1);
        }
        for (int i = 0; i < KS; ++i) {
            mbar_init(smem_addr(&bars.kv_full[i]), 1);
            mbar_init(smem_addr(&bars.kv_empty[i]), 1);
            mbar_init(smem_addr(&bars.fixed[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&bars.s_full[i]), 1);
            mbar_init(smem_addr(&bars.p_full[i]), 4);
            mbar_init(smem_addr(&bars.o_full[i]), 1);
        }
        mbar_init(smem_addr(&bars.drain), 1);
        bars.dead = 0;
        fence_mbar_init();
    }
    if (warp == kIssuer) tmem_alloc<1>(smem_addr(&bars.tmem), 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = bars.tmem;
    const Watch w{&bars.dead, a.waits};
    auto s_col = [](int g) { return (uint32_t)g * KEYS; };
    auto o_col = [](int g) { return 2u * KEYS + (uint32_t)g * DH; };
    int q_filled = 0, kv_filled = 0;             // by the loader's thread

    // the next unit, read by this role
    Place<kInfos> unit_at;
    auto next_unit = [&](Unit& u, bool by_warp) {
        const bool there = w.wait(smem_addr(&bars.unit_full[unit_at.at]), unit_at.parity);
        if (by_warp ? !__all_sync(0xFFFFFFFFu, there) : !there) return false;
        u = bars.units[unit_at.at];
        if (by_warp) __syncwarp();
        if (!by_warp || lane == 0) mbar_arrive<1>(smem_addr(&bars.unit_empty[unit_at.at]));
        unit_at.next();
        return u.rows > 0;
    };
    auto chunks_of = [](int keys) { return (keys + KEYS - 1) / KEYS; };

    if (warp == kLoader) {
        const int nh = a.heads / pack;
        Place<QS> qp;
        Place<KS> kp;
        bool ok = true;
        // one unit, by the elected lane
        auto give = [&](const Unit& u) {
            if (!w.wait(smem_addr(&bars.unit_empty[unit_at.at]), unit_at.parity ^ 1u)) return false;
            bars.units[unit_at.at] = u;
            mbar_arrive<1>(smem_addr(&bars.unit_full[unit_at.at]));
            unit_at.next();
            const int chunks = u.rows > 0 ? chunks_of(u.keys) : 0;
            if (chunks == 0) return true;
            if (!w.wait(smem_addr(&bars.q_empty[qp.at]), qp.parity ^ 1u)) return false;
            uint32_t bar = smem_addr(&bars.q_full[qp.at]);
            mbar_arrive_expect_tx(bar, Sh::kQ + a.waits.extra);
            for (int d = 0; d < Sh::kHalves; ++d)
                tma_load_heads(q_at + qp.at * Sh::kQ + d * kHalfBytes, &mq, d * 64, u.head, (int)u.token, bar);
            qp.next();
            ++q_filled;
            for (int j = 0; j < chunks; ++j) {
                if (!w.wait(smem_addr(&bars.kv_empty[kp.at]), kp.parity ^ 1u)) return false;
                bar = smem_addr(&bars.kv_full[kp.at]);
                mbar_arrive_expect_tx(bar, Sh::kKv + a.waits.extra);
                for (int d = 0; d < Sh::kHalves; ++d) {
                    const uint32_t to = kv_at + kp.at * Sh::kKv + d * Sh::kKeyHalf;
                    tma_load_heads(to, &mk, d * 64, u.kv_head, (int)(u.key + (int64_t)j * KEYS), bar);
                    tma_load_heads(to + Sh::kK, &mv, d * 64, u.kv_head, (int)(u.key + (int64_t)j * KEYS), bar);
                }
                kp.next();
                ++kv_filled;
            }
            return true;
        };
        for (int64_t u0 = blockIdx.x; u0 < n_units && ok; u0 += 32 * (int64_t)gridDim.x) {
            const int64_t mine = u0 + lane * (int64_t)gridDim.x;
            Unit u{0, 0, 0, 0, 0, 0};
            if (mine < n_units) {
                const uint32_t slot = (uint32_t)(mine / nh), y = (uint32_t)(mine - (int64_t)slot * nh);
                uint32_t lo = 0, n = (uint32_t)a.B;      // the sequence: the last whose slots begin there or before
                while (n > 1) {
                    const uint32_t half = n / 2;
                    if (first_slot(a.q_offsets, lo + half, a.B, a.Tq, pack, 7) <= slot) {
                        lo += half;
                        n -= half;
                    } else {
                        n = half;
                    }
                }
                const int64_t tile = (int64_t)slot - first_slot(a.q_offsets, lo, a.B, a.Tq, pack, 7);
                const Span qs = span_of(a.q_offsets, lo, a.B, a.Tq), ks = span_of(a.kv_offsets, lo, a.B, a.Tk);
                const int64_t left = qs.len * pack - tile * 128;
                u.token = qs.at + tile * 128 / pack;
                u.key = ks.at;
                u.rows = tile < 0 || left <= 0 ? 0 : (left < 128 ? (int)left : 128);
                u.keys = (int)ks.len;
                u.head = (int)y * pack;
                u.kv_head = u.head / a.group;
            }
            for (uint32_t todo = __ballot_sync(0xFFFFFFFFu, u.rows > 0); todo && ok; todo &= todo - 1) {
                const int from = __ffs((int)todo) - 1;
                const Unit v{__shfl_sync(0xFFFFFFFFu, u.token, from), __shfl_sync(0xFFFFFFFFu, u.key, from),
                             __shfl_sync(0xFFFFFFFFu, u.rows, from),  __shfl_sync(0xFFFFFFFFu, u.keys, from),
                             __shfl_sync(0xFFFFFFFFu, u.head, from),  __shfl_sync(0xFFFFFFFFu, u.kv_head, from)};
                bool fine = true;
                if (elect_one()) fine = give(v);
                ok = __all_sync(0xFFFFFFFFu, fine);
            }
        }
        if (ok && elect_one()) give(Unit{0, 0, 0, 0, 0, 0});
    } else if (warp == kIssuer) {
        if (elect_one()) {
            Place<QS> qp;
            Place<KS> kp;
            // what a group's weights will multiply: there, first, last, turn of p_full, parity,
            // blocks of 16 keys, stage
            uint32_t pending[2] = {0, 0}, turns = 0;
            auto sums = [&](int g) {
                const uint32_t p = g ? pending[1] : pending[0];
                if (!(p & 1u)) return true;
                (g ? pending[1] : pending[0]) = 0;
                const uint32_t stage = p >> 16, blocks = p >> 8 & 255u;
                if (!w.wait(smem_addr(&bars.fixed[stage]), p >> 4 & 1u)) return false;
                if (!w.wait(smem_addr(&bars.p_full[g]), p >> 3 & 1u)) return false;
                fence_after_sync();
                const uint64_t dv = keys_rows_desc(kv_at + stage * Sh::kKv + Sh::kK, Sh::kKeyHalf);
                const uint32_t id_o = mma_desc(128, DH, kF16, false, true);
                for (uint32_t k = 0; k < blocks; ++k)
                    mma_f16_tmem_a(tmem + o_col(g), tmem + s_col(g) + k * 8, dv + k * desc_step(true), id_o, !(p & 2u) || k > 0);
                mma_commit<1>(smem_addr(&bars.kv_empty[stage]));
                if (p & 4u) mma_commit<1>(smem_addr(&bars.o_full[g]));
                return true;
            };
            Unit u;
            int g = 0;
            bool ok = true;
            for (; ok && next_unit(u, false); g ^= 1) {
                const int chunks = chunks_of(u.keys);
                for (int j = 0; j < chunks && ok; ++j, kp.next()) {
                    if (!(ok = sums(g))) break;
                    // the other group's last may hold the place in the ring that this one needs
                    const uint32_t other = g ? pending[0] : pending[1];
                    if ((other & 1u) && other >> 16 == kp.at && !(ok = sums(g ^ 1))) break;
                    if (j == 0 && !(ok = w.wait(smem_addr(&bars.q_full[qp.at]), qp.parity))) break;
                    if (!(ok = w.wait(smem_addr(&bars.kv_full[kp.at]), kp.parity))) break;
                    fence_after_sync();
                    const int left = u.keys - j * KEYS, blocks = ((left < KEYS ? left : KEYS) + 15) / 16;
                    const uint32_t id_s = mma_desc(128, blocks * 16, kF16, false, false);
#pragma unroll
                    for (int d = 0; d < Sh::kHalves; ++d) {
                        const uint64_t da = tile_desc(q_at + qp.at * Sh::kQ + d * kHalfBytes, false),
                                       db = tile_desc(kv_at + kp.at * Sh::kKv + d * Sh::kKeyHalf, false);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_f16<1>(tmem + s_col(g), da + k * desc_step(false), db + k * desc_step(false), id_s, d + k > 0);
                    }
                    mma_commit<1>(smem_addr(&bars.s_full[g]));
                    if (j == chunks - 1) {
                        mma_commit<1>(smem_addr(&bars.q_empty[qp.at]));
                        qp.next();
                    }
                    (g ? pending[1] : pending[0]) = 1u | (j == 0 ? 2u : 0u) | (j == chunks - 1 ? 4u : 0u) | (turns >> g & 1u) << 3 |
                                                    kp.parity << 4 | (uint32_t)blocks << 8 | kp.at << 16;
                    turns ^= 1u << g;
                }
            }
            // the last units', in their order
            if (ok && (ok = sums(g))) sums(g ^ 1);
        }
    } else if (warp == kFixer) {
        // which keys count; values of those that do not become zeros, because 0 times what they
        // hold may be a NaN
        Place<KS> kp;
        Unit u;
        bool ok = true;
        while (ok && next_unit(u, true)) {
            const int chunks = chunks_of(u.keys);
            for (int j = 0; j < chunks && ok; ++j, kp.next()) {
                const int left = u.keys - j * KEYS, blocks = ((left < KEYS ? left : KEYS) + 15) / 16;
                uint32_t bits[W];
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const int key = i * 32 + lane;
                    bits[i] = __ballot_sync(
                        0xFFFFFFFFu, key < left && (a.kv_ids == nullptr || __ldg(a.kv_ids + u.key + (int64_t)j * KEYS + key) >= 0));
                }
                if (!(ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.kv_full[kp.at]), kp.parity)))) break;
                if (lane == 0)
#pragma unroll
                    for (int i = 0; i < W; ++i) bars.mask[kp.at][i] = bits[i];
                bool any = false;
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const int in = blocks * 16 - i * 32;
                    any |= in > 0 && (~bits[i] & (in >= 32 ? 0xFFFFFFFFu : (1u << in) - 1u));
                }
                if (any) {
                    const uint32_t at = kv_at + kp.at * Sh::kKv + Sh::kK;
#pragma unroll 1
                    for (int i = lane; i < blocks * 16 * 8; i += 32) {
                        const int row = i >> 3;
                        uint32_t word = bits[0];
#pragma unroll
                        for (int x = 1; x < W; ++x) word = (row >> 5) == x ? bits[x] : word;
                        if (!((word >> (row & 31)) & 1u))
#pragma unroll
                            for (int d = 0; d < Sh::kHalves; ++d)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + d * Sh::kKeyHalf + (uint32_t)i * 16u), "r"(0)
                                             : "memory");
                    }
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive<1>(smem_addr(&bars.fixed[kp.at]));
            }
        }
    } else if (warp < kSoftWarps) {
        const int group = warp >> 2, quad = warp & 3;
        const uint32_t mine = tmem + ((uint32_t)quad << 21), s_at = mine + s_col(group), o_at = mine + o_col(group),
                       out = out_at + (uint32_t)warp * 32 * 128;
        const float c = a.scale * kLog2e;
        const float2 c2 = make_float2(c, c);
        Place<KS> kp;
        uint32_t s_turn = 0, o_turn = 0;
        Unit u;
        bool ok = true;
        for (int it = 0; ok && next_unit(u, true); ++it) {
            const int chunks = chunks_of(u.keys);
            if ((it & 1) != group) {
                for (int j = 0; j < chunks; ++j) kp.next();
                continue;
            }
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < chunks && ok; ++j, kp.next(), s_turn ^= 1u) {
                const int left = u.keys - j * KEYS, n = left < KEYS ? left : KEYS;
                // in this order: a wait for `fixed` may not be two fills ahead, and the group sees
                // those of its own units alone; s there means that the fill before was used
                ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.s_full[group]), s_turn) &&
                                                 w.wait(smem_addr(&bars.fixed[kp.at]), kp.parity));
                if (!ok) break;
                fence_after_sync();
                // the first C times 32 keys
                auto weigh = [&](auto count) {
                    constexpr int C = decltype(count)::value;
                    float s[C][32];
#pragma unroll
                    for (int x = 0; x < C; ++x) tmem_ld32(s_at + x * 32, s[x]);
                    uint32_t bits[C];
#pragma unroll
                    for (int x = 0; x < C; ++x) bits[x] = bars.mask[kp.at][x];
#pragma unroll
                    for (int x = 0; x < C; ++x) tmem_wait(s[x]);
                    float high = m;
#pragma unroll
                    for (int x = 0; x < C; ++x) {
                        if (bits[x] != 0xFFFFFFFFu)
#pragma unroll
                            for (int y = 0; y < 32; ++y)
                                if (!((bits[x] >> y) & 1u)) s[x][y] = -INFINITY;
                        float top = s[x][0];
#pragma unroll
                        for (int y = 1; y < 31; y += 2) top = fmaxf(top, fmaxf(s[x][y], s[x][y + 1]));
                        high = fmaxf(high, fmaxf(top, s[x][31]) * c);
                    }
                    const float shrink = m == -INFINITY ? 0.f : ex2(m - high);
                    m = high;
                    if (j > 0) {       // s of this chunk came after the MMAs of o
                        l *= shrink;
#pragma unroll 1
                        for (int d = 0; d < DH; d += 32) {
                            float v[32];
                            tmem_ld32(o_at + d, v);
                            tmem_wait(v);
#pragma unroll
                            for (int y = 0; y < 32; ++y) v[y] *= shrink;
                            tmem_st32(o_at + d, *reinterpret_cast<const uint32_t(*)[32]>(&v));
                        }
                    }
                    const float base = m == -INFINITY ? 0.f : m;
                    const float2 b2 = make_float2(-base, -base);
                    float2 sum = make_float2(0.f, 0.f);
                    uint32_t p[C][16];
#pragma unroll
                    for (int x = 0; x < C; ++x)
#pragma unroll
                        for (int y = 0; y < 32; y += 2) {
                            float2 e = fma_(make_float2(s[x][y], s[x][y + 1]), c2, b2);
                            e.x = ex2(e.x);
                            e.y = ex2(e.y);
                            sum = add_(sum, e);
                            p[x][y / 2] = pack2(e, T());
                        }
#pragma unroll
                    for (int x = 0; x < C; ++x) tmem_st16(s_at + x * 16, p[x]);
                    l += total(sum);
                };
                if (n <= KEYS / 2)
                    weigh(std::integral_constant<int, W / 2>());
                else
                    weigh(std::integral_constant<int, W>());
                tmem_st_wait();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive<1>(smem_addr(&bars.p_full[group]));
            }
            if (ok && chunks > 0) {
                ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.o_full[group]), o_turn));
                o_turn ^= 1u;
            }
            if (!ok) break;
            fence_after_sync();
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const int r = quad * 32 + lane;
            const int64_t token = u.token + r / pack;
            const int head = u.head + r % pack;
            const bool in = r < u.rows, whole = quad * 32 + 32 <= u.rows && pack <= 32;
            T* to = (T*)o.out + token * o.ld + (int64_t)head * a.dh;
#pragma unroll 1
            for (int d = 0; d < DH; d += 64) {
                float v[2][32];
                tmem_ld32(o_at + d, v[0]);
                tmem_ld32(o_at + d + 32, v[1]);
                tmem_wait(v[0]);
                tmem_wait(v[1]);
                if (whole) {
                    if (lane == 0) tma_wait_read<0>();
                    __syncwarp();
                }
#pragma unroll
                for (int y = 0; y < 64; y += 8) {
                    Pack<T, 8> q;
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        const float* x = &v[y >> 5][(y & 31) + 2 * z];
                        q.set(z, chunks > 0 ? mul_(make_float2(x[0], x[1]), make_float2(inv, inv)) : make_float2(0.f, 0.f));
                    }
                    if (whole)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(out + lane * 128 + (((y >> 3) ^ (lane & 7)) << 4)),
                                     "r"(q.w.x), "r"(q.w.y), "r"(q.w.z), "r"(q.w.w)
                                     : "memory");
                    else if (in && d + y < a.dh)
                        q.store(to + d + y);
                }
                if (whole) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_heads(&mo, d, u.head, (int)(u.token + quad * 32 / pack), out);
                        tma_commit();
                    }
                }
            }
            if (in && o.lse) o.lse[token * a.heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
            // the next unit's MMAs write o once this group's weights are there
            fence_before_sync();
        }
        if (lane == 0) tma_wait_all();
    }
    __syncwarp();
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (*(volatile int*)&bars.dead) {
        // a wait ran out: wait once more, bounded, for what is in flight
        const long long begun = clock64();
        auto bounded = [&](uint32_t bar, uint32_t parity) {
            while (!mbar_try_wait(bar, parity) && clock64() - begun < a.waits.cycles) {
            }
        };
        if (warp == kLoader) {                   // the counts are the elected thread's
            for (int i = q_filled > QS ? q_filled - QS : 0; i < q_filled; ++i)
                bounded(smem_addr(&bars.q_full[i % QS]), (uint32_t)(i / QS) & 1u);
            for (int i = kv_filled > KS ? kv_filled - KS : 0; i < kv_filled; ++i)
                bounded(smem_addr(&bars.kv_full[i % KS]), (uint32_t)(i / KS) & 1u);
        }
        if (warp == kIssuer && elect_one()) {
            mma_commit<1>(smem_addr(&bars.drain));
            bounded(smem_addr(&bars.drain), 0);
        }
        __syncwarp();
        __syncthreads();
    }
    if (warp == kIssuer) tmem_free<1>(tmem, 512);
}

template <class T, int DH, int KEYS>
cudaError_t run(const AttendArgs& a, const AttendOut& o, int pack, cudaStream_t s) {
    CUtensorMap mq, mk, mv, mo;
    cudaError_t e = make_head_map(&mq, a.type, a.q, a.Tq, a.heads, a.dh, a.ld_q, pack, 128 / pack);
    if (e == cudaSuccess) e = make_head_map(&mk, a.type, a.k, a.Tk, a.kv_heads, a.dh, a.ld_k, 1, KEYS);
    if (e == cudaSuccess) e = make_head_map(&mv, a.type, a.v, a.Tk, a.kv_heads, a.dh, a.ld_v, 1, KEYS);
    if (e == cudaSuccess) e = make_head_map(&mo, a.type, o.out, a.Tq, a.heads, a.dh, o.ld, pack <= 32 ? pack : 1, pack <= 32 ? 32 / pack : 1);
    if (e == cudaSuccess) e = allow_smem(k_attend_short<T, DH, KEYS>, ShortShape<DH, KEYS>::kSmem);
    if (e != cudaSuccess) return e;
    const int64_t units = slots(a.Tq, a.B, pack, 7) * (a.heads / pack);
    const dim3 grid((unsigned)(units < a.num_sms ? units : a.num_sms));
    return launch_next(k_attend_short<T, DH, KEYS>, grid, dim3(kThreads), ShortShape<DH, KEYS>::kSmem, false, s, mq, mk, mv, mo, a, o, pack,
                       units);
}

}  // namespace

cudaError_t launch_attend_short(const AttendArgs& a, const AttendOut& o, int pack, bool wide, cudaStream_t s) {
    auto go = [&](auto t) {
        using T = decltype(t);
        if (a.dh <= 64) return wide ? run<T, 64, 128>(a, o, pack, s) : run<T, 64, 64>(a, o, pack, s);
        return wide ? run<T, 128, 128>(a, o, pack, s) : run<T, 128, 64>(a, o, pack, s);
    };
    return a.type == IFVS_T_F16 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ifvs
