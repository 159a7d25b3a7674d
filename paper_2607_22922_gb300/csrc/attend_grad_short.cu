// The gradient of attention of many short sequences on the tensor cores (ifvs_attend_grad).
//
// A unit is 64 keys of one sequence and head with all rows of their group, tiles of 128:
//   s = q k^T, dp = do v^T; a thread makes its row's p and ds, which go to shared memory as
//   16-bit tiles [rows][keys]; [p ds]^T [q do], one MMA of 128 x 2 dh, whose quarters p^T do
//   and ds^T q are dv's and dk's sums (the others are not used; two MMAs of 64 keys each take
//   longer, since an MMA has 128 rows); dq = ds k, the same tile of ds along its keys
// Where the unit has all of a sequence's keys, the softmax's sum and delta come from the row
// itself and dq is complete; else from the forward call's lse and output, and k_attend_rows
// makes dq.  Groups of four warps take one unit each and go through them tile by tile by
// turns, so that one's exponentials run beside the other's MMAs.
//
// What bounds a tile is the chain of its waits (rows, s and dp, weights, dq, its rows on their
// way), two of them at a time: 1000 sequences of 60 to 68 queries and up to 65 keys, 8 heads of
// 64 over 2, take 104 to 112 us with k_attend_rows, 2.8 TB/s.  The issuing warp takes whichever group's
// weights come first; in the order of the tiles, with a warp more (128 registers, which spill)
// and all keys of a bundle before its rows it takes 137.
#include "attend_tc.cuh"

namespace ifvs {

namespace {

constexpr int kBatch = 16, kKeys = 64;       // units that are found together; keys of a unit
constexpr uint32_t kWeights = 128 * 128;         // a tile of p or ds
constexpr uint32_t kChunk = 32 * 64;             // 32 rows of 32 elements of dq

template <int DH>
struct BriefShape {
    static constexpr int kHalves = DH / 64;
    static constexpr int kGroups = DH == 64 ? 2 : 1;
    static constexpr int kColumns = 64 + 3 * DH;                         // of TMEM: s, dp (then dq), sums of dk and dv
    static constexpr int kSoft = 4 * kGroups, kLoader = kSoft, kIssuer = kSoft + 1, kFixer = kSoft + 2, kFinder = kSoft + 3,
                         kThreads = (kFinder + 1) * 32;
    static constexpr uint32_t kQ = kHalves * kHalfBytes, kStage = 2 * kQ;            // queries and gradients
    static constexpr uint32_t kKeyHalf = kKeys * 128, kK = kHalves * kKeyHalf, kKv = 2 * kK;
    static constexpr int kQs = DH == 128 ? 2 : 3, kKvs = kGroups + 1;
    static constexpr size_t kSmem = 1024 + kGroups * 2 * kWeights + kQs * kStage + kKvs * kKv + (kGroups == 2 ? kSoft * kChunk : 0);
};

struct BriefUnit {
    int token, key;          // the first row's token, the first key
    int rows;
    int16_t keys, kv_head;
    uint8_t place, parity;   // in the ring of keys
    uint8_t alone;           // whether these are all keys of the sequence
};

template <int QS, int KS, int GROUPS>
struct BriefBars {
    uint64_t batch_full[2], batch_empty[2], q_full[QS], q_fixed[QS], q_empty[QS], kv_full[KS], kv_fixed[KS], kv_empty[KS], s_full[GROUPS],
        p_full[GROUPS], dq_full[GROUPS], dq_read[GROUPS], w_free[GROUPS], drain;
    BriefUnit units[2][kBatch];
    int count[2];            // -1: there are no more
    int some[KS];            // whether a key counts
    alignas(16) float bias[KS][kKeys];   // read four at a time: 0, or -infinity for a key that does not count
    uint32_t tmem;
    Pulse pulse;
};

// whether a phase has ended, without waiting
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity)
                 : "memory");
    return ok != 0;
}

template <int N>
struct Spot {
    uint32_t at = 0, parity = 0;
    __device__ __forceinline__ void next() {
        if (++at == N) {
            at = 0;
            parity ^= 1u;
        }
    }
};

// An operand whose 64-element blocks (M or N) lie `block` bytes apart, its sum along the rows
__device__ __forceinline__ uint64_t along_rows(uint32_t addr, uint32_t block) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(block >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}

template <class T, int DH>
__global__ void __launch_bounds__(BriefShape<DH>::kThreads, 1)
k_grad_short(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ CUtensorMap mk,
             const __grid_constant__ CUtensorMap mv, const __grid_constant__ CUtensorMap mdq, AttendArgs a, AttendGrads g, int log_pack,
             int64_t n_units) {
    using Sh = BriefShape<DH>;
    constexpr int QS = Sh::kQs, KS = Sh::kKvs, GROUPS = Sh::kGroups, H = Sh::kHalves;
    constexpr int kLoader = Sh::kLoader, kIssuer = Sh::kIssuer, kFixer = Sh::kFixer, kFinder = Sh::kFinder;
    constexpr bool kF16 = std::is_same_v<T, __half>;
    __shared__ __align__(16) BriefBars<QS, KS, GROUPS> bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pack = 1 << log_pack;
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    start_dependents();
    const uint32_t w_at = dynamic_smem(), q_at = w_at + GROUPS * 2 * kWeights, kv_at = q_at + QS * Sh::kStage;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&bars.batch_full[i]), 1);
            mbar_init(smem_addr(&bars.batch_empty[i]), Sh::kSoft + 3);
        }
        for (int i = 0; i < QS; ++i) {
            mbar_init(smem_addr(&bars.q_full[i]), 1);
            mbar_init(smem_addr(&bars.q_fixed[i]), 1);
            mbar_init(smem_addr(&bars.q_empty[i]), 1);
        }
        for (int i = 0; i < KS; ++i) {
            mbar_init(smem_addr(&bars.kv_full[i]), 1);
            mbar_init(smem_addr(&bars.kv_fixed[i]), 1);
            mbar_init(smem_addr(&bars.kv_empty[i]), 1);
        }
        for (int i = 0; i < GROUPS; ++i) {
            mbar_init(smem_addr(&bars.s_full[i]), 1);
            mbar_init(smem_addr(&bars.p_full[i]), 4);
            mbar_init(smem_addr(&bars.dq_full[i]), 1);
            mbar_init(smem_addr(&bars.dq_read[i]), 4);
            mbar_init(smem_addr(&bars.w_free[i]), 1);
        }
        mbar_init(smem_addr(&bars.drain), 1);
        bars.pulse.dead = 0;
        bars.pulse.last = (uint32_t)clock();
        fence_mbar_init();
    }
    if (warp == kIssuer) tmem_alloc<1>(smem_addr(&bars.tmem), 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = bars.tmem;
    const UnitWatch w{&bars.pulse, a.waits};
    auto s_col = [](int i) { return (uint32_t)i * Sh::kColumns; };
    auto dp_col = [](int i) { return (uint32_t)i * Sh::kColumns + 64u; };
    // lanes 64 on, columns 0 on: dk; lanes 0 on, columns DH on: dv
    auto sum_col = [](int i) { return (uint32_t)i * Sh::kColumns + 64u + DH; };
    int q_filled = 0, kv_filled = 0;             // by the loader's thread

    // tiles that take MMAs
    auto tiles_of = [](const BriefUnit& u) { return u.keys > 0 ? (u.rows + 127) / 128 : 0; };
    // f(units, how many) for every bundle of up to GROUPS units of a batch.  idle(): called
    // before a batch is waited for; the finder may be waiting for a group that waits for this role.
    auto bundles = [&](bool alone, auto&& idle, auto&& f) {
        uint32_t b = 0, parity = 0;
        for (;;) {
            if (!mbar_try_wait(smem_addr(&bars.batch_full[b]), parity) && !idle()) return false;
            bool ok = w.wait(smem_addr(&bars.batch_full[b]), parity);
            if (!alone) ok = __all_sync(0xFFFFFFFFu, ok);
            const int n = ok ? bars.count[b] : -1;
            if (n < 0) return ok;
            for (int i = 0; i < n; i += GROUPS)
                if (!f(&bars.units[b][i], n - i < GROUPS ? n - i : GROUPS)) return false;
            if (!alone) __syncwarp();
            if (alone || lane == 0) mbar_arrive<1>(smem_addr(&bars.batch_empty[b]));
            b ^= 1u;
            parity ^= b ^ 1u;
        }
    };
    // f(group, tile, unit) for a bundle's tiles, by turns
    auto steps = [&](const BriefUnit* u, int n, auto&& f) {
        int most = 0;
        for (int i = 0; i < n; ++i) most = max(most, tiles_of(u[i]));
        for (int t = 0; t < most; ++t)
            for (int i = 0; i < n; ++i)
                if (t < tiles_of(u[i]) && !f(i, t, u[i])) return false;
        return true;
    };

    auto nothing = [] { return true; };

    if (warp == kFinder) {
        uint32_t b = 0, parity = 1, place = 0, turn = 0;
        const uint32_t grid = gridDim.x;
        // A lane takes a sequence and head: mostly one unit, so that the CTAs have as many each.
        // Of sequences with more keys one unit after the other.
        Span qs{0, 0}, ks{0, 0};
        int head = 0;
        int64_t tile = 0;
        bool some = false;               // this lane has units left
        for (int64_t round = 0;;) {
            if (!__any_sync(0xFFFFFFFFu, some)) {
                if (round * grid >= n_units) break;
                // the CTAs change places from round to round
                const uint32_t seat = (uint32_t)((blockIdx.x + 37u * (uint32_t)((round + lane) % grid)) % grid);
                const int64_t mine = (round + lane) * grid + seat;
                round += kBatch;
                some = lane < kBatch && mine < n_units;
                if (some) {
                    const int64_t seq = mine / a.kv_heads;
                    head = (int)(mine - seq * a.kv_heads);
                    qs = span_of(a.q_offsets, seq, a.B, a.Tq);
                    ks = span_of(a.kv_offsets, seq, a.B, a.Tk);
                    tile = 0;
                }
            }
            BriefUnit u{};
            bool real = false;
            if (some) {
                const int64_t left = ks.len - tile * kKeys;
                u.token = (int)qs.at;
                u.key = (int)(ks.at + tile * kKeys);
                u.rows = (int)(qs.len << log_pack);
                u.keys = (int16_t)(left < kKeys ? left : kKeys);
                u.kv_head = (int16_t)head;
                u.alone = ks.len <= kKeys;
                // without keys the first tile still writes dq
                real = left > 0 || u.rows > 0;
                some = ++tile * kKeys < ks.len;
            }
            const uint32_t there = __ballot_sync(0xFFFFFFFFu, real);
            const uint32_t loads = __ballot_sync(0xFFFFFFFFu, real && tiles_of(u) > 0), below = (1u << lane) - 1u;
            const uint32_t at = place + (uint32_t)__popc(loads & below), all = place + (uint32_t)__popc(loads);
            u.place = (uint8_t)(at % KS);
            u.parity = (uint8_t)((turn + at / KS) & 1u);
            turn += all / KS;
            place = all % KS;
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.batch_empty[b]), parity))) break;
            if (real) bars.units[b][__popc(there & below)] = u;
            if (lane == 0) bars.count[b] = __popc(there);
            __syncwarp();
            if (lane == 0) {
                w.further();
                mbar_arrive<1>(smem_addr(&bars.batch_full[b]));
            }
            b ^= 1u;
            parity ^= b ^ 1u;
        }
        if (__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.batch_empty[b]), parity)) && lane == 0) {
            bars.count[b] = -1;
            mbar_arrive<1>(smem_addr(&bars.batch_full[b]));
        }
    } else if (warp == kLoader) {
        if (elect_one()) {
            Spot<QS> qp;
            Spot<KS> kp;
            // a unit's keys before its first rows: the other roles go by the same order
            bundles(true, nothing, [&](const BriefUnit* u, int n) {
                return steps(u, n, [&](int, int t, const BriefUnit& v) {
                    if (t == 0) {
                        if (!w.wait(smem_addr(&bars.kv_empty[kp.at]), kp.parity ^ 1u)) return false;
                        const uint32_t bar = smem_addr(&bars.kv_full[kp.at]);
                        mbar_arrive_expect_tx(bar, Sh::kKv + a.waits.extra);
                        for (int d = 0; d < H; ++d) {
                            const uint32_t to = kv_at + kp.at * Sh::kKv + d * Sh::kKeyHalf;
                            tma_load_heads(to, &mk, d * 64, v.kv_head, v.key, bar);
                            tma_load_heads(to + Sh::kK, &mv, d * 64, v.kv_head, v.key, bar);
                        }
                        kp.next();
                        ++kv_filled;
                    }
                    if (!w.wait(smem_addr(&bars.q_empty[qp.at]), qp.parity ^ 1u)) return false;
                    const uint32_t bar = smem_addr(&bars.q_full[qp.at]);
                    mbar_arrive_expect_tx(bar, Sh::kStage + a.waits.extra);
                    const int token = v.token + (t * 128 >> log_pack), head = v.kv_head << log_pack;
                    for (int d = 0; d < H; ++d) {
                        const uint32_t to = q_at + qp.at * Sh::kStage + d * kHalfBytes;
                        tma_load_heads(to, &mq, d * 64, head, token, bar);
                        tma_load_heads(to + Sh::kQ, &mdo, d * 64, head, token, bar);
                    }
                    qp.next();
                    ++q_filled;
                    return true;
                });
            });
        }
    } else if (warp == kIssuer) {
        if (elect_one()) {
            Spot<QS> qp;
            const uint32_t id_q = mma_desc(128, DH, kF16, false, true), id_k = mma_desc(128, 2 * DH, kF16, true, true);
            // what waits for a group's weights: there, first and last tile, parity of the unit's
            // place, blocks of 16 keys, place in the ring of rows, place in that of keys
            uint32_t pending[GROUPS] = {}, turns = 0, reads = 0;
            auto of = [&](int i) { return GROUPS == 1 || i == 0 ? pending[0] : pending[GROUPS - 1]; };
            auto put = [&](int i, uint32_t p) { (GROUPS == 1 || i == 0 ? pending[0] : pending[GROUPS - 1]) = p; };
            auto multiply = [&](int i) {         // group i's weights are there
                const uint32_t p = of(i);
                put(i, 0);
                turns ^= 1u << i;
                fence_after_sync();
                const uint32_t stage = p >> 16 & 255u, keys = p >> 24, blocks = p >> 8 & 255u;
                const uint32_t q = q_at + stage * Sh::kStage, k = kv_at + keys * Sh::kKv, weights = w_at + (uint32_t)i * 2 * kWeights;
                const uint64_t da = along_rows(weights, kWeights), dd = along_rows(q, kHalfBytes);
                const bool more = !(p & 2u);
                // dq first: its group waits for it
                const uint64_t sa = tile_desc(weights + kWeights, false), kb = along_rows(k, Sh::kKeyHalf);
                for (uint32_t x = 0; x < blocks; ++x)
                    mma_f16<1>(tmem + dp_col(i), sa + x * desc_step(false), kb + x * desc_step(true), id_q, x > 0);
                mma_commit<1>(smem_addr(&bars.dq_full[i]));
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    mma_f16<1>(tmem + sum_col(i), da + x * desc_step(true), dd + x * desc_step(true), id_k, more || x > 0);
                mma_commit<1>(smem_addr(&bars.w_free[i]));
                mma_commit<1>(smem_addr(&bars.q_empty[stage]));
                if (p & 4u) mma_commit<1>(smem_addr(&bars.kv_empty[keys]));
            };
            // waits for what group i needs; the other group's weights may be there first
            auto wait = [&](int i, uint64_t& barrier, uint32_t parity) {
                const uint32_t bar = smem_addr(&barrier);
                const long long begun = clock64();
                for (;;) {
                    if (mbar_test(bar, parity)) return true;
                    bool other = false;
                    for (int x = 0; x < GROUPS; ++x)
                        if (x != i && (of(x) & 1u)) {
                            other = true;
                            if (mbar_test(smem_addr(&bars.p_full[x]), turns >> x & 1u)) multiply(x);
                        }
                    if (!other || clock64() - begun > a.waits.cycles) return w.wait(bar, parity);
                }
            };
            auto sums = [&](int i) {
                if (!(of(i) & 1u)) return true;
                if (!wait(i, bars.p_full[i], turns >> i & 1u)) return false;
                multiply(i);
                return true;
            };
            auto flush = [&] {
                for (int i = 0; i < GROUPS; ++i)
                    if (!sums(i)) return false;
                return true;
            };
            const bool ok = bundles(true, flush, [&](const BriefUnit* u, int n) {
                return steps(u, n, [&](int i, int t, const BriefUnit& v) {
                    if (!sums(i)) return false;
                    // and another group's last that holds the place for these keys or rows
                    for (int x = 0; x < GROUPS; ++x)
                        if ((of(x) & 1u) && ((t == 0 && of(x) >> 24 == v.place) || (of(x) >> 16 & 255u) == qp.at) && !sums(x)) return false;
                    // dp takes the place of the group's last dq
                    if (!wait(i, bars.dq_read[i], (reads >> i & 1u) ^ 1u)) return false;
                    reads ^= 1u << i;
                    if (t == 0 && !wait(i, bars.kv_fixed[v.place], v.parity)) return false;
                    if (!wait(i, bars.q_full[qp.at], qp.parity)) return false;
                    if (!wait(i, bars.q_fixed[qp.at], qp.parity)) return false;
                    fence_after_sync();
                    const int blocks = (v.keys + 15) / 16;
                    const uint32_t id_s = mma_desc(128, blocks * 16, kF16, false, false);
                    const uint32_t q = q_at + qp.at * Sh::kStage, k = kv_at + v.place * Sh::kKv;
#pragma unroll
                    for (int d = 0; d < H; ++d) {
                        const uint64_t qa = tile_desc(q + d * kHalfBytes, false), kb = tile_desc(k + d * Sh::kKeyHalf, false),
                                       da = tile_desc(q + Sh::kQ + d * kHalfBytes, false),
                                       vb = tile_desc(k + Sh::kK + d * Sh::kKeyHalf, false);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            mma_f16<1>(tmem + s_col(i), qa + x * desc_step(false), kb + x * desc_step(false), id_s, d + x > 0);
                            mma_f16<1>(tmem + dp_col(i), da + x * desc_step(false), vb + x * desc_step(false), id_s, d + x > 0);
                        }
                    }
                    mma_commit<1>(smem_addr(&bars.s_full[i]));
                    put(i, 1u | (t == 0 ? 2u : 0u) | (t == tiles_of(v) - 1 ? 4u : 0u) | (uint32_t)blocks << 8 | qp.at << 16 |
                               (uint32_t)v.place << 24);
                    qp.next();
                    return true;
                });
            });
            if (ok) flush();
        }
    } else if (warp == kFixer) {
        // Which keys count; keys and values of those that do not become zeros, because 0 times
        // what they hold may be a NaN.  Rows behind the sequence become zeros: whatever their p
        // and ds are, they add nothing.  (One warp for both: a thirteenth would leave 128
        // registers a thread, with which the others spill.)
        Spot<QS> qp;
        Spot<KS> kp;
        auto fix_keys = [&](const BriefUnit& u) {
            const int blocks = (u.keys + 15) / 16;
            uint32_t bits[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int key = x * 32 + lane;
                bits[x] = __ballot_sync(0xFFFFFFFFu, key < u.keys && (a.kv_ids == nullptr || __ldg(a.kv_ids + (int64_t)u.key + key) >= 0));
            }
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.kv_full[kp.at]), kp.parity))) return false;
            bool any = false;
            if (lane == 0) bars.some[kp.at] = (bits[0] | bits[1]) != 0;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                bars.bias[kp.at][x * 32 + lane] = (bits[x] >> lane) & 1u ? 0.f : -INFINITY;
                if (x * 32 + lane < blocks * 16 && !((bits[x] >> lane) & 1u)) {
                    any = true;
                    const uint32_t at = kv_at + kp.at * Sh::kKv + (uint32_t)(x * 32 + lane) * 128u;
#pragma unroll
                    for (int d = 0; d < 2 * H; ++d)
#pragma unroll
                        for (int y = 0; y < 8; ++y)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + d * Sh::kKeyHalf + ((y ^ (lane & 7)) << 4)),
                                         "r"(0)
                                         : "memory");
                }
            }
            if (__any_sync(0xFFFFFFFFu, any)) fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive<1>(smem_addr(&bars.kv_fixed[kp.at]));
            kp.next();
            return true;
        };
        bundles(false, nothing, [&](const BriefUnit* units, int n) {
            return steps(units, n, [&](int, int t, const BriefUnit& u) {
                if (t == 0 && !fix_keys(u)) return false;
                if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.q_full[qp.at]), qp.parity))) return false;
                const int rows = u.rows - t * 128;
                if (rows < 128) {
#pragma unroll 1
                    for (int r = lane; r < 128; r += 32)
                        if (r >= rows)
#pragma unroll
                            for (int d = 0; d < 2 * H; ++d)
#pragma unroll
                                for (int y = 0; y < 8; ++y)
                                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(
                                                     q_at + qp.at * Sh::kStage + d * kHalfBytes + (uint32_t)r * 128u + ((y ^ (lane & 7)) << 4)),
                                                 "r"(0)
                                                 : "memory");
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive<1>(smem_addr(&bars.q_fixed[qp.at]));
                qp.next();
                return true;
            });
        });
    } else {
        const int group = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t mine = tmem + ((uint32_t)quad << 21), s_at = mine + s_col(group), dp_at = mine + dp_col(group);
        const uint32_t out = kv_at + KS * Sh::kKv + (uint32_t)warp * kChunk;
        const uint32_t p_row = w_at + (uint32_t)group * 2 * kWeights + (uint32_t)r * 128u;
        const float c = a.scale * kLog2e;
        const float2 c2 = make_float2(c, c);
        uint32_t turn = 0;
        bundles(false, nothing, [&](const BriefUnit* units, int n_units_here) {
            if (group >= n_units_here) return true;
            const BriefUnit u = units[group];
            const int tiles = (u.rows + 127) / 128, head = u.kv_head << log_pack;
            bool counts = false;             // of a key a lane; its place may hold others at the end
            for (int t = 0; t < tiles; ++t) {
                if (lane == 0 && (t & 63) == 63) w.further();
                const int row = t * 128 + r;
                // whole: 32 rows leave by TMA, where there is room for them on their way (one group has none)
                const bool in = row < u.rows, whole = GROUPS == 2 && t * 128 + quad * 32 + 32 <= u.rows && pack <= 32;
                const int64_t token = (int64_t)u.token + (row >> log_pack);
                const int my_head = head + (row & (pack - 1));
                T* to = (T*)g.dq + token * g.ld_dq + (int64_t)my_head * a.dh;
                if (u.keys == 0) {
                    if (in)
                        for (int d = 0; d < a.dh; d += 8) *reinterpret_cast<uint4*>(to + d) = make_uint4(0, 0, 0, 0);
                    continue;
                }
                float lse2 = INFINITY, delta = 0.f;
                if (!u.alone && in) {
                    const float v = __ldg(g.lse + token * a.heads + my_head);
                    if (v != -INFINITY) lse2 = v * kLog2e;
                    const T *x = (const T*)g.out + token * g.ld_out + (int64_t)my_head * a.dh,
                            *y = (const T*)g.d_out + token * g.ld_d_out + (int64_t)my_head * a.dh;
                    float2 sum = make_float2(0.f, 0.f);
#pragma unroll 2
                    for (int d = 0; d < a.dh; d += 8) {
                        Pack<T, 8> p, q;
                        p.load(x + d);
                        q.load(y + d);
#pragma unroll
                        for (int z = 0; z < 4; ++z) sum = fma_(p.get(z), q.get(z), sum);
                    }
                    delta = total(sum);
                }
                // the second wait, over by then, is for the fixer's own stores of what counts.  In this order: the
                // place cannot be filled again before this tile's weights are there
                if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.s_full[group]), turn) &&
                                                 w.wait(smem_addr(&bars.kv_fixed[u.place]), u.parity)))
                    return false;
                fence_after_sync();
                const float* bias = bars.bias[u.place];
                counts = bias[r & 63] == 0.f;
                const bool some = bars.some[u.place] != 0;       // else dq is zero, whatever the scores are
                // the first C times 32 keys; columns behind the last block of 16 hold what was there
                auto weigh = [&](auto count) {
                    constexpr int C = decltype(count)::value;
                    const int most = (u.keys + 15) & ~15;
                    float s[C][32];
#pragma unroll
                    for (int x = 0; x < C; ++x) tmem_ld32(s_at + x * 32, s[x]);
                    float high = -INFINITY;
#pragma unroll
                    for (int x = 0; x < C; ++x) {
                        tmem_wait(s[x]);
#pragma unroll
                        for (int y = 0; y < 32; y += 4) {
                            const float4 b = *reinterpret_cast<const float4*>(bias + x * 32 + y);
                            if (y == 16 && x * 32 + 16 >= most)
#pragma unroll
                                for (int z = 16; z < 32; ++z) s[x][z] = 0.f;
                            float2* v = reinterpret_cast<float2*>(&s[x][y]);
                            v[0] = add_(v[0], make_float2(b.x, b.y));
                            v[1] = add_(v[1], make_float2(b.z, b.w));
                            high = fmaxf(fmaxf(high, fmaxf(s[x][y], s[x][y + 1])), fmaxf(s[x][y + 2], s[x][y + 3]));
                        }
                    }
                    const float base = u.alone ? (high == -INFINITY ? 0.f : high * c) : lse2;
                    const float2 b2 = make_float2(-base, -base);
                    float2 l2 = make_float2(0.f, 0.f), d2 = l2;
#pragma unroll
                    for (int x = 0; x < C; ++x) {
                        float d[32];
                        tmem_ld32(dp_at + x * 32, d);
                        tmem_wait(d);
#pragma unroll
                        for (int y = 0; y < 32; y += 2) {
                            float2 e = fma_(make_float2(s[x][y], s[x][y + 1]), c2, b2);
                            e.x = ex2(e.x);
                            e.y = ex2(e.y);
                            s[x][y] = e.x;
                            s[x][y + 1] = e.y;
                            l2 = add_(l2, e);
                            d2 = fma_(e, x * 32 + y < most ? make_float2(d[y], d[y + 1]) : make_float2(0.f, 0.f), d2);
                        }
                    }
                    float inv = 1.f;
                    if (u.alone) {
                        const float l = total(l2);
                        inv = l == 0.f ? 0.f : 1.f / l;
                        delta = total(d2) * inv;
                    }
                    // the last tile's weights have been multiplied
                    if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.w_free[group]), turn ^ 1u))) return false;
                    const float2 i2 = make_float2(inv, inv), n2 = make_float2(-delta, -delta);
#pragma unroll
                    for (int x = 0; x < C; ++x) {
                        float d[32];
                        tmem_ld32(dp_at + x * 32, d);
                        tmem_wait(d);
#pragma unroll
                        for (int y = 0; y < 32; y += 8) {
                            uint32_t p[4], ds[4];
#pragma unroll
                            for (int z = 0; z < 4; ++z) {
                                const int at = y + 2 * z;
                                const float2 v = mul_(make_float2(s[x][at], s[x][at + 1]), i2);
                                p[z] = pack2(v, T());
                                ds[z] = pack2(mul_(v, add_(make_float2(d[at], d[at + 1]), n2)), T());
                            }
                            const uint32_t at = p_row + (((x * 4 + y / 8) ^ (lane & 7)) << 4);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(p[0]), "r"(p[1]), "r"(p[2]), "r"(p[3])
                                         : "memory");
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + kWeights), "r"(ds[0]), "r"(ds[1]), "r"(ds[2]),
                                         "r"(ds[3])
                                         : "memory");
                        }
                    }
                    return true;
                };
                if (!(u.keys <= 32 ? weigh(std::integral_constant<int, 1>()) : weigh(std::integral_constant<int, 2>()))) return false;
                fence_proxy_async_smem();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive<1>(smem_addr(&bars.p_full[group]));
                if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.dq_full[group]), turn))) return false;
                turn ^= 1u;
                fence_after_sync();
                if (u.alone)
#pragma unroll 1
                    for (int d = 0; d < DH; d += 32) {
                        float v[32];
                        tmem_ld32(dp_at + d, v);
                        tmem_wait(v);
                        if (whole) {
                            if (lane == 0) tma_wait_read<0>();
                            __syncwarp();
                        }
#pragma unroll
                        for (int y = 0; y < 32; y += 8) {
                            Pack<T, 8> q;
#pragma unroll
                            for (int z = 0; z < 4; ++z)
                                q.set(z, some ? mul_(make_float2(v[y + 2 * z], v[y + 2 * z + 1]), make_float2(a.scale, a.scale)) : make_float2(0.f, 0.f));
                            if (whole)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(out + lane * 64 + ((y / 8 ^ (lane >> 1 & 3)) << 4)),
                                             "r"(q.w.x), "r"(q.w.y), "r"(q.w.z), "r"(q.w.w)
                                             : "memory");
                            else if (in && d + y < a.dh)
                                q.store(to + d + y);
                        }
                        if (whole) {
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) {
                                if (d < a.dh) tma_store_heads(&mdq, d, head, u.token + ((t * 128 + quad * 32) >> log_pack), out);
                                tma_commit();
                            }
                        }
                    }
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive<1>(smem_addr(&bars.dq_read[group]));
            }
            // the unit's sums, a key a lane: dv in the first two quarters, dk in the others; their
            // MMAs came after dq's
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.w_free[group]), turn ^ 1u))) return false;
            fence_after_sync();
            {
                const int key = r & 63;
                const bool is_dk = quad >= 2, in = key < u.keys;
                const int64_t row = (int64_t)u.key + key, at = (int64_t)u.kv_head * a.dh;
                T* to = is_dk ? (T*)g.dk + row * g.ld_dk + at : (T*)g.dv + row * g.ld_dv + at;
                const float scale = is_dk ? a.scale : 1.f;
#pragma unroll 1
                for (int d = 0; d < DH; d += 32) {
                    float v[32];
                    tmem_ld32(mine + sum_col(group) + (is_dk ? 0u : (uint32_t)DH) + d, v);
                    tmem_wait(v);
                    if (!in) continue;
#pragma unroll
                    for (int y = 0; y < 32; y += 8) {
                        if (d + y >= a.dh) break;
                        Pack<T, 8> q;
#pragma unroll
                        for (int z = 0; z < 4; ++z)
                            q.set(z, counts ? make_float2(v[y + 2 * z] * scale, v[y + 2 * z + 1] * scale) : make_float2(0.f, 0.f));
                        q.store(to + d + y);
                    }
                }
            }
            fence_before_sync();
            return true;
        });
        // the last rows of dq are read from shared memory until then
        if (lane == 0) tma_wait_all();
    }
    __syncwarp();
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (*(volatile int*)&bars.pulse.dead) {
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

template <class T, int DH>
cudaError_t run(const AttendArgs& a, const AttendGrads& g, cudaStream_t s) {
    CUtensorMap mq, mdo, mk, mv, mdq;
    const int pack = a.group;
    int log_pack = 0;
    while (1 << log_pack < pack) ++log_pack;
    cudaError_t e = make_head_map(&mq, a.type, a.q, a.Tq, a.heads, a.dh, a.ld_q, pack, 128 / pack);
    if (e == cudaSuccess) e = make_head_map(&mdo, a.type, g.d_out, a.Tq, a.heads, a.dh, g.ld_d_out, pack, 128 / pack);
    if (e == cudaSuccess) e = make_head_map(&mk, a.type, a.k, a.Tk, a.kv_heads, a.dh, a.ld_k, 1, kKeys);
    if (e == cudaSuccess) e = make_head_map(&mv, a.type, a.v, a.Tk, a.kv_heads, a.dh, a.ld_v, 1, kKeys);
    if (e == cudaSuccess)
        e = make_head_map(&mdq, a.type, g.dq, a.Tq, a.heads, a.dh, g.ld_dq, pack <= 32 ? pack : 1, pack <= 32 ? 32 / pack : 1, 32);
    if (e == cudaSuccess) e = allow_smem(k_grad_short<T, DH>, BriefShape<DH>::kSmem);
    if (e != cudaSuccess) return e;
    const int64_t units = a.B * a.kv_heads;
    const dim3 grid((unsigned)(units < a.num_sms ? units : a.num_sms));
    return launch_next(k_grad_short<T, DH>, grid, dim3(BriefShape<DH>::kThreads), BriefShape<DH>::kSmem, false, s, mq, mdo, mk, mv, mdq, a, g,
                       log_pack, units);
}

}  // namespace

cudaError_t launch_attend_grad_short(const AttendArgs& a, const AttendGrads& g, cudaStream_t s) {
    auto go = [&](auto t) {
        using T = decltype(t);
        return a.dh <= 64 ? run<T, 64>(a, g, s) : run<T, 128>(a, g, s);
    };
    return a.type == IFVS_T_F16 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ifvs
