// Attention of many short sequences on the tensor cores (ifvs_attend).
//
// Persistent CTAs take units, a tile of 128 rows of one group each, whose keys are mostly one
// chunk of KEYS.  A warp finds units, 16 at a time, a warp loads their queries, keys and values
// by TMA, a warp issues the MMAs, two see to keys that do not count; two or four groups of four warps take units by turns, so
// that one group's exponentials and output run beside the others' MMAs:
//   tensor pipe (two groups):  s_0  s_1 | o_0 s_2 | o_1 s_3 | ...
// What bounds a unit is the chain of its waits (loads, s, weights, o, output), which four
// groups hide better than two.  A thread takes a row's scores 32 at a time, twice: for their
// maximum, then for the weights, which leaves registers for four groups.  Sequences with more keys go on chunk by chunk as in
// attend_tc.cu.  Rows leave through shared memory by TMA, 32 at a time.
//
// 1024 sequences of 120 queries and 0 to 65 keys, 8 heads of 64 over 2: 68 us, 4.0 TB/s.  With
// three stages of queries and six of keys (four and five here) and the MMAs of whichever
// group's weights come first it takes 80: the issuing warp's polls cost the others more than
// they save.
#include "attend_tc.cuh"

namespace ifvs {

namespace {

constexpr int kBatch = 16, kBatches = 2;     // units that are found together; how far ahead

template <int DH, int KEYS>
struct ShortShape {
    static constexpr int kHalves = DH / 64;
    static constexpr int kGroups = DH == 64 && KEYS == 64 ? 4 : 2;       // TMEM: KEYS + DH columns each
    static constexpr int kSoft = 4 * kGroups, kLoader = kSoft, kIssuer = kSoft + 1, kFixer = kSoft + 2,      // warps
                         kFixers = 2, kFinder = kFixer + kFixers, kThreads = (kFinder + 1) * 32;
    static constexpr uint32_t kQ = kHalves * kHalfBytes;                 // 128 rows
    static constexpr uint32_t kKeyHalf = KEYS * 128, kK = kHalves * kKeyHalf, kKv = 2 * kK;
    static constexpr int kQs = DH == 128 ? 2 : (KEYS == 64 ? 4 : 3);
    static constexpr int kKvs = DH == 128 ? (KEYS == 64 ? 3 : 2) : (KEYS == 64 ? 5 : 4);
    static constexpr uint32_t kOut = kSoft * 32 * 128;              // 32 rows of 64 elements a warp
    static constexpr size_t kSmem = 1024 + kQs * kQ + kKvs * kKv + kOut;
};

struct Unit {
    int token, key;          // the first row's token, the first key
    int keys;
    int16_t rows, head, kv_head;
    uint8_t place, parity;   // of its first chunk in the ring of keys
};

template <int QS, int KS, int KEYS, int GROUPS>
struct ShortBars {
    uint64_t batch_full[kBatches], batch_empty[kBatches], q_full[QS], q_empty[QS], kv_full[KS], kv_empty[KS], fixed[KS], s_full[GROUPS],
        p_full[GROUPS], o_full[GROUPS], drain;
    Unit units[kBatches][kBatch];
    int count[kBatches];            // -1: there are no more
    alignas(16) float most[KS][KEYS];    // read four at a time: infinity, or -infinity for a key that does not count
    uint32_t tmem;
    Pulse pulse;
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
__global__ void __launch_bounds__(ShortShape<DH, KEYS>::kThreads, 1)
k_attend_short(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
               const __grid_constant__ CUtensorMap mo, AttendArgs a, AttendOut o, int log_pack, int64_t n_units) {
    using Sh = ShortShape<DH, KEYS>;
    constexpr int QS = Sh::kQs, KS = Sh::kKvs, W = KEYS / 32, GROUPS = Sh::kGroups;
    constexpr int kLoader = Sh::kLoader, kIssuer = Sh::kIssuer, kFixer = Sh::kFixer, kFinder = Sh::kFinder;
    constexpr bool kF16 = std::is_same_v<T, __half>;
    __shared__ __align__(16) ShortBars<QS, KS, KEYS, GROUPS> bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pack = 1 << log_pack;
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const uint32_t q_at = dynamic_smem(), kv_at = q_at + QS * Sh::kQ, out_at = kv_at + KS * Sh::kKv;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kBatches; ++i) {
            mbar_init(smem_addr(&bars.batch_full[i]), 1);
            mbar_init(smem_addr(&bars.batch_empty[i]), Sh::kSoft + 2 + Sh::kFixers);
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
        for (int i = 0; i < GROUPS; ++i) {
            mbar_init(smem_addr(&bars.s_full[i]), 1);
            mbar_init(smem_addr(&bars.p_full[i]), 4);
            mbar_init(smem_addr(&bars.o_full[i]), 1);
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
    // within a unit, and behind other units.  (With the second for all of them the 1024 sequences
    // above take 78 us.)
    const Watch w{&bars.pulse.dead, a.waits};
    const UnitWatch far{&bars.pulse, a.waits};
    auto s_col = [](int g) { return (uint32_t)g * KEYS; };
    auto o_col = [](int g) { return (uint32_t)GROUPS * KEYS + (uint32_t)g * DH; };
    int q_filled = 0, kv_filled = 0;             // by the loader's thread

    auto chunks_of = [](int keys) { return (keys + KEYS - 1) / KEYS; };
    // f(unit) for every step-th unit from the first-th on; by the warp, or (alone) by one of
    // its threads.  idle(): called before a batch is waited for; the finder may be waiting for
    // a group that waits for this role.
    auto units = [&](bool alone, int first, int step, auto&& idle, auto&& f) {
        uint32_t b = 0, parity = 0;
        for (;;) {
            if (!mbar_try_wait(smem_addr(&bars.batch_full[b]), parity) && !idle()) return false;
            bool ok = far.wait(smem_addr(&bars.batch_full[b]), parity);
            if (!alone) ok = __all_sync(0xFFFFFFFFu, ok);
            const int n = ok ? bars.count[b] : -1;
            if (n < 0) return ok;
            for (; first < n; first += step) {
                const Unit u = bars.units[b][first];
                if (!f(u)) return false;
            }
            first -= n;
            if (!alone) __syncwarp();
            if (alone || lane == 0) mbar_arrive<1>(smem_addr(&bars.batch_empty[b]));
            b = (b + 1) % kBatches;
            parity ^= b == 0;
        }
    };

    auto nothing = [] { return true; };

    if (warp == kFinder) {
        const int nh = a.heads >> log_pack;
        uint32_t b = 0, parity = 1, place = 0, turn = 0;
        // Rounds of a slot per CTA; the CTAs change places from round to round, since what the
        // slots hold may repeat with a period that divides the grid's.  (Taking the next eight
        // slots as a CTA comes to them, by a counter, takes 79 us where this takes 65.)
        const uint32_t grid = gridDim.x;
        for (int64_t round = 0; round * grid < n_units; round += kBatch) {
            const uint32_t seat = (uint32_t)((blockIdx.x + 37u * (uint32_t)((round + lane) % grid)) % grid);
            const int64_t mine = (round + lane) * grid + seat;
            Unit u{};
            if (lane < kBatch && mine < n_units) {
                const uint32_t slot = (uint32_t)(mine / nh), y = (uint32_t)(mine - (int64_t)slot * nh);
                uint32_t lo = 0, n = (uint32_t)a.B;      // the sequence: the last whose slots begin there or before
                while (n > 1) {
                    const uint32_t half = n / 2;
                    if (first_slot(a.q_offsets, lo + half, a.B, a.Tq, pack, 7) <= (int64_t)slot) {
                        lo += half;
                        n -= half;
                    } else {
                        n = half;
                    }
                }
                const int64_t tile = (int64_t)slot - first_slot(a.q_offsets, lo, a.B, a.Tq, pack, 7);
                const Span qs = span_of(a.q_offsets, lo, a.B, a.Tq), ks = span_of(a.kv_offsets, lo, a.B, a.Tk);
                const int64_t left = qs.len * pack - tile * 128;
                u.token = (int)(qs.at + (tile * 128 >> log_pack));
                u.key = (int)ks.at;
                u.keys = (int)ks.len;
                u.rows = tile < 0 || left <= 0 ? 0 : (int16_t)(left < 128 ? left : 128);
                u.head = (int16_t)(y << log_pack);
                u.kv_head = (int16_t)((y << log_pack) / a.group);
            }
            const uint32_t there = __ballot_sync(0xFFFFFFFFu, u.rows > 0);
            // places in the ring of keys: chunks before this unit's
            const int mine_chunks = u.rows > 0 ? chunks_of(u.keys) : 0;
            int before = mine_chunks;
#pragma unroll
            for (int x = 1; x < 32; x <<= 1) {
                const int other = __shfl_up_sync(0xFFFFFFFFu, before, x);
                if (lane >= x) before += other;
            }
            const int all = __shfl_sync(0xFFFFFFFFu, before, 31);
            const uint32_t at = place + (uint32_t)(before - mine_chunks);
            u.place = (uint8_t)(at % KS);
            u.parity = (uint8_t)((turn + at / KS) & 1u);
            turn += (place + (uint32_t)all) / KS;
            place = (place + (uint32_t)all) % KS;
            if (!__all_sync(0xFFFFFFFFu, far.wait(smem_addr(&bars.batch_empty[b]), parity))) break;
            if (u.rows > 0) bars.units[b][__popc(there & ((1u << lane) - 1u))] = u;
            if (lane == 0) bars.count[b] = __popc(there);
            __syncwarp();
            if (lane == 0) {
                far.further();
                mbar_arrive<1>(smem_addr(&bars.batch_full[b]));
            }
            b = (b + 1) % kBatches;
            parity ^= b == 0;
        }
        if (__all_sync(0xFFFFFFFFu, far.wait(smem_addr(&bars.batch_empty[b]), parity)) && lane == 0) {
            bars.count[b] = -1;
            mbar_arrive<1>(smem_addr(&bars.batch_full[b]));
        }
    } else if (warp == kLoader) {
        if (elect_one()) {
            Place<QS> qp;
            Place<KS> kp;
            units(true, 0, 1, nothing, [&](const Unit& u) {
                const int chunks = chunks_of(u.keys);
                if (chunks == 0) return true;
                if (!w.wait(smem_addr(&bars.q_empty[qp.at]), qp.parity ^ 1u)) return false;
                uint32_t bar = smem_addr(&bars.q_full[qp.at]);
                mbar_arrive_expect_tx(bar, Sh::kQ + a.waits.extra);
                for (int d = 0; d < Sh::kHalves; ++d)
                    tma_load_heads(q_at + qp.at * Sh::kQ + d * kHalfBytes, &mq, d * 64, u.head, u.token, bar);
                qp.next();
                ++q_filled;
                for (int j = 0; j < chunks; ++j) {
                    if (!w.wait(smem_addr(&bars.kv_empty[kp.at]), kp.parity ^ 1u)) return false;
                    bar = smem_addr(&bars.kv_full[kp.at]);
                    mbar_arrive_expect_tx(bar, Sh::kKv + a.waits.extra);
                    for (int d = 0; d < Sh::kHalves; ++d) {
                        const uint32_t to = kv_at + kp.at * Sh::kKv + d * Sh::kKeyHalf;
                        tma_load_heads(to, &mk, d * 64, u.kv_head, u.key + j * KEYS, bar);
                        tma_load_heads(to + Sh::kK, &mv, d * 64, u.kv_head, u.key + j * KEYS, bar);
                    }
                    kp.next();
                    ++kv_filled;
                }
                return true;
            });
        }
    } else if (warp == kIssuer) {
        if (elect_one()) {
            Place<QS> qp;
            Place<KS> kp;
            // what a group's weights will multiply: there, first, last, turn of p_full, parity,
            // blocks of 16 keys, stage
            uint32_t pending[GROUPS] = {}, turns = 0;
            auto of = [&](int g) {
                uint32_t p = 0;
#pragma unroll
                for (int i = 0; i < GROUPS; ++i) p = i == g ? pending[i] : p;
                return p;
            };
            auto put = [&](int g, uint32_t p) {
#pragma unroll
                for (int i = 0; i < GROUPS; ++i) pending[i] = i == g ? p : pending[i];
            };
            auto sums = [&](int g) {
                const uint32_t p = of(g);
                if (!(p & 1u)) return true;
                put(g, 0);
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
            int g = 0;
            auto flush = [&] {
                bool ok = true;
                for (int i = 0; i < GROUPS && ok; ++i) ok = sums((g + i) % GROUPS);     // in the units' order
                return ok;
            };
            const bool done = units(true, 0, 1, flush, [&](const Unit& u) {
                const int chunks = chunks_of(u.keys);
                bool ok = true;
                for (int j = 0; j < chunks && ok; ++j, kp.next()) {
                    if (!(ok = sums(g))) break;
                    // another group's last may hold the place in the ring that this one needs
                    for (int i = 0; i < GROUPS; ++i) {
                        const uint32_t other = of(i);
                        if ((other & 1u) && other >> 16 == kp.at) ok = ok && sums(i);
                    }
                    if (!ok) break;
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
                    put(g, 1u | (j == 0 ? 2u : 0u) | (j == chunks - 1 ? 4u : 0u) | (turns >> g & 1u) << 3 | kp.parity << 4 |
                               (uint32_t)blocks << 8 | kp.at << 16);
                    turns ^= 1u << g;
                }
                g = g + 1 == GROUPS ? 0 : g + 1;
                return ok;
            });
            if (done) flush();
        }
    } else if (warp >= kFixer) {
        // which keys count; values of those that do not become zeros, because 0 times what they
        // hold may be a NaN.  The fixers take units by turns, but see every chunk arrive.
        Place<KS> kp;
        int it = 0;
        units(false, 0, 1, nothing, [&](const Unit& u) {
            const int chunks = chunks_of(u.keys);
            const bool own = it++ % Sh::kFixers == warp - kFixer;
            bool ok = true;
            for (int j = 0; j < chunks && ok; ++j, kp.next()) {
                const int left = u.keys - j * KEYS, blocks = ((left < KEYS ? left : KEYS) + 15) / 16;
                uint32_t bits[W];
                if (own)
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const int key = i * 32 + lane;
                        bits[i] = __ballot_sync(
                            0xFFFFFFFFu, key < left && (a.kv_ids == nullptr || __ldg(a.kv_ids + (int64_t)u.key + (int64_t)j * KEYS + key) >= 0));
                    }
                ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.kv_full[kp.at]), kp.parity));
                if (!ok) break;
                if (!own) continue;
                bool any = false;
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    bars.most[kp.at][i * 32 + lane] = (bits[i] >> lane) & 1u ? INFINITY : -INFINITY;
                    // a row a lane; of a block of 16 behind the last key the MMAs read nothing
                    if (i * 32 + lane < blocks * 16 && !((bits[i] >> lane) & 1u)) {
                        any = true;
                        const uint32_t at = kv_at + kp.at * Sh::kKv + Sh::kK + (uint32_t)(i * 32 + lane) * 128u;
#pragma unroll
                        for (int d = 0; d < Sh::kHalves; ++d)
#pragma unroll
                            for (int x = 0; x < 8; ++x)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + d * Sh::kKeyHalf + ((x ^ (lane & 7)) << 4)),
                                             "r"(0)
                                             : "memory");
                    }
                }
                if (__any_sync(0xFFFFFFFFu, any)) fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive<1>(smem_addr(&bars.fixed[kp.at]));
            }
            return ok;
        });
    } else {
        const int group = warp >> 2, quad = warp & 3;
        const uint32_t mine = tmem + ((uint32_t)quad << 21), s_at = mine + s_col(group), o_at = mine + o_col(group),
                       out = out_at + (uint32_t)warp * 32 * 128;
        const float c = a.scale * kLog2e;
        const float2 c2 = make_float2(c, c);
        uint32_t s_turn = 0, o_turn = 0;
        units(false, group, GROUPS, nothing, [&](const Unit& u) {
            bool ok = true;
            const int chunks = chunks_of(u.keys);
            Place<KS> kp{u.place, u.parity};
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < chunks && ok; ++j, kp.next(), s_turn ^= 1u) {
                const int left = u.keys - j * KEYS, n = left < KEYS ? left : KEYS;
                // in this order: a wait for `fixed` may not be two fills ahead, and the group sees
                // those of its own units alone; s there means that the fill before was used
                ok = __all_sync(0xFFFFFFFFu, far.wait(smem_addr(&bars.s_full[group]), s_turn) &&
                                                 w.wait(smem_addr(&bars.fixed[kp.at]), kp.parity));
                if (!ok) break;
                fence_after_sync();
                // 32 scores of this row, -infinity for keys that do not count, whatever their score
                // is (the smaller of a NaN and -infinity is -infinity; of a NaN that counts it is
                // infinity, which makes the row a NaN as well)
                auto scores = [&](float(&s)[32], int x) {
                    tmem_ld32(s_at + x * 32, s);
                    const float4* most = reinterpret_cast<const float4*>(bars.most[kp.at] + x * 32);
                    tmem_wait(s);
#pragma unroll
                    for (int y = 0; y < 32; y += 4) {
                        const float4 b = most[y / 4];
                        s[y] = fminf(s[y], b.x);
                        s[y + 1] = fminf(s[y + 1], b.y);
                        s[y + 2] = fminf(s[y + 2], b.z);
                        s[y + 3] = fminf(s[y + 3], b.w);
                    }
                };
                float high = -INFINITY;
#pragma unroll 1
                for (int x = 0; x * 32 < n; ++x) {
                    float s[32];
                    scores(s, x);
                    float top = fmaxf(high, s[0]);
#pragma unroll
                    for (int y = 1; y < 31; y += 2) top = fmaxf(top, fmaxf(s[y], s[y + 1]));
                    high = fmaxf(top, s[31]);
                }
                high = fmaxf(high * c, m);
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
                // the weights of 32 keys take 16 columns: always behind the scores still to come
#pragma unroll 1
                for (int x = 0; x * 32 < n; ++x) {
                    float s[32];
                    scores(s, x);
                    uint32_t p[16];
#pragma unroll
                    for (int y = 0; y < 32; y += 2) {
                        float2 e = fma_(make_float2(s[y], s[y + 1]), c2, b2);
                        e.x = ex2(e.x);
                        e.y = ex2(e.y);
                        sum = add_(sum, e);
                        p[y / 2] = pack2(e, T());
                    }
                    tmem_st16(s_at + x * 16, p);
                }
                l += total(sum);
                tmem_st_wait();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive<1>(smem_addr(&bars.p_full[group]));
                if (lane == 0 && (j & 63) == 63) far.further();
            }
            if (ok && chunks > 0) {
                ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.o_full[group]), o_turn));
                o_turn ^= 1u;
            }
            if (!ok) return false;
            fence_after_sync();
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const int r = quad * 32 + lane;
            const int64_t token = (int64_t)u.token + (r >> log_pack);
            const int head = u.head + (r & (pack - 1));
            const bool in = r < u.rows, whole = quad * 32 + 32 <= u.rows && pack <= 32;
            T* to = (T*)o.out + token * o.ld + (int64_t)head * a.dh;
#pragma unroll 1
            for (int d = 0; d < DH; d += 32) {
                float v[32];
                tmem_ld32(o_at + d, v);
                tmem_wait(v);
                if (whole && (d & 32) == 0) {
                    if (lane == 0) tma_wait_read<0>();
                    __syncwarp();
                }
#pragma unroll
                for (int y = 0; y < 32; y += 8) {
                    Pack<T, 8> q;
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                        q.set(z, chunks > 0 ? mul_(make_float2(v[y + 2 * z], v[y + 2 * z + 1]), make_float2(inv, inv)) : make_float2(0.f, 0.f));
                    if (whole)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                                         out + lane * 128 + (((((uint32_t)d & 32u) + y) >> 3 ^ (lane & 7)) << 4)),
                                     "r"(q.w.x), "r"(q.w.y), "r"(q.w.z), "r"(q.w.w)
                                     : "memory");
                    else if (in && d + y < a.dh)
                        q.store(to + d + y);
                }
                if (whole && (d & 32)) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store_heads(&mo, d - 32, u.head, u.token + (quad * 32 >> log_pack), out);
                        tma_commit();
                    }
                }
            }
            if (in && o.lse) o.lse[token * a.heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
            // the next unit's MMAs write o once this group's weights are there
            fence_before_sync();
            return true;
        });
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

template <class T, int DH, int KEYS>
cudaError_t run(const AttendArgs& a, const AttendOut& o, int pack, cudaStream_t s) {
    CUtensorMap mq, mk, mv, mo;
    cudaError_t e = make_head_map(&mq, a.type, a.q, a.Tq, a.heads, a.dh, a.ld_q, pack, 128 / pack);
    if (e == cudaSuccess) e = make_head_map(&mk, a.type, a.k, a.Tk, a.kv_heads, a.dh, a.ld_k, 1, KEYS);
    if (e == cudaSuccess) e = make_head_map(&mv, a.type, a.v, a.Tk, a.kv_heads, a.dh, a.ld_v, 1, KEYS);
    if (e == cudaSuccess) e = make_head_map(&mo, a.type, o.out, a.Tq, a.heads, a.dh, o.ld, pack <= 32 ? pack : 1, pack <= 32 ? 32 / pack : 1);
    if (e == cudaSuccess) e = allow_smem(k_attend_short<T, DH, KEYS>, ShortShape<DH, KEYS>::kSmem);
    if (e != cudaSuccess) return e;
    int log_pack = 0;
    while (1 << log_pack < pack) ++log_pack;
    const int64_t units = slots(a.Tq, a.B, pack, 7) * (a.heads / pack);
    const dim3 grid((unsigned)(units < a.num_sms ? units : a.num_sms));
    return launch_next(k_attend_short<T, DH, KEYS>, grid, dim3(ShortShape<DH, KEYS>::kThreads), ShortShape<DH, KEYS>::kSmem, false, s, mq, mk, mv, mo,
                       a, o, log_pack, units);
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
