// The gradient of attention of long sequences on the tensor cores (ifvs_attend_grad).
//
// Two kernels, so that every sum has one owner and a fixed order; both make the scores
// again (seven products where a shared pass would take five):
//   k_keys_tc   a CTA owns 128 keys: p^T = exp(k q^T - lse), dp^T = v do^T,
//               dv += p^T do, dk += ds^T q over the rows of their group
//   k_rows_tc   a CTA owns 128 rows: p = exp(q k^T - lse), dp = do v^T, dq += ds k
// Scores and sums are in TMEM; a thread reads 64 scores of its lane, and p and ds go back
// to TMEM as the 16-bit operands of the next MMAs.  Two halves of the threads take half of
// the columns each.  While they take exponentials the tensor pipe makes the other scores:
//   k_keys_tc:  .. dk dp' | dv' s'' | dk' dp'' ..     p' beside dk dp', ds' beside dv' s''
//      DH = 64: .. dk | dv' s'' dp'' | dk' | dv'' ..  TMEM has room for a second dp
//   k_rows_tc:  .. dq s'' | dp'' | dq' s''' ..        p' beside dq s'', ds' beside dp''
// k_rows_tc starts first, since its CTAs mostly have more to do; k_keys_tc's fill the SMs as
// it runs out.
//
// Four sequences of about 1500 x 4250, 8 heads of 64: 223 us, of seven products 820 TFLOP/s;
// apart k_keys_tc takes 143 us and k_rows_tc 102, their tensor pipes active a third of the time:
// the waits between MMAs and exponentials, and a CTA's start and end, which nothing hides since
// it holds all of TMEM.  With one place of dp, made again once ds is there, they take 150 and
// 116, and then with sixteen warps for the exponentials, 32 scores a thread, 155 and 125.
#include "attend_tc.cuh"

namespace ifvs {

namespace {

constexpr int kSoftWarps = 8, kLoader = 8, kIssuer = 9, kFixer = 10, kThreads = 352;

// Shared memory: a resident pair of tiles (keys and values, or queries and gradients) and a
// ring of pairs of the others.
template <int DH>
struct GradShape {
    static constexpr int kHalves = DH / 64;
    static constexpr uint32_t kTile = kHalves * kHalfBytes;           // 128 rows
    static constexpr int kStages = DH == 128 ? 2 : 4;
    static constexpr size_t kSmem = 1024 + (2 + 2 * kStages) * kTile;
};

template <int S>
struct GradBars {
    uint64_t resident, full[S], fixed[S], empty[S], s_full[2], dp_full[2], dp_read, p_full, ds_full, acc_full, drain;
    uint32_t mask[S][4];
    alignas(16) float lse2[S][128], delta[S][128];       // terms of the ring's rows, read four at a time
    uint32_t tmem;
    int dead;
};

template <int S>
__device__ __forceinline__ uint32_t begin(GradBars<S>& b) {
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        mbar_init(smem_addr(&b.resident), 1);
        for (int i = 0; i < S; ++i) {
            mbar_init(smem_addr(&b.full[i]), 1);
            mbar_init(smem_addr(&b.fixed[i]), 1);
            mbar_init(smem_addr(&b.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&b.s_full[i]), 1);
            mbar_init(smem_addr(&b.dp_full[i]), 1);
        }
        mbar_init(smem_addr(&b.dp_read), kSoftWarps);
        mbar_init(smem_addr(&b.p_full), kSoftWarps);
        mbar_init(smem_addr(&b.ds_full), kSoftWarps);
        mbar_init(smem_addr(&b.acc_full), 1);
        mbar_init(smem_addr(&b.drain), 1);
        b.dead = 0;
        fence_mbar_init();
    }
    if (warp == kIssuer) tmem_alloc<1>(smem_addr(&b.tmem), 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    return b.tmem;
}

// filled: stages that the loader's thread armed (its other lanes: 0); armed: whether it armed
// the resident pair
template <int S>
__device__ __forceinline__ void end(GradBars<S>& b, uint32_t tmem, int filled, bool armed, const Waits& waits) {
    const int warp = threadIdx.x >> 5;
    __syncwarp();
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (*(volatile int*)&b.dead) {
        // a wait ran out: wait once more, bounded, for what is in flight
        const long long begun = clock64();
        auto bounded = [&](uint32_t bar, uint32_t parity) {
            while (!mbar_try_wait(bar, parity) && clock64() - begun < waits.cycles) {
            }
        };
        if (warp == kLoader) {
            if (armed) bounded(smem_addr(&b.resident), 0);
            for (int i = filled > S ? filled - S : 0; i < filled; ++i) bounded(smem_addr(&b.full[i % S]), (uint32_t)(i / S) & 1u);
        }
        if (warp == kIssuer && elect_one()) {
            mma_commit<1>(smem_addr(&b.drain));
            bounded(smem_addr(&b.drain), 0);
        }
        __syncwarp();
        __syncthreads();
    }
    if (warp == kIssuer) tmem_free<1>(tmem, 512);
}

// d = a b^T over DH, both 128 rows in shared memory
template <int DH>
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {
#pragma unroll
    for (int h = 0; h < DH / 64; ++h) {
        const uint64_t da = tile_desc(a + h * kHalfBytes, false), db = tile_desc(b + h * kHalfBytes, false);
#pragma unroll
        for (int k = 0; k < 4; ++k) mma_f16<1>(d, da + k * desc_step(false), db + k * desc_step(false), idesc, h + k > 0);
    }
}
// d (+)= x b: x 128 x 128 in TMEM, each half of its columns' operands where that half's scores
// began; b 128 rows in shared memory
__device__ __forceinline__ void mma_sums(uint32_t d, uint32_t x, uint32_t b, uint32_t idesc, bool more) {
    const uint64_t db = rows_desc(b);
#pragma unroll
    for (int k = 0; k < 8; ++k)
        mma_f16_tmem_a(d, x + (k >> 2) * 64 + (k & 3) * 8, db + k * desc_step(true), idesc, more || k > 0);
}

// zeros to the rows of a tile (of `halves` halves) for which !in(row)
template <class In>
__device__ __forceinline__ void clear_rows(uint32_t at, int halves, const In& in) {
#pragma unroll 1
    for (int i = threadIdx.x & 31; i < 128 * halves * 8; i += 32)
        if (!in((i >> 3) & 127))
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + (uint32_t)i * 16u), "r"(0) : "memory");
}

// 64 columns of this warp's lanes
__device__ __forceinline__ void load64(uint32_t at, float (&v)[2][32]) {
    tmem_ld32(at, v[0]);
    tmem_ld32(at + 32, v[1]);
}
__device__ __forceinline__ void wait64(float (&v)[2][32]) {
    tmem_wait(v[0]);
    tmem_wait(v[1]);
}

// ---- delta = out do, per token and head: four lanes each ----------------------------------------
template <class T>
__global__ void __launch_bounds__(256) k_attend_delta(AttendArgs a, AttendGrads g, float* delta) {
    const int64_t row = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 2), n = a.Tq * a.heads;
    const int l = threadIdx.x & 3;
    start_dependents();
    float2 sum = make_float2(0.f, 0.f);
    if (row < n) {
        const int64_t token = row / a.heads, at = (row - token * a.heads) * a.dh;
        for (int c = l * 8; c < a.dh; c += 32) {
            Pack<T, 8> x, y;
            x.load((const T*)g.out + token * g.ld_out + at + c);
            y.load((const T*)g.d_out + token * g.ld_d_out + at + c);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum = fma_(x.get(j), y.get(j), sum);
        }
    }
    float v = total(sum);
    v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
    v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
    if (row < n && l == 0) delta[row] = v;
}

// ---- dk, dv ------------------------------------------------------------------------------------
// TMEM: s^T (then p^T) 0, dp^T (then ds^T) 128, dv 256, dk 256 + DH; for DH = 64 dp^T of odd
// tiles 384
template <class T, int DH>
__global__ void __launch_bounds__(kThreads, 1)
k_keys_tc(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ CUtensorMap mk,
          const __grid_constant__ CUtensorMap mv, AttendArgs a, AttendGrads g, int log_pack, int splits, const float* __restrict__ delta,
          float* part_dk, float* part_dv) {
    using Sh = GradShape<DH>;
    constexpr int S = Sh::kStages, DPS = DH == 64 ? 2 : 1;       // places of dp^T
    constexpr bool kF16 = std::is_same_v<T, __half>;
    __shared__ __align__(16) GradBars<S> bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y, split = blockIdx.z;
    auto dp_col = [](int j) { return DPS == 2 && (j & 1) ? 384u : 128u; };
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const Slot slot = slot_of(a.kv_offsets, a.B, a.Tk, 1, 7, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t key0 = slot.tile * 128;
    if (slot.tile < 0 || key0 >= ks.len) {
        if (last_cta()) wait_before();
        return;
    }
    // tiles of rows, for every part of the group that shares tiles
    const int64_t n_rows = qs.len << log_pack, per_part = (n_rows + 127) / 128, tiles = per_part * (a.group >> log_pack);
    const int64_t t0 = tiles * split / splits, t1 = tiles * (split + 1) / splits;
    const int n = (int)(t1 - t0);
    // a tile's first row and its head, one tile after the other: 64-bit divisions, a tile in
    // the warp that brings the rows' terms, take longer than the tile's MMAs
    struct Tile {
        int64_t row;
        int head;
    };
    auto first_tile = [&] {
        const int64_t part = n > 0 ? t0 / per_part : 0;
        return Tile{(t0 - part * per_part) * 128, hk * a.group + (int)(part << log_pack)};
    };
    auto next_tile = [&](Tile& t) {
        t.row += 128;
        if (t.row >= n_rows) {
            t.row = 0;
            t.head += 1 << log_pack;
        }
    };

    const uint32_t k_at = dynamic_smem(), v_at = k_at + Sh::kTile, ring = v_at + Sh::kTile;
    auto q_of = [&](int stage) { return ring + (uint32_t)stage * 2 * Sh::kTile; };
    const uint32_t tmem = begin(bars);
    const Watch w{&bars.dead, a.waits};
    int filled = 0;

    if (warp == kLoader) {
        if (elect_one() && n > 0) {
            const uint32_t bar = smem_addr(&bars.resident);
            mbar_arrive_expect_tx(bar, 2 * Sh::kTile + a.waits.extra);
            for (int d = 0; d < Sh::kHalves; ++d) {
                tma_load_heads(k_at + d * kHalfBytes, &mk, d * 64, hk, (int)(ks.at + key0), bar);
                tma_load_heads(v_at + d * kHalfBytes, &mv, d * 64, hk, (int)(ks.at + key0), bar);
            }
            Ring<S> r;
            Tile tile = first_tile();
            for (int j = 0; j < n; ++j, r.next(), ++filled, next_tile(tile)) {
                if (!w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u)) break;
                const uint32_t full = smem_addr(&bars.full[r.at]);
                const int head = tile.head, token = (int)(qs.at + (tile.row >> log_pack));
                mbar_arrive_expect_tx(full, 2 * Sh::kTile + a.waits.extra);
                for (int d = 0; d < Sh::kHalves; ++d) {
                    tma_load_heads(q_of(r.at) + d * kHalfBytes, &mq, d * 64, head, token, full);
                    tma_load_heads(q_of(r.at) + Sh::kTile + d * kHalfBytes, &mdo, d * 64, head, token, full);
                }
            }
        }
    } else if (warp == kIssuer) {
        if (elect_one() && n > 0) {
            const uint32_t id_s = mma_desc(128, 128, kF16, false, false), id_o = mma_desc(128, DH, kF16, false, true);
            bool ok = w.wait(smem_addr(&bars.resident), 0);
            auto there = [&](int j) {
                if (!w.wait(smem_addr(&bars.full[j % S]), (uint32_t)(j / S) & 1u)) return false;
                if (!w.wait(smem_addr(&bars.fixed[j % S]), (uint32_t)(j / S) & 1u)) return false;
                fence_after_sync();
                return true;
            };
            auto s_of = [&](int j) {
                mma_rows<DH>(tmem, k_at, q_of(j % S), id_s);
                mma_commit<1>(smem_addr(&bars.s_full[0]));
            };
            auto dp_of = [&](int j) {
                mma_rows<DH>(tmem + dp_col(j), v_at, q_of(j % S) + Sh::kTile, id_s);
                mma_commit<1>(smem_addr(&bars.dp_full[j % DPS]));
            };
            if (ok && (ok = there(0))) {
                s_of(0);
                dp_of(0);
            }
            for (int j = 0; j < n && ok; ++j) {
                if (!(ok = w.wait(smem_addr(&bars.p_full), (uint32_t)j & 1u))) break;
                fence_after_sync();
                mma_sums(tmem + 256, tmem, q_of(j % S) + Sh::kTile, id_o, j > 0);
                if (j + 1 < n) {
                    if (!(ok = there(j + 1))) break;
                    s_of(j + 1);
                    if (DPS == 2) dp_of(j + 1);
                }
                if (!(ok = w.wait(smem_addr(&bars.ds_full), (uint32_t)j & 1u))) break;
                fence_after_sync();
                mma_sums(tmem + 256 + DH, tmem + dp_col(j), q_of(j % S), id_o, j > 0);
                mma_commit<1>(smem_addr(&bars.empty[j % S]));
                if (DPS == 1 && j + 1 < n) dp_of(j + 1);
            }
            if (ok) mma_commit<1>(smem_addr(&bars.acc_full));
        }
    } else if (warp == kFixer) {
        // The rows' terms; rows behind the sequence become zeros with lse infinite, so that
        // their p and ds are 0 whatever they held.  A row without keys has lse = -infinity and
        // no key here that counts: the same.  The next tile's terms are on their way meanwhile.
        float l[4], d[4];
        auto terms = [&](const Tile& t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t row = t.row + i * 32 + lane;
                l[i] = -INFINITY;
                d[i] = 0.f;
                if (row < n_rows) {
                    const int64_t at = (qs.at + (row >> log_pack)) * a.heads + t.head + ((int)row & ((1 << log_pack) - 1));
                    l[i] = __ldg(g.lse + at);
                    d[i] = __ldcg(delta + at);
                }
            }
        };
        Tile tile = first_tile();
        if (n > 0) terms(tile);
        for (int j = 0; j < n; ++j) {
            const int rows = n_rows - tile.row < 128 ? (int)(n_rows - tile.row) : 128;
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.full[j % S]), (uint32_t)(j / S) & 1u))) break;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bars.lse2[j % S][i * 32 + lane] = l[i] == -INFINITY ? -INFINITY : -l[i] * kLog2e;
                bars.delta[j % S][i * 32 + lane] = -d[i];
            }
            next_tile(tile);
            if (j + 1 < n) terms(tile);
            if (rows < 128) {
                clear_rows(q_of(j % S), Sh::kHalves, [&](int r) { return r < rows; });
                clear_rows(q_of(j % S) + Sh::kTile, Sh::kHalves, [&](int r) { return r < rows; });
                fence_proxy_async_smem();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive<1>(smem_addr(&bars.fixed[j % S]));
        }
    } else if (warp < kSoftWarps) {
        const int quad = warp & 3, half = warp >> 2;
        const uint32_t mine = tmem + ((uint32_t)quad << 21) + half * 64;
        const float2 c2 = make_float2(a.scale * kLog2e, a.scale * kLog2e);
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            const uint32_t turn = (uint32_t)j & 1u;
            ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.fixed[j % S]), (uint32_t)(j / S) & 1u) &&
                                             w.wait(smem_addr(&bars.s_full[0]), turn));
            if (!ok) break;
            fence_after_sync();
            float p[2][32], d[2][32];
            load64(mine, p);
            const float4 *lse = reinterpret_cast<const float4*>(&bars.lse2[j % S][half * 64]),
                         *del = reinterpret_cast<const float4*>(&bars.delta[j % S][half * 64]);
            uint32_t w16[32];
            wait64(p);
#pragma unroll
            for (int y = 0; y < 64; y += 4) {
                float* s = &p[y >> 5][y & 31];
                const float4 t = lse[y / 4];
                const float2 e0 = fma_(make_float2(s[0], s[1]), c2, make_float2(t.x, t.y)),
                             e1 = fma_(make_float2(s[2], s[3]), c2, make_float2(t.z, t.w));
                s[0] = ex2(e0.x);
                s[1] = ex2(e0.y);
                s[2] = ex2(e1.x);
                s[3] = ex2(e1.y);
                w16[y / 2] = pack2(make_float2(s[0], s[1]), T());
                w16[y / 2 + 1] = pack2(make_float2(s[2], s[3]), T());
            }
            tmem_st32(mine, w16);
            tmem_st_wait();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive<1>(smem_addr(&bars.p_full));
            ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.dp_full[j % DPS]), (uint32_t)(j / DPS) & 1u));
            if (!ok) break;
            fence_after_sync();
            load64(mine + dp_col(j), d);
            wait64(d);
#pragma unroll
            for (int y = 0; y < 64; y += 4) {
                const float *x = &d[y >> 5][y & 31], *s = &p[y >> 5][y & 31];
                const float4 t = del[y / 4];
                w16[y / 2] = pack2(mul_(make_float2(s[0], s[1]), add_(make_float2(x[0], x[1]), make_float2(t.x, t.y))), T());
                w16[y / 2 + 1] = pack2(mul_(make_float2(s[2], s[3]), add_(make_float2(x[2], x[3]), make_float2(t.z, t.w))), T());
            }
            tmem_st32(mine + dp_col(j), w16);
            tmem_st_wait();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive<1>(smem_addr(&bars.ds_full));
        }
        if (ok && n > 0) ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full), 0));
        if (ok) {
            fence_after_sync();
            const int64_t key = key0 + quad * 32 + lane;
            const bool in = key < ks.len, counts = in && n > 0 && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key) >= 0);
            const int64_t row = ks.at + key, part = (((int64_t)split * a.Tk + row) * a.kv_heads + hk) * a.dh;
            // half 0 writes dv, half 1 dk
            T* to = half ? (T*)g.dk + row * g.ld_dk + (int64_t)hk * a.dh : (T*)g.dv + row * g.ld_dv + (int64_t)hk * a.dh;
            float* to_part = (half ? part_dk : part_dv) + part;
            const float scale = half ? a.scale : 1.f;
            const uint32_t acc = tmem + ((uint32_t)quad << 21) + 256 + half * DH;
#pragma unroll 1
            for (int d = 0; d < DH; d += 32) {
                float v[32];
                if (n > 0) {
                    tmem_ld32(acc + d, v);
                    tmem_wait(v);
                }
                if (!in) continue;
#pragma unroll
                for (int y = 0; y < 32; ++y) v[y] = counts ? v[y] * scale : 0.f;
#pragma unroll
                for (int y = 0; y < 32; y += 8) {
                    if (d + y >= a.dh) break;
                    if (splits > 1) {
                        float4* p = reinterpret_cast<float4*>(to_part + d + y);
                        p[0] = make_float4(v[y], v[y + 1], v[y + 2], v[y + 3]);
                        p[1] = make_float4(v[y + 4], v[y + 5], v[y + 6], v[y + 7]);
                    } else {
                        Pack<T, 8> q;
#pragma unroll
                        for (int z = 0; z < 4; ++z) q.set(z, make_float2(v[y + 2 * z], v[y + 2 * z + 1]));
                        q.store(to + d + y);
                    }
                }
            }
        }
    }
    end(bars, tmem, filled, filled > 0, a.waits);
    if (last_cta()) wait_before();
}

// ---- dq ----------------------------------------------------------------------------------------
// TMEM: s of even tiles 0, of odd ones 128 (then ds), dp 256, dq 384
template <class T, int DH>
__global__ void __launch_bounds__(kThreads, 1)
k_rows_tc(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mdo, const __grid_constant__ CUtensorMap mk,
          const __grid_constant__ CUtensorMap mv, AttendArgs a, AttendGrads g, int log_pack, const float* __restrict__ delta) {
    using Sh = GradShape<DH>;
    constexpr int S = Sh::kStages;
    constexpr bool kF16 = std::is_same_v<T, __half>;
    __shared__ __align__(16) GradBars<S> bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pack = 1 << log_pack, h0 = blockIdx.y * pack, hk = h0 / a.group;
    const Slot slot = slot_of(a.q_offsets, a.B, a.Tq, pack, 7, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t row0 = slot.tile * 128, left = qs.len * pack - row0;
    if (slot.tile < 0 || left <= 0) {
        if (last_cta()) wait_before();
        return;
    }
    const int rows = left < 128 ? (int)left : 128, n = (int)((ks.len + 127) / 128);

    const uint32_t q_at = dynamic_smem(), do_at = q_at + Sh::kTile, ring = do_at + Sh::kTile;
    auto k_of = [&](int stage) { return ring + (uint32_t)stage * 2 * Sh::kTile; };
    const uint32_t tmem = begin(bars);
    wait_before();           // delta; with it there k_keys_tc may start
    start_dependents();
    const Watch w{&bars.dead, a.waits};
    int filled = 0;

    if (warp == kLoader) {
        if (elect_one() && n > 0) {
            const uint32_t bar = smem_addr(&bars.resident);
            const int token = (int)(qs.at + (row0 >> log_pack));
            mbar_arrive_expect_tx(bar, 2 * Sh::kTile + a.waits.extra);
            for (int d = 0; d < Sh::kHalves; ++d) {
                tma_load_heads(q_at + d * kHalfBytes, &mq, d * 64, h0, token, bar);
                tma_load_heads(do_at + d * kHalfBytes, &mdo, d * 64, h0, token, bar);
            }
            Ring<S> r;
            for (int j = 0; j < n; ++j, r.next(), ++filled) {
                if (!w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u)) break;
                const uint32_t full = smem_addr(&bars.full[r.at]);
                mbar_arrive_expect_tx(full, 2 * Sh::kTile + a.waits.extra);
                for (int d = 0; d < Sh::kHalves; ++d) {
                    tma_load_heads(k_of(r.at) + d * kHalfBytes, &mk, d * 64, hk, (int)(ks.at + (int64_t)j * 128), full);
                    tma_load_heads(k_of(r.at) + Sh::kTile + d * kHalfBytes, &mv, d * 64, hk, (int)(ks.at + (int64_t)j * 128), full);
                }
            }
        }
    } else if (warp == kIssuer) {
        if (elect_one() && n > 0) {
            const uint32_t id_s = mma_desc(128, 128, kF16, false, false), id_o = mma_desc(128, DH, kF16, false, true);
            bool ok = w.wait(smem_addr(&bars.resident), 0);
            auto s_of = [&](int j) {
                if (!w.wait(smem_addr(&bars.full[j % S]), (uint32_t)(j / S) & 1u)) return false;
                if (!w.wait(smem_addr(&bars.fixed[j % S]), (uint32_t)(j / S) & 1u)) return false;
                fence_after_sync();
                mma_rows<DH>(tmem + (j & 1) * 128, q_at, k_of(j % S), id_s);
                mma_commit<1>(smem_addr(&bars.s_full[j & 1]));
                return true;
            };
            auto dp_of = [&](int j) {
                mma_rows<DH>(tmem + 256, do_at, k_of(j % S) + Sh::kTile, id_s);
                mma_commit<1>(smem_addr(&bars.dp_full[0]));
            };
            if (ok && (ok = s_of(0))) {
                dp_of(0);
                if (n > 1) ok = s_of(1);
            }
            for (int j = 0; j < n && ok; ++j) {
                if (j + 1 < n) {         // as soon as dp is in registers
                    if (!(ok = w.wait(smem_addr(&bars.dp_read), (uint32_t)j & 1u))) break;
                    fence_after_sync();
                    dp_of(j + 1);
                }
                if (!(ok = w.wait(smem_addr(&bars.ds_full), (uint32_t)j & 1u))) break;
                fence_after_sync();
                mma_sums(tmem + 384, tmem + (j & 1) * 128, k_of(j % S), id_o, j > 0);
                mma_commit<1>(smem_addr(&bars.empty[j % S]));
                if (j + 2 < n) ok = s_of(j + 2);
            }
            if (ok) mma_commit<1>(smem_addr(&bars.acc_full));
        }
    } else if (warp == kFixer) {
        // which keys count; keys that do not become zeros, because 0 times what they hold may
        // be a NaN (their values meet dp alone, which is not used)
        for (int j = 0; j < n; ++j) {
            uint32_t bits[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t key = (int64_t)j * 128 + i * 32 + lane;
                bits[i] = __ballot_sync(0xFFFFFFFFu, key < ks.len && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key) >= 0));
            }
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.full[j % S]), (uint32_t)(j / S) & 1u))) break;
            if (lane == 0)
#pragma unroll
                for (int i = 0; i < 4; ++i) bars.mask[j % S][i] = bits[i];
            if ((bits[0] & bits[1] & bits[2] & bits[3]) != 0xFFFFFFFFu) {
                clear_rows(k_of(j % S), Sh::kHalves, [&](int r) {
                    return ((r < 32 ? bits[0] : r < 64 ? bits[1] : r < 96 ? bits[2] : bits[3]) >> (r & 31)) & 1u;
                });
                fence_proxy_async_smem();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive<1>(smem_addr(&bars.fixed[j % S]));
        }
    } else if (warp < kSoftWarps) {
        const int quad = warp & 3, half = warp >> 2, r = quad * 32 + lane;
        const uint32_t mine = tmem + ((uint32_t)quad << 21) + half * 64;
        const float2 c2 = make_float2(a.scale * kLog2e, a.scale * kLog2e);
        const int64_t token = qs.at + ((row0 + r) >> log_pack);
        const int head = h0 + ((int)(row0 + r) & (pack - 1));
        float lse2 = -INFINITY, del = 0.f;       // negated; a row without keys: p = 0
        if (r < rows) {
            const float v = __ldg(g.lse + token * a.heads + head);
            if (v != -INFINITY) lse2 = -v * kLog2e;
            del = -__ldcg(delta + token * a.heads + head);
        }
        const float2 l2 = make_float2(lse2, lse2), d2 = make_float2(del, del);
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.fixed[j % S]), (uint32_t)(j / S) & 1u) &&
                                             w.wait(smem_addr(&bars.s_full[j & 1]), (uint32_t)(j / 2) & 1u));
            if (!ok) break;
            fence_after_sync();
            float p[2][32], d[2][32];
            const uint32_t at = mine + (j & 1) * 128;
            load64(at, p);
            const uint32_t b0 = bars.mask[j % S][half * 2], b1 = bars.mask[j % S][half * 2 + 1];
            wait64(p);
#pragma unroll
            for (int y = 0; y < 64; y += 2) {
                float* s = &p[y >> 5][y & 31];
                const float2 e = fma_(make_float2(s[0], s[1]), c2, l2);
                s[0] = ex2(e.x);
                s[1] = ex2(e.y);
            }
            ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.dp_full[0]), (uint32_t)j & 1u));
            if (!ok) break;
            fence_after_sync();
            load64(mine + 256, d);
            wait64(d);
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive<1>(smem_addr(&bars.dp_read));
#pragma unroll
            for (int y = 0; y < 64; y += 2) {
                float *x = &d[y >> 5][y & 31], *s = &p[y >> 5][y & 31];
                const float2 v = mul_(make_float2(s[0], s[1]), add_(make_float2(x[0], x[1]), d2));
                x[0] = v.x;
                x[1] = v.y;
            }
            if ((b0 & b1) != 0xFFFFFFFFu)
#pragma unroll
                for (int y = 0; y < 64; ++y)
                    if (!(((y < 32 ? b0 : b1) >> (y & 31)) & 1u)) d[y >> 5][y & 31] = 0.f;
            uint32_t w16[32];
#pragma unroll
            for (int y = 0; y < 64; y += 2) w16[y / 2] = pack2(make_float2(d[y >> 5][y & 31], d[y >> 5][(y & 31) + 1]), T());
            tmem_st32(at, w16);
            tmem_st_wait();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive<1>(smem_addr(&bars.ds_full));
        }
        if (ok && n > 0) ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full), 0));
        if (ok) {
            fence_after_sync();
            T* to = (T*)g.dq + token * g.ld_dq + (int64_t)head * a.dh;
            const uint32_t acc = tmem + ((uint32_t)quad << 21) + 384;
#pragma unroll 1
            for (int d = half * (DH / 2); d < (half + 1) * (DH / 2); d += 32) {
                float v[32];
                if (n > 0) {
                    tmem_ld32(acc + d, v);
                    tmem_wait(v);
                }
                if (r >= rows) continue;
#pragma unroll
                for (int y = 0; y < 32; y += 8) {
                    if (d + y >= a.dh) break;
                    Pack<T, 8> q;
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                        q.set(z, n > 0 ? make_float2(v[y + 2 * z] * a.scale, v[y + 2 * z + 1] * a.scale) : make_float2(0.f, 0.f));
                    q.store(to + d + y);
                }
            }
        }
    }
    end(bars, tmem, filled, filled > 0, a.waits);
}

template <class T, int DH>
cudaError_t run(const AttendArgs& a, const AttendGrads& g, int pack, int splits, float* delta, float* part_dk, float* part_dv,
                cudaStream_t s) {
    CUtensorMap mq, mdo, mk, mv;
    cudaError_t e = make_head_map(&mq, a.type, a.q, a.Tq, a.heads, a.dh, a.ld_q, pack, 128 / pack);
    if (e == cudaSuccess) e = make_head_map(&mdo, a.type, g.d_out, a.Tq, a.heads, a.dh, g.ld_d_out, pack, 128 / pack);
    if (e == cudaSuccess) e = make_head_map(&mk, a.type, a.k, a.Tk, a.kv_heads, a.dh, a.ld_k, 1, 128);
    if (e == cudaSuccess) e = make_head_map(&mv, a.type, a.v, a.Tk, a.kv_heads, a.dh, a.ld_v, 1, 128);
    if (e == cudaSuccess) e = allow_smem(k_keys_tc<T, DH>, GradShape<DH>::kSmem);
    if (e == cudaSuccess) e = allow_smem(k_rows_tc<T, DH>, GradShape<DH>::kSmem);
    if (e != cudaSuccess) return e;
    int log_pack = 0;
    while (1 << log_pack < pack) ++log_pack;
    e = launch_next(k_attend_delta<T>, dim3((unsigned)((a.Tq * a.heads + 63) / 64)), dim3(256), 0, false, s, a, g, delta);
    if (e != cudaSuccess) return e;
    e = launch_next(k_rows_tc<T, DH>, dim3((unsigned)slots(a.Tq, a.B, pack, 7), (unsigned)(a.heads / pack)), dim3(kThreads),
                    GradShape<DH>::kSmem, true, s, mq, mdo, mk, mv, a, g, log_pack, (const float*)delta);
    if (e != cudaSuccess) return e;
    return launch_next(k_keys_tc<T, DH>, dim3((unsigned)slots(a.Tk, a.B, 1, 7), (unsigned)a.kv_heads, (unsigned)splits), dim3(kThreads),
                       GradShape<DH>::kSmem, true, s, mq, mdo, mk, mv, a, g, log_pack, splits, (const float*)delta, part_dk, part_dv);
}

}  // namespace

cudaError_t launch_attend_grad_tc(const AttendArgs& a, const AttendGrads& g, int pack, int splits, float* delta, float* part_dk,
                                  float* part_dv, cudaStream_t s) {
    auto go = [&](auto t) {
        using T = decltype(t);
        return a.dh <= 64 ? run<T, 64>(a, g, pack, splits, delta, part_dk, part_dv, s)
                          : run<T, 128>(a, g, pack, splits, delta, part_dk, part_dv, s);
    };
    return a.type == IFVS_T_F16 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ifvs
