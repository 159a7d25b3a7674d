// The gated feed-forward block and its gradient (ifvs_ffn, ifvs_ffn_grad).
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wo^T
//   dh = dy Wo, dg = dh u act'(g), du = dh act(g)
//   dx = [dg du] W_in, dW_in = [dg du]^T x, dWo = dy^T h          (W_in = [Wg; Wu])
//
// k_hidden makes h with both projections in one accumulator tile (128 tokens x
// FT gate columns and the same FT up columns), k_hidden_grad makes h, dg and du
// from x and dy with three (g, u and dh all sum over D), so that nothing of the
// hidden layer is kept from the forward call.  h, dg and du are rounded to the
// arrays' type between the products, because the tensor cores multiply 16-bit
// operands (and k_few keeps to it): against float64 y and the gradients are off by
// 0.0022 to 0.0024 of their norm in bfloat16, where rounding the outputs alone
// takes 0.0017 (float16 0.0003 and 0.0002).  k_products makes the other
// products, those of the gradient in one launch.  All are persistent: a CTA, or
// a pair of CTAs that share one MMA of 256 rows, takes tiles; a warp fills a
// ring of operand stages by TMA, a warp issues the MMAs, the others turn
// accumulators into 16-bit tiles in shared memory and store them by TMA.
#include "few.cuh"
#include "products.cuh"

namespace ifvs {

namespace {

// ---- h = act(x Wg^T) * (x Wu^T) ------------------------------------------------------
// Bound by the tensor pipe: 17408 x 960 x 2560 (171 GFLOP) 92 us, 1.86 PFLOP/s, the
// pipe 87 % active.
// FT hidden columns per tile: gate rows and up rows of W_in side by side in B.  In
// a pair the first CTA holds the gate's rows, the second the up projection's.
template <int CG, int FT>
struct HiddenShape {
    static constexpr int kEpi = FT / 16;                 // a warp: 32 rows x 64 columns
    static constexpr uint32_t kStage = kABytes + 2 * FT / CG * 128, kOut = kEpi * kOutBytes;
    static constexpr int kStages = stages_of(kStage, kOut);
    static constexpr size_t kSmem = smem_of(kStage, kOut);
};

template <int CG, int FT>
__device__ __forceinline__ void load_projections(uint32_t dst, const CUtensorMap* mw, int f, int F, int k, int rank, uint32_t bar) {
    if constexpr (CG == 1) {
        tma_load<CG>(dst, mw, k, f, bar);
        tma_load<CG>(dst + FT * 128, mw, k, F + f, bar);
    } else {
        tma_load<CG>(dst, mw, k, rank * F + f, bar);
    }
}

template <int ACT, int CG, int FT>
__global__ void __launch_bounds__(HiddenShape<CG, FT>::kEpi * 32 + 64, 1)
k_hidden(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw,
         const __grid_constant__ CUtensorMap mh, Grid g, bool f16, Waits waits) {
    using Sh = HiddenShape<CG, FT>;
    constexpr int EPI = Sh::kEpi, S = Sh::kStages;
    __shared__ __align__(8) Bars<S> bars;
    const uint32_t ring = dynamic_smem(), out = ring + S * Sh::kStage;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    const uint32_t tmem = setup<CG, EPI>(bars);
    const Watch w{&bars.dead, waits};
    const int tiles = g.m_tiles * g.n_tiles, first = blockIdx.x / CG, step = gridDim.x / CG;
    int filled = 0;

    if (warp == EPI) {
        if (elect_one()) {
            Ring<S> r;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step) {
                const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
                for (int k = 0; k < g.k_steps; ++k, r.next(), ++filled) {
                    if (!(ok = w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u))) break;
                    const uint32_t a = ring + r.at * Sh::kStage, bar = smem_addr(&bars.full[r.at]);
                    if (rank == 0) mbar_arrive_expect_tx(bar, CG * Sh::kStage + waits.extra);
                    tma_load<CG>(a, &mx, k * kStepK, (mn.x * CG + rank) * kRows, bar);
                    load_projections<CG, FT>(a + kABytes, &mw, mn.y * FT, g.cols, k * kStepK, rank, bar);
                }
            }
            start_dependents();
        }
    } else if (warp == EPI + 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = mma_desc(CG * kRows, 2 * FT, f16, false, false);
            const Operands o(ring, ring + kABytes, false, false);
            Ring<S> r;
            Ring<2> acc;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step, acc.next()) {
                if (!(ok = w.wait(smem_addr(&bars.acc_empty[acc.at]), acc.parity ^ 1u))) break;
                fence_after_sync();
                for (int k = 0; k < g.k_steps; ++k, r.next()) {
                    if (!(ok = w.wait(smem_addr(&bars.full[r.at]), r.parity))) break;
                    fence_after_sync();
                    o.mma<CG>(tmem + acc.at * 256, r.at * Sh::kStage, idesc, k == 0);
                    mma_commit<CG>(smem_addr(&bars.empty[r.at]));
                }
                if (ok) mma_commit<CG>(smem_addr(&bars.acc_full[acc.at]));
            }
        }
    } else {
        OutTile<1> o{out + (uint32_t)warp * kOutBytes};
        const int quad = warp & 3, part = (warp >> 2) * 64;
        Ring<2> acc;
        for (int t = first; t < tiles; t += step, acc.next()) {
            const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
            const int row = (mn.x * CG + rank) * kRows + quad * 32, col = mn.y * FT + part;
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full[acc.at]), acc.parity))) break;
            fence_after_sync();
            const uint32_t tm = tmem + acc.at * 256 + part + ((uint32_t)quad << 21);
            o.begin(lane);
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
                float a[32], u[32];
                tmem_ld32(tm + c, a);
                tmem_ld32(tm + FT + c, u);
                tmem_wait(a);
                tmem_wait(u);
                if (c == 32) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive<CG>(smem_addr(&bars.acc_empty[acc.at]));
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    float v, slope;
                    activation<ACT>(a[j], v, slope);
                    u[j] *= v;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    o.put(lane, c / 8 + j, pack16(u[8 * j], u[8 * j + 1], f16), pack16(u[8 * j + 2], u[8 * j + 3], f16),
                          pack16(u[8 * j + 4], u[8 * j + 5], f16), pack16(u[8 * j + 6], u[8 * j + 7], f16));
            }
            o.store(lane, &mh, col, row, row < g.rows && col < g.cols);
        }
        if (lane == 0) tma_wait_all();
    }
    finish<CG, EPI>(bars, tmem, filled, rank == 0, waits);
}

// ---- h, dg, du from x and dy ---------------------------------------------------------
// Per tile first dh = dy Wo (FT columns), then g and u (2 FT).  TMEM: g | u in
// columns FT .. 3 FT - 1; dh in the first FT or from 3 FT by turns, so that the
// next tile's dh accumulates while this tile's values are read.  16411 x 1024 x 4096
// (413 GFLOP) 267 us, 1.55 PFLOP/s, the tensor pipe 68 % active.  Shared memory
// allows 86 %: per 64 of the sum 56 KB come in by TMA and are read by the MMAs, 112
// KB or 896 clocks at 128 bytes each, against 768 clocks of MMAs.  What holds the
// rest has not been measured; g | u are read before the next tile's may begin.
template <int CG, int FT>
struct GradShape {
    static constexpr int kEpi = FT / 16;
    static constexpr uint32_t kStage = kABytes + 2 * FT / CG * 128, kOut = kEpi * 2 * kOutBytes;
    static constexpr uint32_t kDhBytes = kABytes + FT / CG * 128;      // of a stage of dh
    static constexpr int kStages = stages_of(kStage, kOut);
    static constexpr size_t kSmem = smem_of(kStage, kOut);
};

template <int ACT, int CG, int FT>
__global__ void __launch_bounds__(GradShape<CG, FT>::kEpi * 32 + 64, 1)
k_hidden_grad(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mdy,
              const __grid_constant__ CUtensorMap mw, const __grid_constant__ CUtensorMap mwo,
              const __grid_constant__ CUtensorMap mh, const __grid_constant__ CUtensorMap mdg,
              const __grid_constant__ CUtensorMap mdu, Grid g, bool f16, Waits waits) {
    using Sh = GradShape<CG, FT>;
    constexpr int EPI = Sh::kEpi, S = Sh::kStages;
    __shared__ __align__(8) Bars<S> bars;     // of the accumulators' barriers the first pair alone
    const uint32_t ring = dynamic_smem(), out = ring + S * Sh::kStage;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    const uint32_t tmem = setup<CG, EPI>(bars);
    const Watch w{&bars.dead, waits};
    const int tiles = g.m_tiles * g.n_tiles, first = blockIdx.x / CG, step = gridDim.x / CG;
    int filled = 0;

    if (warp == EPI) {
        if (elect_one()) {
            Ring<S> r;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step) {
                const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
                const int row = (mn.x * CG + rank) * kRows;
                for (int k = 0; k < 2 * g.k_steps; ++k, r.next(), ++filled) {
                    if (!(ok = w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u))) break;
                    const uint32_t a = ring + r.at * Sh::kStage, bar = smem_addr(&bars.full[r.at]);
                    if (k < g.k_steps) {
                        if (rank == 0) mbar_arrive_expect_tx(bar, CG * Sh::kDhBytes + waits.extra);
                        tma_load<CG>(a, &mdy, k * kStepK, row, bar);
                        load_tile<CG>(true, a + kABytes, &mwo, mn.y * FT + rank * (FT / CG), FT / CG, k * kStepK, bar);
                    } else {
                        const int kk = (k - g.k_steps) * kStepK;
                        if (rank == 0) mbar_arrive_expect_tx(bar, CG * Sh::kStage + waits.extra);
                        tma_load<CG>(a, &mx, kk, row, bar);
                        load_projections<CG, FT>(a + kABytes, &mw, mn.y * FT, g.cols, kk, rank, bar);
                    }
                }
            }
            start_dependents();
        }
    } else if (warp == EPI + 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t id_gu = mma_desc(CG * kRows, 2 * FT, f16, false, false);
            const uint32_t id_dh = mma_desc(CG * kRows, FT, f16, false, true);
            const Operands of_gu(ring, ring + kABytes, false, false), of_dh(ring, ring + kABytes, false, true);
            Ring<S> r;
            uint32_t parity = 0;
            int turn = 0;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step, ++turn, parity ^= 1u) {
                // dh's place was read two tiles ago, before the g | u of the last tile
                for (int k = 0; k < 2 * g.k_steps; ++k, r.next()) {
                    if (k == g.k_steps) {
                        if (!(ok = w.wait(smem_addr(&bars.acc_empty[0]), parity ^ 1u))) break;
                        fence_after_sync();
                    }
                    if (!(ok = w.wait(smem_addr(&bars.full[r.at]), r.parity))) break;
                    fence_after_sync();
                    if (k < g.k_steps)
                        of_dh.mma<CG>(tmem + (turn & 1 ? 3 * FT : 0), r.at * Sh::kStage, id_dh, k == 0);
                    else
                        of_gu.mma<CG>(tmem + FT, r.at * Sh::kStage, id_gu, k == g.k_steps);
                    mma_commit<CG>(smem_addr(&bars.empty[r.at]));
                }
                if (ok) mma_commit<CG>(smem_addr(&bars.acc_full[0]));
            }
        }
    } else {
        OutTile<2> o{out + (uint32_t)warp * 2 * kOutBytes};
        const int quad = warp & 3, part = (warp >> 2) * 64;
        uint32_t parity = 0;
        int turn = 0;
        for (int t = first; t < tiles; t += step, ++turn, parity ^= 1u) {
            const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
            const int row = (mn.x * CG + rank) * kRows + quad * 32, col = mn.y * FT + part;
            const bool in = row < g.rows && col < g.cols;
            // g | u come after dh in the order of the MMAs
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full[0]), parity))) break;
            fence_after_sync();
            const uint32_t tm = tmem + part + ((uint32_t)quad << 21), td = tm + (turn & 1 ? 3 * FT : 0);
            uint32_t h[32], dg[32], du[32];
#pragma unroll
            for (int c = 0; c < 64; c += 32) {
                float a[32], u[32], d[32];
                tmem_ld32(tm + FT + c, a);
                tmem_ld32(tm + 2 * FT + c, u);
                tmem_ld32(td + c, d);
                tmem_wait(a);
                tmem_wait(u);
                tmem_wait(d);
                if (c == 32) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive<CG>(smem_addr(&bars.acc_empty[0]));
                }
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    float v0, s0, v1, s1;
                    activation<ACT>(a[j], v0, s0);
                    activation<ACT>(a[j + 1], v1, s1);
                    h[(c + j) / 2] = pack16(v0 * u[j], v1 * u[j + 1], f16);
                    dg[(c + j) / 2] = pack16(d[j] * u[j] * s0, d[j + 1] * u[j + 1] * s1, f16);
                    du[(c + j) / 2] = pack16(d[j] * v0, d[j + 1] * v1, f16);
                }
            }
            auto give = [&](const uint32_t (&q)[32], const CUtensorMap* map) {
                o.begin(lane);
#pragma unroll
                for (int j = 0; j < 8; ++j) o.put(lane, j, q[4 * j], q[4 * j + 1], q[4 * j + 2], q[4 * j + 3]);
                o.store(lane, map, col, row, in);
            };
            give(h, &mh);
            give(dg, &mdg);
            give(du, &mdu);
        }
        if (lane == 0) tma_wait_all();
    }
    finish<CG, EPI>(bars, tmem, filled, rank == 0, waits);
}

// ---- a few tokens ----------------------------------------------------------------------
// Up to kFewTokens tokens: the weights are read once and bound the call, and a
// tile of 128 tokens would leave most SMs without one.  Both kernels' GPU time,
// weights from memory, here against the tensor cores: 960 x 2560 1 token 8.0 us
// against 15.4, 2 tokens 8.7 against 15.0, 4 tokens 9.4 against 15.1; 128 x 344 3.6,
// 4.0 and 4.3 against 8.7.  Compiled for 8 tokens, 5 to 8 take 20 us against 15.3
// at 960 x 2560 and 7.4 against 8.7 at 128 x 344 (for 16: 35 and 9).
// The hidden values from both projections' sums; the output's.
template <int ACT>
struct HiddenOf {
    static constexpr int kRows = 2;
    static constexpr bool kChained = false;
    __device__ __forceinline__ float operator()(const float (&s)[2], int, int) const {
        float v, slope;
        activation<ACT>(s[0], v, slope);
        return v * s[1];
    }
};
struct SumOf {
    static constexpr int kRows = 1;
    static constexpr bool kChained = true;
    __device__ __forceinline__ float operator()(const float (&s)[1], int, int) const { return s[0]; }
};

// ---- host -------------------------------------------------------------------------
template <class T>
cudaError_t ffn_few(const FfnArgs& a, const void* x, void* y, void* h, cudaStream_t s) {
    const cudaError_t e = with_act(a.act, [&](auto act) {
        return launch_few((const T*)x, (const T*)a.w_in, (T*)h, (int)a.T, a.F, a.D, a.num_sms, HiddenOf<act()>(), s);
    });
    return e != cudaSuccess ? e : launch_few((const T*)h, (const T*)a.w_out, (T*)y, (int)a.T, a.D, a.F, a.num_sms, SumOf(), s);
}

}  // namespace

namespace {
TileArgs tile_args(const FfnArgs& a) { return {a.type, a.num_sms, a.waits}; }
bool hidden_pairs(const FfnArgs& a) { return use_pairs(tile_args(a), a.T, 2 * (int64_t)a.F, a.D); }
bool out_pairs(const FfnArgs& a) { return use_pairs(tile_args(a), a.T, a.D, a.F); }
// The gradient's products together.  The weights' sum over the tokens: few tokens
// are over before a pair has started (960 x 2560, pairs against single CTAs: 128
// tokens 35 us against 30, 512 42 against 39, 4096 116 against 149).
bool grad_pairs(const FfnArgs& a) {
    return a.T > 512 && (use_pairs(tile_args(a), a.T, a.D, 2 * (int64_t)a.F) || use_pairs(tile_args(a), 2 * (int64_t)a.F, a.D, a.T));
}
}  // namespace

size_t ffn_bytes(const FfnArgs& a) {
    return padded((size_t)a.T * a.F * 2) + (a.T > 0 ? Plan::part_bytes(tile_args(a), a.T, a.D, a.F, out_pairs(a)) : 0);
}
size_t ffn_grad_bytes(const FfnArgs& a) {
    if (a.T == 0) return 0;
    const bool p = grad_pairs(a);
    return padded((size_t)a.T * a.F * 2) + padded((size_t)a.T * a.F * 4) + Plan::part_bytes(tile_args(a), a.T, a.D, 2 * (int64_t)a.F, p) +
           Plan::part_bytes(tile_args(a), 2 * (int64_t)a.F, a.D, a.T, p) + Plan::part_bytes(tile_args(a), a.D, a.F, a.T, p);
}

cudaError_t launch_ffn(const FfnArgs& a, const void* x, void* y, uint8_t* work, cudaStream_t s) {
    if (a.T <= kFewTokens)
        return a.type == IFVS_T_F16 ? ffn_few<__half>(a, x, y, work, s) : ffn_few<__nv_bfloat16>(a, x, y, work, s);
    CUtensorMap mx, mw, mh;
    auto run = [&](auto act, auto cg, auto ft) {
        using Sh = HiddenShape<cg(), ft()>;
        cudaError_t e = make_map(&mx, a.type, x, a.T, a.D, a.D, kRows);
        if (e == cudaSuccess) e = make_map(&mw, a.type, a.w_in, 2 * (int64_t)a.F, a.D, a.D, ft());
        if (e == cudaSuccess) e = make_map(&mh, a.type, work, a.T, a.F, a.F, 32);
        if (e != cudaSuccess) return e;
        const Grid g{ceil_div(a.T, kRows * cg()), ceil_div(a.F, ft()), ceil_div(a.D, kStepK), (int)a.T, a.F};
        return launch_tiles<cg()>(k_hidden<act(), cg(), ft()>, (int64_t)g.m_tiles * g.n_tiles, a.num_sms, Sh::kEpi * 32 + 64,
                                  Sh::kSmem, false, s, mx, mw, mh, g, a.type == IFVS_T_F16, a.waits);
    };
    const cudaError_t e = with_act(a.act, [&](auto act) {
        return hidden_pairs(a) ? run(act, std::integral_constant<int, 2>(), std::integral_constant<int, 128>())
                                                   : run(act, std::integral_constant<int, 1>(), std::integral_constant<int, 64>());
    });
    if (e != cudaSuccess) return e;
    Plan plan(tile_args(a), out_pairs(a), work + padded((size_t)a.T * a.F * 2));
    plan.add(a.T, a.D, a.F, work, false, a.w_out, false, y);
    return plan.launch(true, s);
}

cudaError_t launch_ffn_grad(const FfnArgs& a, const void* x, const void* dy, void* dx, void* d_w_in, void* d_w_out,
                            uint8_t* work, cudaStream_t s) {
    const int64_t D = a.D, F = a.F;
    if (a.T == 0) {
        const cudaError_t e = cudaMemsetAsync(d_w_in, 0, (size_t)(2 * F * D) * 2, s);
        return e != cudaSuccess ? e : cudaMemsetAsync(d_w_out, 0, (size_t)(D * F) * 2, s);
    }
    uint8_t *h = work, *dgu = work + padded((size_t)a.T * F * 2);
    auto run = [&](auto act, auto cg, auto ft) {
        using Sh = GradShape<cg(), ft()>;
        CUtensorMap mx, mdy, mw, mwo, mh, mdg, mdu;
        cudaError_t e = make_map(&mx, a.type, x, a.T, D, D, kRows);
        auto then = [&](cudaError_t r) { e = e == cudaSuccess ? r : e; };
        then(make_map(&mdy, a.type, dy, a.T, D, D, kRows));
        then(make_map(&mw, a.type, a.w_in, 2 * F, D, D, ft()));
        then(make_map(&mwo, a.type, a.w_out, D, F, F, 64));
        then(make_map(&mh, a.type, h, a.T, F, F, 32));
        then(make_map(&mdg, a.type, dgu, a.T, F, 2 * F, 32));
        then(make_map(&mdu, a.type, dgu + F * 2, a.T, F, 2 * F, 32));
        if (e != cudaSuccess) return e;
        const Grid g{ceil_div(a.T, kRows * cg()), ceil_div(F, ft()), ceil_div(D, kStepK), (int)a.T, a.F};
        return launch_tiles<cg()>(k_hidden_grad<act(), cg(), ft()>, (int64_t)g.m_tiles * g.n_tiles, a.num_sms,
                                  Sh::kEpi * 32 + 64, Sh::kSmem, false, s, mx, mdy, mw, mwo, mh, mdg, mdu, g,
                                  a.type == IFVS_T_F16, a.waits);
    };
    const cudaError_t e = with_act(a.act, [&](auto act) {
        return hidden_pairs(a) ? run(act, std::integral_constant<int, 2>(), std::integral_constant<int, 128>())
                                        : run(act, std::integral_constant<int, 1>(), std::integral_constant<int, 64>());
    });
    if (e != cudaSuccess) return e;
    // the longest sums first
    Plan plan(tile_args(a), grad_pairs(a), dgu + padded((size_t)a.T * F * 4));
    auto d_in = [&] { plan.add(2 * F, D, a.T, dgu, true, x, true, d_w_in); };
    auto d_out = [&] { plan.add(D, F, a.T, dy, true, h, true, d_w_out); };
    if (a.T >= 2 * F) {
        d_in();
        d_out();
        plan.add(a.T, D, 2 * F, dgu, false, a.w_in, true, dx);
    } else {
        plan.add(a.T, D, 2 * F, dgu, false, a.w_in, true, dx);
        d_in();
        d_out();
    }
    return plan.launch(true, s);
}

}  // namespace ifvs
