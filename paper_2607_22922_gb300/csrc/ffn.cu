// The gated feed-forward block and its gradient (ifvs_ffn, ifvs_ffn_grad).
//
//   g = x Wg^T, u = x Wu^T, h = act(g) u, y = h Wo^T
//   dh = dy Wo, dg = dh u act'(g), du = dh act(g)
//   dx = [dg du] W_in, dW_in = [dg du]^T x, dWo = dy^T h          (W_in = [Wg; Wu])
//
// k_hidden makes h with both projections in one accumulator tile (128 tokens x
// 128 gate columns and the same 128 up columns), k_hidden_grad makes h, dg and
// du from x and dy with three (g, u and dh all sum over D), so that nothing of
// the hidden layer is kept from the forward call.  The other products are
// k_product.  All are persistent: one CTA per SM takes tiles; a warp fills a
// ring of operand stages by TMA, a warp issues the MMAs, the others turn
// accumulators into 16-bit tiles in shared memory and store them by TMA.
#include "umma.cuh"

namespace ifvs {

namespace {

constexpr uint32_t kRowTile = 128;                        // rows of an accumulator tile
constexpr uint32_t kABytes = kRowTile * 128;              // a stage's A tile
constexpr uint32_t kBBytes = 256 * 128;                   // a stage's B tile (up to 256 columns)
constexpr uint32_t kStageBytes = kABytes + kBBytes;
constexpr uint32_t kOutBytes = 32 * 128;                  // 32 rows x 64 columns of output

// act(g) and act'(g)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& v, float& slope) {
    if (ACT == IFVS_ACT_RELU) {
        v = g > 0.f ? g : 0.f;
        slope = g > 0.f ? 1.f : 0.f;
    } else if (ACT == IFVS_ACT_SILU) {
        const float p = __fdividef(1.f, 1.f + __expf(-g));
        v = g * p;
        slope = p * (1.f + g * (1.f - p));
    } else {
        const float p = 0.5f * erfcf(-0.70710678f * g);
        v = g * p;
        slope = p + g * 0.39894228f * __expf(-0.5f * g * g);
    }
}

// Barriers of a CTA: operand stages, accumulator slots, the last MMAs
template <int S, int SLOTS>
struct Bars {
    uint64_t full[S], empty[S], acc_full[SLOTS], acc_empty[SLOTS], drain;
};

// What every kernel here starts with; returns the TMEM base (512 columns).
// Warps 0 .. EPI - 1: epilogue, EPI: TMA, EPI + 1: MMA.
template <int EPI, int S, int SLOTS>
__device__ __forceinline__ uint32_t setup(Bars<S, SLOTS>& b, uint32_t* tmem, int* dead) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(smem_addr(&b.full[i]), 1);
            mbar_init(smem_addr(&b.empty[i]), 1);
        }
        for (int i = 0; i < SLOTS; ++i) {
            mbar_init(smem_addr(&b.acc_full[i]), 1);
            mbar_init(smem_addr(&b.acc_empty[i]), EPI);
        }
        mbar_init(smem_addr(&b.drain), 1);
        *dead = 0;
        fence_mbar_init();
    }
    if (threadIdx.x / 32 == EPI + 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    return *tmem;
}

// The end of a kernel: with everything in order the roles have waited for
// their own work; a dead CTA waits here for what it had in flight.
template <int EPI, int S, int SLOTS>
__device__ __forceinline__ void finish(Bars<S, SLOTS>& b, uint32_t tmem, const int* dead, int filled) {
    __syncwarp();
    __syncthreads();
    if (*(volatile const int*)dead) {
        auto bounded = [](uint32_t bar, uint32_t parity) {
            const long long t0 = clock64();
            while (!mbar_try_wait(bar, parity) && clock64() - t0 < kWaitCycles) {
            }
        };
        if (threadIdx.x == EPI * 32)
            for (int i = max(0, filled - S); i < filled; ++i) bounded(smem_addr(&b.full[i % S]), (uint32_t)(i / S) & 1u);
        if (threadIdx.x == EPI * 32 + 32) {
            mma_commit(smem_addr(&b.drain));
            bounded(smem_addr(&b.drain), 0);
        }
        __syncthreads();
    }
    if (threadIdx.x / 32 == EPI + 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// K-major tiles: `rows` rows from `row`; MN-major: `rows` columns from `row`.
// k: the first of the stage's 64 along the sum.
template <bool MN>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, int row, int rows, int k, uint32_t bar) {
    if (MN) {
#pragma unroll 1
        for (int i = 0; i < rows; i += 64) tma_load(dst + (uint32_t)i * 128u, map, row + i, k, bar);
    } else {
        tma_load(dst, map, k, row, bar);
    }
}

// the four MMAs of a stage
template <bool A_MN, bool B_MN>
__device__ __forceinline__ void mma_stage(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool first) {
    const uint64_t da = tile_desc(a, A_MN), db = tile_desc(b, B_MN);
#pragma unroll
    for (uint32_t i = 0; i < kStepK / 16; ++i)
        mma_f16(d, da + i * desc_step(A_MN), db + i * desc_step(B_MN), idesc, !first || i > 0);
}

// This warp's 32 rows x 64 columns of 16-bit output: `words` packed pairs go to
// the staging tile (swizzled), a TMA store takes it.  BUFS tiles per warp.
template <int BUFS>
struct OutTile {
    uint32_t base;      // of this warp's staging tiles
    uint32_t at = 0;
    __device__ __forceinline__ void begin(int lane) {
        if (lane == 0) tma_wait_read<BUFS - 1>();
        __syncwarp();
    }
    // 8 columns (16 bytes) `chunk` of this lane's row
    __device__ __forceinline__ void put(int lane, int chunk, uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + at * kOutBytes + lane * 128 +
                                                                      ((chunk ^ (lane & 7)) << 4)),
                     "r"(w0), "r"(w1), "r"(w2), "r"(w3)
                     : "memory");
    }
    __device__ __forceinline__ void store(int lane, const CUtensorMap* map, int col, int row, bool in) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            if (in) tma_store(map, col, row, base + at * kOutBytes);
            tma_commit();
        }
        at = at + 1 == BUFS ? 0 : at + 1;
    }
};

struct Grid {
    int m_tiles, n_tiles, k_steps;
    int rows, cols;      // of the output
};

__device__ __forceinline__ uint32_t dynamic_smem() {
    extern __shared__ uint8_t raw[];
    return (smem_addr(raw) + 1023u) & ~1023u;
}

// ---- C = A B^T in 16 bits ----------------------------------------------------------
// A K-major [rows][K] or MN-major [K][rows]; B the same with `cols`.
constexpr int kProductStages = 4;

template <bool A_MN, bool B_MN, int BN>
__global__ void __launch_bounds__(192, 1)
k_product(const __grid_constant__ CUtensorMap ma, const __grid_constant__ CUtensorMap mb,
          const __grid_constant__ CUtensorMap mc, Grid g, bool f16, int* err) {
    constexpr int EPI = 4, S = kProductStages;
    __shared__ __align__(8) Bars<S, 2> bars;
    __shared__ uint32_t tmem_slot;
    __shared__ int dead;
    const uint32_t ring = dynamic_smem(), out = ring + S * kStageBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = setup<EPI>(bars, &tmem_slot, &dead);
    const Watch w{&dead, err};
    const int tiles = g.m_tiles * g.n_tiles;
    int filled = 0;
    wait_before();

    if (warp == EPI) {
        if (lane == 0) {
            Ring<S> r;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
                const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
                for (int k = 0; k < g.k_steps; ++k, r.next(), ++filled) {
                    if (!(ok = w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u))) break;
                    const uint32_t a = ring + r.at * kStageBytes, bar = smem_addr(&bars.full[r.at]);
                    mbar_arrive_expect_tx(bar, kABytes + BN * 128);
                    load_tile<A_MN>(a, &ma, mn.x * kRowTile, kRowTile, k * kStepK, bar);
                    load_tile<B_MN>(a + kABytes, &mb, mn.y * BN, BN, k * kStepK, bar);
                }
            }
            start_dependents();
        }
    } else if (warp == EPI + 1) {
        if (lane == 0) {
            const uint32_t idesc = mma_desc(BN, f16, A_MN, B_MN);
            Ring<S> r;
            Ring<2> acc;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x, acc.next()) {
                if (!(ok = w.wait(smem_addr(&bars.acc_empty[acc.at]), acc.parity ^ 1u))) break;
                fence_after_sync();
                for (int k = 0; k < g.k_steps; ++k, r.next()) {
                    if (!(ok = w.wait(smem_addr(&bars.full[r.at]), r.parity))) break;
                    fence_after_sync();
                    const uint32_t a = ring + r.at * kStageBytes;
                    mma_stage<A_MN, B_MN>(tmem + acc.at * 256, a, a + kABytes, idesc, k == 0);
                    mma_commit(smem_addr(&bars.empty[r.at]));
                }
                mma_commit(smem_addr(&bars.acc_full[acc.at]));
            }
        }
    } else {
        OutTile<2> o{out + (uint32_t)warp * 2 * kOutBytes};
        Ring<2> acc;
        for (int t = blockIdx.x; t < tiles; t += gridDim.x, acc.next()) {
            const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
            const int row = mn.x * (int)kRowTile + warp * 32;
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full[acc.at]), acc.parity))) break;
            fence_after_sync();
            const uint32_t tm = tmem + acc.at * 256 + ((uint32_t)warp << 21);
#pragma unroll 1
            for (int c = 0; c < BN; c += 64) {
                float v[2][32];
                tmem_ld32(tm + c, v[0]);
                tmem_ld32(tm + c + 32, v[1]);
                o.begin(lane);
                tmem_wait(v[0]);
                tmem_wait(v[1]);
                if (c + 64 == BN) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_addr(&bars.acc_empty[acc.at]));
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float* q = &v[j >> 2][(j & 3) * 8];
                    o.put(lane, j, pack16(q[0], q[1], f16), pack16(q[2], q[3], f16), pack16(q[4], q[5], f16),
                          pack16(q[6], q[7], f16));
                }
                const int col = mn.y * BN + c;
                o.store(lane, &mc, col, row, row < g.rows && col < g.cols);
            }
        }
        if (lane == 0) tma_wait_all();
    }
    finish<EPI>(bars, tmem, &dead, filled);
}

// ---- h = act(x Wg^T) * (x Wu^T) ------------------------------------------------------
constexpr int kHiddenEpi = 8;

template <int ACT>
__global__ void __launch_bounds__(kHiddenEpi * 32 + 64, 1)
k_hidden(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw,
         const __grid_constant__ CUtensorMap mh, Grid g, bool f16, int* err) {
    constexpr int EPI = kHiddenEpi, S = 4;
    __shared__ __align__(8) Bars<S, 2> bars;
    __shared__ uint32_t tmem_slot;
    __shared__ int dead;
    const uint32_t ring = dynamic_smem(), out = ring + S * kStageBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = setup<EPI>(bars, &tmem_slot, &dead);
    const Watch w{&dead, err};
    const int tiles = g.m_tiles * g.n_tiles;
    int filled = 0;

    if (warp == EPI) {
        if (lane == 0) {
            Ring<S> r;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
                const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
                for (int k = 0; k < g.k_steps; ++k, r.next(), ++filled) {
                    if (!(ok = w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u))) break;
                    const uint32_t a = ring + r.at * kStageBytes, bar = smem_addr(&bars.full[r.at]);
                    mbar_arrive_expect_tx(bar, kStageBytes);
                    tma_load(a, &mx, k * kStepK, mn.x * kRowTile, bar);
                    tma_load(a + kABytes, &mw, k * kStepK, mn.y * 128, bar);
                    tma_load(a + kABytes + kBBytes / 2, &mw, k * kStepK, g.cols + mn.y * 128, bar);
                }
            }
            start_dependents();
        }
    } else if (warp == EPI + 1) {
        if (lane == 0) {
            const uint32_t idesc = mma_desc(256, f16, false, false);
            Ring<S> r;
            Ring<2> acc;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x, acc.next()) {
                if (!(ok = w.wait(smem_addr(&bars.acc_empty[acc.at]), acc.parity ^ 1u))) break;
                fence_after_sync();
                for (int k = 0; k < g.k_steps; ++k, r.next()) {
                    if (!(ok = w.wait(smem_addr(&bars.full[r.at]), r.parity))) break;
                    fence_after_sync();
                    const uint32_t a = ring + r.at * kStageBytes;
                    mma_stage<false, false>(tmem + acc.at * 256, a, a + kABytes, idesc, k == 0);
                    mma_commit(smem_addr(&bars.empty[r.at]));
                }
                mma_commit(smem_addr(&bars.acc_full[acc.at]));
            }
        }
    } else {
        OutTile<1> o{out + (uint32_t)warp * kOutBytes};
        const int quad = warp & 3, half = (warp >> 2) * 64;
        Ring<2> acc;
        for (int t = blockIdx.x; t < tiles; t += gridDim.x, acc.next()) {
            const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
            const int row = mn.x * (int)kRowTile + quad * 32, col = mn.y * 128 + half;
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full[acc.at]), acc.parity))) break;
            fence_after_sync();
            const uint32_t tm = tmem + acc.at * 256 + half + ((uint32_t)quad << 21);
            o.begin(lane);
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
                float a[32], u[32];
                tmem_ld32(tm + c, a);
                tmem_ld32(tm + 128 + c, u);
                tmem_wait(a);
                tmem_wait(u);
                if (c == 32) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_addr(&bars.acc_empty[acc.at]));
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
    finish<EPI>(bars, tmem, &dead, filled);
}

// ---- h, dg, du from x and dy ---------------------------------------------------------
// Per tile first dh = dy Wo (128 columns), then g and u (256).  TMEM: g | u at
// columns 128 .. 383; dh in the first or the last 128 by turns, so that the next
// tile's dh accumulates while this tile's values are read.
constexpr int kGradStages = 3;

template <int ACT>
__global__ void __launch_bounds__(kHiddenEpi * 32 + 64, 1)
k_hidden_grad(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mdy,
              const __grid_constant__ CUtensorMap mw, const __grid_constant__ CUtensorMap mwo,
              const __grid_constant__ CUtensorMap mh, const __grid_constant__ CUtensorMap mdg,
              const __grid_constant__ CUtensorMap mdu, Grid g, bool f16, int* err) {
    constexpr int EPI = kHiddenEpi, S = kGradStages;
    __shared__ __align__(8) Bars<S, 2> bars;     // slot 0: g | u, slot 1: dh (both places)
    __shared__ uint32_t tmem_slot;
    __shared__ int dead;
    const uint32_t ring = dynamic_smem(), out = ring + S * kStageBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tmem = setup<EPI>(bars, &tmem_slot, &dead);
    const Watch w{&dead, err};
    const int tiles = g.m_tiles * g.n_tiles;
    int filled = 0;

    if (warp == EPI) {
        if (lane == 0) {
            Ring<S> r;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
                const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
                for (int k = 0; k < 2 * g.k_steps; ++k, r.next(), ++filled) {
                    if (!(ok = w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u))) break;
                    const uint32_t a = ring + r.at * kStageBytes, bar = smem_addr(&bars.full[r.at]);
                    if (k < g.k_steps) {
                        mbar_arrive_expect_tx(bar, kABytes + kBBytes / 2);
                        tma_load(a, &mdy, k * kStepK, mn.x * kRowTile, bar);
                        load_tile<true>(a + kABytes, &mwo, mn.y * 128, 128, k * kStepK, bar);
                    } else {
                        const int kk = (k - g.k_steps) * kStepK;
                        mbar_arrive_expect_tx(bar, kStageBytes);
                        tma_load(a, &mx, kk, mn.x * kRowTile, bar);
                        tma_load(a + kABytes, &mw, kk, mn.y * 128, bar);
                        tma_load(a + kABytes + kBBytes / 2, &mw, kk, g.cols + mn.y * 128, bar);
                    }
                }
            }
            start_dependents();
        }
    } else if (warp == EPI + 1) {
        if (lane == 0) {
            const uint32_t id_gu = mma_desc(256, f16, false, false), id_dh = mma_desc(128, f16, false, true);
            Ring<S> r;
            uint32_t parity = 0;
            int turn = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x, ++turn, parity ^= 1u) {
                // dh's place was read two tiles ago, before the g | u of the last tile
                for (int k = 0; k < 2 * g.k_steps; ++k, r.next()) {
                    if (k == g.k_steps) {
                        mma_commit(smem_addr(&bars.acc_full[1]));
                        if (!(ok = w.wait(smem_addr(&bars.acc_empty[0]), parity ^ 1u))) break;
                        fence_after_sync();
                    }
                    if (!(ok = w.wait(smem_addr(&bars.full[r.at]), r.parity))) break;
                    fence_after_sync();
                    const uint32_t a = ring + r.at * kStageBytes;
                    if (k < g.k_steps)
                        mma_stage<false, true>(tmem + (turn & 1 ? 384 : 0), a, a + kABytes, id_dh, k == 0);
                    else
                        mma_stage<false, false>(tmem + 128, a, a + kABytes, id_gu, k == g.k_steps);
                    mma_commit(smem_addr(&bars.empty[r.at]));
                }
                mma_commit(smem_addr(&bars.acc_full[0]));
            }
        }
    } else {
        OutTile<2> o{out + (uint32_t)warp * 2 * kOutBytes};
        const int quad = warp & 3, half = (warp >> 2) * 64;
        uint32_t parity = 0;
        int turn = 0;
        for (int t = blockIdx.x; t < tiles; t += gridDim.x, ++turn, parity ^= 1u) {
            const int2 mn = tile_of(t, g.m_tiles, g.n_tiles);
            const int row = mn.x * (int)kRowTile + quad * 32, col = mn.y * 128 + half;
            const bool in = row < g.rows && col < g.cols;
            // g | u come after dh in the order of the MMAs
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full[0]), parity))) break;
            fence_after_sync();
            const uint32_t tm = tmem + half + ((uint32_t)quad << 21), td = tm + (turn & 1 ? 384 : 0);
            uint32_t h[32], dg[32], du[32];
#pragma unroll
            for (int c = 0; c < 64; c += 32) {
                float a[32], u[32], d[32];
                tmem_ld32(tm + 128 + c, a);
                tmem_ld32(tm + 256 + c, u);
                tmem_ld32(td + c, d);
                tmem_wait(a);
                tmem_wait(u);
                tmem_wait(d);
                if (c == 32) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_addr(&bars.acc_empty[0]));
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
    finish<EPI>(bars, tmem, &dead, filled);
}

// ---- host -------------------------------------------------------------------------
constexpr size_t kProductSmem = 1024 + kProductStages * kStageBytes + 4 * 2 * kOutBytes;
constexpr size_t kHiddenSmem = 1024 + 4 * kStageBytes + kHiddenEpi * kOutBytes;
constexpr size_t kGradSmem = 1024 + kGradStages * kStageBytes + kHiddenEpi * 2 * kOutBytes;

template <class K>
cudaError_t allow_smem(K* kernel, size_t bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// C [rows][cols] = A B^T over K
template <bool A_MN, bool B_MN>
cudaError_t product(const FfnArgs& a, int64_t rows, int64_t cols, int64_t K, const void* A, const void* B, void* C,
                    cudaStream_t s) {
    constexpr int BN = 256;
    CUtensorMap ma, mb, mc;
    cudaError_t e = A_MN ? make_map(&ma, a.type, A, K, rows, rows, 64) : make_map(&ma, a.type, A, rows, K, K, kRowTile);
    if (e == cudaSuccess) e = B_MN ? make_map(&mb, a.type, B, K, cols, cols, 64) : make_map(&mb, a.type, B, cols, K, K, BN);
    if (e == cudaSuccess) e = make_map(&mc, a.type, C, rows, cols, cols, 32);
    if (e == cudaSuccess) e = allow_smem(k_product<A_MN, B_MN, BN>, kProductSmem);
    if (e != cudaSuccess) return e;
    const Grid g{ceil_div(rows, kRowTile), ceil_div(cols, BN), ceil_div(K, kStepK), (int)rows, (int)cols};
    const int64_t tiles = (int64_t)g.m_tiles * g.n_tiles;
    return launch_kernel(k_product<A_MN, B_MN, BN>, dim3((unsigned)(tiles < a.num_sms ? tiles : a.num_sms)), dim3(192),
                         kProductSmem, true, s, ma, mb, mc, g, a.type == IFVS_T_F16, a.err);
}

// f(constant) for the activation
template <class Fn>
cudaError_t with_act(int act, const Fn& f) {
    if (act == IFVS_ACT_SILU) return f(std::integral_constant<int, IFVS_ACT_SILU>());
    if (act == IFVS_ACT_GELU) return f(std::integral_constant<int, IFVS_ACT_GELU>());
    return f(std::integral_constant<int, IFVS_ACT_RELU>());
}

}  // namespace

cudaError_t make_map(CUtensorMap* map, int type, const void* p, int64_t rows, int64_t cols, int64_t stride,
                     int box_rows) {
    static const auto encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            fn = nullptr;
        return (decltype(&cuTensorMapEncodeTiled))fn;
    }();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, step[2] = {1, 1};
    const CUresult r = encode(map, type == IFVS_T_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                              2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

size_t ffn_bytes(const FfnArgs& a) { return (size_t)a.T * a.F * 2; }
size_t ffn_grad_bytes(const FfnArgs& a) { return (size_t)a.T * a.F * 6; }

cudaError_t launch_ffn(const FfnArgs& a, const void* x, void* y, uint8_t* work, cudaStream_t s) {
    CUtensorMap mx, mw, mh;
    cudaError_t e = make_map(&mx, a.type, x, a.T, a.D, a.D, kRowTile);
    if (e == cudaSuccess) e = make_map(&mw, a.type, a.w_in, 2 * (int64_t)a.F, a.D, a.D, 128);
    if (e == cudaSuccess) e = make_map(&mh, a.type, work, a.T, a.F, a.F, 32);
    if (e != cudaSuccess) return e;
    const Grid g{ceil_div(a.T, kRowTile), ceil_div(a.F, 128), ceil_div(a.D, kStepK), (int)a.T, a.F};
    const int64_t tiles = (int64_t)g.m_tiles * g.n_tiles;
    e = with_act(a.act, [&](auto act) {
        const cudaError_t r = allow_smem(k_hidden<act()>, kHiddenSmem);
        return r != cudaSuccess ? r
                                : launch_kernel(k_hidden<act()>, dim3((unsigned)(tiles < a.num_sms ? tiles : a.num_sms)),
                                                dim3(kHiddenEpi * 32 + 64), kHiddenSmem, false, s, mx, mw, mh, g,
                                                a.type == IFVS_T_F16, a.err);
    });
    if (e != cudaSuccess) return e;
    return product<false, false>(a, a.T, a.D, a.F, work, a.w_out, y, s);
}

cudaError_t launch_ffn_grad(const FfnArgs& a, const void* x, const void* dy, void* dx, void* d_w_in, void* d_w_out,
                            uint8_t* work, cudaStream_t s) {
    const int64_t D = a.D, F = a.F;
    if (a.T == 0) {
        const cudaError_t e = cudaMemsetAsync(d_w_in, 0, (size_t)(2 * F * D) * 2, s);
        return e != cudaSuccess ? e : cudaMemsetAsync(d_w_out, 0, (size_t)(D * F) * 2, s);
    }
    uint8_t *h = work, *dgu = work + (size_t)a.T * F * 2;
    CUtensorMap mx, mdy, mw, mwo, mh, mdg, mdu;
    cudaError_t e = make_map(&mx, a.type, x, a.T, D, D, kRowTile);
    auto then = [&](cudaError_t r) { e = e == cudaSuccess ? r : e; };
    then(make_map(&mdy, a.type, dy, a.T, D, D, kRowTile));
    then(make_map(&mw, a.type, a.w_in, 2 * F, D, D, 128));
    then(make_map(&mwo, a.type, a.w_out, D, F, F, 64));
    then(make_map(&mh, a.type, h, a.T, F, F, 32));
    then(make_map(&mdg, a.type, dgu, a.T, F, 2 * F, 32));
    then(make_map(&mdu, a.type, dgu + F * 2, a.T, F, 2 * F, 32));
    if (e != cudaSuccess) return e;
    const Grid g{ceil_div(a.T, kRowTile), ceil_div(F, 128), ceil_div(D, kStepK), (int)a.T, a.F};
    const int64_t tiles = (int64_t)g.m_tiles * g.n_tiles;
    e = with_act(a.act, [&](auto act) {
        const cudaError_t r = allow_smem(k_hidden_grad<act()>, kGradSmem);
        return r != cudaSuccess ? r
                                : launch_kernel(k_hidden_grad<act()>, dim3((unsigned)(tiles < a.num_sms ? tiles : a.num_sms)),
                                                dim3(kHiddenEpi * 32 + 64), kGradSmem, false, s, mx, mdy, mw, mwo, mh, mdg,
                                                mdu, g, a.type == IFVS_T_F16, a.err);
    });
    if (e == cudaSuccess) e = product<false, true>(a, a.T, D, 2 * F, dgu, a.w_in, dx, s);
    if (e == cudaSuccess) e = product<true, true>(a, 2 * F, D, a.T, dgu, x, d_w_in, s);
    if (e == cudaSuccess) e = product<true, true>(a, D, F, a.T, dy, h, d_w_out, s);
    return e;
}

}  // namespace ifvs
