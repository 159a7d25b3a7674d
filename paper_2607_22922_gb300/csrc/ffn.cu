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
#include "umma.cuh"

namespace ifvs {

namespace {

constexpr int kRows = 128;                                // rows of a CTA's accumulator tile
constexpr uint32_t kABytes = kRows * 128;                 // a stage's A tile
constexpr uint32_t kOutBytes = 32 * 128;                  // 32 rows x 64 columns of output
constexpr int kMaxStages = 8;
constexpr size_t kMaxSmem = 227 * 1024 - 512;             // beside the static shared memory

// act(g) and act'(g)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& v, float& slope) {
    if (ACT == IFVS_ACT_RELU) {
        v = g <= 0.f ? 0.f : g;              // a NaN passes
        slope = g > 0.f ? 1.f : v;
    } else if (ACT == IFVS_ACT_SILU) {
        const float p = __fdividef(1.f, 1.f + __expf(-g));
        v = g * p;
        slope = p * (1.f + g * (1.f - p));
    } else {
        // Phi by Abramowitz and Stegun 7.1.26: erfc(x) = (a1 t + .. + a5 t^5) e^(-x^2),
        // t = 1 / (1 + p x), within 1.5e-7; here x = |g| / sqrt(2), so that the
        // exponential serves the density too
        const float e = __expf(-0.5f * g * g), t = __fdividef(1.f, fmaf(0.3275911f * 0.70710678f, fabsf(g), 1.f));
        float q = fmaf(t, 1.061405429f, -1.453152027f);
        q = fmaf(t, q, 1.421413741f);
        q = fmaf(t, q, -0.284496736f);
        q = fmaf(t, q, 0.254829592f);
        q *= 0.5f * t * e;
        const float p = g < 0.f ? q : 1.f - q;
        v = g * p;
        slope = fmaf(0.39894228f * g, e, p);
    }
}

// Barriers of a CTA: operand stages, accumulator slots, the last MMAs
template <int S>
struct Bars {
    uint64_t full[S], empty[S], acc_full[2], acc_empty[2], drain;
    uint32_t tmem;
    int dead;
};

// What every kernel here starts with; returns the TMEM base (512 columns).
// Warps 0 .. EPI - 1: epilogue, EPI: TMA, EPI + 1: MMA (of a pair the first CTA's).
template <int CG, int EPI, int S>
__device__ __forceinline__ uint32_t setup(Bars<S>& b) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(smem_addr(&b.full[i]), 1);
            mbar_init(smem_addr(&b.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&b.acc_full[i]), 1);
            mbar_init(smem_addr(&b.acc_empty[i]), EPI * CG);
        }
        mbar_init(smem_addr(&b.drain), 1);
        b.dead = 0;
        fence_mbar_init();
    }
    if (threadIdx.x / 32 == EPI + 1) tmem_alloc<CG>(smem_addr(&b.tmem), 512);
    fence_before_sync();
    __syncthreads();
    if constexpr (CG == 2) pair_sync();      // the other CTA's barriers are there
    fence_after_sync();
    return b.tmem;
}

// The end of a kernel: with everything in order the roles have waited for
// their own work; a dead CTA waits here, bounded, for what it had in flight: a
// warp for all of its copies, a thread for its MMAs.
template <int CG, int EPI, int S>
__device__ __forceinline__ void finish(Bars<S>& b, uint32_t tmem, int filled, bool issues, const Waits& waits) {
    __syncwarp();
    __syncthreads();
    if (*(volatile int*)&b.dead) {
        const long long t0 = clock64();
        auto bounded = [&](uint32_t bar, uint32_t parity) {
            while (!mbar_try_wait(bar, parity) && clock64() - t0 < waits.cycles) {
            }
        };
        if (threadIdx.x / 32 == EPI && issues)       // `filled` is the elected thread's
            for (int i = max(0, filled - S); i < filled; ++i) bounded(smem_addr(&b.full[i % S]), (uint32_t)(i / S) & 1u);
        if (threadIdx.x / 32 == EPI + 1 && issues && elect_one()) {
            mma_commit<CG>(smem_addr(&b.drain));
            bounded(smem_addr(&b.drain), 0);
        }
        __syncwarp();
        __syncthreads();
    }
    if constexpr (CG == 2) pair_sync();      // nothing of the pair uses this CTA's memory any more
    if (threadIdx.x / 32 == EPI + 1) tmem_free<CG>(tmem, 512);
}

// K-major tiles: `rows` rows from `row`; MN-major: `rows` columns from `row`.
// k: the first of the stage's 64 along the sum.
template <int CG>
__device__ __forceinline__ void load_tile(bool mn_major, uint32_t dst, const CUtensorMap* map, int row, int rows, int k,
                                          uint32_t bar) {
    if (mn_major) {
#pragma unroll 1
        for (int i = 0; i < rows; i += 64) tma_load<CG>(dst + (uint32_t)i * 128u, map, row + i, k, bar);
    } else {
        tma_load<CG>(dst, map, k, row, bar);
    }
}

// The operands' descriptors at the ring's first stage; a stage further on differs
// in the address alone
struct Operands {
    uint64_t a, b, step_a, step_b;
    __device__ __forceinline__ Operands(uint32_t at_a, uint32_t at_b, bool a_mn, bool b_mn)
        : a(tile_desc(at_a, a_mn)), b(tile_desc(at_b, b_mn)), step_a(desc_step(a_mn)), step_b(desc_step(b_mn)) {}
    // the four MMAs of the stage `offset` bytes into the ring
    template <int CG>
    __device__ __forceinline__ void mma(uint32_t d, uint32_t offset, uint32_t idesc, bool first) const {
        const uint64_t da = a + (offset >> 4), db = b + (offset >> 4);
#pragma unroll
        for (uint32_t i = 0; i < kStepK / 16; ++i) mma_f16<CG>(d, da + i * step_a, db + i * step_b, idesc, !first || i > 0);
    }
};

// This warp's 32 rows x 64 columns of 16-bit output: packed pairs go to the
// staging tile (swizzled), a TMA store takes it.  BUFS tiles per warp.
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
    int m_tiles, n_tiles, k_steps;     // m_tiles of CG x 128 rows
    int rows, cols;                    // of the output
};

__device__ __forceinline__ uint32_t dynamic_smem() {
    extern __shared__ uint8_t raw[];
    return (smem_addr(raw) + 1023u) & ~1023u;
}

// stages that fit beside the staging tiles
constexpr int stages_of(uint32_t stage_bytes, uint32_t out_bytes) {
    const int n = (int)((kMaxSmem - 1024 - out_bytes) / stage_bytes);
    return n < kMaxStages ? n : kMaxStages;
}
constexpr size_t smem_of(uint32_t stage_bytes, uint32_t out_bytes) {
    return 1024 + (size_t)stages_of(stage_bytes, out_bytes) * stage_bytes + out_bytes;
}

// ---- products C = A B^T in 16 bits ---------------------------------------------------
// Bound by the tensor pipe and, in a long run, by power: the gradient's three
// products at 16411 x 1024 x 4096 (688 GFLOP) 372 us, 1.85 PFLOP/s, the pipe 96.4 %
// active at 1.69 GHz.
// A K-major [rows][K] or MN-major [K][rows]; B the same with `cols`.  Up to three
// products in one launch, items (tiles, or parts of a tile's sum) in their order.
struct Product {
    CUtensorMap a, b, c;
    Grid g;
    int splits;          // parts of the sum; more than one: float32 parts in `parts`, added by k_join_parts
    int items;           // tiles x splits
    bool a_mn, b_mn;
    float* parts;        // [splits][rows][cols]
};
struct Products {
    Product p[3];
    int n, items;
};

template <int CG, int BN>
struct ProductShape {
    static constexpr uint32_t kB = BN / CG * 128, kStage = kABytes + kB, kOut = 4 * 2 * kOutBytes;
    static constexpr int kStages = stages_of(kStage, kOut);
    static constexpr size_t kSmem = smem_of(kStage, kOut);
};

struct Item {
    const Product* p;
    int m, n, split, k0, k1;
};
__device__ __forceinline__ Item item_of(const Products& all, int i) {
    int j = 0;
    while (j + 1 < all.n && i >= all.p[j].items) i -= all.p[j++].items;
    Item t;
    t.p = &all.p[j];
    const Grid& g = t.p->g;
    const int tile = i / t.p->splits;
    t.split = i - tile * t.p->splits;
    const int2 mn = tile_of(tile, g.m_tiles, g.n_tiles);
    t.m = mn.x;
    t.n = mn.y;
    t.k0 = (int)((int64_t)g.k_steps * t.split / t.p->splits);
    t.k1 = (int)((int64_t)g.k_steps * (t.split + 1) / t.p->splits);
    return t;
}

template <int CG, int BN>
__global__ void __launch_bounds__(192, 1) k_products(const __grid_constant__ Products all, bool f16, Waits waits) {
    using Sh = ProductShape<CG, BN>;
    constexpr int EPI = 4, S = Sh::kStages;
    __shared__ __align__(8) Bars<S> bars;
    const uint32_t ring = dynamic_smem(), out = ring + S * Sh::kStage;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    const uint32_t tmem = setup<CG, EPI>(bars);
    const Watch w{&bars.dead, waits};
    const int first = blockIdx.x / CG, step = gridDim.x / CG;
    int filled = 0;
    wait_before();

    if (warp == EPI) {
        if (elect_one()) {
            Ring<S> r;
            bool ok = true;
            for (int i = first; i < all.items && ok; i += step) {
                const Item t = item_of(all, i);
                const bool a_mn = t.p->a_mn, b_mn = t.p->b_mn;
                const int row = (t.m * CG + rank) * kRows, col = t.n * BN + rank * (BN / CG);
                for (int k = t.k0; k < t.k1; ++k, r.next(), ++filled) {
                    if (!(ok = w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u))) break;
                    const uint32_t a = ring + r.at * Sh::kStage, bar = smem_addr(&bars.full[r.at]);
                    if (rank == 0) mbar_arrive_expect_tx(bar, CG * Sh::kStage + waits.extra);
                    load_tile<CG>(a_mn, a, &t.p->a, row, kRows, k * kStepK, bar);
                    load_tile<CG>(b_mn, a + kABytes, &t.p->b, col, BN / CG, k * kStepK, bar);
                }
            }
            start_dependents();
        }
    } else if (warp == EPI + 1) {
        if (rank == 0 && elect_one()) {
            Ring<S> r;
            Ring<2> acc;
            bool ok = true;
            for (int i = first; i < all.items && ok; i += step, acc.next()) {
                const Item t = item_of(all, i);
                const bool a_mn = t.p->a_mn, b_mn = t.p->b_mn;
                const uint32_t idesc = mma_desc(CG * kRows, BN, f16, a_mn, b_mn);
                if (!(ok = w.wait(smem_addr(&bars.acc_empty[acc.at]), acc.parity ^ 1u))) break;
                fence_after_sync();
                const Operands o(ring, ring + kABytes, a_mn, b_mn);
                for (int k = t.k0; k < t.k1; ++k, r.next()) {
                    if (!(ok = w.wait(smem_addr(&bars.full[r.at]), r.parity))) break;
                    fence_after_sync();
                    o.mma<CG>(tmem + acc.at * 256, r.at * Sh::kStage, idesc, k == t.k0);
                    mma_commit<CG>(smem_addr(&bars.empty[r.at]));
                }
                if (ok) mma_commit<CG>(smem_addr(&bars.acc_full[acc.at]));
            }
        }
    } else {
        OutTile<2> o{out + (uint32_t)warp * 2 * kOutBytes};
        Ring<2> acc;
        for (int i = first; i < all.items; i += step, acc.next()) {
            const Item t = item_of(all, i);
            const Grid& g = t.p->g;
            const int row = (t.m * CG + rank) * kRows + warp * 32;
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full[acc.at]), acc.parity))) break;
            fence_after_sync();
            const uint32_t tm = tmem + acc.at * 256 + ((uint32_t)warp << 21);
#pragma unroll 1
            for (int c = 0; c < BN; c += 64) {
                const int col = t.n * BN + c;
                float v[2][32];
                tmem_ld32(tm + c, v[0]);
                tmem_ld32(tm + c + 32, v[1]);
                if (t.p->splits == 1) o.begin(lane);
                tmem_wait(v[0]);
                tmem_wait(v[1]);
                if (c + 64 == BN) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive<CG>(smem_addr(&bars.acc_empty[acc.at]));
                }
                if (t.p->splits > 1) {
                    if (row + lane < g.rows) {
                        float* to = t.p->parts + ((int64_t)t.split * g.rows + row + lane) * g.cols + col;
#pragma unroll
                        for (int j = 0; j < 64; j += 4)      // columns are a multiple of 8
                            if (col + j < g.cols)
                                *reinterpret_cast<float4*>(to + j) = *reinterpret_cast<float4*>(&v[j >> 5][j & 31]);
                    }
                    continue;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float* q = &v[j >> 2][(j & 3) * 8];
                    o.put(lane, j, pack16(q[0], q[1], f16), pack16(q[2], q[3], f16), pack16(q[4], q[5], f16),
                          pack16(q[6], q[7], f16));
                }
                o.store(lane, &t.p->c, col, row, row < g.rows && col < g.cols);
            }
        }
        if (lane == 0) tma_wait_all();
    }
    finish<CG, EPI>(bars, tmem, filled, rank == 0, waits);
}

// C = the sum of the parts, in order; up to three products
struct Parts {
    const float* parts[3];
    void* c[3];
    int64_t n[3];        // values, a multiple of 8
    int splits[3];
};
template <class T>
__global__ void __launch_bounds__(256) k_join_parts(Parts p) {
    wait_before();
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const int j = blockIdx.y;
    if (i >= p.n[j]) return;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = 0; s < p.splits[j]; ++s) {
        const float4 q = __ldcg(reinterpret_cast<const float4*>(p.parts[j] + s * p.n[j] + i));
        v.x += q.x;
        v.y += q.y;
        v.z += q.z;
        v.w += q.w;
    }
    *reinterpret_cast<uint2*>((T*)p.c[j] + i) = make_uint2(pack2(make_float2(v.x, v.y), T()), pack2(make_float2(v.z, v.w), T()));
}

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
// at 960 x 2560 and 7.4 against 8.7 at 128 x 344 (for 16: 35 and 9).  A row of
// weights (PAIR:
// the gate's row and the up projection's) is spread over the lanes of one or
// more warps, 16 bytes a lane and access, against every token's row.
constexpr int kFewTokens = 4;

template <class T>
struct FewArgs {
    const T *x, *w;      // x [tokens][K], w [rows][K] (PAIR: [2 rows][K])
    T* out;              // [tokens][rows]
    int tokens, rows, K;
    int cta_rows;        // rows per CTA of 8 warps: 8 / cta_rows warps share one
};

template <class T, bool PAIR, int ACT, int TT>
__global__ void __launch_bounds__(256) k_few(FewArgs<T> a) {
    constexpr int NW = PAIR ? 2 : 1, AHEAD = 4;
    __shared__ float sums[8][NW * TT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int share = 8 / a.cta_rows, part = warp % share, row = blockIdx.x * a.cta_rows + warp / share;
    const int chunks = a.K / 8;
    const bool in = row < a.rows;
    const T* w[NW];
#pragma unroll
    for (int r = 0; r < NW; ++r) w[r] = a.w + ((int64_t)r * a.rows + (in ? row : 0)) * a.K;
    float2 acc[NW][TT];
#pragma unroll
    for (int r = 0; r < NW; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[r][t] = make_float2(0.f, 0.f);
    bool waited = false;
    if constexpr (PAIR) start_dependents();
    for (int c0 = part * 32 + lane; c0 < chunks; c0 += share * 32 * AHEAD) {
        Pack<T, 8> v[AHEAD][NW];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int r = 0; r < NW; ++r) v[k][r].load(w[r] + (int64_t)min(c0 + k * share * 32, chunks - 1) * 8);
        // the weights are on their way before the kernel that makes x has ended
        if (!PAIR && !waited) wait_before();
        waited = true;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int c = c0 + k * share * 32;
            if (c >= chunks) break;
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                Pack<T, 8> x;
                const T* from = a.x + (int64_t)min(t, a.tokens - 1) * a.K + c * 8;
                if constexpr (PAIR)
                    x.load(from);
                else             // written by the kernel before, which this one may have started beside
                    x.w = __ldcg(reinterpret_cast<const uint4*>(from));
#pragma unroll
                for (int r = 0; r < NW; ++r)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[r][t] = fma_(v[k][r].get(j), x.get(j), acc[r][t]);
            }
        }
    }
    if (!PAIR && !waited) wait_before();
#pragma unroll
    for (int r = 0; r < NW; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const float s = warp_sum(total(acc[r][t]));
            if (lane == 0) sums[warp][r * TT + t] = s;
        }
    __syncthreads();
    if (part == 0 && in)
        for (int t = lane; t < a.tokens; t += 32) {
            float s[NW];
#pragma unroll
            for (int r = 0; r < NW; ++r) {
                s[r] = 0.f;
                for (int k = 0; k < share; ++k) s[r] += sums[warp + k][r * TT + t];
            }
            float v = s[0];
            if constexpr (PAIR) {
                float slope;
                activation<ACT>(s[0], v, slope);
                v *= s[1];
            }
            a.out[(int64_t)t * a.rows + row] = from_f32<T>(v);
        }
}

// ---- host -------------------------------------------------------------------------
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// f(constant) for the activation
template <class Fn>
cudaError_t with_act(int act, const Fn& f) {
    if (act == IFVS_ACT_SILU) return f(std::integral_constant<int, IFVS_ACT_SILU>());
    if (act == IFVS_ACT_GELU) return f(std::integral_constant<int, IFVS_ACT_GELU>());
    return f(std::integral_constant<int, IFVS_ACT_RELU>());
}

// A persistent launch: at most one CTA per SM, in clusters of CG
template <int CG, class... P, class... A>
cudaError_t launch_tiles(void (*kernel)(P...), int64_t items, int num_sms, int threads, size_t smem, bool chain,
                         cudaStream_t s, const A&... args) {
    cudaError_t e = allow_smem(kernel, smem);
    if (e != cudaSuccess) return e;
    const int64_t most = num_sms / CG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((items < most ? items : most) * CG));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {(unsigned)CG, 1u, 1u};
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = chain ? 2 : 1;
    e = next_launch();
    return e != cudaSuccess ? e : cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Products of one launch, in the order they are added
struct Plan {
    const FfnArgs& a;
    bool pairs;          // 256 x 256 tiles of CTA pairs; else 128 x 128
    uint8_t* work;       // for parts of sums
    Products all;
    Parts parts;
    int joined = 0;
    cudaError_t e = cudaSuccess;
    explicit Plan(const FfnArgs& a_, bool pairs_, uint8_t* work_) : a(a_), pairs(pairs_), work(work_) {
        all.n = all.items = 0;
    }

    int rows_tile() const { return pairs ? 256 : 128; }
    // C [rows][cols] = A B^T over K
    void add(int64_t rows, int64_t cols, int64_t K, const void* A, bool a_mn, const void* B, bool b_mn, void* C) {
        Product& p = all.p[all.n++];
        auto then = [&](cudaError_t r) { e = e == cudaSuccess ? r : e; };
        then(a_mn ? make_map(&p.a, a.type, A, K, rows, rows, 64) : make_map(&p.a, a.type, A, rows, K, K, kRows));
        then(b_mn ? make_map(&p.b, a.type, B, K, cols, cols, 64) : make_map(&p.b, a.type, B, cols, K, K, 128));
        then(make_map(&p.c, a.type, C, rows, cols, cols, 32));
        p.g = Grid{ceil_div(rows, rows_tile()), ceil_div(cols, rows_tile()), ceil_div(K, kStepK), (int)rows, (int)cols};
        p.a_mn = a_mn;
        p.b_mn = b_mn;
        p.splits = splits_of(a, rows, cols, K, pairs);
        p.items = p.g.m_tiles * p.g.n_tiles * p.splits;
        p.parts = nullptr;
        all.items += p.items;
        if (p.splits > 1) {
            p.parts = (float*)work;
            work += (size_t)p.splits * rows * cols * sizeof(float);
            parts.parts[joined] = p.parts;
            parts.c[joined] = C;
            parts.n[joined] = rows * cols;
            parts.splits[joined++] = p.splits;
        }
    }
    // Parts of a tile's sum: where the tiles leave SMs without work, at least four
    // stages each.  A sum of any length is cut below 2^16 stages, which bounds
    // every wait for a tile.
    static int splits_of(const FfnArgs& a, int64_t rows, int64_t cols, int64_t K, bool pairs) {
        const int tile = pairs ? 256 : 128, steps = ceil_div(K, kStepK);
        const int64_t tiles = (int64_t)ceil_div(rows, tile) * ceil_div(cols, tile), slots = a.num_sms / (pairs ? 2 : 1);
        int64_t n = slots / tiles;
        if (n > steps / 4) n = steps / 4;
        if (n > 32) n = 32;
        const int64_t least = ((int64_t)steps + 65535) / 65536;
        return (int)(n > least ? n : (least > 1 ? least : 1));
    }
    static size_t part_bytes(const FfnArgs& a, int64_t rows, int64_t cols, int64_t K, bool pairs) {
        const int n = splits_of(a, rows, cols, K, pairs);
        return n > 1 ? (size_t)n * rows * cols * sizeof(float) : 0;
    }
    cudaError_t launch(bool chain, cudaStream_t s) {
        if (e != cudaSuccess) return e;
        const bool f16 = a.type == IFVS_T_F16;
        e = pairs ? launch_tiles<2>(k_products<2, 256>, all.items, a.num_sms, 192, ProductShape<2, 256>::kSmem, chain, s, all,
                                    f16, a.waits)
                  : launch_tiles<1>(k_products<1, 128>, all.items, a.num_sms, 192, ProductShape<1, 128>::kSmem, chain, s, all,
                                    f16, a.waits);
        if (e != cudaSuccess || joined == 0) return e;
        int64_t most = 0;
        for (int j = 0; j < joined; ++j) most = parts.n[j] > most ? parts.n[j] : most;
        const dim3 grid((unsigned)((most + 1023) / 1024), (unsigned)joined);
        return f16 ? launch_next(k_join_parts<__half>, grid, dim3(256), 0, true, s, parts)
                   : launch_next(k_join_parts<__nv_bfloat16>, grid, dim3(256), 0, true, s, parts);
    }
};

// Pairs of CTAs where their tiles fill the device, or half of it where each sums
// over 1024 or more.  Forward pass, pairs against single CTAs: 8192 tokens x 960 x
// 2560 76 us against 93; 2048 x 1536 x 5120 67 against 81; 1024 x 1536 x 5120 (24
// tiles of the output) 57 against 45; 4096 x 128 x 344 11.8 against 11.1.
bool use_pairs(const FfnArgs& a, int64_t rows, int64_t cols, int64_t K) {
    return (int64_t)ceil_div(rows, 256) * ceil_div(cols, 256) >= a.num_sms / (K >= 1024 ? 4 : 2);
}

template <class T, bool PAIR, int ACT>
cudaError_t launch_few(const FfnArgs& a, const void* x, const void* w, void* out, int rows, int K, cudaStream_t s) {
    FewArgs<T> f{(const T*)x, (const T*)w, (T*)out, (int)a.T, rows, K, 8};
    while (f.cta_rows > 1 && ceil_div(rows, f.cta_rows) < 2 * a.num_sms) f.cta_rows /= 2;
    const dim3 grid((unsigned)ceil_div(rows, f.cta_rows));
    auto go = [&](auto tt) { return launch_next(k_few<T, PAIR, ACT, tt()>, grid, dim3(256), 0, !PAIR, s, f); };
    if (a.T == 1) return go(std::integral_constant<int, 1>());
    if (a.T == 2) return go(std::integral_constant<int, 2>());
    return go(std::integral_constant<int, kFewTokens>());
}

template <class T>
cudaError_t ffn_few(const FfnArgs& a, const void* x, void* y, void* h, cudaStream_t s) {
    const cudaError_t e = with_act(a.act, [&](auto act) { return launch_few<T, true, act()>(a, x, a.w_in, h, a.F, a.D, s); });
    return e != cudaSuccess ? e : launch_few<T, false, IFVS_ACT_RELU>(a, h, a.w_out, y, a.D, a.F, s);
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

namespace {
size_t padded(size_t n) { return (n + 255) / 256 * 256; }
bool hidden_pairs(const FfnArgs& a) { return use_pairs(a, a.T, 2 * (int64_t)a.F, a.D); }
bool out_pairs(const FfnArgs& a) { return use_pairs(a, a.T, a.D, a.F); }
// The gradient's products together.  The weights' sum over the tokens: few tokens
// are over before a pair has started (960 x 2560, pairs against single CTAs: 128
// tokens 35 us against 30, 512 42 against 39, 4096 116 against 149).
bool grad_pairs(const FfnArgs& a) {
    return a.T > 512 && (use_pairs(a, a.T, a.D, 2 * (int64_t)a.F) || use_pairs(a, 2 * (int64_t)a.F, a.D, a.T));
}
}  // namespace

size_t ffn_bytes(const FfnArgs& a) {
    return padded((size_t)a.T * a.F * 2) + (a.T > 0 ? Plan::part_bytes(a, a.T, a.D, a.F, out_pairs(a)) : 0);
}
size_t ffn_grad_bytes(const FfnArgs& a) {
    if (a.T == 0) return 0;
    const bool p = grad_pairs(a);
    return padded((size_t)a.T * a.F * 2) + padded((size_t)a.T * a.F * 4) + Plan::part_bytes(a, a.T, a.D, 2 * (int64_t)a.F, p) +
           Plan::part_bytes(a, 2 * (int64_t)a.F, a.D, a.T, p) + Plan::part_bytes(a, a.D, a.F, a.T, p);
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
    Plan plan(a, out_pairs(a), work + padded((size_t)a.T * a.F * 2));
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
    Plan plan(a, grad_pairs(a), dgu + padded((size_t)a.T * F * 4));
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
