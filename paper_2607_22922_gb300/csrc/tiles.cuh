// Persistent tile kernels on the tensor cores: what the feed-forward block, the
// products of their gradients and the linear layer share.  A CTA, or a pair of CTAs
// that share one MMA of 256 rows, takes tiles of the output; a warp fills a ring of
// operand stages by TMA, a warp issues the MMAs, the others turn accumulators into
// 16-bit tiles in shared memory and store them by TMA.
#pragma once

#include "umma.cuh"

namespace ifvs {

constexpr int kRows = 128;                                // rows of a CTA's accumulator tile
constexpr uint32_t kABytes = kRows * 128;                 // a stage's A tile
constexpr uint32_t kOutBytes = 32 * 128;                  // 32 rows x 64 columns of output
constexpr int kMaxStages = 8;
constexpr size_t kMaxSmem = 227 * 1024 - 512;             // beside the static shared memory

// act(g) and act'(g)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& v, float& slope) {
    if (ACT == IFVS_ACT_NONE) {
        v = g;
        slope = 1.f;
    } else if (ACT == IFVS_ACT_RELU) {
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

// ---- host -------------------------------------------------------------------------
inline int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }


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

// What a launch of tiles goes by
struct TileArgs {
    int type, num_sms;
    Waits waits;
};

// Pairs of CTAs where their tiles fill the device, or half of it where each sums
// over 1024 or more.  Forward pass, pairs against single CTAs: 8192 tokens x 960 x
// 2560 76 us against 93; 2048 x 1536 x 5120 67 against 81; 1024 x 1536 x 5120 (24
// tiles of the output) 57 against 45; 4096 x 128 x 344 11.8 against 11.1.
inline bool use_pairs(const TileArgs& a, int64_t rows, int64_t cols, int64_t K) {
    return (int64_t)ceil_div(rows, 256) * ceil_div(cols, 256) >= a.num_sms / (K >= 1024 ? 4 : 2);
}

}  // namespace ifvs
