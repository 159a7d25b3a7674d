// A linear layer with bias, activation and residual in its epilogue (ifvs_linear,
// ifvs_linear_grad).
//
//   z = x W^T + b, y = act(z) + residual
//   dz = dy act'(z), dx = dz W, dW = dz^T x, db = sum over the tokens of dz
//
// k_linear accumulates a tile of z in TMEM and makes y (or, from dy, dz) of it, so
// that z is never stored: the gradient computes it again.  dz is rounded to the
// arrays' type, because the next products multiply 16-bit operands; without an
// activation it is dy itself.  dx, dW and db are one launch of k_products.
#include "few.cuh"
#include "products.cuh"

namespace ifvs {

namespace {

// What the epilogue does beside the activation and bias
enum Mode { kForward = 0, kSlope = 1 };

struct Epilogue {
    const void *bias, *other;    // [cols] or null; kForward: the residual or null, kSlope: dy, [rows][cols]
    bool f16;
};

__device__ __forceinline__ float2 unpack16(uint32_t w, bool f16) { return f16 ? unpack2(w, __half()) : unpack2(w, __nv_bfloat16()); }

// 8 columns' bias, the same in every lane
__device__ __forceinline__ uint4 bias_of(const Epilogue& e, int col, int cols) {
    return e.bias && col < cols ? __ldg(reinterpret_cast<const uint4*>((const uint16_t*)e.bias + col)) : make_uint4(0, 0, 0, 0);
}

__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 pair_ex2(float2 x) {
    float2 y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(x.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(x.y));
    return y;
}

// g Phi(g) and its slope, two values at a time.  The lower tail is a product, so that it keeps
// its leading digits however small it is:
//   Phi(-x) = e^(-x^2 / 2) R(x), R(x) = erfcx(x / sqrt(2)) / 2 = Q(t), t = 1 / (1 + 0.29 x)
// and Q, of degree 6, was fitted to R over 0 <= x <= 13.4, where the exponential vanishes: within
// 8.3e-8 of Phi where it is large, within 1.2e-5 of its own value where it is small.  (Phi as 1/2 +
// (1/2 - tail) loses all digits from -5 down.  17408 x 960 -> 2560 with the residual takes 80.3 us,
// with that 80.5; with t P(t), P of degree 6, 81.9.)
__device__ __forceinline__ void gelu(float2 g, float2& v, float2& slope) {
    auto both2 = [](float c) { return make_float2(c, c); };
    const float2 e = pair_ex2(mul_(mul_(g, g), both2(-0.5f * 1.44269504f)));
    const float2 d = fma_(make_float2(fabsf(g.x), fabsf(g.y)), both2(0.29f), both2(1.f));
    const float2 t = make_float2(rcp(d.x), rcp(d.y));
    float2 q = fma_(t, both2(-0.0930059254f), both2(0.301860571f));
    q = fma_(t, q, both2(-0.120859757f));
    q = fma_(t, q, both2(0.202541292f));
    q = fma_(t, q, both2(0.0905459449f));
    q = fma_(t, q, both2(0.119104102f));
    q = fma_(t, q, both2(-0.000186309364f));
    const float2 tail = mul_(e, q);
    const float2 p = make_float2(g.x < 0.f ? tail.x : 1.f - tail.x, g.y < 0.f ? tail.y : 1.f - tail.y);
    v = mul_(g, p);
    slope = fma_(mul_(g, both2(0.39894228f)), e, p);
}

// act and act' of two values, two float32 operations per instruction: the epilogue of 17408 x
// 960 -> 2560 with GELU takes 16 instructions a value one by one, 11 so.
template <int ACT>
__device__ __forceinline__ void activations(float2 g, float2& v, float2& slope) {
    auto both2 = [](float c) { return make_float2(c, c); };
    if constexpr (ACT == IFVS_ACT_SILU) {
        const float2 e = pair_ex2(mul_(g, both2(-1.44269504f))), d = add_(e, both2(1.f)), p = make_float2(rcp(d.x), rcp(d.y));
        v = mul_(g, p);
        slope = fma_(v, fma_(p, both2(-1.f), both2(1.f)), p);
    } else if constexpr (ACT == IFVS_ACT_GELU) {
        gelu(g, v, slope);
    } else {
        activation<ACT>(g.x, v.x, slope.x);
        activation<ACT>(g.y, v.y, slope.y);
    }
}

template <int ACT, int MODE>
__device__ __forceinline__ float2 finish_two(float2 z, float2 other) {
    float2 v, slope;
    activations<ACT>(z, v, slope);
    return MODE == kSlope ? mul_(slope, other) : add_(v, other);
}

// ---- tiles -------------------------------------------------------------------------
// BN columns of the output per tile; 8 epilogue warps, each 32 rows x BN / 2 columns, 32
// columns at a time.  A warp's two buffers of 32 x 32 hold the residual (or dy), brought by
// TMA, then the output in its place.  More room there would take a stage of the ring: with
// five instead of six 17408 x 960 -> 2560 takes 7 us more.  Without residual and activation that
// takes 53 us, with GELU 67, with the residual 67, with both 81; a residual through registers
// (83), or asked of L2 a tile ahead (82), takes no less: the operands alone take 64 bytes a
// clock of an SM's way to L2.
constexpr uint32_t kChunkBytes = 32 * 64;
template <int CG, int BN>
struct LinearShape {
    static constexpr int kEpi = 8;
    static constexpr uint32_t kStage = kABytes + BN / CG * 128, kOut = kEpi * 2 * kChunkBytes;
    static constexpr int kStages = stages_of(kStage, kOut);
    static constexpr size_t kSmem = smem_of(kStage, kOut);
};

template <int ACT, int MODE, int CG, int BN>
__global__ void __launch_bounds__(LinearShape<CG, BN>::kEpi * 32 + 64, 1)
k_linear(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw,
         const __grid_constant__ CUtensorMap my, const __grid_constant__ CUtensorMap mo, Grid g, int splits, float* parts, Epilogue e,
         Waits waits) {
    using Sh = LinearShape<CG, BN>;
    constexpr int EPI = Sh::kEpi, S = Sh::kStages;
    __shared__ __align__(8) Bars<S> bars;
    __shared__ __align__(8) uint64_t other_full[EPI][2];
    const uint32_t ring = dynamic_smem(), out = ring + S * Sh::kStage;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    if (threadIdx.x == 0)
        for (int i = 0; i < 2 * EPI; ++i) mbar_init(smem_addr(&other_full[0][0] + i), 1);
    const uint32_t tmem = setup<CG, EPI>(bars);
    const Watch w{&bars.dead, waits};
    const int items = g.m_tiles * g.n_tiles * splits, first = blockIdx.x / CG, step = gridDim.x / CG;
    int filled = 0;
    auto k_of = [&](int split) { return (int)((int64_t)g.k_steps * split / splits); };

    if (warp == EPI) {
        if (elect_one()) {
            Ring<S> r;
            bool ok = true;
            for (int i = first; i < items && ok; i += step) {
                const int2 mn = tile_of(i / splits, g.m_tiles, g.n_tiles);
                const int row = (mn.x * CG + rank) * kRows, col = mn.y * BN + rank * (BN / CG);
                for (int k = k_of(i % splits), k1 = k_of(i % splits + 1); k < k1; ++k, r.next(), ++filled) {
                    if (!(ok = w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u))) break;
                    const uint32_t a = ring + r.at * Sh::kStage, bar = smem_addr(&bars.full[r.at]);
                    if (rank == 0) mbar_arrive_expect_tx(bar, CG * Sh::kStage + waits.extra);
                    tma_load<CG>(a, &mx, k * kStepK, row, bar);
                    tma_load<CG>(a + kABytes, &mw, k * kStepK, col, bar);
                }
            }
            start_dependents();
        }
    } else if (warp == EPI + 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = mma_desc(CG * kRows, BN, e.f16, false, false);
            const Operands o(ring, ring + kABytes, false, false);
            Ring<S> r;
            Ring<2> acc;
            bool ok = true;
            for (int i = first; i < items && ok; i += step, acc.next()) {
                if (!(ok = w.wait(smem_addr(&bars.acc_empty[acc.at]), acc.parity ^ 1u))) break;
                fence_after_sync();
                const int k0 = k_of(i % splits), k1 = k_of(i % splits + 1);
                for (int k = k0; k < k1; ++k, r.next()) {
                    if (!(ok = w.wait(smem_addr(&bars.full[r.at]), r.parity))) break;
                    fence_after_sync();
                    o.mma<CG>(tmem + acc.at * 256, r.at * Sh::kStage, idesc, k == k0);
                    mma_commit<CG>(smem_addr(&bars.empty[r.at]));
                }
                if (ok) mma_commit<CG>(smem_addr(&bars.acc_full[acc.at]));
            }
        }
    } else {
        const uint32_t mine = out + (uint32_t)warp * 2 * kChunkBytes;
        const int quad = warp & 3, part = (warp >> 2) * (BN / 2);
        auto row_of = [&](int2 mn) { return (mn.x * CG + rank) * kRows + quad * 32; };
        const bool fetches = e.other && splits == 1;
        // into buffer n mod 2, once its last store has been read
        int asked = 0, taken = 0;
        auto fetch = [&](int2 mn, int c) {
            if (lane == 0) {
                tma_wait_read<0>();
                const uint32_t bar = smem_addr(&other_full[warp][asked & 1]);
                mbar_arrive_expect_tx(bar, kChunkBytes + waits.extra);
                tma_load<1>(mine + (asked & 1) * kChunkBytes, &mo, mn.y * BN + part + c, row_of(mn), bar);
            }
            ++asked;
        };
        if (fetches && first < items) fetch(tile_of(first, g.m_tiles, g.n_tiles), 0);
        Ring<2> acc;
        bool ok = true;
        int turn = 0;
        for (int i = first; i < items && ok; i += step, acc.next()) {
            const int2 mn = tile_of(i / splits, g.m_tiles, g.n_tiles);
            const int row = row_of(mn), col0 = mn.y * BN + part;
            if (!(ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full[acc.at]), acc.parity)))) break;
            fence_after_sync();
            const uint32_t tm = tmem + acc.at * 256 + part + ((uint32_t)quad << 21);
#pragma unroll 1
            for (int c = 0; c < BN / 2; c += 32, turn ^= 1) {
                const int col = col0 + c;
                float z[32];
                tmem_ld32(tm + c, z);
                uint4 b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = bias_of(e, col + 8 * j, g.cols);
                tmem_wait(z);
                if (c + 32 == BN / 2) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive<CG>(smem_addr(&bars.acc_empty[acc.at]));
                }
                if (splits > 1) {
                    if (row + lane < g.rows) {
                        float* to = parts + ((int64_t)(i % splits) * g.rows + row + lane) * g.cols + col;
#pragma unroll
                        for (int j = 0; j < 32; j += 4)      // columns are a multiple of 8
                            if (col + j < g.cols) *reinterpret_cast<float4*>(to + j) = *reinterpret_cast<float4*>(&z[j]);
                    }
                    continue;
                }
                float2 v[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint32_t bw = reinterpret_cast<const uint32_t*>(&b[j / 4])[j & 3];
                    float2 slope;
                    activations<ACT>(add_(make_float2(z[2 * j], z[2 * j + 1]), unpack16(bw, e.f16)), v[j], slope);
                    if (MODE == kSlope) v[j] = slope;
                }
                if (fetches) {
                    if (c + 32 < BN / 2)
                        fetch(mn, c + 32);
                    else if (i + step < items)
                        fetch(tile_of(i + step, g.m_tiles, g.n_tiles), 0);
                    ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&other_full[warp][taken & 1]), (uint32_t)(taken >> 1) & 1u));
                    if (!ok) break;
                    ++taken;
                } else {
                    if (lane == 0) tma_wait_read<1>();
                    __syncwarp();
                }
                const uint32_t at = mine + turn * kChunkBytes + lane * 64, key = (lane >> 1) & 3;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t to = at + ((j ^ key) << 4);
                    uint32_t q[4];
                    if (fetches) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]) : "r"(to) : "memory");
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float2 r = v[4 * j + k];
                        if (fetches) {
                            const float2 other = unpack16(q[k], e.f16);
                            r = MODE == kSlope ? mul_(r, other) : add_(r, other);
                        }
                        q[k] = pack16(r.x, r.y, e.f16);
                    }
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3]) : "memory");
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (row < g.rows && col < g.cols) tma_store(&my, col, row, mine + turn * kChunkBytes);
                    tma_commit();
                }
            }
        }
        if (lane == 0) tma_wait_all();
        // a wait ran out: what is on its way has to land before the CTA ends
        if (*(volatile int*)&bars.dead) {
            const long long begun = clock64();
            for (; taken < asked; ++taken)
                while (!mbar_try_wait(smem_addr(&other_full[warp][taken & 1]), (uint32_t)(taken >> 1) & 1u) &&
                       clock64() - begun < waits.cycles) {
                }
        }
    }
    finish<CG, EPI>(bars, tmem, filled, rank == 0, waits);
}

// The epilogue of sums that were made in parts, added in order
template <class T, int ACT, int MODE>
__global__ void __launch_bounds__(256) k_linear_join(const float* parts, int splits, int64_t n, int cols, Epilogue e, T* out) {
    wait_before();
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= n) return;
    float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) {
        const float4 q = __ldcg(reinterpret_cast<const float4*>(parts + s * n + i));
        z[0] += q.x;
        z[1] += q.y;
        z[2] += q.z;
        z[3] += q.w;
    }
    const int col = (int)(i % cols);
    uint2 q;
    uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float2 b = make_float2(0.f, 0.f), o = b;
        if (e.bias) b = unpack2(__ldg((const uint32_t*)e.bias + (col >> 1) + k), T());
        if (e.other) o = unpack2(__ldg((const uint32_t*)e.other + (i >> 1) + k), T());
        w[k] = pack2(finish_two<ACT, MODE>(add_(make_float2(z[2 * k], z[2 * k + 1]), b), o), T());
    }
    *reinterpret_cast<uint2*>(out + i) = q;
}

// ---- a few tokens (few.cuh) ------------------------------------------------------------
template <class T, int ACT>
struct LinearOf {
    static constexpr int kRows = 1;
    static constexpr bool kChained = false;
    const T *bias, *residual;
    int rows;
    __device__ __forceinline__ float operator()(const float (&s)[1], int t, int row) const {
        const float z = s[0] + (bias ? to_f32(__ldg(bias + row)) : 0.f);
        float v, slope;
        if constexpr (ACT == IFVS_ACT_GELU) {        // as the tiles have it
            float2 two, slopes;
            gelu(make_float2(z, z), two, slopes);
            v = two.x;
        } else {
            activation<ACT>(z, v, slope);
        }
        return residual ? v + to_f32(__ldg(residual + (int64_t)t * rows + row)) : v;
    }
};

// ---- host -------------------------------------------------------------------------------
TileArgs tile_args(const LinearArgs& a) { return {a.type, a.num_sms, a.waits}; }
bool linear_pairs(const LinearArgs& a) { return use_pairs(tile_args(a), a.T, a.D_out, a.D_in); }
size_t z_part_bytes(const LinearArgs& a) { return padded(Plan::part_bytes(tile_args(a), a.T, a.D_out, a.D_in, linear_pairs(a))); }
// the gradient's two products together
bool grad_pairs(const LinearArgs& a) {
    return a.T > 512 &&
           (use_pairs(tile_args(a), a.T, a.D_in, a.D_out) || use_pairs(tile_args(a), a.D_out, a.D_in, a.T));
}

template <class Fn>
cudaError_t with_any_act(int act, const Fn& f) {
    return act == IFVS_ACT_NONE ? f(std::integral_constant<int, IFVS_ACT_NONE>()) : with_act(act, f);
}

// out = the epilogue of x W^T; parts: z_part_bytes of workspace
template <int ACT, int MODE>
cudaError_t run_tiles(const LinearArgs& a, const void* x, const void* other, void* out, float* parts, cudaStream_t s) {
    const Epilogue e{a.bias, other, a.type == IFVS_T_F16};
    const bool pairs = linear_pairs(a);
    const int splits = Plan::splits_of(tile_args(a), a.T, a.D_out, a.D_in, pairs);
    auto run = [&](auto cg, auto bn) {
        using Sh = LinearShape<cg(), bn()>;
        CUtensorMap mx, mw, my, mo;
        cudaError_t r = make_map(&mx, a.type, x, a.T, a.D_in, a.D_in, kRows);
        if (r == cudaSuccess) r = make_map(&mw, a.type, a.w, a.D_out, a.D_in, a.D_in, bn() / cg());
        if (r == cudaSuccess) r = make_map(&my, a.type, out, a.T, a.D_out, a.D_out, 32, 32);
        mo = my;
        if (r == cudaSuccess && other) r = make_map(&mo, a.type, other, a.T, a.D_out, a.D_out, 32, 32);
        if (r != cudaSuccess) return r;
        const Grid g{ceil_div(a.T, kRows * cg()), ceil_div(a.D_out, bn()), ceil_div(a.D_in, kStepK), (int)a.T, a.D_out};
        return launch_tiles<cg()>(k_linear<ACT, MODE, cg(), bn()>, (int64_t)g.m_tiles * g.n_tiles * splits, a.num_sms,
                                  Sh::kEpi * 32 + 64, Sh::kSmem, false, s, mx, mw, my, mo, g, splits, parts, e, a.waits);
    };
    const cudaError_t r = pairs ? run(std::integral_constant<int, 2>(), std::integral_constant<int, 256>())
                                : run(std::integral_constant<int, 1>(), std::integral_constant<int, 128>());
    if (r != cudaSuccess || splits == 1) return r;
    const int64_t n = a.T * a.D_out;
    const dim3 grid((unsigned)((n + 1023) / 1024));
    return e.f16 ? launch_next(k_linear_join<__half, ACT, MODE>, grid, dim3(256), 0, true, s, (const float*)parts, splits, n, a.D_out,
                               e, (__half*)out)
                 : launch_next(k_linear_join<__nv_bfloat16, ACT, MODE>, grid, dim3(256), 0, true, s, (const float*)parts, splits, n,
                               a.D_out, e, (__nv_bfloat16*)out);
}

}  // namespace

size_t linear_bytes(const LinearArgs& a) { return a.T <= kFewTokens ? 0 : z_part_bytes(a); }
size_t linear_grad_bytes(const LinearArgs& a) {
    if (a.T == 0) return 0;
    const bool p = grad_pairs(a), act = a.act != IFVS_ACT_NONE;
    return (act ? padded((size_t)a.T * a.D_out * 2) + z_part_bytes(a) : 0) +
           (a.bias ? Plan::sums_bytes(tile_args(a), a.D_out) : 0) + Plan::part_bytes(tile_args(a), a.T, a.D_in, a.D_out, p) +
           Plan::part_bytes(tile_args(a), a.D_out, a.D_in, a.T, p);
}

cudaError_t launch_linear(const LinearArgs& a, const void* x, const void* residual, void* y, uint8_t* work, cudaStream_t s) {
    return with_any_act(a.act, [&](auto act) {
        if (a.T <= kFewTokens) {
            auto few = [&](auto t) {
                using T = decltype(t);
                return launch_few((const T*)x, (const T*)a.w, (T*)y, (int)a.T, a.D_out, a.D_in, a.num_sms,
                                  LinearOf<T, act()>{(const T*)a.bias, (const T*)residual, a.D_out}, s);
            };
            return a.type == IFVS_T_F16 ? few(__half()) : few(__nv_bfloat16());
        }
        return run_tiles<act(), kForward>(a, x, residual, y, (float*)work, s);
    });
}

cudaError_t launch_linear_grad(const LinearArgs& a, const void* x, const void* dy, void* dx, void* d_w, void* d_bias, uint8_t* work,
                               cudaStream_t s) {
    if (a.T == 0) {
        const cudaError_t e = cudaMemsetAsync(d_w, 0, (size_t)a.D_out * a.D_in * 2, s);
        return e != cudaSuccess || !d_bias ? e : cudaMemsetAsync(d_bias, 0, (size_t)a.D_out * 2, s);
    }
    const void* dz = dy;
    bool chain = false;
    if (a.act != IFVS_ACT_NONE) {
        uint8_t* to = work;
        work += padded((size_t)a.T * a.D_out * 2);
        const cudaError_t e = with_act(a.act, [&](auto act) { return run_tiles<act(), kSlope>(a, x, dy, to, (float*)work, s); });
        if (e != cudaSuccess) return e;
        work += z_part_bytes(a);
        dz = to;
        chain = true;
    }
    // the longer sums first
    Plan plan(tile_args(a), grad_pairs(a), work);
    auto weights = [&] { plan.add(a.D_out, a.D_in, a.T, dz, true, x, true, d_w); };
    if (a.T >= a.D_out) weights();
    plan.add(a.T, a.D_in, a.D_out, dz, false, a.w, true, dx);
    if (a.T < a.D_out) weights();
    if (d_bias) plan.add_sums(dz, a.T, a.D_out, d_bias);
    return plan.launch(chain, s);
}

}  // namespace ifvs
