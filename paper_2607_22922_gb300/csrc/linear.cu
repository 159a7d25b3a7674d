// A linear layer with bias, activation and residual in its epilogue (ifvs_linear,
// ifvs_linear_grad).
//
//   z = x W^T + b, y = act(z) + residual
//   dz = dy act'(z), dx = dz W, dW = dz^T x, db = sum over the tokens of dz
//
// k_linear accumulates a tile of z in TMEM and makes y (or, from dy, dz) of it, so
// that z is never stored: the gradient computes it again.  dz is rounded to the
// arrays' type, because the next products multiply 16-bit operands; without an
// activation it is dy itself.  dx and dW are one launch of k_products.
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

template <int ACT, int MODE>
__device__ __forceinline__ float finish_one(float z, float other) {
    float v, slope;
    activation<ACT>(z, v, slope);
    return MODE == kSlope ? slope * other : v + other;
}

// ---- tiles -------------------------------------------------------------------------
// BN columns of the output per tile; 8 epilogue warps, each 32 rows x BN / 2 columns.
template <int CG, int BN>
struct LinearShape {
    static constexpr int kEpi = 8;
    static constexpr uint32_t kStage = kABytes + BN / CG * 128, kOut = kEpi * kOutBytes;
    static constexpr int kStages = stages_of(kStage, kOut);
    static constexpr size_t kSmem = smem_of(kStage, kOut);
};

template <int ACT, int MODE, int CG, int BN>
__global__ void __launch_bounds__(LinearShape<CG, BN>::kEpi * 32 + 64, 1)
k_linear(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw,
         const __grid_constant__ CUtensorMap my, Grid g, int splits, float* parts, Epilogue e, Waits waits) {
    using Sh = LinearShape<CG, BN>;
    constexpr int EPI = Sh::kEpi, S = Sh::kStages;
    __shared__ __align__(8) Bars<S> bars;
    const uint32_t ring = dynamic_smem(), out = ring + S * Sh::kStage;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
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
        OutTile<1> o{out + (uint32_t)warp * kOutBytes};
        const int quad = warp & 3, part = (warp >> 2) * (BN / 2);
        Ring<2> acc;
        for (int i = first; i < items; i += step, acc.next()) {
            const int2 mn = tile_of(i / splits, g.m_tiles, g.n_tiles);
            const int row = (mn.x * CG + rank) * kRows + quad * 32, col0 = mn.y * BN + part;
            // this lane's row of the residual or of dy, 32 columns ahead of their use
            uint4 ahead[4];
            auto fetch = [&](int col) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    ahead[j] = e.other && row + lane < g.rows && col + 8 * j < g.cols
                                   ? __ldg(reinterpret_cast<const uint4*>((const uint16_t*)e.other +
                                                                          (int64_t)(row + lane) * g.cols + col + 8 * j))
                                   : make_uint4(0, 0, 0, 0);
            };
            if (splits == 1) fetch(col0);
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.acc_full[acc.at]), acc.parity))) break;
            fence_after_sync();
            const uint32_t tm = tmem + acc.at * 256 + part + ((uint32_t)quad << 21);
#pragma unroll 1
            for (int c = 0; c < BN / 2; c += 32) {
                const int col = col0 + c;
                float z[32];
                tmem_ld32(tm + c, z);
                uint4 other[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) other[j] = ahead[j];
                if (splits == 1 && c + 32 < BN / 2) fetch(col + 32);
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
                if ((c & 32) == 0) o.begin(lane);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 b = bias_of(e, col + 8 * j, g.cols);
                    const uint32_t bw[4] = {b.x, b.y, b.z, b.w}, ow[4] = {other[j].x, other[j].y, other[j].z, other[j].w};
                    uint32_t q[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 bf = unpack16(bw[k], e.f16), of = unpack16(ow[k], e.f16);
                        q[k] = pack16(finish_one<ACT, MODE>(z[8 * j + 2 * k] + bf.x, of.x),
                                      finish_one<ACT, MODE>(z[8 * j + 2 * k + 1] + bf.y, of.y), e.f16);
                    }
                    o.put(lane, (c & 32) / 8 + j, q[0], q[1], q[2], q[3]);
                }
                if (c & 32) o.store(lane, &my, col - 32, row, row < g.rows && col - 32 < g.cols);
            }
        }
        if (lane == 0) tma_wait_all();
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
        w[k] = pack2(make_float2(finish_one<ACT, MODE>(z[2 * k] + b.x, o.x), finish_one<ACT, MODE>(z[2 * k + 1] + b.y, o.y)), T());
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
        float v, slope;
        activation<ACT>(s[0] + (bias ? to_f32(__ldg(bias + row)) : 0.f), v, slope);
        return residual ? v + to_f32(__ldg(residual + (int64_t)t * rows + row)) : v;
    }
};

// ---- the bias's gradient: sums over the tokens -------------------------------------------
// A CTA adds the rows of its part for 256 columns, 8 a lane; its 8 warps take rows by
// turns and are added in order, and so are the parts.
constexpr int kBiasCols = 256, kBiasAhead = 4;
template <class T>
__global__ void __launch_bounds__(256) k_bias_parts(const T* __restrict__ dz, int64_t rows, int cols, int n_parts, float* parts,
                                                    T* out) {
    __shared__ float sums[8][kBiasCols];
    wait_before();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = blockIdx.x * kBiasCols + lane * 8;
    const int64_t r0 = rows * blockIdx.y / n_parts, r1 = rows * (blockIdx.y + 1) / n_parts;
    float2 acc[4] = {};
    if (col < cols)
        for (int64_t r = r0 + warp; r < r1; r += 8 * kBiasAhead) {
            Pack<T, 8> v[kBiasAhead];
#pragma unroll
            for (int k = 0; k < kBiasAhead; ++k)       // dz may be the work of the kernel before
                v[k].w = r + 8 * k < r1 ? __ldcg(reinterpret_cast<const uint4*>(dz + (r + 8 * k) * cols + col)) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < kBiasAhead; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = add_(acc[j], v[k].get(j));
        }
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<float2*>(&sums[warp][lane * 8 + 2 * j]) = acc[j];
    __syncthreads();
    const int c = blockIdx.x * kBiasCols + threadIdx.x;
    if (c >= cols) return;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += sums[k][threadIdx.x];
    if (n_parts == 1)
        out[c] = from_f32<T>(s);
    else
        parts[(int64_t)blockIdx.y * cols + c] = s;
}
template <class T>
__global__ void __launch_bounds__(256) k_bias_join(const float* parts, int n_parts, int cols, T* out) {
    __shared__ float sums[8][33];
    wait_before();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < cols)
#pragma unroll 8
        for (int p = warp; p < n_parts; p += 8) s += __ldcg(parts + (int64_t)p * cols + c);
    sums[warp][lane] = s;
    __syncthreads();
    if (warp || c >= cols) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += sums[k][lane];
    out[c] = from_f32<T>(s);
}

// ---- host -------------------------------------------------------------------------------
TileArgs tile_args(const LinearArgs& a) { return {a.type, a.num_sms, a.waits}; }
bool linear_pairs(const LinearArgs& a) { return use_pairs(tile_args(a), a.T, a.D_out, a.D_in); }
int bias_parts(const LinearArgs& a) {
    const int64_t wanted = 4 * a.num_sms / ceil_div(a.D_out, kBiasCols), most = ceil_div(a.T, 64);
    const int64_t n = wanted < most ? wanted : most;
    return (int)(n < 1 ? 1 : n);
}
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
        CUtensorMap mx, mw, my;
        cudaError_t r = make_map(&mx, a.type, x, a.T, a.D_in, a.D_in, kRows);
        if (r == cudaSuccess) r = make_map(&mw, a.type, a.w, a.D_out, a.D_in, a.D_in, bn() / cg());
        if (r == cudaSuccess) r = make_map(&my, a.type, out, a.T, a.D_out, a.D_out, 32);
        if (r != cudaSuccess) return r;
        const Grid g{ceil_div(a.T, kRows * cg()), ceil_div(a.D_out, bn()), ceil_div(a.D_in, kStepK), (int)a.T, a.D_out};
        return launch_tiles<cg()>(k_linear<ACT, MODE, cg(), bn()>, (int64_t)g.m_tiles * g.n_tiles * splits, a.num_sms,
                                  Sh::kEpi * 32 + 64, Sh::kSmem, false, s, mx, mw, my, g, splits, parts, e, a.waits);
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

template <class T>
cudaError_t run_bias(const LinearArgs& a, const void* dz, void* d_bias, float* parts, bool chain, cudaStream_t s) {
    const int n = bias_parts(a);
    const dim3 grid((unsigned)ceil_div(a.D_out, kBiasCols), (unsigned)n);
    const cudaError_t r = launch_next(k_bias_parts<T>, grid, dim3(256), 0, chain, s, (const T*)dz, a.T, a.D_out, n, parts, (T*)d_bias);
    if (r != cudaSuccess || n == 1) return r;
    return launch_next(k_bias_join<T>, dim3((unsigned)ceil_div(a.D_out, 32)), dim3(256), 0, true, s, (const float*)parts, n, a.D_out,
                       (T*)d_bias);
}

}  // namespace

size_t linear_bytes(const LinearArgs& a) { return a.T <= kFewTokens ? 0 : z_part_bytes(a); }
size_t linear_grad_bytes(const LinearArgs& a) {
    if (a.T == 0) return 0;
    const bool p = grad_pairs(a), act = a.act != IFVS_ACT_NONE;
    return (act ? padded((size_t)a.T * a.D_out * 2) + z_part_bytes(a) : 0) +
           (a.bias ? padded((size_t)bias_parts(a) * a.D_out * 4) : 0) +
           padded(Plan::part_bytes(tile_args(a), a.T, a.D_in, a.D_out, p)) +
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
    if (d_bias) {
        const cudaError_t e = a.type == IFVS_T_F16 ? run_bias<__half>(a, dz, d_bias, (float*)work, chain, s)
                                                   : run_bias<__nv_bfloat16>(a, dz, d_bias, (float*)work, chain, s);
        if (e != cudaSuccess) return e;
        work += padded((size_t)bias_parts(a) * a.D_out * 4);
        chain = true;
    }
    // the longer sums first
    Plan plan(tile_args(a), grad_pairs(a), work);
    auto weights = [&] { plan.add(a.D_out, a.D_in, a.T, dz, true, x, true, d_w); };
    if (a.T >= a.D_out) weights();
    plan.add(a.T, a.D_in, a.D_out, dz, false, a.w, true, dx);
    if (a.T < a.D_out) weights();
    return plan.launch(chain, s);
}

}  // namespace ifvs
