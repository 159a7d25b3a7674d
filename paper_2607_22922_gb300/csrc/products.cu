// Products C = A B^T in 16 bits (products.cuh).
#include "products.cuh"

namespace ifvs {

namespace {

// Bound by the tensor pipe and, in a long run, by power: the feed-forward gradient's three
// products at 16411 x 1024 x 4096 (688 GFLOP) 372 us, 1.85 PFLOP/s, the pipe 96.4 %
// active at 1.69 GHz.
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

// The epilogue's four warps' share of the row sums: they take rows by turns, 8 columns a lane,
// and are added in order through `scratch` (4 KB of shared memory).
template <class T>
__device__ __forceinline__ void add_rows(const RowSums& r, uint32_t scratch) {
    const int cta = blockIdx.x, part = cta % r.n_parts, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (cta / r.n_parts >= r.n_phases) return;
    const int64_t r0 = r.rows * part / r.n_parts, r1 = r.rows * (part + 1) / r.n_parts;
    constexpr int AHEAD = 8;
#pragma unroll 1
    for (int c0 = cta / r.n_parts * 256; c0 < r.cols; c0 += r.n_phases * 256) {
        const int col = c0 + lane * 8;
        float2 acc[4] = {};
        if (col < r.cols)
#pragma unroll 1
            for (int64_t row = r0 + warp; row < r1; row += 4 * AHEAD) {
                Pack<T, 8> v[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)       // may be the work of the kernel before
                    v[k].w = row + 4 * k < r1 ? __ldcg(reinterpret_cast<const uint4*>((const T*)r.from + (row + 4 * k) * r.cols + col))
                                              : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = add_(acc[j], v[k].get(j));
            }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(scratch + (warp * 256 + lane * 8 + 2 * j) * 4), "f"(acc[j].x), "f"(acc[j].y)
                         : "memory");
        asm volatile("bar.sync 1, 128;" ::: "memory");
        const int t = threadIdx.x * 2;
        if (c0 + t < r.cols) {
            float2 s = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float2 v;
                asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(scratch + (k * 256 + t) * 4) : "memory");
                s = add_(s, v);
            }
            *reinterpret_cast<float2*>(r.parts + (int64_t)part * r.cols + c0 + t) = s;
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
    }
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
        if (all.sums.from) {
            if (f16)
                add_rows<__half>(all.sums, out);
            else
                add_rows<__nv_bfloat16>(all.sums, out);
        }
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

template <class T>
__global__ void __launch_bounds__(256) k_join_parts(const __grid_constant__ Parts p) {
    wait_before();
    const int j = blockIdx.y;
    // the row sums are few values of many parts: eight lanes share four of them
    const bool shared = j == p.sums;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, i = (shared ? t / 8 : t) * 4;
    const int first = shared ? (int)(t & 7) : 0, step = shared ? 8 : 1;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const int splits = i < p.n[j] ? p.splits[j] : 0;
#pragma unroll 8
    for (int s = first; s < splits; s += step) {
        const float4 q = __ldcg(reinterpret_cast<const float4*>(p.parts[j] + s * p.n[j] + i));
        v.x += q.x;
        v.y += q.y;
        v.z += q.z;
        v.w += q.w;
    }
    if (shared)
#pragma unroll
        for (int x = 1; x < 8; x <<= 1) {
            v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, x);
            v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, x);
            v.z += __shfl_xor_sync(0xFFFFFFFFu, v.z, x);
            v.w += __shfl_xor_sync(0xFFFFFFFFu, v.w, x);
        }
    if (i >= p.n[j] || first > 0) return;
    *reinterpret_cast<uint2*>((T*)p.c[j] + i) = make_uint2(pack2(make_float2(v.x, v.y), T()), pack2(make_float2(v.z, v.w), T()));
}

}  // namespace

cudaError_t make_map(CUtensorMap* map, int type, const void* p, int64_t rows, int64_t cols, int64_t stride,
                     int box_rows, int box_cols) {
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
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, step[2] = {1, 1};
    const CUresult r = encode(map, type == IFVS_T_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                              2, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              box_cols == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t Plan::launch(bool chain, cudaStream_t s) {
    if (e != cudaSuccess) return e;
    const bool f16 = a.type == IFVS_T_F16;
    e = pairs ? launch_tiles<2>(k_products<2, 256>, all.items, a.num_sms, 192, ProductShape<2, 256>::kSmem, chain, s, all,
                                f16, a.waits)
              : launch_tiles<1>(k_products<1, 128>, all.items, a.num_sms, 192, ProductShape<1, 128>::kSmem, chain, s, all,
                                f16, a.waits);
    if (e != cudaSuccess || joined == 0) return e;
    int64_t most = 0;
    for (int j = 0; j < joined; ++j) {
        const int64_t n = j == parts.sums ? parts.n[j] * 8 : parts.n[j];
        most = n > most ? n : most;
    }
    const dim3 grid((unsigned)((most + 1023) / 1024), (unsigned)joined);
    return f16 ? launch_next(k_join_parts<__half>, grid, dim3(256), 0, true, s, parts)
               : launch_next(k_join_parts<__nv_bfloat16>, grid, dim3(256), 0, true, s, parts);
}

}  // namespace ifvs
