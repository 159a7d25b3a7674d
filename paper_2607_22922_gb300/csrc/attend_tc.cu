// Attention of long sequences on the tensor cores (ifvs_attend).
//
// A CTA takes 256 rows of one group, as two tiles of 128, and the keys of one split, 128
// at a time.  Scores s = q k^T and outputs o accumulate in TMEM; a thread reads its row's
// 128 scores, takes the exponentials and puts them back as 16-bit operands, from where the
// next MMA multiplies them with the values.  The tiles take turns, so that the MMAs of one
// run while the other's exponentials are taken:
//   tensor pipe:  s_a  s_b | o_a s_a' | o_b s_b' | ...
// The running maximum is raised, and o rescaled by the threads that hold its rows, only
// where a score exceeds it by 2^8: until then the weights are at most 2^8 and as exact.
//
// 4099 queries x 17 403 keys, 8 heads of 128 in bfloat16: 232 us, 1.26 PFLOP/s, on 128 of the
// 152 SMs (plan_of in attend.cu); their tensor pipes are active 64 % of the time, the rest are
// the waits between the MMAs and the exponentials of one tile.  With all weights of a tile at once
// for their MMAs it takes 246, with a quarter at a time 245; with all and twice the warps, half of a row's scores a thread and
// the maximum by way of shared memory, 354.
#include "attend_tc.cuh"

namespace ifvs {

namespace {

constexpr int kSoftWarps = 8, kLoader = 8, kIssuer = 9, kFixer = 10, kThreads = 352;
constexpr int kMasks = 8;
constexpr float kSlack = 8.f;

template <int DH>
struct TcShapes {
    static constexpr int kHalves = DH / 64;
    static constexpr uint32_t kTile = kHalves * kHalfBytes;           // 128 rows
    static constexpr int kSlots = DH == 128 ? 4 : 8;                  // of keys and values by turns
    static constexpr size_t kSmem = 1024 + (2 + kSlots) * kTile;
};

template <int S>
struct TcBars {
    uint64_t full[S], empty[S], fixed[S], mask_ready[kMasks], q_full, s_full[2], p_full[2][2], o_full[2], drain;
    uint32_t mask[kMasks][4];
    uint32_t tmem;
    int dead;
};

struct TcWork {
    int64_t row0, q_at, k_at, k_len;
    int rows;                 // of the tiles, at most 256
    int64_t t0, t1;           // tiles of keys
};

template <class T, int DH>
__global__ void __launch_bounds__(kThreads, 1)
k_attend_tc(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
            AttendArgs a, AttendOut o, int pack, int splits, float* part_out, float* part_lse) {
    using Sh = TcShapes<DH>;
    constexpr int S = Sh::kSlots;
    constexpr bool kF16 = std::is_same_v<T, __half>;
    __shared__ __align__(8) TcBars<S> bars;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, split = blockIdx.z;
    // head of the group's first row, and its keys'
    const int h0 = blockIdx.y * pack, hk = h0 / a.group;
    check_offsets(a.q_offsets, a.B, a.Tq, a.waits.err);
    check_offsets(a.kv_offsets, a.B, a.Tk, a.waits.err);
    const Slot slot = slot_of(a.q_offsets, a.B, a.Tq, pack, 8, blockIdx.x);
    const Span qs = span_of(a.q_offsets, slot.b, a.B, a.Tq), ks = span_of(a.kv_offsets, slot.b, a.B, a.Tk);
    const int64_t row0 = slot.tile * 256, left = qs.len * pack - row0;
    if (slot.tile < 0 || left <= 0) return;
    const int rows = left < 256 ? (int)left : 256, n_tiles = rows > 128 ? 2 : 1;
    const int64_t tiles = (ks.len + 127) / 128, t0 = tiles * split / splits, t1 = tiles * (split + 1) / splits;
    const int n = (int)(t1 - t0);

    const uint32_t q_at = dynamic_smem(), ring = q_at + 2 * Sh::kTile;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            mbar_init(smem_addr(&bars.full[i]), 1);
            mbar_init(smem_addr(&bars.empty[i]), 1);
            mbar_init(smem_addr(&bars.fixed[i]), 1);
        }
        for (int i = 0; i < kMasks; ++i) mbar_init(smem_addr(&bars.mask_ready[i]), 1);
        mbar_init(smem_addr(&bars.q_full), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&bars.s_full[i]), 1);
            for (int x = 0; x < 2; ++x) mbar_init(smem_addr(&bars.p_full[i][x]), 4);
            mbar_init(smem_addr(&bars.o_full[i]), 1);
        }
        mbar_init(smem_addr(&bars.drain), 1);
        bars.dead = 0;
        fence_mbar_init();
    }
    if (warp == kIssuer) tmem_alloc<1>(smem_addr(&bars.tmem), 512);
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = bars.tmem;
    const Watch w{&bars.dead, a.waits};
    int filled = 0;                              // slots, by the loader's thread
    auto s_col = [](int i) { return (uint32_t)i * 128u; };
    auto o_col = [](int i) { return 256u + (uint32_t)i * DH; };

    if (warp == kLoader) {
        if (elect_one() && n > 0) {
            const int token = (int)(qs.at + row0 / pack), step = 128 / pack;
            mbar_arrive_expect_tx(smem_addr(&bars.q_full), n_tiles * Sh::kTile + a.waits.extra);
            for (int i = 0; i < n_tiles; ++i)
                for (int d = 0; d < Sh::kHalves; ++d)
                    tma_load_heads(q_at + i * Sh::kTile + d * kHalfBytes, &mq, d * 64, h0, token + i * step, smem_addr(&bars.q_full));
            Ring<S> r;
            bool ok = true;
            for (int j = 0; j < 2 * n && ok; ++j, r.next(), ++filled) {
                if (!(ok = w.wait(smem_addr(&bars.empty[r.at]), r.parity ^ 1u))) break;
                const uint32_t bar = smem_addr(&bars.full[r.at]);
                mbar_arrive_expect_tx(bar, Sh::kTile + a.waits.extra);
                for (int d = 0; d < Sh::kHalves; ++d)
                    tma_load_heads(ring + r.at * Sh::kTile + d * kHalfBytes, j & 1 ? &mv : &mk, d * 64, hk,
                                   (int)(ks.at + (t0 + j / 2) * 128), bar);
            }
        }
    } else if (warp == kIssuer) {
        if (elect_one() && n > 0) {
            const uint32_t id_s = mma_desc(128, 128, kF16, false, false), id_o = mma_desc(128, DH, kF16, false, true);
            bool ok = w.wait(smem_addr(&bars.q_full), 0);
            auto slot_at = [&](int j) { return (uint32_t)(j % S); };
            auto parity = [&](int j) { return (uint32_t)(j / S) & 1u; };
            // s_i of tile j; slot 2 j holds its keys
            auto scores = [&](int i, int j) {
                const uint32_t at = ring + slot_at(2 * j) * Sh::kTile;
#pragma unroll
                for (int d = 0; d < Sh::kHalves; ++d) {
                    const uint64_t da = tile_desc(q_at + i * Sh::kTile + d * kHalfBytes, false), db = tile_desc(at + d * kHalfBytes, false);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        mma_f16<1>(tmem + s_col(i), da + k * desc_step(false), db + k * desc_step(false), id_s, d + k > 0);
                }
                mma_commit<1>(smem_addr(&bars.s_full[i]));
            };
            auto keys_there = [&](int j) {
                if (!w.wait(smem_addr(&bars.full[slot_at(2 * j)]), parity(2 * j))) return false;
                fence_after_sync();
                return true;
            };
            if (ok) {
                fence_after_sync();
                if ((ok = keys_there(0))) {
                    for (int i = 0; i < n_tiles; ++i) scores(i, 0);
                    mma_commit<1>(smem_addr(&bars.empty[slot_at(0)]));
                }
            }
            for (int j = 0; j < n && ok; ++j) {
                const int v = 2 * j + 1;
                if (!(ok = w.wait(smem_addr(&bars.full[slot_at(v)]), parity(v)))) break;
                if (!(ok = w.wait(smem_addr(&bars.fixed[slot_at(v)]), parity(v)))) break;
                if (j + 1 < n && !(ok = keys_there(j + 1))) break;
                const uint64_t dv = rows_desc(ring + slot_at(v) * Sh::kTile);
                for (int i = 0; i < n_tiles && ok; ++i) {
                    for (int x = 0; x < 2; ++x) {
                        if (!(ok = w.wait(smem_addr(&bars.p_full[i][x]), (uint32_t)j & 1u))) break;
                        fence_after_sync();
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_f16_tmem_a(tmem + o_col(i), tmem + s_col(i) + (4 * x + k) * 8, dv + (4 * x + k) * desc_step(true), id_o,
                                           j > 0 || x + k > 0);
                    }
                    if (!ok) break;
                    if (i == n_tiles - 1) mma_commit<1>(smem_addr(&bars.empty[slot_at(v)]));
                    if (j + 1 < n)
                        scores(i, j + 1);
                    else
                        mma_commit<1>(smem_addr(&bars.o_full[i]));
                }
                if (ok && j + 1 < n) mma_commit<1>(smem_addr(&bars.empty[slot_at(2 * j + 2)]));
            }
        }
    } else if (warp == kFixer) {
        // which keys count, for the threads that take the exponentials; values of those that
        // do not become zeros, because 0 times what they hold may be a NaN
        for (int j = 0; j < n; ++j) {
            uint32_t bits[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t key = (t0 + j) * 128 + i * 32 + lane;
                bits[i] = __ballot_sync(0xFFFFFFFFu, key < ks.len && (a.kv_ids == nullptr || __ldg(a.kv_ids + ks.at + key) >= 0));
            }
            if (lane == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) bars.mask[j % kMasks][i] = bits[i];
                mbar_arrive<1>(smem_addr(&bars.mask_ready[j % kMasks]));
            }
            const int v = 2 * j + 1;
            if (!__all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.full[v % S]), (uint32_t)(v / S) & 1u))) break;
            if ((bits[0] & bits[1] & bits[2] & bits[3]) != 0xFFFFFFFFu) {
                const uint32_t at = ring + (v % S) * Sh::kTile;
#pragma unroll 1
                for (int i = lane; i < 128 * Sh::kHalves * 8; i += 32) {
                    const int row = (i >> 3) & 127;
                    const uint32_t word = row < 32 ? bits[0] : row < 64 ? bits[1] : row < 96 ? bits[2] : bits[3];
                    if (!((word >> (row & 31)) & 1u))
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at + (uint32_t)i * 16u), "r"(0) : "memory");
                }
                fence_proxy_async_smem();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive<1>(smem_addr(&bars.fixed[v % S]));
        }
    } else if (warp < kSoftWarps && (warp >> 2) < n_tiles) {
        const int i = warp >> 2, quad = warp & 3, r = i * 128 + quad * 32 + lane;
        const uint32_t mine = (uint32_t)quad << 21, s_at = tmem + s_col(i) + mine, o_at = tmem + o_col(i) + mine;
        const float c = a.scale * kLog2e;
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.s_full[i]), (uint32_t)j & 1u));
            if (!ok) break;
            fence_after_sync();
            float s[4][32];
#pragma unroll
            for (int x = 0; x < 4; ++x) tmem_ld32(s_at + x * 32, s[x]);
            ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.mask_ready[j % kMasks]), (uint32_t)(j / kMasks) & 1u));
            if (!ok) break;
            uint32_t bits[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) bits[x] = bars.mask[j % kMasks][x];
#pragma unroll
            for (int x = 0; x < 4; ++x) tmem_wait(s[x]);
            if ((bits[0] & bits[1] & bits[2] & bits[3]) != 0xFFFFFFFFu)
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int y = 0; y < 32; ++y)
                        if (!((bits[x] >> y) & 1u)) s[x][y] = -INFINITY;
            float top[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                top[x] = s[x][0];
#pragma unroll
                for (int y = 1; y < 31; y += 2) top[x] = fmaxf(top[x], fmaxf(s[x][y], s[x][y + 1]));
                top[x] = fmaxf(top[x], s[x][31]);
            }
            const float high = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * c;
            const bool raise = high > m + kSlack || (m == -INFINITY && high > m);
            if (__any_sync(0xFFFFFFFFu, raise)) {
                const float shrink = raise ? ex2(m - high) : 1.f;
                if (raise) m = high;
                l *= shrink;
                if (j > 0)       // s of this tile came after the MMAs of o
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
            const float2 c2 = make_float2(c, c), b2 = make_float2(-base, -base);
            float2 sum[2] = {};
#pragma unroll
            for (int x = 0; x < 4; x += 2) {
                uint32_t p[32];
#pragma unroll
                for (int y = 0; y < 64; y += 2) {
                    float* at = &s[x + (y >> 5)][y & 31];
                    float2 e = fma_(make_float2(at[0], at[1]), c2, b2);
                    e.x = ex2(e.x);
                    e.y = ex2(e.y);
                    sum[(y >> 1) & 1] = add_(sum[(y >> 1) & 1], e);
                    p[y / 2] = pack2(e, T());
                }
                tmem_st32(s_at + x * 16, p);
                // half of the weights: their MMAs run beside the other half's exponentials
                tmem_st_wait();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive<1>(smem_addr(&bars.p_full[i][x / 2]));
            }
            l += total(add_(sum[0], sum[1]));
        }
        if (ok && n > 0) ok = __all_sync(0xFFFFFFFFu, w.wait(smem_addr(&bars.o_full[i]), 0));
        if (ok) {
            fence_after_sync();
            const float inv = l == 0.f ? 0.f : 1.f / l, ln = l == 0.f ? -INFINITY : m + log2f(l);
            const int64_t row = row0 + r, token = qs.at + row / pack;
            const int head = h0 + (int)(row % pack);
            const bool in = r < rows;
            const int64_t to = ((int64_t)split * a.Tq + token) * a.heads + head;
            T* out = (T*)o.out + token * o.ld + (int64_t)head * a.dh;
#pragma unroll 1
            for (int d = 0; d < DH; d += 32) {
                float v[32];
                if (n > 0) {
                    tmem_ld32(o_at + d, v);
                    tmem_wait(v);
                }
#pragma unroll
                for (int y = 0; y < 32; ++y) v[y] = n > 0 ? v[y] * inv : 0.f;
                if (!in) continue;
#pragma unroll
                for (int y = 0; y < 32; y += 8) {
                    if (d + y >= a.dh) break;
                    if (splits > 1) {
                        float4* p = reinterpret_cast<float4*>(part_out + to * a.dh + d + y);
                        p[0] = make_float4(v[y], v[y + 1], v[y + 2], v[y + 3]);
                        p[1] = make_float4(v[y + 4], v[y + 5], v[y + 6], v[y + 7]);
                    } else {
                        Pack<T, 8> q;
#pragma unroll
                        for (int z = 0; z < 4; ++z) q.set(z, make_float2(v[y + 2 * z], v[y + 2 * z + 1]));
                        q.store(out + d + y);
                    }
                }
            }
            if (in && splits > 1)
                part_lse[to] = ln;
            else if (in && o.lse)
                o.lse[to] = ln * kLn2;
        }
    }
    __syncwarp();
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (*(volatile int*)&bars.dead) {
        // a wait ran out: wait once more, bounded, for what is in flight
        const long long begun = clock64();
        auto bounded = [&](uint32_t bar, uint32_t parity) {
            while (!mbar_try_wait(bar, parity) && clock64() - begun < a.waits.cycles) {
            }
        };
        if (warp == kLoader && n > 0) {          // `filled` is the elected thread's
            bounded(smem_addr(&bars.q_full), 0);
            for (int i = filled > S ? filled - S : 0; i < filled; ++i) bounded(smem_addr(&bars.full[i % S]), (uint32_t)(i / S) & 1u);
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
cudaError_t run(const AttendArgs& a, const AttendOut& o, int pack, int splits, float* part_out, float* part_lse, cudaStream_t s) {
    CUtensorMap mq, mk, mv;
    cudaError_t e = make_head_map(&mq, a.type, a.q, a.Tq, a.heads, a.dh, a.ld_q, pack, 128 / pack);
    if (e == cudaSuccess) e = make_head_map(&mk, a.type, a.k, a.Tk, a.kv_heads, a.dh, a.ld_k, 1, 128);
    if (e == cudaSuccess) e = make_head_map(&mv, a.type, a.v, a.Tk, a.kv_heads, a.dh, a.ld_v, 1, 128);
    if (e == cudaSuccess) e = allow_smem(k_attend_tc<T, DH>, TcShapes<DH>::kSmem);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)slots(a.Tq, a.B, pack, 8), (unsigned)(a.heads / pack), (unsigned)splits);
    return launch_next(k_attend_tc<T, DH>, grid, dim3(kThreads), TcShapes<DH>::kSmem, false, s, mq, mk, mv, a, o, pack, splits,
                       part_out, part_lse);
}

}  // namespace

cudaError_t make_head_map(CUtensorMap* map, int type, const void* p, int64_t T, int heads, int dh, int64_t ld, int box_heads,
                          int box_rows, int box_dims) {
    static const auto encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            fn = nullptr;
        return (decltype(&cuTensorMapEncodeTiled))fn;
    }();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {(cuuint64_t)dh, (cuuint64_t)heads, (cuuint64_t)T},
                     strides[2] = {(cuuint64_t)dh * 2, (cuuint64_t)ld * 2};
    const cuuint32_t box[3] = {(cuuint32_t)box_dims, (cuuint32_t)box_heads, (cuuint32_t)box_rows}, step[3] = {1, 1, 1};
    const CUresult r = encode(map, type == IFVS_T_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                              3, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              box_dims == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t launch_attend_tc(const AttendArgs& a, const AttendOut& o, int pack, int splits, float* part_out, float* part_lse,
                             cudaStream_t s) {
    auto go = [&](auto t) {
        using T = decltype(t);
        return a.dh <= 64 ? run<T, 64>(a, o, pack, splits, part_out, part_lse, s) : run<T, 128>(a, o, pack, splits, part_out, part_lse, s);
    };
    return a.type == IFVS_T_F16 ? go(__half()) : go(__nv_bfloat16());
}

}  // namespace ifvs
