// Matrix products of a few tokens, on the CUDA cores: the weights are read once and
// bound the call.
#pragma once

#include "layers.cuh"

namespace ifvs {

constexpr int kFewTokens = 4;

// A row of weights (two of them, for an Epi of two) is spread over the lanes of one or
// more warps, 16 bytes a lane and access, against every token's row.
template <class T>
struct FewArgs {
    const T *x, *w;      // x [tokens][K], w [rows][K] ([kRows rows][K])
    T* out;              // [tokens][rows]
    int tokens, rows, K;
    int cta_rows;        // rows per CTA of 8 warps: 8 / cta_rows warps share one
};

// Epi: what becomes of the sums.  kRows: rows of weights per row of the output, `rows`
// apart; kChained: x comes from the kernel before, which this one may have started
// beside; operator()(sums, token, row): the output, in float32.
template <class T, class Epi, int TT>
__global__ void __launch_bounds__(256) k_few(FewArgs<T> a, Epi epi) {
    constexpr int NW = Epi::kRows, AHEAD = 4;
    constexpr bool kChained = Epi::kChained;
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
    if constexpr (!kChained) start_dependents();
    for (int c0 = part * 32 + lane; c0 < chunks; c0 += share * 32 * AHEAD) {
        Pack<T, 8> v[AHEAD][NW];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int r = 0; r < NW; ++r) v[k][r].load(w[r] + (int64_t)min(c0 + k * share * 32, chunks - 1) * 8);
        // the weights are on their way before the kernel that makes x has ended
        if (kChained && !waited) wait_before();
        waited = true;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int c = c0 + k * share * 32;
            if (c >= chunks) break;
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                Pack<T, 8> x;
                const T* from = a.x + (int64_t)min(t, a.tokens - 1) * a.K + c * 8;
                if constexpr (!kChained)
                    x.load(from);
                else
                    x.w = __ldcg(reinterpret_cast<const uint4*>(from));
#pragma unroll
                for (int r = 0; r < NW; ++r)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[r][t] = fma_(v[k][r].get(j), x.get(j), acc[r][t]);
            }
        }
    }
    if (kChained && !waited) wait_before();
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
            a.out[(int64_t)t * a.rows + row] = from_f32<T>(epi(s, t, row));
        }
}

// CTAs of 8 warps over the rows: 8 rows a CTA, fewer where they would leave SMs without one
template <class T, class Epi>
inline cudaError_t launch_few(const T* x, const T* w, T* out, int tokens, int rows, int K, int num_sms, const Epi& epi,
                              cudaStream_t s) {
    FewArgs<T> f{x, w, out, tokens, rows, K, 8};
    while (f.cta_rows > 1 && (rows + f.cta_rows - 1) / f.cta_rows < 2 * num_sms) f.cta_rows /= 2;
    const dim3 grid((unsigned)((rows + f.cta_rows - 1) / f.cta_rows));
    auto go = [&](auto tt) { return launch_next(k_few<T, Epi, tt()>, grid, dim3(256), 0, Epi::kChained, s, f, epi); };
    if (tokens == 1) return go(std::integral_constant<int, 1>());
    if (tokens == 2) return go(std::integral_constant<int, 2>());
    return go(std::integral_constant<int, kFewTokens>());
}

}  // namespace ifvs
