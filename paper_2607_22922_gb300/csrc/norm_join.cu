// The norm after a block, its gate, the residual and the norm before the next
// block in one pass, and the gradients (ifvs_norm_join, ifvs_norm_join_grad).
#include "layers.cuh"

namespace ifvs {

namespace {

// a warp per token
template <class T>
__global__ void k_norm_join(JoinArgs a, const T* __restrict__ x, const T* __restrict__ y, T* __restrict__ xo,
                            T* __restrict__ no) {
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    check_offsets(a.offsets, a.B, a.T, a.err);
    if (t >= a.T) return;
    const int64_t b = sequence_of(a.offsets, a.B, t);
    const T* gate = (const T*)a.gate;
    const T* wp = (const T*)a.w_post;
    const T* wn = (const T*)a.w_pre;
    x += t * a.D;
    float iy = 0.f;
    if (y) {
        y += t * a.D;
        float q = 0.f;
        for (int d = lane; d < a.D; d += 32) q += to_f32(y[d]) * to_f32(y[d]);
        iy = rsqrtf(warp_sum(q) / a.D + a.eps);
    }
    auto joined = [&](int d) {
        float v = a.rho * to_f32(x[d]);
        if (y) v += (gate ? to_f32(gate[b * a.D + d]) : 1.f) * to_f32(wp[d]) * to_f32(y[d]) * iy;
        return v;
    };
    float q = 0.f;
    for (int d = lane; d < a.D; d += 32) {
        const float v = joined(d);
        q += v * v;
        if (xo) xo[t * a.D + d] = from_f32<T>(v);
    }
    if (!no) return;
    const float ix = rsqrtf(warp_sum(q) / a.D + a.eps);
    for (int d = lane; d < a.D; d += 32) no[t * a.D + d] = from_f32<T>(to_f32(wn[d]) * joined(d) * ix);
}

// per token: 1 / rms(x_out), the term of the norm's gradient along x_out, 1 / rms(y)
struct Stats {
    float ix, c, iy;
};

template <class T>
__device__ __forceinline__ float d_joined(const JoinArgs& a, const JoinGrads& g, const Stats& s, int64_t i, int d) {
    float v = g.d_x_out ? to_f32(((const T*)g.d_x_out)[i]) : 0.f;
    if (g.d_n)
        v += s.ix * (to_f32(((const T*)g.d_n)[i]) * to_f32(((const T*)a.w_pre)[d]) - to_f32(((const T*)g.x_out)[i]) * s.c);
    return v;
}

// dx, dy and the statistics: a warp per token
template <class T>
__global__ void k_join_rows(JoinArgs a, JoinGrads g, Stats* __restrict__ stats) {
    const int lane = threadIdx.x & 31;
    const int64_t t = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    check_offsets(a.offsets, a.B, a.T, a.err);
    if (t >= a.T) return;
    const int64_t b = sequence_of(a.offsets, a.B, t);
    const T* x = (const T*)g.x_out + t * a.D;
    const T* y = g.y ? (const T*)g.y + t * a.D : nullptr;
    Stats s{0.f, 0.f, 0.f};
    if (g.d_n) {
        float q = 0.f, p = 0.f;
        for (int d = lane; d < a.D; d += 32) {
            const float v = to_f32(x[d]);
            q += v * v;
            p += v * to_f32(((const T*)g.d_n)[t * a.D + d]) * to_f32(((const T*)a.w_pre)[d]);
        }
        s.ix = rsqrtf(warp_sum(q) / a.D + a.eps);
        s.c = s.ix * s.ix * warp_sum(p) / a.D;
    }
    if (y) {
        float q = 0.f;
        for (int d = lane; d < a.D; d += 32) q += to_f32(y[d]) * to_f32(y[d]);
        s.iy = rsqrtf(warp_sum(q) / a.D + a.eps);
    }
    if (lane == 0) stats[t] = s;
    auto du = [&](int d) {
        const float gt = a.gate ? to_f32(((const T*)a.gate)[b * a.D + d]) : 1.f;
        return gt * to_f32(((const T*)a.w_post)[d]) * d_joined<T>(a, g, s, t * a.D + d, d);
    };
    float m = 0.f;
    for (int d = lane; d < a.D; d += 32) {
        ((T*)g.dx)[t * a.D + d] = from_f32<T>(a.rho * d_joined<T>(a, g, s, t * a.D + d, d));
        if (y) m += du(d) * to_f32(y[d]) * s.iy;
    }
    if (!y) return;
    m = warp_sum(m) / a.D;
    for (int d = lane; d < a.D; d += 32)
        ((T*)g.dy)[t * a.D + d] = from_f32<T>(s.iy * (du(d) - to_f32(y[d]) * s.iy * m));
}

// sums[b] = sum over the tokens of sequence b of d x_out * u, and d_gate: a thread per entry
template <class T>
__global__ void k_join_gate(JoinArgs a, JoinGrads g, const Stats* __restrict__ stats, float* __restrict__ sums) {
    const int64_t b = blockIdx.x;
    const int64_t t0 = a.offsets ? max((int64_t)0, a.offsets[b]) : 0, t1 = a.offsets ? min(a.T, a.offsets[b + 1]) : a.T;
    for (int d = threadIdx.x; d < a.D; d += blockDim.x) {
        float s = 0.f;
        for (int64_t t = t0; t < t1; ++t)
            s += d_joined<T>(a, g, stats[t], t * a.D + d, d) * to_f32(((const T*)g.y)[t * a.D + d]) * stats[t].iy;
        sums[b * a.D + d] = s;
        if (g.d_gate) ((T*)g.d_gate)[b * a.D + d] = from_f32<T>(to_f32(((const T*)a.w_post)[d]) * s);
    }
}

// the norms' weights: a thread per column
template <class T>
__global__ void k_join_weights(JoinArgs a, JoinGrads g, const Stats* __restrict__ stats, const float* __restrict__ sums) {
    const int d = blockIdx.x * blockDim.x + threadIdx.x;
    if (d >= a.D) return;
    if (g.d_w_post) {
        float s = 0.f;
        for (int64_t b = 0; b < a.B; ++b)
            s += (a.gate ? to_f32(((const T*)a.gate)[b * a.D + d]) : 1.f) * sums[b * a.D + d];
        ((T*)g.d_w_post)[d] = from_f32<T>(s);
    }
    if (g.d_w_pre) {
        float s = 0.f;
        for (int64_t t = 0; t < a.T; ++t)
            s += to_f32(((const T*)g.d_n)[t * a.D + d]) * to_f32(((const T*)g.x_out)[t * a.D + d]) * stats[t].ix;
        ((T*)g.d_w_pre)[d] = from_f32<T>(s);
    }
}

}  // namespace

cudaError_t launch_norm_join(const JoinArgs& a, const void* x, const void* y, void* x_out, void* n_out,
                             cudaStream_t s) {
    return with_type(a.type, [&](auto z) {
        using T = decltype(z);
        k_norm_join<T><<<(unsigned)((a.T + 7) / 8), 256, 0, s>>>(a, (const T*)x, (const T*)y, (T*)x_out, (T*)n_out);
        return cudaGetLastError();
    });
}

size_t norm_join_grad_bytes(const JoinArgs& a) { return (size_t)a.T * sizeof(Stats) + (size_t)a.B * a.D * 4 + 256; }

cudaError_t launch_norm_join_grad(const JoinArgs& a, const JoinGrads& g, uint8_t* work, cudaStream_t s) {
    float* sums = (float*)work;
    Stats* stats = (Stats*)(work + (size_t)a.B * a.D * 4);
    return with_type(a.type, [&](auto z) {
        using T = decltype(z);
        if (a.T > 0) k_join_rows<T><<<(unsigned)((a.T + 7) / 8), 256, 0, s>>>(a, g, stats);
        if (g.y) k_join_gate<T><<<(unsigned)a.B, 256, 0, s>>>(a, g, stats, sums);
        k_join_weights<T><<<(unsigned)((a.D + 63) / 64), 64, 0, s>>>(a, g, stats, sums);
        return cudaGetLastError();
    });
}

}  // namespace ifvs
