// The gated feed-forward block and its gradient (ifvs_ffn, ifvs_ffn_grad).
#include "layers.cuh"

namespace ifvs {

namespace {

// act(g) and act'(g)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& v, float& slope) {
    if (ACT == IFVS_ACT_RELU) {
        v = g > 0.f ? g : 0.f;
        slope = g > 0.f ? 1.f : 0.f;
    } else if (ACT == IFVS_ACT_SILU) {
        const float p = 1.f / (1.f + __expf(-g));
        v = g * p;
        slope = p * (1.f + g * (1.f - p));
    } else {
        const float p = 0.5f * erfcf(-0.70710678f * g);
        v = g * p;
        slope = p + g * 0.39894228f * __expf(-0.5f * g * g);
    }
}

// C[m][n] = sum_k A(m, k) B(n, k); an operand's element (i, k) at i * si + k * sk
template <class T, class TC>
__global__ void k_product(int64_t M, int64_t N, int64_t K, const T* __restrict__ A, int64_t am, int64_t ak,
                          const T* __restrict__ B, int64_t bn, int64_t bk, TC* __restrict__ C) {
    __shared__ float sa[16][65], sb[16][65];
    const int tid = threadIdx.x;
    const int64_t m0 = (int64_t)blockIdx.y * 64, n0 = (int64_t)blockIdx.x * 64;
    const int tm = tid / 16 * 4, tn = tid % 16 * 4;
    float c[4][4] = {};
    for (int64_t k0 = 0; k0 < K; k0 += 16) {
        for (int i = tid; i < 1024; i += 256) {
            const int r = i / 16, k = i % 16;
            const bool in = k0 + k < K;
            sa[k][r] = in && m0 + r < M ? to_f32(A[(m0 + r) * am + (k0 + k) * ak]) : 0.f;
            sb[k][r] = in && n0 + r < N ? to_f32(B[(n0 + r) * bn + (k0 + k) * bk]) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < 16; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) c[i][j] += sa[k][tm + i] * sb[k][tn + j];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (m0 + tm + i < M && n0 + tn + j < N) C[(m0 + tm + i) * N + n0 + tn + j] = from_f32<TC>(c[i][j]);
}

template <class T, class TC>
cudaError_t product(int64_t M, int64_t N, int64_t K, const void* A, int64_t am, int64_t ak, const void* B, int64_t bn,
                    int64_t bk, void* C, cudaStream_t s) {
    // rows of tiles along y, at most 65535 of them a launch
    for (int64_t m = 0; m < M; m += 65535 * 64) {
        const int64_t rows = M - m < 65535 * 64 ? M - m : 65535 * 64;
        k_product<T, TC><<<dim3((unsigned)((N + 63) / 64), (unsigned)((rows + 63) / 64)), 256, 0, s>>>(
            rows, N, K, (const T*)A + m * am, am, ak, (const T*)B, bn, bk, (TC*)C + m * N);
    }
    return cudaGetLastError();
}

// h = act(g) u; with dh: dg | du beside it
template <class T, int ACT>
__global__ void k_gate(int64_t T_, int F, const float* __restrict__ gu, const float* __restrict__ dh, T* __restrict__ h,
                       T* __restrict__ dgu) {
    const int64_t n = T_ * F;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t t = i / F, f = i % F;
        const float g = gu[t * 2 * F + f], u = gu[t * 2 * F + F + f];
        float v, slope;
        activation<ACT>(g, v, slope);
        h[i] = from_f32<T>(v * u);
        if (dh) {
            dgu[t * 2 * F + f] = from_f32<T>(dh[i] * u * slope);
            dgu[t * 2 * F + F + f] = from_f32<T>(dh[i] * v);
        }
    }
}

template <class T>
cudaError_t gate(const FfnArgs& a, const float* gu, const float* dh, T* h, T* dgu, cudaStream_t s) {
    const unsigned grid = (unsigned)(a.num_sms * 8);
    if (a.act == IFVS_ACT_SILU)
        k_gate<T, IFVS_ACT_SILU><<<grid, 256, 0, s>>>(a.T, a.F, gu, dh, h, dgu);
    else if (a.act == IFVS_ACT_GELU)
        k_gate<T, IFVS_ACT_GELU><<<grid, 256, 0, s>>>(a.T, a.F, gu, dh, h, dgu);
    else
        k_gate<T, IFVS_ACT_RELU><<<grid, 256, 0, s>>>(a.T, a.F, gu, dh, h, dgu);
    return cudaGetLastError();
}

template <class Fn>
cudaError_t with_type16(int type, const Fn& f) {
    return type == IFVS_T_F16 ? f(__half()) : f(__nv_bfloat16());
}

}  // namespace

size_t ffn_bytes(const FfnArgs& a) { return (size_t)a.T * a.F * (8 + 2); }
size_t ffn_grad_bytes(const FfnArgs& a) { return (size_t)a.T * a.F * (8 + 4 + 2 + 4); }

cudaError_t launch_ffn(const FfnArgs& a, const void* x, void* y, uint8_t* work, cudaStream_t s) {
    return with_type16(a.type, [&](auto z) {
        using T = decltype(z);
        const int64_t D = a.D, F = a.F;
        float* gu = (float*)work;
        T* h = (T*)(work + (size_t)a.T * F * 8);
        cudaError_t e = product<T, float>(a.T, 2 * F, D, x, D, 1, a.w_in, D, 1, gu, s);
        if (e == cudaSuccess) e = gate<T>(a, gu, nullptr, h, nullptr, s);
        if (e == cudaSuccess) e = product<T, T>(a.T, D, F, h, F, 1, a.w_out, F, 1, y, s);
        return e;
    });
}

cudaError_t launch_ffn_grad(const FfnArgs& a, const void* x, const void* dy, void* dx, void* d_w_in, void* d_w_out,
                            uint8_t* work, cudaStream_t s) {
    return with_type16(a.type, [&](auto z) {
        using T = decltype(z);
        const int64_t D = a.D, F = a.F;
        const size_t n = (size_t)a.T * F;
        float *gu = (float*)work, *dh = (float*)(work + n * 8);
        T *h = (T*)(work + n * 12), *dgu = (T*)(work + n * 14);
        cudaError_t e = cudaSuccess;
        auto then = [&](cudaError_t r) { e = e == cudaSuccess ? r : e; };
        if (a.T > 0) {
            then(product<T, float>(a.T, 2 * F, D, x, D, 1, a.w_in, D, 1, gu, s));
            then(product<T, float>(a.T, F, D, dy, D, 1, a.w_out, 1, F, dh, s));
            then(gate<T>(a, gu, dh, h, dgu, s));
            then(product<T, T>(a.T, D, 2 * F, dgu, 2 * F, 1, a.w_in, 1, D, dx, s));
        }
        then(product<T, T>(2 * F, D, a.T, dgu, 1, 2 * F, x, 1, D, d_w_in, s));
        then(product<T, T>(D, F, a.T, dy, 1, D, h, 1, F, d_w_out, s));
        return e;
    });
}

}  // namespace ifvs
