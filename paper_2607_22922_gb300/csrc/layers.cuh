// Layers of a predicate encoder: what their kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "internal.cuh"

namespace ifvs {

// The handle's error words: one per error, so that a kernel's plain store of 1
// takes back no other
constexpr int kErrId = 0;        // a token id outside -1..V-1
constexpr int kErrOffsets = 1;   // offsets that break their rules
constexpr int kErrWait = 2;      // a bounded wait ran out
constexpr int kErrWords = 3;

inline size_t padded(size_t n) { return (n + 255) / 256 * 256; }
inline size_t elem_bytes(int type) { return type == IFVS_T_F32 ? 4 : 2; }

// ---- element types --------------------------------------------------------
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// ---- pairs of floats: two float32 operations per instruction -----------------
__device__ __forceinline__ uint64_t bits(float2 v) { return *reinterpret_cast<uint64_t*>(&v); }
__device__ __forceinline__ float2 pair(uint64_t v) { return *reinterpret_cast<float2*>(&v); }
__device__ __forceinline__ float2 fma_(float2 a, float2 b, float2 c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)), "l"(bits(c)));
    return pair(d);
}
__device__ __forceinline__ float2 mul_(float2 a, float2 b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)));
    return pair(d);
}
__device__ __forceinline__ float2 add_(float2 a, float2 b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits(a)), "l"(bits(b)));
    return pair(d);
}
__device__ __forceinline__ float fma_(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float mul_(float a, float b) { return a * b; }
__device__ __forceinline__ float add_(float a, float b) { return a + b; }
__device__ __forceinline__ float total(float2 v) { return v.x + v.y; }
__device__ __forceinline__ float total(float v) { return v; }
template <class F>
__device__ __forceinline__ F both(float v);
template <>
__device__ __forceinline__ float both<float>(float v) { return v; }
template <>
__device__ __forceinline__ float2 both<float2>(float v) { return make_float2(v, v); }

// two 16-bit elements <-> a pair of floats
__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }
__device__ __forceinline__ uint32_t pack2(float2 v, __nv_bfloat16) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(v.y), "f"(v.x));
    return d;
}
__device__ __forceinline__ uint32_t pack2(float2 v, __half) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(v.y), "f"(v.x));
    return d;
}

// N consecutive elements, in one access of 16, 8, 4 or 2 bytes, as N / 2 pairs of
// floats or (N = 1) one float
template <class T, int N>
struct Pack {
    static constexpr int kBytes = N * (int)sizeof(T);
    using Word = std::conditional_t<kBytes == 16, uint4, std::conditional_t<kBytes == 8, uint2, std::conditional_t<kBytes == 4, uint32_t, uint16_t>>>;
    using F = std::conditional_t<N == 1, float, float2>;
    static constexpr int kF = N == 1 ? 1 : N / 2;
    Word w;
    __device__ __forceinline__ void load(const T* p) { w = __ldg(reinterpret_cast<const Word*>(p)); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Word*>(p) = w; }
    // not to be read again soon
    __device__ __forceinline__ void store_stream(T* p) const { __stcs(reinterpret_cast<Word*>(p), w); }
    __device__ __forceinline__ F get(int i) const {
        if constexpr (N == 1) {
            return to_f32(*reinterpret_cast<const T*>(&w));
        } else if constexpr (sizeof(T) == 4) {
            return reinterpret_cast<const float2*>(&w)[i];
        } else {
            return unpack2(reinterpret_cast<const uint32_t*>(&w)[i], T());
        }
    }
    __device__ __forceinline__ void set(int i, F v) {
        if constexpr (N == 1) {
            *reinterpret_cast<T*>(&w) = from_f32<T>(v);
        } else if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float2*>(&w)[i] = v;
        } else {
            reinterpret_cast<uint32_t*>(&w)[i] = pack2(v, T());
        }
    }
};

// One thread of a converged warp, always the same.  Where it is asked for this
// way the compiler knows that one thread runs the branch; under `lane == 0` it
// issues every MMA and TMA instruction in a loop over the warp's active
// threads: 513 clocks per 4 MMAs of 128 columns with their wait and commit
// instead of 257, which is what the tensor pipe takes.
__device__ __forceinline__ bool elect_one() {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0u;
}

// Calls f with a value of the element type that `type` names
template <class Fn>
inline cudaError_t with_type(int type, const Fn& f) {
    if (type == IFVS_T_F32) return f(float());
    if (type == IFVS_T_F16) return f(__half());
    return f(__nv_bfloat16());
}

// Dynamic shared memory beyond the 48 KB, static included (at most 17 KB in these
// kernels), that a kernel may have unasked
template <class K>
inline cudaError_t allow_smem(K* kernel, size_t bytes) {
    return bytes <= 31 * 1024 ? cudaSuccess
                              : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

// What a kernel's waits for its copies go by
struct Waits {
    int* err;               // the error words
    uint32_t extra;         // bytes that barriers expect beyond the copies' (0 but in tests)
    long long cycles;       // a wait's bound
};

// Failure injection for tests of calls that fail on their way: the launch that the
// calling thread's count reaches 0 at is not made and fails (layers.cu sets the
// count; 0: none does).
extern thread_local int launches_to_failure;
inline cudaError_t next_launch() {
    return launches_to_failure > 0 && --launches_to_failure == 0 ? cudaErrorLaunchOutOfResources : cudaSuccess;
}
// launch_kernel, as one of a call's launches
template <class K, class... A>
inline cudaError_t launch_next(K* kernel, dim3 grid, dim3 block, size_t smem, bool chain, cudaStream_t s, A... args) {
    const cudaError_t e = next_launch();
    return e != cudaSuccess ? e : launch_kernel(kernel, grid, block, smem, chain, s, args...);
}

// ---- launchers --------------------------------------------------------------
struct EmbedArgs {
    const int32_t* ids;
    int64_t T, V;
    int D, type;
    float scale;
    Waits waits;
    int num_sms;
};
cudaError_t launch_embed(const EmbedArgs& a, const void* table, void* out, cudaStream_t s);
size_t embed_grad_bytes(const EmbedArgs& a);
cudaError_t launch_embed_grad(const EmbedArgs& a, const void* d_out, void* d_table, uint8_t* work, cudaStream_t s);

struct JoinArgs {
    int64_t T, B;
    int D, type;
    const int64_t* offsets;      // null: B = 1
    const int64_t* given;        // the caller's, of any B: to be checked, or null
    const void *gate, *w_post, *w_pre;
    float rho, eps;
    Waits waits;
    int num_sms;
};
cudaError_t launch_norm_join(const JoinArgs& a, const void* x, const void* y, void* x_out, void* n_out,
                             cudaStream_t s);
struct JoinGrads {
    const void *x_out, *y, *d_x_out, *d_n;
    void *dx, *dy, *d_gate, *d_w_post, *d_w_pre;
};
size_t norm_join_grad_bytes(const JoinArgs& a);
cudaError_t launch_norm_join_grad(const JoinArgs& a, const JoinGrads& g, uint8_t* work, cudaStream_t s);

struct FfnArgs {
    int64_t T;
    int D, F, type, act;
    const void *w_in, *w_out;
    Waits waits;
    int num_sms;
};
size_t ffn_bytes(const FfnArgs& a);
cudaError_t launch_ffn(const FfnArgs& a, const void* x, void* y, uint8_t* work, cudaStream_t s);
size_t ffn_grad_bytes(const FfnArgs& a);
cudaError_t launch_ffn_grad(const FfnArgs& a, const void* x, const void* dy, void* dx, void* d_w_in, void* d_w_out,
                            uint8_t* work, cudaStream_t s);

struct LinearArgs {
    int64_t T;
    int D_in, D_out, type, act;
    const void *w, *bias;        // bias: or null
    Waits waits;
    int num_sms;
};
size_t linear_bytes(const LinearArgs& a);
cudaError_t launch_linear(const LinearArgs& a, const void* x, const void* residual, void* y, uint8_t* work, cudaStream_t s);
size_t linear_grad_bytes(const LinearArgs& a);
cudaError_t launch_linear_grad(const LinearArgs& a, const void* x, const void* dy, void* dx, void* d_w, void* d_bias,
                               uint8_t* work, cudaStream_t s);

cudaError_t launch_dropout(const void* x, const void* residual, int64_t n, int type, uint32_t below, float scale, uint64_t seed,
                           uint64_t step, const int64_t* more_steps, void* out, cudaStream_t s);

// Reports offsets that break their rules; the whole grid (x) calls it.
__device__ __forceinline__ void check_offsets(const int64_t* __restrict__ offsets, int64_t B, int64_t T, int* err) {
    if (offsets == nullptr) return;
    bool bad = false;
    for (int64_t b = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; b < B; b += (int64_t)gridDim.x * blockDim.x) {
        const int64_t lo = __ldg(offsets + b), hi = __ldg(offsets + b + 1);
        bad |= hi < lo || (b == 0 && lo != 0) || (b == B - 1 && hi != T);
    }
    if (bad) err[kErrOffsets] = 1;
}

// the sequence of token t: the last b with offsets[b] <= t, within 0..B-1
// whatever the offsets hold
__device__ __forceinline__ int64_t sequence_of(const int64_t* __restrict__ offsets, int64_t B, int64_t t) {
    if (offsets == nullptr || B == 1) return 0;
    int64_t lo = 0, hi = B;      // offsets[lo] <= t (assumed of 0), hi: beyond
    while (hi - lo > 1) {
        const int64_t m = (lo + hi) >> 1;
        if (__ldg(offsets + m) <= t)
            lo = m;
        else
            hi = m;
    }
    return lo;
}

}  // namespace ifvs
