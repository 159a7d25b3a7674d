// Dropout whose mask is never stored (ifvs_dropout): element i keeps its value iff the
// random word i of (seed, step) is at least p 2^32, so that the backward pass, the
// same call on the gradient, finds the same elements.
#include "layers.cuh"
#include "philox.h"

namespace ifvs {

namespace {

struct DropArgs {
    const void *x, *residual;
    void* out;
    int64_t n;
    RoundKeys keys;
    uint64_t step;
    const int64_t* more_steps;
    uint32_t below;      // words below it drop their element
    float scale;
};

// Ten rounds of two 32 x 32-bit products make four words; at 16 bits an element they bound
// the call, not memory: 163 847 x 960 in bfloat16 take 125 us, 5.0 TB/s, where their bytes take 93.
// A thread takes CH chunks of 16 bytes of x, a grid's width apart.  WIDE: all arrays
// begin on 16 bytes; else elements come one by one.
template <class T, bool RES, bool WIDE, int CH>
__global__ void __launch_bounds__(256) k_dropout(const __grid_constant__ DropArgs a) {
    constexpr int E = 16 / (int)sizeof(T);
    using P = Pack<T, E>;
    const T *x = (const T*)a.x, *res = (const T*)a.residual;
    T* out = (T*)a.out;
    const int64_t first = ((int64_t)blockIdx.x * CH * 256 + threadIdx.x) * E;
    P v[CH], r[CH];
    auto at = [&](int c) { return first + (int64_t)c * 256 * E; };
    if constexpr (WIDE) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (at(c) + E <= a.n) {
                v[c].load(x + at(c));
                if constexpr (RES) r[c].load(res + at(c));
            }
    }
    // a CTA's blocks of four words are a power of two and begin at a multiple of it: their
    // numbers' high halves are one, and so are the products with it
    const uint64_t block0 = (uint64_t)blockIdx.x * (CH * 256 * E / 4);
    const uint32_t low = (uint32_t)block0 + threadIdx.x * (E / 4), high = (uint32_t)(block0 >> 32);
    const uint64_t step = a.step + (a.more_steps ? (uint64_t)__ldg(a.more_steps) : 0u);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int64_t i = at(c);
        if (i >= a.n) return;
        uint32_t w[E];
#pragma unroll
        for (int j = 0; j < E; j += 4) {
            const Words q = philox(low + (uint32_t)(c * 256 * E + j) / 4, high, step, a.keys);
#pragma unroll
            for (int k = 0; k < 4; ++k) w[j + k] = q.w[k];
        }
        // one rounding; what is dropped may be anything
        auto one = [&](float value, float base, uint32_t word) {
            // predicated, not selected: comparisons, selections and the generator's exclusive
            // ors share a pipe
            float y = base;
            if constexpr (RES)
                asm("{\n\t.reg .pred p;\n\tsetp.ge.u32 p, %1, %2;\n\t@p fma.rn.f32 %0, %3, %4, %0;\n\t}"
                    : "+f"(y)
                    : "r"(word), "r"(a.below), "f"(value), "f"(a.scale));
            else
                asm("{\n\t.reg .pred p;\n\tsetp.ge.u32 p, %1, %2;\n\t@p mul.rn.f32 %0, %3, %4;\n\t}"
                    : "+f"(y)
                    : "r"(word), "r"(a.below), "f"(value), "f"(a.scale));
            return y;
        };
        if (WIDE && i + E <= a.n) {
#pragma unroll
            for (int j = 0; j < E / 2; ++j) {
                const float2 p = v[c].get(j), q = RES ? r[c].get(j) : make_float2(0.f, 0.f);
                v[c].set(j, make_float2(one(p.x, q.x, w[2 * j]), one(p.y, q.y, w[2 * j + 1])));
            }
            v[c].store(out + i);
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (i + j < a.n) out[i + j] = from_f32<T>(one(to_f32(x[i + j]), RES ? to_f32(res[i + j]) : 0.f, w[j]));
        }
    }
}

bool wide(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

cudaError_t launch_dropout(const void* x, const void* residual, int64_t n, int type, uint32_t below, float scale, uint64_t seed,
                           uint64_t step, const int64_t* more_steps, void* out, cudaStream_t s) {
    const DropArgs a{x, residual, out, n, round_keys(seed), step, more_steps, below, scale};
    return with_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int CH = 2;
        constexpr int64_t kPer = 256 * CH * (16 / (int64_t)sizeof(T));
        const dim3 grid((unsigned)((n + kPer - 1) / kPer));
        const bool w = wide(x) && wide(out) && wide(residual);
        auto go = [&](auto res, auto wd) { return launch_next(k_dropout<T, res(), wd(), CH>, grid, dim3(256), 0, false, s, a); };
        if (residual) return w ? go(std::true_type(), std::true_type()) : go(std::true_type(), std::false_type());
        return w ? go(std::false_type(), std::true_type()) : go(std::false_type(), std::false_type());
    });
}

}  // namespace ifvs
