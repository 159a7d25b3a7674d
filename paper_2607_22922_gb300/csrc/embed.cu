// Embedding lookup with scaling and its gradient (ifvs_embed, ifvs_embed_grad).
#include "layers.cuh"

namespace ifvs {

namespace {

// out[t] = scale table[ids[t]]: a CTA per token
template <class T>
__global__ void k_embed(const T* __restrict__ table, EmbedArgs a, T* __restrict__ out) {
    const int64_t t = blockIdx.x;
    const int id = a.ids[t];
    const bool ok = id >= 0 && id < a.V;
    if (!ok && id != -1 && threadIdx.x == 0) *a.err = kErrId;
    for (int d = threadIdx.x; d < a.D; d += blockDim.x)
        out[t * a.D + d] = from_f32<T>(ok ? a.scale * to_f32(table[(int64_t)id * a.D + d]) : 0.f);
}

// d_table[v]: a CTA per row of the table looks through all ids
template <class T>
__global__ void k_embed_grad(const T* __restrict__ d_out, EmbedArgs a, T* __restrict__ d_table) {
    const int64_t v = blockIdx.x;
    for (int d0 = 0; d0 < a.D; d0 += blockDim.x) {
        const int d = d0 + threadIdx.x;
        float sum = 0.f;
        for (int64_t t = 0; t < a.T; ++t) {
            const int id = __ldg(a.ids + t);
            if (v == 0 && d == 0 && (id < -1 || id >= a.V)) *a.err = kErrId;
            if (id == v && d < a.D) sum += to_f32(d_out[t * a.D + d]);
        }
        if (d < a.D) d_table[v * a.D + d] = from_f32<T>(a.scale * sum);
    }
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs& a, const void* table, void* out, cudaStream_t s) {
    return with_type(a.type, [&](auto z) {
        using T = decltype(z);
        k_embed<T><<<(unsigned)a.T, 128, 0, s>>>((const T*)table, a, (T*)out);
        return cudaGetLastError();
    });
}

size_t embed_grad_bytes(const EmbedArgs&) { return 0; }

cudaError_t launch_embed_grad(const EmbedArgs& a, const void* d_out, void* d_table, uint8_t*, cudaStream_t s) {
    return with_type(a.type, [&](auto z) {
        using T = decltype(z);
        k_embed_grad<T><<<(unsigned)a.V, 128, 0, s>>>((const T*)d_out, a, (T*)d_table);
        return cudaGetLastError();
    });
}

}  // namespace ifvs
