// Counter-based random words, in a form that a host compiler takes too: tests hold
// them to the published answers.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define IFVS_HD __host__ __device__ __forceinline__
#else
#define IFVS_HD inline
#endif

namespace ifvs {

struct Words {
    uint32_t w[4];
};

// Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers:
// as easy as 1, 2, 3", SC 2011): the counter is `block` and `step`, 64 bits each, the
// key is `seed`.  Words of different counters are independent, so that a word costs no
// memory and is the same whoever computes it.
IFVS_HD Words philox(uint64_t block, uint64_t step, uint64_t seed) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)step, c3 = (uint32_t)(step >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#ifdef __CUDACC__
#pragma unroll
#endif
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

}  // namespace ifvs
