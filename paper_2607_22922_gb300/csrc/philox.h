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

struct RoundKeys {
    uint32_t k[10][2];
};
IFVS_HD RoundKeys round_keys(uint64_t seed) {
    RoundKeys r;
    for (int i = 0; i < 10; ++i) {
        r.k[i][0] = (uint32_t)seed + (uint32_t)i * 0x9E3779B9u;
        r.k[i][1] = (uint32_t)(seed >> 32) + (uint32_t)i * 0xBB67AE85u;
    }
    return r;
}

// Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers:
// as easy as 1, 2, 3", SC 2011): the counter is a block's number and `step`, 64 bits
// each, the round keys come from the seed.  Words of different counters are independent,
// so that a word costs no memory and is the same whoever computes it.
IFVS_HD Words philox(uint32_t block_low, uint32_t block_high, uint64_t step, const RoundKeys& keys) {
    uint32_t c0 = block_low, c1 = block_high, c2 = (uint32_t)step, c3 = (uint32_t)(step >> 32);
#ifdef __CUDACC__
#pragma unroll
#endif
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ keys.k[r][0];
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ keys.k[r][1];
        c3 = (uint32_t)a;
    }
    return {{c0, c1, c2, c3}};
}

}  // namespace ifvs
