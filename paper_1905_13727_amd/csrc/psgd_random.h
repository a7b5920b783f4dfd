// The counter-based generator of dropout and of the random mask: Philox4x32 with ten rounds (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", SC 2011).  Four words from a 128-bit counter and a 64-bit key, nothing
// carried from one call to the next, so that a backward pass or a replay draws again what it needs and no mask is stored.
#ifndef PSGD_RANDOM_H
#define PSGD_RANDOM_H

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace psgd {

struct Draw {   // key and the upper half of the counter, the same in every lane
    unsigned k0, k1, c2, c3;
};

// rng: {seed, offset} in device memory, so that a captured graph draws anew once the caller has moved the offset on
typedef unsigned DrawWords __attribute__((ext_vector_type(4)));
__device__ __forceinline__ DrawWords words_ahead(const uint64_t* __restrict__ rng, uint64_t offset) {
    const uint64_t seed = rng[0], at = rng[1] + offset;
    return DrawWords{(unsigned)seed, (unsigned)(seed >> 32), (unsigned)at, (unsigned)(at >> 32)};
}
__device__ __forceinline__ Draw make_draw(const DrawWords& w) {
    Draw d;
    d.k0 = __builtin_amdgcn_readfirstlane(w[0]);
    d.k1 = __builtin_amdgcn_readfirstlane(w[1]);
    d.c2 = __builtin_amdgcn_readfirstlane(w[2]);
    d.c3 = __builtin_amdgcn_readfirstlane(w[3]);
    return d;
}
__device__ __forceinline__ Draw make_draw(const uint64_t* __restrict__ rng, uint64_t offset) { return make_draw(words_ahead(rng, offset)); }

struct Words {
    unsigned w[4];
};

__device__ __forceinline__ Words philox(const Draw& d, unsigned c0, unsigned c1) {
    unsigned c2 = d.c2, c3 = d.c3, k0 = d.k0, k1 = d.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        const unsigned n0 = (unsigned)(b >> 32) ^ c1 ^ k0, n2 = (unsigned)(a >> 32) ^ c3 ^ k1;
        c1 = (unsigned)b;
        c3 = (unsigned)a;
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

// Dropout: sixteen bits an element, eight columns a call; element j of the eight is dropped where its half word is below
// `below`.  Sixteen bits make p a multiple of 2^-16; thirty-two would need twice the calls, which bf16 data does not hide.
__device__ __forceinline__ bool dropped(const Words& x, int j, unsigned below) {
    const unsigned w = x.w[j >> 1];
    return ((j & 1) ? w >> 16 : w & 0xffffu) < below;
}

struct DropArgs {
    const uint64_t* rng = nullptr;
    uint64_t offset = 0;
    unsigned below = 0;    // 0: no dropout
    float factor = 1.f;    // of the elements that stay: 65536 / (65536 - below); 0 where none does
};

}  // namespace psgd

#endif
