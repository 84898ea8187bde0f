// Counter-based random bits: Philox4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lrd {

struct Words4 { uint32_t w0, w1, w2, w3; };

// Four words for a counter of 128 bits and a key of 64: any element's bits are computed where they are needed.
__device__ __forceinline__ Words4 philox4x32(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {c0, c1, c2, c3};
}

// Which elements a dropout keeps.  Element i of the dense array has 16 bits: half (i & 1) of word (i >> 1 & 3) for the counter
// (i / 8, call), key = seed; it is dropped where they are below `below` = round(65536 p).  16 bits and not 32: one generator
// call (20 multiplications of quarter rate) serves eight elements, so that it stays under the time of their memory traffic; p is
// then a multiple of 2^-16, and the scale 65536 / (65536 - below) is that p's, so that the mean is kept.
struct DropRng {
    const uint64_t* state;      // device memory: seed, call
    uint32_t below;             // 0: nothing is dropped, and state is not read
    float scale;
};
struct DropKey {
    uint32_t k0, k1, c2, c3;
    DropKey() = default;
    __device__ __forceinline__ explicit DropKey(const uint64_t* state)
    {
        const uint64_t seed = state[0], call = state[1];
        k0 = (uint32_t)seed; k1 = (uint32_t)(seed >> 32);
        c2 = (uint32_t)call; c3 = (uint32_t)(call >> 32);
    }
    __device__ __forceinline__ Words4 eight(uint64_t group) const { return philox4x32((uint32_t)group, (uint32_t)(group >> 32), c2, c3, k0, k1); }
};
// The bits of element e = 0 .. 7 of a group (e known at compile time or not).
__device__ __forceinline__ uint32_t drop_bits(Words4 w, int e)
{
    const uint32_t lo = (e & 2) ? w.w1 : w.w0, hi = (e & 2) ? w.w3 : w.w2, v = (e & 4) ? hi : lo;
    return (e & 1) ? v >> 16 : v & 0xffffu;
}

}  // namespace lrd
