// Philox4x32-10, the counter-based generator of Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3"
// (SC 2011), as the dropout kernels use it (internal).  Ten rounds of two 32 x 32 -> 64 bit products on a counter of four words,
// the two key words moved on by constants; every bit of the four output words is a random bit of (counter, key).
#pragma once
#include "common.cuh"

namespace hn {

struct DropArgs {
    const long long *rng;     // device: [0] seed (the key), [1] step (counter word 2, its low 32 bits); nullptr: nothing is dropped
    unsigned site;            // counter word 3: which dropout of a step
    unsigned threshold;       // an element is dropped where its 16 bits are below
    float scale;              // 65536 / (65536 - threshold): the kept elements
};

// false: p is not a probability below 1 (dropout.cu)
bool drop_args(float p, const long long *rng, int site, DropArgs *d);

// The factors of the eight elements [8 octet, 8 octet + 8) of a tensor, 16 bits each: low half of word 0, high half of word 0, ...
struct DropKey {
    unsigned k0, k1, step, site, threshold;                  // threshold: in the upper half of the word
    DropKey() = default;
    __device__ __forceinline__ explicit DropKey(const DropArgs &d) : site(d.site), threshold(d.threshold << 16)
    {
        HN_G(d.rng, 16);
        const long long seed = __ldg(d.rng);
        k0 = (unsigned)seed; k1 = (unsigned)((unsigned long long)seed >> 32);
        step = (unsigned)__ldg(d.rng + 1);
    }
    // the words of U octets, `apart` from one another; the key words of a round are formed once for all
    template <int U> __device__ __forceinline__ void words(long long octet, long long apart, uint4 (&w)[U]) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned long long o = (unsigned long long)(octet + u * apart);
            w[u] = make_uint4((unsigned)o, (unsigned)(o >> 32), step, site);
        }
        unsigned a = k0, b = k1;
#pragma unroll
        for (int r = 0; r < 10; ++r, a += 0x9E3779B9u, b += 0xBB67AE85u)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned long long p0 = (unsigned long long)w[u].x * 0xD2511F53u, p1 = (unsigned long long)w[u].z * 0xCD9E8D57u;
                w[u] = make_uint4((unsigned)(p1 >> 32) ^ w[u].y ^ a, (unsigned)p1, (unsigned)(p0 >> 32) ^ w[u].w ^ b, (unsigned)p0);
            }
    }
    // whether the element of a word's lower and of its upper half stays (an upper half is compared together with the lower: it decides)
    __device__ __forceinline__ bool low(unsigned w) const { return w << 16 >= threshold; }
    __device__ __forceinline__ bool high(unsigned w) const { return w >= threshold; }
    // bit e set: element e of the octet stays
    __device__ __forceinline__ unsigned bits(const uint4 &w) const
    {
        const unsigned v[4] = {w.x, w.y, w.z, w.w};
        unsigned m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (low(v[j])) m |= 1u << (2 * j);
            if (high(v[j])) m |= 2u << (2 * j);
        }
        return m;
    }
    __device__ __forceinline__ unsigned keep(long long octet) const
    {
        uint4 w[1];
        words(octet, 0, w);
        return bits(w[0]);
    }
};

}  // namespace hn
