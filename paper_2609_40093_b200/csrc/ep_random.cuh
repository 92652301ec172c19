// Dropout from a counter-based generator: what is dropped follows from the element's place, the seed and the step, so no mask
// is stored and the gradient makes the same one again.
//
// Philox4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten rounds of
// two 32 x 32 -> 64 bit products and three-way xors. One call's four words serve the eight elements of a 16-byte vector, 16
// bits each: 60 instructions instead of 120 with a word per element, and with 120 the generator, not memory, would bound an
// elementwise pass. A probability is therefore kept to a multiple of 2^-16, and the scale of what is kept follows that multiple,
// so that the mean is right.
#pragma once

#include "ep_common.cuh"

namespace ep {

struct DropoutArgs {
    const unsigned long long *state;      // device: seed, step; NULL: no dropout
    uint32_t edge;                        // an element is dropped where its 16 bits, as the upper half of a word, are below this
    uint32_t site;
    float scale;
    int all;                              // p = 1: everything is dropped
};

// What a call is given, as the kernels take it. p = 0 (or NULL) is no dropout.
inline int dropout_args(const ep_dropout_t *d, DropoutArgs *a)
{
    *a = DropoutArgs{};
    if (!d) return EP_OK;
    if (!(d->p >= 0.0 && d->p <= 1.0)) return EP_ERR_INVALID_ARG;             // NaN too
    if (!d->state) return EP_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(d->state) & 7u) return EP_ERR_INVALID_ARG;
    const long edge = (long)nearbyint(d->p * 65536.0);
    if (edge == 0) return EP_OK;
    a->state = reinterpret_cast<const unsigned long long *>(d->state);
    a->site = d->site;
    a->all = edge == 65536;
    a->edge = a->all ? 0u : (uint32_t)edge << 16;
    a->scale = a->all ? 0.f : (float)(65536.0 / (65536 - edge));
    return EP_OK;
}

#ifdef __CUDACC__

struct Dropout {
    uint32_t k0, k1, step, edge, site;
    float scale;
    bool all;

    __device__ __forceinline__ Dropout(const DropoutArgs &a) : k0(0), k1(0), step(0), edge(a.edge), site(a.site), scale(a.scale), all(a.all != 0)
    {
        if (a.state) {
            const unsigned long long seed = *a.state;
            k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32), step = (uint32_t)a.state[1];
        }
    }

    // The words of N vectors, round by round, so that they share a round's keys (and the first product of the step).
    template <int N>
    __device__ __forceinline__ void words(const unsigned long long (&v)[N], uint32_t (&w)[N][4]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) w[n][0] = (uint32_t)v[n], w[n][1] = (uint32_t)(v[n] >> 32), w[n][2] = step, w[n][3] = site;
#pragma unroll
        for (uint32_t i = 0; i < 10; ++i) {
            const uint32_t a = k0 + i * 0x9E3779B9u, b = k1 + i * 0xBB67AE85u;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const unsigned long long p = (unsigned long long)w[n][0] * 0xD2511F53u, q = (unsigned long long)w[n][2] * 0xCD9E8D57u;
                w[n][0] = (uint32_t)(q >> 32) ^ w[n][1] ^ a, w[n][1] = (uint32_t)q;
                w[n][2] = (uint32_t)(p >> 32) ^ w[n][3] ^ b, w[n][3] = (uint32_t)p;
            }
        }
    }

    // Two packed elements, 0 where the word's halves say so.
    __device__ __forceinline__ uint32_t masked(uint32_t pair, uint32_t word) const
    {
        return pair & (((word << 16) >= edge ? 0x0000ffffu : 0u) | (word >= edge ? 0xffff0000u : 0u));
    }

    // The eight elements of vector v of the row-major array: 0 where dropped (whatever they hold), scaled elsewhere.
    __device__ __forceinline__ void apply(float (&f)[8], unsigned long long v) const
    {
        const unsigned long long one[1] = {v};
        uint32_t w[1][4];
        words(one, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = (w[0][i] << 16) >= edge && !all ? f[2 * i] * scale : 0.f;
            f[2 * i + 1] = w[0][i] >= edge && !all ? f[2 * i + 1] * scale : 0.f;
        }
    }
};

#endif  // __CUDACC__

}  // namespace ep
