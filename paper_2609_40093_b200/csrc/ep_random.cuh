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

    __device__ __forceinline__ uint4 words(unsigned long long v) const
    {
        uint32_t c0 = (uint32_t)v, c1 = (uint32_t)(v >> 32), c2 = step, c3 = site;
#pragma unroll
        for (uint32_t i = 0; i < 10; ++i) {
            const unsigned long long p = (unsigned long long)c0 * 0xD2511F53u, q = (unsigned long long)c2 * 0xCD9E8D57u;
            const uint32_t n0 = (uint32_t)(q >> 32) ^ c1 ^ (k0 + i * 0x9E3779B9u), n2 = (uint32_t)(p >> 32) ^ c3 ^ (k1 + i * 0xBB67AE85u);
            c0 = n0, c1 = (uint32_t)q, c2 = n2, c3 = (uint32_t)p;
        }
        return make_uint4(c0, c1, c2, c3);
    }

    // The eight elements of vector v of the row-major array: 0 where dropped (whatever they hold), scaled elsewhere.
    __device__ __forceinline__ void apply(float (&f)[8], unsigned long long v) const
    {
        const uint4 w = words(v);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = (u[i] << 16) >= edge && !all ? f[2 * i] * scale : 0.f;
            f[2 * i + 1] = u[i] >= edge && !all ? f[2 * i + 1] * scale : 0.f;
        }
    }
};

#endif  // __CUDACC__

}  // namespace ep
