// The router: expert scores, top-k picks and weights from logits, the balance loss over them, and the gradient of both.
//
//   score      softmax: s_e = exp(l_e - max) / sum          sigmoid: s_e = 1 / (1 + exp(-l_e))
//   order      by l_e, or by s_e + bias_e where a selection bias is given; equal values by ascending expert id
//   weight     w_k = scale * s_k, divided by the sum of the token's picked scores if they are renormalised
//   balance    f_e = E * count_e / sum(counts), P_e = mean over tokens of p_e, loss = coef * sum_e f_e P_e
//              (p = s for softmax, s / sum(s) for sigmoid); the counts are constants of the gradient
//
// One warp owns a token and holds its row in registers: NV values a lane, four neighbouring experts at a time, so that a
// row of 128 fp32 logits is one 16-byte load per lane. A token's row is read once and nothing of size E is written in the
// forward pass.
//
// Picks. The least of the maxima of 2, 4 or 8 groups of lanes (K up to 8, up to 8 values a lane), or the K-th largest of the 32 lanes'
// maxima, bounds the K-th largest value from below, so the values that reach it hold all the picks. They are few (some 20 for 8 of
// 256): one per lane in the order of the ids, they go through K rounds of a warp-wide maximum over order-preserving integer keys and a
// ballot of its holders, about 6 instructions a round. (Rounds over all NV values of a lane, for rows where more than 64 values reach
// the bound, take 45 at E = 256.)
//
// For the balance loss a warp adds up its tokens' probabilities by itself and a CTA, one per SM, its warps' sums, both in a
// fixed order; a CTA adds its sums to one of kRows rows of 64-bit whole numbers of 2^-shift, whose sum does not depend on the
// order: the same bits every time. The CTA that comes last adds the rows and leaves zeros. At 4096 x 128 this takes 4.5 us on top of
// the picks' 4.0; one row per CTA, read by the last one, 7.1 (an SM reads some 60 bytes a cycle); a second kernel, a cluster of
// eight CTAs, 5.4 and 3 us of the host's time for its launch; a single row of atomics 5.5.
#include "ep_common.cuh"

namespace ep {
namespace {

constexpr int kBalanceCtas = 148;          // at most: one per SM
constexpr int kRows = 8;                   // that the CTAs' sums are spread over
constexpr uint32_t kDead = 0x007fffffu;    // key of -inf: an expert that may not be picked

enum { kRoute = 0, kRouteBalance = 1, kBalance = 2 };

struct RouteArgs {
    const void *logits;
    const float *bias;
    int32_t *topk_idx;                    // written (route) or read (balance alone)
    float *topk_weights;
    unsigned long long *sums;             // [kRows][E] sums of probabilities in units of 2^-shift; zero between calls, as all of the workspace
    int32_t *sum_counts;                  // [kRows][E] picks; then: tokens, CTAs that are done
    int32_t *expert_counts, *tokens;      // the loss's outputs
    float *mean_probs, *loss;
    int32_t *status;
    int T, E, K, scoring, renormalize, vec, vec_bias, shift;
    float scale, coef;
};

__device__ __forceinline__ float value(const float *p, size_t i) { return __ldg(p + i); }
__device__ __forceinline__ float value(const __nv_bfloat16 *p, size_t i)
{
    return __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t *>(p) + i) << 16);
}
__device__ __forceinline__ void value4(const float *p, size_t i, float (&v)[4])
{
    const float4 t = __ldg(reinterpret_cast<const float4 *>(p + i));
    v[0] = t.x, v[1] = t.y, v[2] = t.z, v[3] = t.w;
}
__device__ __forceinline__ void value4(const __nv_bfloat16 *p, size_t i, float (&v)[4])
{
    const uint2 t = __ldg(reinterpret_cast<const uint2 *>(p + i));
    v[0] = bf16_lo(t.x), v[1] = bf16_hi(t.x), v[2] = bf16_lo(t.y), v[3] = bf16_hi(t.y);
}

// The expert of a lane's j-th value.
template <int NV>
__device__ __forceinline__ int expert_of(int j, int lane)
{
    return NV < 4 ? j * 32 + lane : (j >> 2) * 128 + lane * 4 + (j & 3);
}

// A row of logits, -inf past E.
template <int NV, class T>
__device__ __forceinline__ void load_row(const T *row, int E, int lane, int vec, float (&l)[NV])
{
    if (NV >= 4 && vec) {
#pragma unroll
        for (int j = 0; j < NV; j += 4) {
            const int e = expert_of<NV>(j, lane);
            float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (e < E) value4(row, e, v);
#pragma unroll
            for (int c = 0; c < 4; ++c) l[(j + c) % NV] = v[c];
        }
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = expert_of<NV>(j, lane);
            l[j] = e < E ? value(row, e) : -INFINITY;
        }
    }
}

// NaN and +inf, which may not be picked either, become -inf. Returns whether there were any (of this lane's).
template <int NV>
__device__ __forceinline__ bool clean_row(float (&l)[NV])
{
    bool bad = false;
#pragma unroll
    for (int j = 0; j < NV; ++j) bad |= !(l[j] < INFINITY);
    if (__any_sync(kFullMask, bad)) {                     // hardly ever
#pragma unroll
        for (int j = 0; j < NV; ++j) l[j] = l[j] < INFINITY ? l[j] : -INFINITY;
    }
    return bad;
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v = fmaxf(v, __shfl_xor_sync(kFullMask, v, d));
    return v;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(kFullMask, v, d);
    return v;
}

// Order-preserving integer of a float: kDead for -inf, larger for every other number; -0 counts as +0.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const int b = __float_as_int(v + 0.f);
    return (uint32_t)(b ^ ((b >> 31) | 0x80000000));
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

// A score of every expert of a row: two or four instructions a value where the functions to the last bit take forty (they took
// 65536 x 256 with the loss and the gradient from 144 us to 120). Off by less than 2^-20 of the largest score; a small score relative to itself
// by 2 + 1.16 |l - top| (sigmoid: |l|) units in the last place, 103 at 87. They feed sums, and choose who may be among the picks; a
// pick's own score, and what decides between picks, is exact_score. Against 64 bits the loss's probabilities and gradients of 4096 x
// 128 and 65536 x 256 logits err by 5 to 10 % more than with the functions to the last bit.
__device__ __forceinline__ float rough_score(bool soft, float l, float top)
{
    return soft ? __expf(l - top) : __fdividef(1.f, 1.f + __expf(-l));
}

// The score (softmax: before the division by the row's sum) of one expert. exp(-l) overflows below -88; there the sigmoid is exp(l)
// to the last bit.
__device__ __forceinline__ float exact_score(bool soft, float l, float top)
{
    const bool low = l < -80.f;
    const float e = expf(soft ? l - top : low ? l : -l);
    return soft || low ? e : 1.f / (1.f + e);
}

// Renormalised weights are ratios of the picked scores. Those of a softmax are ratios of exp(l), and so, below logits of -40 and to the last
// bit, are those of sigmoids: there they come from the logits' differences to the largest pick, because the scores themselves
// and the reciprocal of their sum leave fp32's normal range at -87 (for a softmax where a bias picks that far below the largest logit).
// At kNoScore and below every sigmoid is 0 in fp32, and so are the weights.
constexpr float kNoScore = -103.97f;

// The same for the probabilities of the balance loss, a sigmoid over the sum of its row: where that sum is below kSmallSum the scores
// are taken as 2^-64 exp(l - most), whose ratios are theirs, and beside which 1 - score is 1 as it is beside theirs.
constexpr float kSmallSum = 0x1p-57f;
template <int N>
__device__ __forceinline__ void scale_small_sigmoids(const float (&l)[N], float most, float (&s)[N])
{
    if (most > kNoScore) {
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = 0x1p-64f * __expf(l[j] - most);
    }
}

// K rounds of "the largest key, and of its holders the lowest id": lane k gets the k-th's id. `N` keys a lane, of ids that ascend
// with the position in the lane.
template <int N, class Id>
__device__ __forceinline__ int pick_rounds(uint32_t (&key)[N], Id id_of, int K, int lane)
{
    int id = -1;
    for (int k = 0; k < K; ++k) {
        uint32_t best = key[0];
        int at = 0;
#pragma unroll
        for (int j = 1; j < N; ++j)
            if (key[j] > best) best = key[j], at = j;
        const uint32_t m = __reduce_max_sync(kFullMask, best);
        if (m <= kDead) break;                                                // no expert left
        const int e = __reduce_min_sync(kFullMask, best == m ? id_of(at) : 0x7fffffff);
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (id_of(j) == e) key[j] = 0u;
        if (lane == k) id = e;
    }
    return id;
}

// The same for one key a lane, ids ascending with the lane: the lowest lane that holds the maximum holds the lowest id.
__device__ __forceinline__ void pick_listed(uint32_t key, int e, float q, int K, int lane, int &id, float &got)
{
    const int rounds = min(K, __popc(__ballot_sync(kFullMask, key > kDead)));
    int from = 0;
    for (int k = 0; k < rounds; ++k) {
        const uint32_t m = __reduce_max_sync(kFullMask, key);
        const int src = __ffs(__ballot_sync(kFullMask, key == m)) - 1;
        if (lane == src) key = 0u;
        if (lane == k) from = src;
    }
    got = __shfl_sync(kFullMask, q, from);
    e = __shfl_sync(kFullMask, e, from);
    id = lane < rounds ? e : -1;
}

// Lane k's pick out of a row: its id (-1: none left). `rough` holds a value per expert that is off by at most `slack` of 1 + itself from
// what orders them; exact(logit, id, q) gives that value's key and in q what the caller wants of the pick, which comes back in
// `got`. `list`: 2 kListed words of shared memory of this warp.
constexpr int kListed = 64;

template <int NV, class T, class Exact>
__device__ __forceinline__ int pick(const float (&l)[NV], const float (&rough)[NV], float slack, Exact exact, const T *row, int E, int K, int lane,
                                    uint32_t *list, float &got)
{
    int id = -1;
    if (NV == 1) {                                                            // a key per lane is what the list below would be
        float q;
        pick_listed(l[0] > -INFINITY ? exact(l[0], lane, q) : 0u, lane, q, K, lane, id, got);
        return id;
    }
    // the warp in at least K groups of lanes: the least of the groups' maxima is reached by K values
    float best = rough[0];
#pragma unroll
    for (int j = 1; j < NV; ++j) best = fmaxf(best, rough[j]);
    float bound;
    if (K <= 8 && NV <= 8) {
        best = fmaxf(best, __shfl_xor_sync(kFullMask, best, 1));
        best = fmaxf(best, __shfl_xor_sync(kFullMask, best, 2));              // 8 groups of 4
        if (K <= 4) best = fmaxf(best, __shfl_xor_sync(kFullMask, best, 4));  // 4 groups of 8
        if (K <= 2) best = fmaxf(best, __shfl_xor_sync(kFullMask, best, 8));  // 2 groups of 16
        bound = of_key(__reduce_min_sync(kFullMask, key_of(best)));
    } else {                                                                  // the K-th largest of the lanes' maxima: closer
        uint32_t top = key_of(best), m = 0u;
        for (int k = 0; k < K; ++k) {
            m = __reduce_max_sync(kFullMask, top);
            if (m <= kDead) break;
            if (lane == __ffs(__ballot_sync(kFullMask, top == m)) - 1) top = 0u;
        }
        bound = of_key(max(m, kDead));
    }
    bound -= slack * (1.f + fabsf(bound));
    bound = fmaxf(bound, -3.4028235e38f);                                     // where a group is empty: every value that may be picked
    // what reaches it, in the order of the ids
    int count = 0;
    constexpr int kStep = NV < 4 ? 1 : 4;                                     // a lane's neighbouring experts
#pragma unroll
    for (int j = 0; j < NV; j += kStep) {
        if (NV > 8) {
            float most = rough[j];
#pragma unroll
            for (int c = 1; c < kStep; ++c) most = fmaxf(most, rough[(j + c) % NV]);
            if (!__any_sync(kFullMask, most >= bound)) continue;
        }
        int at = count;
#pragma unroll
        for (int c = 0; c < kStep; ++c) {
            const unsigned who = __ballot_sync(kFullMask, rough[j + c] >= bound);
            at += __popc(who & lanemask_lt());
            count += __popc(who);
        }
#pragma unroll
        for (int c = 0; c < kStep; ++c)
            if (rough[j + c] >= bound) {
                if (at < kListed) list[at] = __float_as_uint(l[j + c]), list[kListed + at] = expert_of<NV>(j + c, lane);
                ++at;
            }
    }
    __syncwarp();
    if (count <= 32) {
        const bool in = lane < count;
        const int e = in ? (int)list[kListed + lane] : 0;
        float q = 0.f;
        pick_listed(in ? exact(__uint_as_float(list[lane]), e, q) : 0u, e, q, K, lane, id, got);
    } else {
        float q;
        if (count <= kListed) {
            const int e0 = (int)list[kListed + lane], e1 = lane + 32 < count ? (int)list[kListed + 32 + lane] : 0x7ffffffe;
            uint32_t two[2] = {exact(__uint_as_float(list[lane]), e0, q),
                               lane + 32 < count ? exact(__uint_as_float(list[lane + 32]), e1, q) : 0u};
            id = pick_rounds<2>(two, [&](int j) { return j ? e1 : e0; }, K, lane);
        } else if (NV <= 8) {
            uint32_t key[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) key[j] = l[j] > -INFINITY ? exact(l[j], expert_of<NV>(j, lane), q) : kDead;
            id = pick_rounds<NV>(key, [&](int j) { return expert_of<NV>(j, lane); }, K, lane);
        } else {                                                              // the row again, once per pick: what follows the pick before
            uint32_t last_key = 0xffffffffu;
            int last_e = -1;
            for (int k = 0; k < K; ++k) {
                uint32_t best = kDead;
                int at = 0x7fffffff;
#pragma unroll 1
                for (int e = lane; e < E; e += 32) {
                    const float x = value(row, e);
                    const uint32_t o = x < INFINITY && x > -INFINITY ? exact(x, e, q) : kDead;
                    const bool after = o < last_key || (o == last_key && e > last_e);
                    if (after && o > best) best = o, at = e;
                }
                const uint32_t m = __reduce_max_sync(kFullMask, best);
                if (m <= kDead) break;
                last_key = m;
                last_e = __reduce_min_sync(kFullMask, best == m ? at : 0x7fffffff);
                if (lane == k) id = last_e;
            }
        }
        if (id >= 0) exact(value(row, id), id, got);
    }
    __syncwarp();                                                             // the list is free again
    return id;
}

// The end of a kernel with a balance loss: `sums` holds the warps' sums of probabilities, [warp][value of a lane][lane], `counts` the
// CTA's picks and, at E, its tokens. All threads call it; `shared` (the start of the dynamic shared memory) is free.
template <int NV, int kWarps>
__device__ __forceinline__ void finish_balance(const RouteArgs &a, float *shared, const float *sums, int *counts)
{
    constexpr int kPadded = NV * 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __shared__ bool last;
    __syncthreads();
    for (int i = threadIdx.x; i < kPadded; i += blockDim.x) {
        const int e = expert_of<NV>(i >> 5, i & 31);
        if (e < a.E) {
            float v = 0.f;
#pragma unroll 8
            for (int w = 0; w < kWarps; ++w) v += sums[(size_t)w * kPadded + i];
            const size_t at = (size_t)(blockIdx.x % kRows) * a.E + e;
            if (v > 0.f) atomicAdd(a.sums + at, __float2ull_rn(ldexpf(v, a.shift)));
            if (counts[e]) atomicAdd(a.sum_counts + at, counts[e]);
        }
    }
    int32_t *total = a.sum_counts + (size_t)kRows * a.E;                  // tokens, CTAs
    if (threadIdx.x == 0 && counts[a.E]) atomicAdd(total, counts[a.E]);
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(total + 1, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int n = __ldcg(total);
    const float unit = n ? ldexpf(1.f, -a.shift) / (float)n : 0.f;
    float dot = 0.f;                                                      // sum of count * (mean probability)
    int picks = 0;
    for (int e = threadIdx.x; e < a.E; e += blockDim.x) {
        unsigned long long p[kRows];
        int k[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) p[r] = __ldcg(a.sums + (size_t)r * a.E + e), k[r] = __ldcg(a.sum_counts + (size_t)r * a.E + e);
#pragma unroll
        for (int r = 0; r < kRows; ++r) a.sums[(size_t)r * a.E + e] = 0ull, a.sum_counts[(size_t)r * a.E + e] = 0;
#pragma unroll
        for (int r = 1; r < kRows; ++r) p[0] += p[r], k[0] += k[r];
        const float mean = __ull2float_rn(p[0]) * unit;
        a.mean_probs[e] = mean;
        a.expert_counts[e] = k[0];
        dot += (float)k[0] * mean;
        picks += k[0];
    }
    dot = warp_sum(dot);
    picks = __reduce_add_sync(kFullMask, picks);
    __syncthreads();
    if (lane == 0) shared[warp] = dot, counts[warp] = picks;
    __syncthreads();
    if (warp == 0) {
        dot = warp_sum(lane < kWarps ? shared[lane] : 0.f);
        picks = __reduce_add_sync(kFullMask, lane < kWarps ? counts[lane] : 0);
        if (lane == 0) {
            *a.loss = picks ? a.coef * (float)a.E / (float)picks * dot : 0.f;
            *a.tokens = n;
            total[0] = total[1] = 0;
        }
    }
}

// Warps per CTA. With a balance loss one CTA fills an SM as far as the registers allow.
__host__ __device__ constexpr int route_warps(int nv, bool balance)
{
    return !balance ? (nv > 32 ? 4 : 8) : nv <= 8 ? 32 : nv <= 16 ? 24 : nv <= 32 ? 16 : 8;
}

template <class T, int NV, int MODE>
__global__ void __launch_bounds__(route_warps(NV, MODE != kRoute) * 32)
route_kernel(const RouteArgs a)
{
    extern __shared__ float shared[];
    constexpr bool kBal = MODE != kRoute;
    constexpr int kWarps = route_warps(NV, kBal), kPadded = NV * 32;
    constexpr bool kInRegisters = NV <= 16;                                   // where a warp keeps its sums of probabilities
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t *list = reinterpret_cast<uint32_t *>(shared) + warp * 2 * kListed;
    float *sums = shared + kWarps * 2 * kListed;                                       // [warp][value of a lane][lane]
    float *mine = sums + (size_t)warp * kPadded;
    int *counts = reinterpret_cast<int *>(sums + (size_t)kWarps * kPadded);   // [E + 1], and at least [kWarps]
    float psum[kInRegisters ? NV : 1];
    if (kBal) {
        if (kInRegisters) {
#pragma unroll
            for (int j = 0; j < NV; ++j) psum[j % (kInRegisters ? NV : 1)] = 0.f;
        } else {
            for (int i = lane; i < kPadded; i += 32) mine[i] = 0.f;
        }
        for (int i = threadIdx.x; i <= a.E; i += blockDim.x) counts[i] = 0;
        __syncthreads();
    }
    const bool soft = a.scoring == EP_SCORE_SOFTMAX;
    const bool all = kBal || a.bias || (soft && !a.renormalize);              // are scores needed beyond the picked ones?
    int tokens = 0;
    bool bad = false, bad_index = false;
    for (unsigned t = blockIdx.x * kWarps + warp; t < (unsigned)a.T; t += gridDim.x * kWarps) {   // T < 2^31: no wrap
        const T *row = static_cast<const T *>(a.logits) + (size_t)t * a.E;
        float l[NV];
        load_row<NV>(row, a.E, lane, a.vec, l);
        bad |= clean_row<NV>(l);
        float top = l[0];
#pragma unroll
        for (int j = 1; j < NV; ++j) top = fmaxf(top, l[j]);
        const bool live = __any_sync(kFullMask, top > -INFINITY);             // does the token have an expert at all?
        if (soft) top = warp_max(top);
        int id = -1;
        if (MODE == kBalance && lane < a.K) {
            id = __ldg(a.topk_idx + (size_t)t * a.K + lane);
            if (id < -1 || id >= a.E) bad_index = true, id = -1;
        }
        bool counted = live && (MODE != kBalance || __any_sync(kFullMask, id >= 0));

        // ---- scores
        float s[NV], sum = 1.f;
        if (all && live) {
#pragma unroll
            for (int j = 0; j < NV; ++j) s[j] = rough_score(soft, l[j], top);
            if (kBal || soft) {
                sum = 0.f;
#pragma unroll
                for (int j = 0; j < NV; ++j) sum += s[j];
                sum = warp_sum(sum);
                if (kBal && !soft && sum < kSmallSum) {                       // hardly ever
                    scale_small_sigmoids<NV>(l, warp_max(top), s);
                    sum = 0.f;
#pragma unroll
                    for (int j = 0; j < NV; ++j) sum += s[j];
                    sum = warp_sum(sum);
                }
            }
        }
        float rough[MODE != kBalance ? NV : 1];                               // what orders the picks, where there is a bias
        if (MODE != kBalance && a.bias && live) {
            float(&v)[NV] = reinterpret_cast<float(&)[NV]>(rough);
            load_row<NV>(a.bias, a.E, lane, a.vec_bias, v);                   // -inf past E
            const float inv = soft ? __fdividef(1.f, sum) : 1.f;
            float most = -INFINITY;
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = l[j] > -INFINITY ? s[j] * inv + v[j] : -INFINITY;
            bad |= clean_row<NV>(v);
#pragma unroll
            for (int j = 0; j < NV; ++j) most = fmaxf(most, v[j]);
            counted = __any_sync(kFullMask, most > -INFINITY);                // a bias of -inf masks too
        }
        if (kBal && counted) {
            const float inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;         // sigmoids of logits below -103.97 are 0
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (kInRegisters) psum[j % (kInRegisters ? NV : 1)] += s[j] * inv;
                else mine[j * 32 + lane] += s[j] * inv;
            }
            ++tokens;
        }
        if (MODE != kBalance) {
            float w = 0.f;                                                    // the pick's score
            if (live && a.bias) {
                id = pick<NV>(l, reinterpret_cast<float(&)[NV]>(rough), 0x1p-18f, [&](float x, int e, float &q) {
                    q = exact_score(soft, x, top);
                    const float o = (soft ? q / sum : q) + __ldg(a.bias + e);
                    return o < INFINITY ? key_of(o) : kDead;
                }, row, a.E, a.K, lane, list, w);
            } else if (live) {
                id = pick<NV>(l, l, 0.f, [](float x, int, float &q) { q = x; return key_of(x); }, row, a.E, a.K, lane, list, w);
                w = exact_score(soft, w, top);
            }
            if (id < 0) w = 0.f;
            if (a.renormalize) {
                float picked = warp_sum(w);
                if (picked < kSmallSum) {                                     // hardly ever
                    const float x = id >= 0 ? value(row, id) : -INFINITY, most = warp_max(x);
                    if (soft || most > kNoScore) {
                        w = id >= 0 ? expf(x - most) : 0.f;
                        picked = warp_sum(w);
                    }
                }
                w = picked > 0.f ? w / picked : 0.f;
            } else if (soft) {
                w /= sum;
            }
            if (lane < a.K) {
                a.topk_idx[(size_t)t * a.K + lane] = id;
                a.topk_weights[(size_t)t * a.K + lane] = w * a.scale;
            }
        }
        if (kBal && id >= 0) atomicAdd(counts + id, 1);                       // whole numbers: the order does not matter
    }
    if (a.status) {
        if (bad) atomicOr(a.status, EP_STATUS_BAD_LOGIT);
        if (bad_index) atomicOr(a.status, EP_STATUS_BAD_INDEX);
    }
    if (kBal) {
        if (kInRegisters) {
#pragma unroll
            for (int j = 0; j < NV; ++j) mine[j * 32 + lane] = psum[j % (kInRegisters ? NV : 1)];
        }
        if (lane == 0 && tokens) atomicAdd(counts + a.E, tokens);
        finish_balance<NV, kWarps>(a, shared, sums, counts);
    }
}

// ---- few experts -------------------------------------------------------------------------------------------------
// Up to 16 experts and many tokens: a thread per token, its row in registers, the picks by plain scans over them. A warp per token
// leaves most lanes idle there, but its chain is shorter: us with a warp -> a thread per token, forward / with the loss / gradient,
//   8 experts, top 2:    4096 tokens 2.8 -> 2.4 / 7.1 -> 7.7 / 3.8 -> 3.8     16384 6.0 -> 2.6 / 11.7 -> 7.8 / 8.1 -> 3.8
//   16, sigmoid + bias, top 8: 16384 8.1 -> 9.1 / 14.1 -> 20.8 / 8.1 -> 7.5   65536 25.9 -> 12.7 / 34.4 -> 23.5 / 23.4 -> 9.5
// hence from 2048 tokens per expert on.

constexpr int kFew = 16, kFewWarps = 8, kFewCtas = 4 * 148;

template <int NE, class T>
__device__ __forceinline__ void load_few(const T *row, int E, int vec, float (&l)[NE])
{
#pragma unroll
    for (int j = 0; j < NE; j += 4) {
        float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (vec) {
            if (j < E) value4(row, j, v);
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (j + c < E) v[c] = value(row, j + c);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) l[j + c] = v[c];
    }
}

// Cleans the row; the largest logit (-inf: no expert), the scores (softmax: before the division by their sum) and their sum.
template <int NE>
__device__ __forceinline__ float score_few(float (&l)[NE], bool soft, float (&s)[NE], float &sum, bool &bad)
{
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < NE; ++j) {
        if (!(l[j] < INFINITY)) bad = true, l[j] = -INFINITY;
        top = fmaxf(top, l[j]);
    }
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < NE; ++j) {
        s[j] = top == -INFINITY ? 0.f : rough_score(soft, l[j], top);
        sum += s[j];
    }
    if (!soft && sum < kSmallSum) {                                           // hardly ever
        scale_small_sigmoids<NE>(l, top, s);
        sum = 0.f;
#pragma unroll
        for (int j = 0; j < NE; ++j) sum += s[j];
    }
    return top;
}

template <class T, int NE, int MODE>
__global__ void __launch_bounds__(kFewWarps * 32)
route_few_kernel(const RouteArgs a)
{
    constexpr bool kBal = MODE != kRoute;
    __shared__ float shared[kFewWarps * 64], sums[kFewWarps * 32];
    __shared__ int counts[kFew + 1 > kFewWarps ? kFew + 1 : kFewWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool soft = a.scoring == EP_SCORE_SOFTMAX;
    float psum[NE];
    int cnt[NE], tokens = 0;
    if (kBal) {
#pragma unroll
        for (int j = 0; j < NE; ++j) psum[j] = 0.f, cnt[j] = 0;
        if (threadIdx.x <= a.E) counts[threadIdx.x] = 0;
        __syncthreads();
    }
    bool bad = false, bad_index = false;
    for (unsigned t = blockIdx.x * blockDim.x + threadIdx.x; t < (unsigned)a.T; t += gridDim.x * blockDim.x) {
        float l[NE], s[NE], sum;
        load_few<NE>(static_cast<const T *>(a.logits) + (size_t)t * a.E, a.E, a.vec, l);
        const float top = score_few<NE>(l, soft, s, sum, bad);
        bool counted = top > -INFINITY;
        if (MODE == kBalance) {
            bool any = false;
            for (int k = 0; k < a.K; ++k) {
                const int id = __ldg(a.topk_idx + (size_t)t * a.K + k);
                bad_index |= id < -1 || id >= a.E;
                any |= id >= 0 && id < a.E;
#pragma unroll
                for (int j = 0; j < NE; ++j) cnt[j] += id == j && j < a.E;
            }
            counted &= any;
        } else {
            uint32_t key[NE];
            if (a.bias) {
#pragma unroll
                for (int j = 0; j < NE; ++j) {
                    float v = -INFINITY;
                    if (l[j] > -INFINITY) {
                        v = exact_score(soft, l[j], top);
                        v = (soft ? v / sum : v) + __ldg(a.bias + j);
                        if (!(v < INFINITY)) bad = true, v = -INFINITY;
                    }
                    key[j] = key_of(v);
                }
            } else {
#pragma unroll
                for (int j = 0; j < NE; ++j) key[j] = key_of(l[j]);
            }
            float w[kFew], picked = 0.f;
            int32_t *ids = a.topk_idx + (size_t)t * a.K;
            float *weights = a.topk_weights + (size_t)t * a.K;
            const int rounds = min(a.K, kFew);
#pragma unroll 1
            for (int k = 0; k < rounds; ++k) {                                // rolled: sixteen copies outgrew the instruction cache
                uint32_t best = kDead;
                int at = -1;
                float x = 0.f;
#pragma unroll
                for (int j = 0; j < NE; ++j)
                    if (key[j] > best) best = key[j], at = j, x = l[j];       // the lowest id of equal keys
#pragma unroll
                for (int j = 0; j < NE; ++j)
                    if (at == j) {
                        key[j] = 0u;
                        if (kBal) ++cnt[j];
                    }
                if (k == 0) counted = at >= 0;                                // a bias may mask what the logits did not
                w[k] = at >= 0 ? exact_score(soft, x, top) : 0.f;
                picked += w[k];
                ids[k] = at;
            }
            if (a.renormalize && picked < kSmallSum) {                        // hardly ever
                const T *row = static_cast<const T *>(a.logits) + (size_t)t * a.E;
                float most = -INFINITY;
#pragma unroll 1
                for (int k = 0; k < rounds; ++k)
                    if (ids[k] >= 0) most = fmaxf(most, value(row, ids[k]));
                if (soft || most > kNoScore) {
                    picked = 0.f;
#pragma unroll 1
                    for (int k = 0; k < rounds; ++k) {
                        w[k] = ids[k] >= 0 ? expf(value(row, ids[k]) - most) : 0.f;
                        picked += w[k];
                    }
                }
            }
            const float by = a.renormalize ? picked : soft ? sum : 1.f;
#pragma unroll 1
            for (int k = 0; k < a.K; ++k) {
                if (k >= rounds) ids[k] = -1;
                weights[k] = k < rounds && by > 0.f ? w[k] / by * a.scale : 0.f;
            }
        }
        if (kBal && counted) {
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
            for (int j = 0; j < NE; ++j) psum[j] += s[j] * inv;
            ++tokens;
        }
    }
    if (a.status) {
        if (bad) atomicOr(a.status, EP_STATUS_BAD_LOGIT);
        if (bad_index) atomicOr(a.status, EP_STATUS_BAD_INDEX);
    }
    if (kBal) {
#pragma unroll
        for (int j = 0; j < NE; ++j) {
            const float p = warp_sum(psum[j]);
            const int c = __reduce_add_sync(kFullMask, cnt[j]);
            if (lane == 0) {
                sums[warp * 32 + j] = p;
                if (j < a.E && c) atomicAdd(counts + j, c);
            }
        }
        tokens = __reduce_add_sync(kFullMask, tokens);
        if (lane == 0 && tokens) atomicAdd(counts + a.E, tokens);
        finish_balance<1, kFewWarps>(a, shared, sums, counts);
    }
}

// ---- gradient ----------------------------------------------------------------------------------------------------

struct RouteGradArgs {
    const void *logits;
    const int32_t *topk_idx;
    const float *d_weights;               // NULL: the loss alone
    const int32_t *counts, *tokens;       // NULL: the weights alone
    const float *d_loss;
    void *dlogits;
    int T, E, K, scoring, renormalize, vec;
    float scale, coef;
};

// One warp per token; the row, its scores and the gradient of the probabilities (the same for every token) stay in registers.
// Bound by memory at large batches: a row is read and a row is written.
constexpr int route_grad_ctas(int nv) { return nv <= 8 ? 5 : nv <= 12 ? 4 : nv <= 16 ? 3 : 2; }   // per SM

template <class T, int NV>
__global__ void __launch_bounds__(NV <= 32 ? 256 : 128, route_grad_ctas(NV))
route_grad_kernel(const RouteGradArgs a)
{
    extern __shared__ float4 shared4[];
    constexpr int kWarps = NV <= 32 ? 8 : 4, kPadded = NV * 32 < 128 ? 128 : NV * 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float *at_pick = reinterpret_cast<float *>(shared4) + (size_t)warp * kPadded;   // the weights' part at the picks, 0 elsewhere
    __shared__ int total;
    const bool soft = a.scoring == EP_SCORE_SOFTMAX, balance = a.counts != nullptr;
    for (int i = lane; i < kPadded; i += 32) at_pick[i] = 0.f;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    float f[NV];                                                              // gradient of the probabilities
#pragma unroll
    for (int j = 0; j < NV; ++j) f[j] = 0.f;
    if (balance) {
        int n = 0;
        for (int e = threadIdx.x; e < a.E; e += blockDim.x) n += __ldg(a.counts + e);
        n = __reduce_add_sync(kFullMask, n);
        if (lane == 0) atomicAdd(&total, n);
        __syncthreads();
        const int tokens = __ldg(a.tokens);
        const float unit = total && tokens ? __ldg(a.d_loss) * a.coef / (float)tokens * ((float)a.E / (float)total) : 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = expert_of<NV>(j, lane);
            if (e < a.E) f[j] = unit * (float)__ldg(a.counts + e);
        }
    }
    // the next token's row, picks and gradients are requested before this one's are used
    constexpr bool kAhead = NV <= 8;
    float l_next[kAhead ? NV : 1], dw_next = 0.f;
    int id_next = -1;
    const auto fetch = [&](unsigned t, float (&l)[kAhead ? NV : 1], int &id, float &dw) {
        if (kAhead) load_row<NV>(static_cast<const T *>(a.logits) + (size_t)t * a.E, a.E, lane, a.vec, reinterpret_cast<float (&)[NV]>(l));
        id = lane < a.K ? __ldg(a.topk_idx + (size_t)t * a.K + lane) : -1;
        dw = lane < a.K && a.d_weights ? __ldg(a.d_weights + (size_t)t * a.K + lane) : 0.f;
    };
    const unsigned first = blockIdx.x * kWarps + warp, stride = gridDim.x * kWarps, T_ = a.T;
    if (first < T_) fetch(first, l_next, id_next, dw_next);
    for (unsigned t = first; t < T_; t += stride) {
        const T *row = static_cast<const T *>(a.logits) + (size_t)t * a.E;
        T *out = static_cast<T *>(a.dlogits) + (size_t)t * a.E;
        float l[NV];
        if (kAhead) {
#pragma unroll
            for (int j = 0; j < NV; ++j) l[j] = l_next[j % (kAhead ? NV : 1)];
        } else {
            load_row<NV>(row, a.E, lane, a.vec, l);
        }
        int id = id_next >= 0 && id_next < a.E ? id_next : -1;
        const float dw = id >= 0 ? a.scale * dw_next : 0.f;
        if (t + stride < T_) fetch(t + stride, l_next, id_next, dw_next);
        clean_row<NV>(l);
        float top = l[0];
#pragma unroll
        for (int j = 1; j < NV; ++j) top = fmaxf(top, l[j]);
        if (soft) top = warp_max(top);
        const bool counted = __any_sync(kFullMask, top > -INFINITY) && __any_sync(kFullMask, id >= 0);
        if (!soft && balance && !__any_sync(kFullMask, top >= -40.f)) {       // hardly ever: scale_small_sigmoids, in place
            const float most = warp_max(top), shift = most > kNoScore ? most + 44.361420f : 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) l[j] -= shift;
        }
        float s[NV], sum = 0.f, inv = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) s[j] = counted ? rough_score(soft, l[j], top) : 0.f;
        if (soft || balance) {
#pragma unroll
            for (int j = 0; j < NV; ++j) sum += s[j];
            sum = warp_sum(sum);
            inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;
        }
        // The weights' part: the gradient of a picked score times that score. Renormalised, with r = score / (sum of the picked), it
        // is r (dw - sum r dw), which sums to 0; nothing is divided by the sum and multiplied by a score again, which would be
        // inf * 0 where both are tiny, nor by a softmax's denominator, which cancels.
        float picked_dot = 0.f;
        if (a.d_weights) {
            float x = id >= 0 && counted ? value(row, id) : -INFINITY, base = top, part;
            if (!(x < INFINITY)) x = -INFINITY;
            bool as_exp = soft;
            if (a.renormalize && !__any_sync(kFullMask, x >= (soft ? top - 40.f : -40.f))) {      // hardly ever
                base = warp_max(x);
                as_exp = soft || base > kNoScore;
            }
            const float v = x > -INFINITY ? exact_score(as_exp, x, base) : 0.f;
            if (a.renormalize) {
                const float picked = warp_sum(v), dot = warp_sum(dw * v);
                part = picked > 0.f ? (dw - dot / picked) * __fdividef(v, picked) : 0.f;
            } else {
                part = soft ? dw * v * inv : dw * v;
                if (soft) picked_dot = warp_sum(part);
            }
            if (id >= 0) at_pick[id] = part;                                  // a token's picks are distinct
            __syncwarp();
        }
        float dot = 0.f;
        if (balance) {
#pragma unroll
            for (int j = 0; j < NV; ++j) dot += s[j] * f[j];
            dot = warp_sum(dot) * inv;
        }
        float d[NV];
#pragma unroll
        for (int j = 0; j < NV; j += NV < 4 ? 1 : 4) {
            float k[4] = {0.f, 0.f, 0.f, 0.f};
            if (a.d_weights) {
                if (NV < 4) {
                    k[0] = at_pick[expert_of<NV>(j, lane)];
                } else {
                    const float4 q = *reinterpret_cast<const float4 *>(at_pick + expert_of<NV>(j, lane));
                    k[0] = q.x, k[1] = q.y, k[2] = q.z, k[3] = q.w;
                }
            }
#pragma unroll
            for (int c = 0; c < (NV < 4 ? 1 : 4); ++c) {
                const int i = (j + c) % NV;
                const float p = s[i] * inv, g = balance ? f[i] - dot : 0.f;
                d[i] = soft ? p * (g - picked_dot) + k[c] : (p * g + k[c]) * (1.f - s[i]);
            }
        }
        if (a.d_weights) {
            __syncwarp();
            if (id >= 0) at_pick[id] = 0.f;
            __syncwarp();
        }
        if (NV >= 4 && a.vec) {
#pragma unroll
            for (int j = 0; j < NV; j += 4) {
                const int e = expert_of<NV>(j, lane);
                if (e < a.E) {
                    if (sizeof(T) == 4)
                        *reinterpret_cast<float4 *>(reinterpret_cast<float *>(out) + e) =
                            make_float4(d[j], d[(j + 1) % NV], d[(j + 2) % NV], d[(j + 3) % NV]);
                    else
                        *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(out) + e) =
                            make_uint2(pack_bf16x2(d[j], d[(j + 1) % NV]), pack_bf16x2(d[(j + 2) % NV], d[(j + 3) % NV]));
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int e = expert_of<NV>(j, lane);
                if (e < a.E) out[e] = (T)d[j];
            }
        }
    }
}

template <class T, int NE>
__global__ void __launch_bounds__(kFewWarps * 32)
route_few_grad_kernel(const RouteGradArgs a)
{
    const bool soft = a.scoring == EP_SCORE_SOFTMAX, balance = a.counts != nullptr;
    float f[NE];                                                              // gradient of the probabilities
#pragma unroll
    for (int j = 0; j < NE; ++j) f[j] = 0.f;
    if (balance) {
        int total = 0;
#pragma unroll
        for (int j = 0; j < NE; ++j)
            if (j < a.E) {
                const int c = __ldg(a.counts + j);
                total += c;
                f[j] = (float)c;
            }
        const int tokens = __ldg(a.tokens);
        const float unit = total && tokens ? __ldg(a.d_loss) * a.coef / (float)tokens * ((float)a.E / (float)total) : 0.f;
#pragma unroll
        for (int j = 0; j < NE; ++j) f[j] *= unit;
    }
    for (unsigned t = blockIdx.x * blockDim.x + threadIdx.x; t < (unsigned)a.T; t += gridDim.x * blockDim.x) {
        float l[NE], s[NE], sum;
        bool bad = false;
        load_few<NE>(static_cast<const T *>(a.logits) + (size_t)t * a.E, a.E, a.vec, l);
        const float top = score_few<NE>(l, soft, s, sum, bad);
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        float k_grad[NE] /* at the picks: dw, then the weights' part */, v[NE] /* their scores */, picked = 0.f, dot = 0.f, picked_dot = 0.f;
        bool any = false;
#pragma unroll
        for (int j = 0; j < NE; ++j) k_grad[j] = 0.f, v[j] = 0.f;
        unsigned chosen = 0u;
#pragma unroll 1
        for (int k = 0; k < a.K; ++k) {
            const int id = __ldg(a.topk_idx + (size_t)t * a.K + k);
            if (id < 0 || id >= a.E) continue;
            any = true;
            chosen |= 1u << id;
            if (!a.d_weights) continue;
            const float dw = a.scale * __ldg(a.d_weights + (size_t)t * a.K + k);
            float x = -INFINITY;
#pragma unroll
            for (int j = 0; j < NE; ++j)
                if (id == j) x = l[j];
            const float score = x > -INFINITY ? exact_score(soft, x, top) * (soft && !a.renormalize ? inv : 1.f) : 0.f;
#pragma unroll
            for (int j = 0; j < NE; ++j)
                if (id == j) k_grad[j] = dw, v[j] = score;                    // a token's picks are distinct
            picked += score;
            dot += dw * score;
        }
        const bool counted = top > -INFINITY && any;
        if (a.d_weights && a.renormalize) {                                   // as above
            float most = -INFINITY;
#pragma unroll
            for (int j = 0; j < NE; ++j)
                if ((chosen >> j) & 1u) most = fmaxf(most, l[j]);
            if (soft ? most < top - 40.f : most < -40.f && most > kNoScore) { // hardly ever: the scores above will do otherwise
                picked = dot = 0.f;
#pragma unroll
                for (int j = 0; j < NE; ++j) {
                    v[j] = ((chosen >> j) & 1u) && l[j] > -INFINITY ? expf(l[j] - most) : 0.f;
                    picked += v[j], dot += k_grad[j] * v[j];
                }
            }
            const float by = picked > 0.f ? 1.f / picked : 0.f, mean = picked > 0.f ? dot / picked : 0.f;
#pragma unroll
            for (int j = 0; j < NE; ++j) k_grad[j] = (k_grad[j] - mean) * (v[j] * by);
        } else if (a.d_weights) {
#pragma unroll
            for (int j = 0; j < NE; ++j) {
                k_grad[j] *= v[j];
                if (soft) picked_dot += k_grad[j];
            }
        }
        float p_dot = 0.f;
#pragma unroll
        for (int j = 0; j < NE; ++j) p_dot += s[j] * f[j];
        p_dot *= inv;
        T *out = static_cast<T *>(a.dlogits) + (size_t)t * a.E;
        float d[NE];
#pragma unroll
        for (int j = 0; j < NE; ++j) {
            const float p = s[j] * inv, g = balance ? f[j] - p_dot : 0.f;
            d[j] = !counted ? 0.f : soft ? p * (g - picked_dot) + k_grad[j] : (p * g + k_grad[j]) * (1.f - s[j]);
        }
#pragma unroll
        for (int j = 0; j < NE; j += 4) {
            if (a.vec) {
                if (j < a.E) {
                    if (sizeof(T) == 4)
                        *reinterpret_cast<float4 *>(reinterpret_cast<float *>(out) + j) = make_float4(d[j], d[j + 1], d[j + 2], d[j + 3]);
                    else
                        *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(out) + j) =
                            make_uint2(pack_bf16x2(d[j], d[j + 1]), pack_bf16x2(d[j + 2], d[j + 3]));
                }
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (j + c < a.E) out[j + c] = (T)d[j + c];
            }
        }
    }
}

// ---- host side ---------------------------------------------------------------------------------------------------

int check_router(const ep_router_t *r)
{
    if (!r) return EP_ERR_NULL;
    if (r->num_tokens < 0 || r->num_experts < 1 || r->num_experts > kMaxExperts || r->top_k < 1 || r->top_k > kMaxTopK ||
        (int64_t)r->num_tokens * r->top_k >= (int64_t(1) << 31) || (r->logits_dtype != EP_DTYPE_F32 && r->logits_dtype != EP_DTYPE_BF16) ||
        (r->scoring != EP_SCORE_SOFTMAX && r->scoring != EP_SCORE_SIGMOID))
        return EP_ERR_INVALID_ARG;
    return EP_OK;
}

int values_per_lane(int E)
{
    for (const int nv : {1, 2, 4, 8, 12, 16, 24, 32, 64})
        if (nv * 32 >= E) return nv;
    return 128;
}

bool thread_per_token(const ep_router_t &r) { return r.num_experts <= kFew && r.num_tokens >= 2048 * r.num_experts; }

int balance_ctas(const ep_router_t &r)
{
    const bool few = thread_per_token(r);
    const int want = ceil_div(r.num_tokens, few ? kFewWarps * 32 : route_warps(values_per_lane(r.num_experts), true));
    const int most = few ? kFewCtas : kBalanceCtas;
    return want < most ? (want < 1 ? 1 : want) : most;
}

bool rows_of_vectors(const ep_router_t &r, const void *p)   // may a lane load four neighbouring logits at once?
{
    return r.num_experts % 4 == 0 && (reinterpret_cast<uintptr_t>(p) % (r.logits_dtype == EP_DTYPE_F32 ? 16 : 8)) == 0;
}

template <class Kernel>
int allow_smem(Kernel kernel, size_t bytes)
{
    if (bytes > 48 * 1024) EP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    return EP_OK;
}

template <class T, int NV, int MODE>
int launch_route(const RouteArgs &a, int ctas, cudaStream_t stream)
{
    constexpr int kWarps = route_warps(NV, MODE != kRoute);
    if (MODE == kRoute) ctas = ceil_div(a.T, kWarps);
    const size_t smem = ((size_t)kWarps * 2 * kListed + (MODE == kRoute ? 0 : (size_t)kWarps * NV * 32 + a.E + 1 + kWarps)) * 4;
    const int rc = allow_smem(route_kernel<T, NV, MODE>, smem);
    if (rc != EP_OK) return rc;
    route_kernel<T, NV, MODE><<<ctas, kWarps * 32, smem, stream>>>(a);
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

template <class T, int NV>
int launch_route_grad(const RouteGradArgs &a, cudaStream_t stream)
{
    constexpr int kWarps = NV <= 32 ? 8 : 4, kPadded = NV * 32 < 128 ? 128 : NV * 32;
    const size_t smem = (size_t)kWarps * kPadded * 4;
    const int rc = allow_smem(route_grad_kernel<T, NV>, smem);
    if (rc != EP_OK) return rc;
    int ctas = ceil_div(a.T, kWarps);
    if (ctas > route_grad_ctas(NV) * 148) ctas = route_grad_ctas(NV) * 148;   // one wave
    route_grad_kernel<T, NV><<<ctas, kWarps * 32, smem, stream>>>(a);
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

// Calls f.run<T, values per lane>() or, with few experts, f.few<T, values per thread>() for the router's type and size.
template <class F>
int for_router(const ep_router_t &r, F f)
{
    const bool f32 = r.logits_dtype == EP_DTYPE_F32;
    if (thread_per_token(r) && r.num_experts <= 8) return f32 ? f.template few<float, 8>() : f.template few<__nv_bfloat16, 8>();
    if (thread_per_token(r)) return f32 ? f.template few<float, kFew>() : f.template few<__nv_bfloat16, kFew>();
    switch (values_per_lane(r.num_experts)) {
#define EP_CASE(nv) case nv: return f32 ? f.template run<float, nv>() : f.template run<__nv_bfloat16, nv>();
        EP_CASE(1) EP_CASE(2) EP_CASE(4) EP_CASE(8) EP_CASE(12) EP_CASE(16) EP_CASE(24) EP_CASE(32) EP_CASE(64)
    default: return f32 ? f.template run<float, 128>() : f.template run<__nv_bfloat16, 128>();
#undef EP_CASE
    }
}

template <class T, int NE, int MODE>
int launch_few(const RouteArgs &a, int ctas, cudaStream_t stream)
{
    if (MODE == kRoute) ctas = ceil_div(a.T, kFewWarps * 32);
    route_few_kernel<T, NE, MODE><<<ctas, kFewWarps * 32, 0, stream>>>(a);
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

template <class T, int NE>
int launch_few_grad(const RouteGradArgs &a, cudaStream_t stream)
{
    const int ctas = ceil_div(a.T, kFewWarps * 32);
    route_few_grad_kernel<T, NE><<<ctas < kFewCtas ? ctas : kFewCtas, kFewWarps * 32, 0, stream>>>(a);
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

template <int MODE>
struct RunRoute {
    const RouteArgs &a;
    int ctas;
    cudaStream_t stream;
    template <class T, int NV> int run() const { return launch_route<T, NV, MODE>(a, ctas, stream); }
    template <class T, int NE> int few() const { return launch_few<T, NE, MODE>(a, ctas, stream); }
};
struct RunRouteGrad {
    const RouteGradArgs &a;
    cudaStream_t stream;
    template <class T, int NV> int run() const { return launch_route_grad<T, NV>(a, stream); }
    template <class T, int NE> int few() const { return launch_few_grad<T, NE>(a, stream); }
};

int check_balance(const ep_balance_t *b)
{
    return b->expert_counts && b->tokens && b->mean_probs && b->loss ? EP_OK : EP_ERR_NULL;
}

int run_route(const ep_router_t &r, RouteArgs &a, const ep_balance_t *b, bool pick, void *workspace, size_t workspace_bytes,
              cudaStream_t stream)
{
    a.T = r.num_tokens, a.E = r.num_experts, a.K = r.top_k, a.scoring = r.scoring, a.renormalize = r.renormalize, a.scale = r.scale;
    a.vec = rows_of_vectors(r, a.logits);
    a.vec_bias = r.num_experts % 4 == 0 && aligned16(a.bias);
    if (!b) {
        if (r.num_tokens == 0) return EP_OK;
        return for_router(r, RunRoute<kRoute>{a, 0, stream});
    }
    if (!workspace) return EP_ERR_NULL;
    if (!aligned16(workspace)) return EP_ERR_INVALID_ARG;
    if (workspace_bytes < ep_route_workspace_bytes(&r)) return EP_ERR_CAPACITY;
    a.sums = static_cast<unsigned long long *>(workspace);
    a.sum_counts = reinterpret_cast<int32_t *>(a.sums + (size_t)kRows * a.E);
    a.shift = 62;                                                             // T probabilities of at most 1 and a little fit 63 bits
    for (int64_t t = a.T; t > 0; t >>= 1) --a.shift;
    a.expert_counts = b->expert_counts, a.tokens = b->tokens, a.mean_probs = b->mean_probs, a.loss = b->loss;
    a.coef = r.balance_coef;
    const int ctas = balance_ctas(r);
    return pick ? for_router(r, RunRoute<kRouteBalance>{a, ctas, stream}) : for_router(r, RunRoute<kBalance>{a, ctas, stream});
}

}  // namespace
}  // namespace ep

extern "C" size_t ep_route_workspace_bytes(const ep_router_t *r)
{
    using namespace ep;
    if (check_router(r) != EP_OK) return 0;
    return ((size_t)kRows * r->num_experts * 12 + 8 + 15) & ~size_t(15);
}

extern "C" int ep_route(const ep_router_t *r, const void *logits, const float *bias, int32_t *topk_idx, float *topk_weights,
                        const ep_balance_t *balance, int32_t *status, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace ep;
    int rc = check_router(r);
    if (rc != EP_OK) return rc;
    if (balance && (rc = check_balance(balance)) != EP_OK) return rc;
    if (r->num_tokens && (!logits || !topk_idx || !topk_weights)) return EP_ERR_NULL;
    RouteArgs a = {};
    a.logits = logits;
    a.bias = bias;
    a.topk_idx = topk_idx;
    a.topk_weights = topk_weights;
    a.status = status;
    return run_route(*r, a, balance, true, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int ep_balance_loss(const ep_router_t *r, const void *logits, const int32_t *topk_idx, const ep_balance_t *balance,
                               int32_t *status, void *workspace, size_t workspace_bytes, void *stream)
{
    using namespace ep;
    int rc = check_router(r);
    if (rc != EP_OK) return rc;
    if (!balance) return EP_ERR_NULL;
    if ((rc = check_balance(balance)) != EP_OK) return rc;
    if (r->num_tokens && (!logits || !topk_idx)) return EP_ERR_NULL;
    RouteArgs a = {};
    a.logits = logits;
    a.topk_idx = const_cast<int32_t *>(topk_idx);
    a.status = status;
    return run_route(*r, a, balance, false, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int ep_route_backward(const ep_router_t *r, const void *logits, const int32_t *topk_idx, const float *d_weights,
                                 const ep_balance_t *balance, const float *d_loss, void *dlogits, void *stream)
{
    using namespace ep;
    const int rc = check_router(r);
    if (rc != EP_OK) return rc;
    if (!d_weights && !balance) return EP_ERR_INVALID_ARG;                    // nothing to take the gradient of
    if (balance && (!balance->expert_counts || !balance->tokens || !d_loss)) return EP_ERR_NULL;
    if (r->num_tokens == 0) return EP_OK;
    if (!logits || !topk_idx || !dlogits) return EP_ERR_NULL;
    RouteGradArgs a = {};
    a.logits = logits;
    a.topk_idx = topk_idx;
    a.d_weights = d_weights;
    if (balance) a.counts = balance->expert_counts, a.tokens = balance->tokens, a.d_loss = d_loss;
    a.dlogits = dlogits;
    a.T = r->num_tokens, a.E = r->num_experts, a.K = r->top_k, a.scoring = r->scoring, a.renormalize = r->renormalize;
    a.scale = r->scale, a.coef = r->balance_coef;
    a.vec = rows_of_vectors(*r, logits) && rows_of_vectors(*r, dlogits);
    return for_router(*r, RunRouteGrad{a, static_cast<cudaStream_t>(stream)});
}
