// The router: expert scores, top-k picks and weights from logits, the balance loss over them, and the gradient of both.
//
//   score      softmax: s_e = exp(l_e - max) / sum          sigmoid: s_e = 1 / (1 + exp(-l_e))
//   order      by l_e, or by s_e + bias_e where a selection bias is given; equal values by ascending expert id
//   weight     w_k = scale * s_k, divided by the sum of the token's picked scores if they are renormalised
//   balance    f_e = E * count_e / sum(counts), P_e = mean over tokens of p_e, loss = coef * sum_e f_e P_e
//              (p = s for softmax, s / sum(s) for sigmoid); the counts are constants of the gradient
//
// One warp owns a token and holds its row in registers: NV values a lane, four neighbouring experts at a time, so that a
// row of 128 fp32 logits is one 16-byte load per lane. The picks are K rounds of a warp-wide maximum over order-preserving
// integer keys and a warp-wide minimum over the ids that hold it. A token's row is read once and nothing of size E is
// written in the forward pass. For the balance loss a warp adds its tokens' probabilities into a row of shared memory of
// its own (no atomics, a fixed order of additions), a CTA writes its sums once, and one small cluster adds the CTAs' rows
// in their order: the same bits every time.
#include "ep_common.cuh"

#include <cooperative_groups.h>

namespace ep {
namespace {

constexpr int kMaxRouteCtas = 296;
constexpr int kFinishCtas = 8, kFinishThreads = 256;

enum { kRoute = 0, kRouteBalance = 1, kBalance = 2 };

struct RouteArgs {
    const void *logits;
    const float *bias;
    int32_t *topk_idx;                    // written (route) or read (balance alone)
    float *topk_weights;
    float *partial;                       // [ctas][E] sums of probabilities
    int32_t *partial_counts;              // [ctas][E + 1] picks, tokens
    int32_t *status;
    int T, E, K, scoring, renormalize, vec;
    float scale;
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

// A row of logits; an expert that may not be picked (-inf, NaN, +inf, or past E) comes as -inf. Returns whether a NaN or +inf was seen.
template <int NV, class T>
__device__ __forceinline__ bool load_row(const T *row, int E, int lane, int vec, float (&l)[NV])
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
    bool bad = false;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const bool ok = l[j] < INFINITY;                 // false for NaN and +inf
        bad |= !ok;
        l[j] = ok ? l[j] : -INFINITY;
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

// Order-preserving integer of a float: -inf is the smallest that occurs and maps to 0; -0 counts as +0.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);
    return v == -INFINITY ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k); }

// exp(-l) overflows below -88; there the sigmoid is exp(l) to the last bit (0 for -inf)
__device__ __forceinline__ float sigmoid(float l) { return l < -80.f ? expf(l) : 1.f / (1.f + expf(-l)); }

template <class T, int NV, int MODE>
__global__ void __launch_bounds__(NV <= 32 ? 256 : 128)
route_kernel(const RouteArgs a)
{
    extern __shared__ float shared[];
    constexpr bool kBal = MODE != kRoute;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int padded = NV * 32;
    float *mine = shared + (size_t)warp * padded;                             // this warp's sums, in the order of its lanes' values
    int *counts = reinterpret_cast<int *>(shared + (size_t)warps * padded);   // [E + 1]
    if (kBal) {
        for (int i = lane; i < padded; i += 32) mine[i] = 0.f;
        for (int i = threadIdx.x; i <= a.E; i += blockDim.x) counts[i] = 0;
        __syncthreads();
    }
    int tokens = 0;
    bool bad = false, bad_index = false;
    for (int t = blockIdx.x * warps + warp; t < a.T; t += gridDim.x * warps) {
        const T *row = static_cast<const T *>(a.logits) + (size_t)t * a.E;
        float l[NV];
        bad |= load_row<NV>(row, a.E, lane, a.vec, l);
        float top = l[0];
#pragma unroll
        for (int j = 1; j < NV; ++j) top = fmaxf(top, l[j]);
        top = warp_max(top);
        const bool live = top > -INFINITY;                                    // does the token have an expert at all?
        int id = -1;
        if (MODE == kBalance && lane < a.K) {
            id = __ldg(a.topk_idx + (size_t)t * a.K + lane);
            if (id < -1 || id >= a.E) bad_index = true, id = -1;
        }
        const bool counted = live && (MODE != kBalance || __any_sync(kFullMask, id >= 0));

        // ---- probabilities
        const bool soft = a.scoring == EP_SCORE_SOFTMAX;
        const bool all = kBal || a.bias || (soft && !a.renormalize);          // are scores needed beyond the picked ones?
        float s[NV], sum = 1.f;
        if (all && live) {
            sum = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                s[j] = soft ? expf(l[j] - top) : sigmoid(l[j]);
                sum += s[j];
            }
            sum = warp_sum(sum);
            if (kBal && counted) {
                const float inv = sum > 0.f ? 1.f / sum : 0.f;                // sigmoids of very negative logits can all be 0
#pragma unroll
                for (int j = 0; j < NV; ++j) mine[j * 32 + lane] += s[j] * inv;
                if (lane == 0) ++tokens;
            }
        }
        if (MODE != kBalance) {
            // ---- picks: lane k ends up with the k-th
            uint32_t key[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int e = expert_of<NV>(j, lane);
                float v = l[j];
                if (a.bias && e < a.E && v > -INFINITY) {
                    v = (soft ? s[j] / sum : s[j]) + __ldg(a.bias + e);
                    if (!(v < INFINITY)) bad = true, v = -INFINITY;
                }
                key[j] = key_of(v);
            }
            uint32_t my_key = 0u;
            for (int k = 0; k < a.K; ++k) {
                uint32_t best = key[0];
                int at = 0;
#pragma unroll
                for (int j = 1; j < NV; ++j)
                    if (key[j] > best) best = key[j], at = j;                 // ids ascend with j
                const uint32_t m = __reduce_max_sync(kFullMask, best);
                if (m == 0u) break;                                           // no expert left
                const int e = __reduce_min_sync(kFullMask, best == m ? expert_of<NV>(at, lane) : 0x7fffffff);
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (expert_of<NV>(j, lane) == e) key[j] = 0u;
                if (lane == k) id = e, my_key = m;
            }
            // ---- weights of the picks
            float w = 0.f;
            if (id >= 0) {
                const float v = a.bias ? value(row, id) : of_key(my_key);
                w = soft ? expf(v - top) : sigmoid(v);
            }
            const float picked = warp_sum(w);
            if (a.renormalize) w = picked > 0.f ? w / picked : 0.f;
            else if (soft) w /= sum;
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
        if (lane == 0 && tokens) atomicAdd(counts + a.E, tokens);
        __syncthreads();
        for (int i = threadIdx.x; i < padded; i += blockDim.x) {
            const int e = expert_of<NV>(i >> 5, i & 31);
            if (e < a.E) {
                float v = 0.f;
                for (int w = 0; w < warps; ++w) v += shared[(size_t)w * padded + i];
                a.partial[(size_t)blockIdx.x * a.E + e] = v;
            }
        }
        for (int i = threadIdx.x; i <= a.E; i += blockDim.x) a.partial_counts[(size_t)blockIdx.x * (a.E + 1) + i] = counts[i];
    }
}

// Adds the CTAs' rows: counts, mean probabilities, loss. One cluster; each CTA owns a run of experts, eight warps split the rows.
__global__ void __launch_bounds__(kFinishThreads) __cluster_dims__(kFinishCtas, 1, 1)
balance_finish_kernel(const float *partial, const int32_t *partial_counts, int ctas, int E, float coef, int32_t *expert_counts,
                      int32_t *tokens_out, float *mean_probs, float *loss)
{
    namespace cg = cooperative_groups;
    constexpr int kWarps = kFinishThreads / 32;
    __shared__ float psum[kWarps][32];
    __shared__ int csum[kWarps][32];
    __shared__ float share_dot;
    __shared__ int share_count, share_tokens;
    cg::cluster_group cluster = cg::this_cluster();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = cluster.block_rank();
    pdl_wait();
    if (threadIdx.x == 0) share_tokens = 0;
    __syncthreads();
    int n = 0;
    for (int c = threadIdx.x; c < ctas; c += kFinishThreads) n += partial_counts[(size_t)c * (E + 1) + E];
    n = __reduce_add_sync(kFullMask, n);
    if (lane == 0 && n) atomicAdd(&share_tokens, n);
    __syncthreads();
    const int tokens = share_tokens;
    const float inv = tokens ? 1.f / (float)tokens : 0.f;
    float dot = 0.f;                                                          // warp 0: sum of count * (sum of probabilities)
    int count = 0;
    for (int base = rank * 32; base < E; base += kFinishCtas * 32) {
        const int e = base + lane;
        float p = 0.f;
        int k = 0;
        if (e < E) {
#pragma unroll 8
            for (int c = warp; c < ctas; c += kWarps) {
                p += partial[(size_t)c * E + e];
                k += partial_counts[(size_t)c * (E + 1) + e];
            }
        }
        psum[warp][lane] = p;
        csum[warp][lane] = k;
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (int w = 1; w < kWarps; ++w) p += psum[w][lane], k += csum[w][lane];
            if (e < E) {
                expert_counts[e] = k;
                mean_probs[e] = p * inv;
                dot += (float)k * (p * inv);
                count += k;
            }
        }
        __syncthreads();
    }
    if (warp == 0) {
        dot = warp_sum(dot);
        count = __reduce_add_sync(kFullMask, count);
        if (lane == 0) share_dot = dot, share_count = count;
    }
    cluster.sync();
    if (rank == 0 && threadIdx.x == 0) {
        float d = 0.f;
        int c = 0;
        for (int r = 0; r < kFinishCtas; ++r) d += *cluster.map_shared_rank(&share_dot, r), c += *cluster.map_shared_rank(&share_count, r);
        *loss = c ? coef * (float)E / (float)c * d : 0.f;
        *tokens_out = tokens;
    }
    cluster.sync();                                                           // the other CTAs' words stay until they are read
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

template <class T, int NV>
__global__ void __launch_bounds__(NV <= 32 ? 256 : 128)
route_grad_kernel(const RouteGradArgs a)
{
    extern __shared__ float shared[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int padded = NV * 32;
    float *at_pick = shared + (size_t)warp * padded;                          // gradient of the picked scores, 0 elsewhere
    float *f = shared + (size_t)warps * padded;                               // gradient of the probabilities, in the order of the lanes' values
    __shared__ int total;
    const bool soft = a.scoring == EP_SCORE_SOFTMAX, balance = a.counts != nullptr;
    for (int i = lane; i < padded; i += 32) at_pick[i] = 0.f;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    if (balance) {
        int n = 0;
        for (int e = threadIdx.x; e < a.E; e += blockDim.x) n += __ldg(a.counts + e);
        n = __reduce_add_sync(kFullMask, n);
        if (lane == 0) atomicAdd(&total, n);
        __syncthreads();
        const int tokens = __ldg(a.tokens);
        const float unit = total && tokens ? __ldg(a.d_loss) * a.coef / (float)tokens * ((float)a.E / (float)total) : 0.f;
        for (int i = threadIdx.x; i < padded; i += blockDim.x) {
            const int e = expert_of<NV>(i >> 5, i & 31);
            f[i] = e < a.E ? unit * (float)__ldg(a.counts + e) : 0.f;
        }
        __syncthreads();
    }
    for (int t = blockIdx.x * warps + warp; t < a.T; t += gridDim.x * warps) {
        const T *row = static_cast<const T *>(a.logits) + (size_t)t * a.E;
        T *out = static_cast<T *>(a.dlogits) + (size_t)t * a.E;
        float l[NV];
        load_row<NV>(row, a.E, lane, a.vec, l);
        int id = -1;
        float dw = 0.f;
        if (lane < a.K) {
            id = __ldg(a.topk_idx + (size_t)t * a.K + lane);
            if (id < 0 || id >= a.E) id = -1;
            if (id >= 0 && a.d_weights) dw = a.scale * __ldg(a.d_weights + (size_t)t * a.K + lane);
        }
        float top = l[0];
#pragma unroll
        for (int j = 1; j < NV; ++j) top = fmaxf(top, l[j]);
        top = warp_max(top);
        const bool counted = top > -INFINITY && __any_sync(kFullMask, id >= 0);
        float s[NV], sum = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            s[j] = !counted ? 0.f : soft ? expf(l[j] - top) : sigmoid(l[j]);
            sum += s[j];
        }
        sum = warp_sum(sum);
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        // gradient with respect to the picked scores
        float mine = 0.f, picked_dot = 0.f;
        if (a.d_weights) {
            float v = 0.f;
            if (id >= 0 && counted) {
                v = value(row, id);
                v = !(v < INFINITY) || v == -INFINITY ? 0.f : soft ? expf(v - top) * inv : sigmoid(v);
            }
            if (a.renormalize) {
                const float picked = warp_sum(v), dot = warp_sum(dw * v);
                mine = picked > 0.f ? (dw - dot / picked) / picked : 0.f;
            } else {
                mine = dw;
            }
            picked_dot = warp_sum(mine * v);
            if (id >= 0) at_pick[id] = mine;                                  // a token's picks are distinct
            __syncwarp();
        }
        float dot = 0.f;
        if (balance) {
#pragma unroll
            for (int j = 0; j < NV; ++j) dot += s[j] * f[j * 32 + lane];
            dot = warp_sum(dot) * inv;
        }
        float d[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = expert_of<NV>(j, lane);
            const float p = s[j] * inv, g = balance ? f[j * 32 + lane] - dot : 0.f, k = a.d_weights ? at_pick[e] : 0.f;
            d[j] = soft ? p * (g + (k - picked_dot)) : (p * g + s[j] * k) * (1.f - s[j]);
        }
        __syncwarp();
        if (a.d_weights && id >= 0) at_pick[id] = 0.f;
        __syncwarp();
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

int route_warps(int E) { return E <= 1024 ? 8 : 4; }

int route_ctas(const ep_router_t &r)
{
    const int want = ceil_div(r.num_tokens, route_warps(r.num_experts));
    return want < kMaxRouteCtas ? (want < 1 ? 1 : want) : kMaxRouteCtas;
}

int values_per_lane(int E)
{
    int nv = 1;
    while (nv * 32 < E) nv *= 2;
    return nv;
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
    const int warps = route_warps(a.E);
    const size_t smem = MODE == kRoute ? 0 : ((size_t)warps * NV * 32 + a.E + 1) * 4;
    const int rc = allow_smem(route_kernel<T, NV, MODE>, smem);
    if (rc != EP_OK) return rc;
    route_kernel<T, NV, MODE><<<ctas, warps * 32, smem, stream>>>(a);
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

template <class T, int NV>
int launch_route_grad(const RouteGradArgs &a, cudaStream_t stream)
{
    const int warps = route_warps(a.E);
    const size_t smem = ((size_t)warps + 1) * NV * 32 * 4;
    const int rc = allow_smem(route_grad_kernel<T, NV>, smem);
    if (rc != EP_OK) return rc;
    int ctas = ceil_div(a.T, warps);
    if (ctas > 4 * 148) ctas = 4 * 148;
    route_grad_kernel<T, NV><<<ctas, warps * 32, smem, stream>>>(a);
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

// Calls f.template operator()<T, NV>() for the router's type and size.
template <class F>
int for_router(const ep_router_t &r, F f)
{
    const bool f32 = r.logits_dtype == EP_DTYPE_F32;
    switch (values_per_lane(r.num_experts)) {
#define EP_CASE(nv) case nv: return f32 ? f.template run<float, nv>() : f.template run<__nv_bfloat16, nv>();
        EP_CASE(1) EP_CASE(2) EP_CASE(4) EP_CASE(8) EP_CASE(16) EP_CASE(32) EP_CASE(64)
    default: return f32 ? f.template run<float, 128>() : f.template run<__nv_bfloat16, 128>();
#undef EP_CASE
    }
}

template <int MODE>
struct RunRoute {
    const RouteArgs &a;
    int ctas;
    cudaStream_t stream;
    template <class T, int NV> int run() const { return launch_route<T, NV, MODE>(a, ctas, stream); }
};
struct RunRouteGrad {
    const RouteGradArgs &a;
    cudaStream_t stream;
    template <class T, int NV> int run() const { return launch_route_grad<T, NV>(a, stream); }
};

int check_balance(const ep_balance_t *b)
{
    return b->expert_counts && b->tokens && b->mean_probs && b->loss ? EP_OK : EP_ERR_NULL;
}

// The route kernel in the given mode, then (with a balance) the cluster that adds up.
int run_route(const ep_router_t &r, RouteArgs &a, const ep_balance_t *b, bool pick, void *workspace, size_t workspace_bytes,
              cudaStream_t stream)
{
    a.T = r.num_tokens, a.E = r.num_experts, a.K = r.top_k, a.scoring = r.scoring, a.renormalize = r.renormalize, a.scale = r.scale;
    a.vec = rows_of_vectors(r, a.logits);
    int ctas = route_ctas(r);
    if (!b) {
        if (r.num_tokens == 0) return EP_OK;
        return for_router(r, RunRoute<kRoute>{a, ceil_div(a.T, route_warps(a.E)), stream});
    }
    if (!workspace) return EP_ERR_NULL;
    if (!aligned16(workspace)) return EP_ERR_INVALID_ARG;
    if (workspace_bytes < ep_route_workspace_bytes(&r)) return EP_ERR_CAPACITY;
    a.partial = static_cast<float *>(workspace);
    a.partial_counts = reinterpret_cast<int32_t *>(a.partial + (size_t)ctas * a.E);
    const int rc = pick ? for_router(r, RunRoute<kRouteBalance>{a, ctas, stream}) : for_router(r, RunRoute<kBalance>{a, ctas, stream});
    if (rc != EP_OK) return rc;
    EP_CUDA_TRY(launch_pdl(balance_finish_kernel, dim3(kFinishCtas), dim3(kFinishThreads), 0, stream, (const float *)a.partial,
                           (const int32_t *)a.partial_counts, ctas, a.E, r.balance_coef, b->expert_counts, b->tokens, b->mean_probs,
                           b->loss));
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

}  // namespace
}  // namespace ep

extern "C" size_t ep_route_workspace_bytes(const ep_router_t *r)
{
    using namespace ep;
    if (check_router(r) != EP_OK) return 0;
    return ((size_t)route_ctas(*r) * (2 * (size_t)r->num_experts + 1) * 4 + 15) & ~size_t(15);
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
