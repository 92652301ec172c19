// Rows sorted by expert and back with weights, as a training step needs them: ep_sort, ep_sort_backward, ep_combine_residual,
// ep_combine_backward; and ep_dropout. Two row kernels, each the other's gradient:
//
//   spread   dst[slot[t][k]] = w[t][k] * v[t]                       d[t][k] = <v[t], table[slot[t][k]]>
//            (ep_sort: v = x, no d; ep_combine_backward: v = drop(dy), table = out)
//   gather   y[t] = add[t] + drop(sum_k w[t][k] * table[slot[t][k]])       d[t][k] = <v[t], table[slot[t][k]]>
//            (ep_combine_residual: no d; ep_sort_backward: v = x, no drop)
//
// A group of G threads (32, 64, 128 or 512) owns a token, a thread 16-byte columns of it. Every row named is read once and the
// products for d are taken on the way. Sums are fp32 in ascending k; a d is the sum of a thread's columns, then of the group's
// threads in a fixed tree: the same bits every time. Slots and weights sit one per lane and travel by warp shuffle.
//
// Both are bound by memory: 8192 tokens of 7168 elements, 8 picks, 173 us (gather, with residual and dropout: 6.7 TB/s) and 306 us (spread
// with its products: 6.5 TB/s).
#include <cmath>

#include "ep_random.cuh"

namespace ep {
namespace {

constexpr int kBlock = 128, kWide = 512;   // threads of a CTA; kWide where a whole CTA of that many has a token
template <int G>
constexpr int kBlockOf = G > kBlock ? G : kBlock;
constexpr int kChunk = 8;   // rows in flight per column

// CTAs per SM that the compiler leaves registers for. Left to itself it takes 125 and more where there are products, to have several
// columns' loads under way in one thread; seven CTAs with 72 each and one column are faster (gather with products, 8192 tokens of
// 1024 elements, 4 picks: 22.3 us with 72, 23.7 with 80, 25.5 with 64, 34.5 with 125). More than 8 picks with products, 4096 tokens of 2048
// elements, gather and spread: 12 picks 47 and 72 us with four CTAs, 58 and 81 with three, 44 and 69 with five; 24 picks 121 and 147 with three, 153 and
// 147 with two, 143 and 135 with four. Without products, 12 picks: 37 and 37 with seven (gather) and twelve (spread), 41 and 37 with five and eight.
constexpr int resident(bool spread, int chunks, bool dots) { return !dots ? (spread ? 12 : 7) : chunks == 1 ? 7 : chunks == 2 ? 4 : 3; }

struct RowArgs {
    const uint4 *v;             // [T] rows
    const uint4 *add;           // gather: [T] rows, may be NULL
    const uint4 *table;         // rows by slot
    uint4 *out;                 // spread: rows by slot; gather: [T] rows
    long long rows;             // of the table, or the destination
    const int32_t *slot;
    const float *weights;       // NULL: unit weights, a row that several picks name counts once
    float *dots;
    int T, K, vec_per_row;
    int32_t *status;
    DropoutArgs drop;
};

// 16 bytes that nothing else will read; the destination may be the same memory, so not through the read-only path.
__device__ __forceinline__ uint4 ld_once(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
// Sums of eight values over a warp, nine shuffles: lane l returns the sum of value (l >> 2).
__device__ __forceinline__ float warp_sums8(float (&d)[8])
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float give = lane & 16 ? d[i] : d[i + 4], keep = lane & 16 ? d[i + 4] : d[i];
        d[i] = keep + __shfl_xor_sync(kFullMask, give, 16);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float give = lane & 8 ? d[i] : d[i + 2], keep = lane & 8 ? d[i + 2] : d[i];
        d[i] = keep + __shfl_xor_sync(kFullMask, give, 8);
    }
    const float give = lane & 4 ? d[0] : d[1], keep = lane & 4 ? d[1] : d[0];
    float s = keep + __shfl_xor_sync(kFullMask, give, 4);
    s += __shfl_xor_sync(kFullMask, s, 2);
    return s + __shfl_xor_sync(kFullMask, s, 1);
}

// A token's picks, one per lane.
struct Picks {
    int32_t slot;               // -1: nothing to read or write
    float w;
    int first;                  // the lowest pick that names the same row
    unsigned mask;              // the picks whose row is visited: those that are their row's first
};

// SHARED_ONCE: a row that several picks name is visited once, with the sum of their weights (in ascending k).
template <bool SHARED_ONCE>
__device__ __forceinline__ Picks load_picks(const RowArgs &a, int t)
{
    const int lane = threadIdx.x & 31;
    Picks p;
    p.slot = -1, p.w = 0.f;
    if (t < a.T && lane < a.K) {
        p.slot = __ldg(a.slot + (size_t)t * a.K + lane);
        p.w = a.weights ? __ldg(a.weights + (size_t)t * a.K + lane) : 1.f;
        if (p.slot >= a.rows) {
            if (a.status) atomicOr(a.status, EP_STATUS_CAPACITY);
            p.slot = -1;
        }
        if (p.slot < 0) p.slot = -1, p.w = 0.f;
    }
    const unsigned same = __match_any_sync(kFullMask, p.slot);
    p.first = __ffs(same) - 1;
    if (SHARED_ONCE && a.weights && __any_sync(kFullMask, p.slot >= 0 && p.first != lane)) {
        float sum = 0.f;
        for (int k = 0; k < a.K; ++k) {
            const float w = __shfl_sync(kFullMask, p.w, k);
            if ((same >> k) & 1u) sum += w;
        }
        p.w = sum;
    }
    const bool visit = p.slot >= 0 && (p.first == lane || !(SHARED_ONCE || !a.weights));
    p.mask = __ballot_sync(kFullMask, visit);
    return p;
}

// d[t][k] from the threads' partial sums: over the warp, then over the group's warps.
template <int G, int CHUNKS, bool SHARED_ONCE>
__device__ __forceinline__ void store_dots(const RowArgs &a, const Picks &p, float (&dot)[CHUNKS][kChunk], int t)
{
    __shared__ float part[kBlockOf<G> / 32][CHUNKS * kChunk];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const float s = warp_sums8(dot[c]);
        if ((lane & 3) == 0) part[warp][c * kChunk + (lane >> 2)] = s;
    }
    if (G > 32) __syncthreads(); else __syncwarp();
    const int g = threadIdx.x % G, w0 = warp - g / 32;
    if (t < a.T && g < a.K) {                                            // the group's first warp: its lanes hold the picks
        const int from = SHARED_ONCE ? p.first : g;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < G / 32; ++w) s += part[w0 + w][from];
        a.dots[(size_t)t * a.K + g] = p.slot < 0 ? 0.f : s;
    }
}

template <int G, int CHUNKS, bool DOTS>
__global__ void __launch_bounds__(kBlockOf<G>, G > kBlock ? 1 : resident(true, CHUNKS, DOTS))
spread_rows_kernel(const RowArgs a)
{
    const int g = threadIdx.x % G, t = blockIdx.x * (kBlockOf<G> / G) + threadIdx.x / G;
    pdl_trigger();                                                       // the next kernel's CTAs may take the places that get free
    pdl_wait();                                                          // nothing is read or written before this
    const Picks p = load_picks<true>(a, t);
    const Dropout drop(a.drop);
    const bool copy = !a.weights && !a.drop.state;
    float dot[CHUNKS][kChunk];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < kChunk; ++j) dot[c][j] = 0.f;

    if (p.mask) {
        const uint4 *const own = a.v + (size_t)t * a.vec_per_row;
        uint4 next = make_uint4(0u, 0u, 0u, 0u);                         // without d, a column ahead
        if (!DOTS && g < a.vec_per_row) next = ld_once(own + g);
#pragma unroll 1
        for (int base = 0; base < a.vec_per_row; base += G) {            // trip count uniform over the warp
            const int col = base + g;
            const bool live = col < a.vec_per_row;
            uint4 mine = next;
            if (DOTS && live) mine = ld_once(own + col);
            if (!DOTS && col + G < a.vec_per_row) next = ld_once(own + col + G);
            uint4 row[kChunk];
            const auto request = [&](int c) {
#pragma unroll
                for (int j = 0; j < kChunk; ++j) {
                    const int32_t s = __shfl_sync(kFullMask, p.slot, c * kChunk + j);
                    if (live && ((p.mask >> (c * kChunk + j)) & 1u)) row[j] = ld_once(a.table + (size_t)s * a.vec_per_row + col);
                }
            };
            if (DOTS) request(0);
            float f[8];
            unpack8(mine, f);
            if (a.drop.state) drop.apply(f, (size_t)t * a.vec_per_row + col);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if (DOTS && c > 0) request(c);
#pragma unroll
                for (int j = 0; j < kChunk; ++j) {
                    const int k = c * kChunk + j;
                    const int32_t s = __shfl_sync(kFullMask, p.slot, k);
                    const float w = __shfl_sync(kFullMask, p.w, k);
                    if (live && ((p.mask >> k) & 1u)) {
                        if (DOTS) {
                            float r[8];
                            unpack8(row[j], r);
#pragma unroll
                            for (int i = 0; i < 8; ++i) dot[c][j] = fmaf(f[i], r[i], dot[c][j]);
                        }
                        float o[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) o[i] = w * f[i];
                        if (a.out) st_stream(a.out + (size_t)s * a.vec_per_row + col, copy ? mine : pack8(o));
                    }
                }
            }
        }
    }
    if (DOTS) store_dots<G, CHUNKS, true>(a, p, dot, t);
}

template <int G, int CHUNKS, bool DOTS>
__global__ void __launch_bounds__(kBlockOf<G>, G > kBlock ? 1 : resident(false, CHUNKS, DOTS))
gather_rows_kernel(const RowArgs a)
{
    const int g = threadIdx.x % G, t = blockIdx.x * (kBlockOf<G> / G) + threadIdx.x / G;
    pdl_trigger();
    pdl_wait();
    const Picks p = load_picks<false>(a, t);
    const Dropout drop(a.drop);
    float dot[CHUNKS][kChunk];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < kChunk; ++j) dot[c][j] = 0.f;

    const auto request = [&](uint4 &to, int k, int col) {
        const int32_t s = __shfl_sync(kFullMask, p.slot, k);
        if (col < a.vec_per_row && ((p.mask >> k) & 1u)) to = ld_once(a.table + (size_t)s * a.vec_per_row + col);
    };
    const auto fold = [&](float (&acc)[8], const float (&f)[8], float &d, const uint4 &row, int k, bool live) {
        const float w = __shfl_sync(kFullMask, p.w, k);
        if (live && ((p.mask >> k) & 1u)) {
            float r[8];
            unpack8(row, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc[i] = fmaf(w, r[i], acc[i]);
                if (DOTS) d = fmaf(f[i], r[i], d);
            }
        }
    };
    const auto finish = [&](float (&acc)[8], const uint4 &add, size_t at) {
        if (a.drop.state) drop.apply(acc, at);
        if (a.add) {
            float r[8];
            unpack8(add, r);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += r[i];
        }
        st_stream(a.out + at, pack8(acc));
    };
    if (t < a.T) {
        const size_t first = (size_t)t * a.vec_per_row;
        const auto request_own = [&](uint4 &mine, uint4 &add, int col) {
            if (col < a.vec_per_row) {
                if (DOTS) mine = ld_once(a.v + first + col);
                if (a.add) add = ld_once(a.add + first + col);
            }
        };
        uint4 row[kChunk], mine = make_uint4(0u, 0u, 0u, 0u), add = mine;
        if (CHUNKS == 1 && !DOTS) {
            // the next column's rows are requested half by half as this column's are used, so that loads stay in flight during the
            // arithmetic (with products that takes too many registers: 4096 tokens of 2048 elements, 8 picks, 64 us instead of 50)
            request_own(mine, add, g);
#pragma unroll
            for (int k = 0; k < kChunk; ++k) request(row[k], k, g);
            for (int base = 0; base < a.vec_per_row; base += G) {
                const int col = base + g;
                const bool live = col < a.vec_per_row;
                float f[8], acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (DOTS) unpack8(mine, f);
                const uint4 extra = add;
                request_own(mine, add, col + G);
#pragma unroll
                for (int h = 0; h < kChunk; h += 4) {
#pragma unroll
                    for (int k = h; k < h + 4; ++k) fold(acc, f, dot[0][k], row[k], k, live);
#pragma unroll
                    for (int k = h; k < h + 4; ++k) request(row[k], k, col + G);
                }
                if (live && a.out) finish(acc, extra, first + col);
            }
        } else {
#pragma unroll 1
            for (int base = 0; base < a.vec_per_row; base += G) {            // (unrolled, it takes 125 registers, and twice the time)
                const int col = base + g;
                const bool live = col < a.vec_per_row;
                float f[8], acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                request_own(mine, add, col);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) request(row[j], c * kChunk + j, col);
                    if (DOTS && c == 0) unpack8(mine, f);
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) fold(acc, f, dot[c][j], row[j], c * kChunk + j, live);
                }
                if (live && a.out) finish(acc, add, first + col);
            }
        }
    }
    if (DOTS) store_dots<G, CHUNKS, false>(a, p, dot, t);
}

template <template <int, int, bool> class Kernel, int CHUNKS, bool DOTS>
int launch_group(const RowArgs &a, bool few_columns, cudaStream_t stream)
{
    const int vpr = a.vec_per_row;
    cudaError_t e;
    // Threads per token: a row's columns are dealt out to more threads as there are more of them. Gather with products has a thread do one
    // column after the other, and wants few (8192 x 1024 elements, 4 picks: 22.3 us with 128 threads, 29.3 with 64; the others 10 % and
    // more the other way round).
    // Few tokens: 512 threads for each, so that all of a row's columns are under way at once. With at most a token per SM that is faster
    // for all (140 tokens of 4096 elements, 8 picks: gradients 6.0 -> 3.2 and 6.3 -> 3.7 us); with more, CTAs that read the table hold too many
    // registers (560 x 2160, 7 picks: 8.0 -> 9.3), while those that only write gain on (7.5 -> 5.2; 1000 x 7168, 8 picks: 27.5 -> 22.6).
    if (vpr > kBlock && a.T <= (a.table ? 148 : 8 * 148))
        e = launch_pdl(Kernel<kWide, CHUNKS, DOTS>::get(), dim3(a.T), dim3(kWide), 0, stream, a);
    else if (vpr <= 64)
        e = launch_pdl(Kernel<32, CHUNKS, DOTS>::get(), dim3(ceil_div(a.T, kBlock / 32)), dim3(kBlock), 0, stream, a);
    else if (vpr < (few_columns ? 65 : 256))
        e = launch_pdl(Kernel<64, CHUNKS, DOTS>::get(), dim3(ceil_div(a.T, kBlock / 64)), dim3(kBlock), 0, stream, a);
    else
        e = launch_pdl(Kernel<128, CHUNKS, DOTS>::get(), dim3(a.T), dim3(kBlock), 0, stream, a);
    EP_CUDA_TRY(e);
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}
template <template <int, int, bool> class Kernel, bool DOTS>
int launch_chunks(const RowArgs &a, bool few_columns, cudaStream_t stream)
{
    // The kernel for 16 picks is there because the one for 32 is slower (12 picks of 4096 x 2048 with products: 90 us gather and 91 spread, 47 and 72).
    return a.K <= 8    ? launch_group<Kernel, 1, DOTS>(a, few_columns, stream)
           : a.K <= 16 ? launch_group<Kernel, 2, DOTS>(a, few_columns, stream)
                       : launch_group<Kernel, 4, DOTS>(a, few_columns, stream);
}
template <int G, int CHUNKS, bool DOTS>
struct Spread {
    static auto get() { return spread_rows_kernel<G, CHUNKS, DOTS>; }
};
template <int G, int CHUNKS, bool DOTS>
struct Gather {
    static auto get() { return gather_rows_kernel<G, CHUNKS, DOTS>; }
};
int launch_spread(const RowArgs &a, cudaStream_t stream)
{
    return a.dots ? launch_chunks<Spread, true>(a, false, stream) : launch_chunks<Spread, false>(a, false, stream);
}
int launch_gather(const RowArgs &a, cudaStream_t stream)
{
    return a.dots ? launch_chunks<Gather, true>(a, true, stream) : launch_chunks<Gather, false>(a, false, stream);
}

// ---- dropout of whole rows ----------------------------------------------------------------------------------------

// Bound by memory with a residual (65536 rows of 7168: 399 us, 7.1 TB/s), by the instructions of the generator without (322 us, 5.8 TB/s; a
// vector at a time, each with its own round keys, 350). Four vectors a thread need more registers than leave enough warps (367 us), and
// CTAs that stay and ask for the next vectors ahead were not faster (340 to 413).
constexpr int kDropThreads = 128, kDropVecs = 3;

__global__ void __launch_bounds__(kDropThreads)
dropout_kernel(const uint4 *x, const uint4 *residual, uint4 *y, const int32_t *limit, long long rows, int vec_per_row, const DropoutArgs args)
{
    pdl_trigger();
    pdl_wait();
    if (limit) rows = max(0ll, min(rows, (long long)__ldg(limit)));
    const long long total = rows * vec_per_row, first = (long long)blockIdx.x * (kDropThreads * kDropVecs) + threadIdx.x;
    if (first >= total) return;
    const Dropout drop(args);
    uint4 v[kDropVecs], r[kDropVecs];
    unsigned long long place[kDropVecs];
    uint32_t w[kDropVecs][4];
#pragma unroll
    for (int i = 0; i < kDropVecs; ++i) {
        const long long at = first + i * kDropThreads;
        place[i] = at;
        if (at < total) {
            v[i] = ld_once(x + at);
            if (residual) r[i] = ld_once(residual + at);
        }
    }
    if (args.state) drop.words(place, w);
    const float scale = args.state ? drop.scale : 1.f;
#pragma unroll
    for (int i = 0; i < kDropVecs; ++i) {
        const long long at = first + i * kDropThreads;
        if (at < total) {
            if (args.state) {
                v[i] = make_uint4(drop.masked(v[i].x, w[i][0]), drop.masked(v[i].y, w[i][1]), drop.masked(v[i].z, w[i][2]), drop.masked(v[i].w, w[i][3]));
                if (drop.all) v[i] = make_uint4(0u, 0u, 0u, 0u);
            }
            float f[8], g[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            unpack8(v[i], f);
            if (residual) unpack8(r[i], g);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = fmaf(f[j], scale, g[j]);
            st_stream(y + at, pack8(f));
        }
    }
}

// The checks and arguments that the four row calls share.
int row_args(const ep_shape_t *shape, const int32_t *slot, const float *weights, int64_t rows, int32_t *status, RowArgs *a)
{
    const int rc = check_shape(shape, true);
    if (rc != EP_OK) return rc;
    if (rows < 0) return EP_ERR_INVALID_ARG;
    if (shape->num_tokens > 0 && !slot) return EP_ERR_NULL;
    *a = RowArgs{};
    a->slot = slot, a->weights = weights, a->rows = rows, a->status = status;
    a->T = shape->num_tokens, a->K = shape->top_k, a->vec_per_row = shape->hidden / 8;
    return EP_OK;
}

}  // namespace
}  // namespace ep

extern "C" int ep_sort(const ep_shape_t *shape, const void *x, const int32_t *slot, const float *weights, void *sorted, int64_t sorted_rows,
                       int32_t *status, void *stream)
{
    using namespace ep;
    RowArgs a;
    const int rc = row_args(shape, slot, weights, sorted_rows, status, &a);
    if (rc != EP_OK || a.T == 0) return rc;
    if (!x || !sorted) return EP_ERR_NULL;
    if (!aligned16(x) || !aligned16(sorted)) return EP_ERR_INVALID_ARG;
    a.v = static_cast<const uint4 *>(x);
    a.out = static_cast<uint4 *>(sorted);
    return launch_spread(a, static_cast<cudaStream_t>(stream));
}

extern "C" int ep_sort_backward(const ep_shape_t *shape, const void *d_sorted, int64_t sorted_rows, const int32_t *slot, const float *weights,
                                const void *x, const void *add, void *dx, float *d_weights, int32_t *status, void *stream)
{
    using namespace ep;
    RowArgs a;
    const int rc = row_args(shape, slot, weights, sorted_rows, status, &a);
    if (rc != EP_OK) return rc;
    if (d_weights && !weights) return EP_ERR_INVALID_ARG;                // unit weights have no gradient
    if (a.T == 0) return EP_OK;
    if (!d_sorted || (d_weights && !x) || (!dx && !d_weights)) return EP_ERR_NULL;
    if (!aligned16(d_sorted) || !aligned16(x) || !aligned16(add) || !aligned16(dx)) return EP_ERR_INVALID_ARG;
    a.table = static_cast<const uint4 *>(d_sorted);
    a.v = static_cast<const uint4 *>(x);
    a.add = static_cast<const uint4 *>(dx ? add : nullptr);
    a.out = static_cast<uint4 *>(dx);
    a.dots = d_weights;
    return launch_gather(a, static_cast<cudaStream_t>(stream));
}

extern "C" int ep_combine_residual(const ep_shape_t *shape, const void *out, int64_t out_rows, const int32_t *slot, const float *topk_weights,
                                   const void *residual, const ep_dropout_t *dropout, void *y, int32_t *status, void *stream)
{
    using namespace ep;
    RowArgs a;
    int rc = row_args(shape, slot, topk_weights, out_rows, status, &a);
    if (rc == EP_OK) rc = dropout_args(dropout, &a.drop);
    if (rc != EP_OK || a.T == 0) return rc;
    if (!out || !topk_weights || !y) return EP_ERR_NULL;
    if (!aligned16(out) || !aligned16(residual) || !aligned16(y)) return EP_ERR_INVALID_ARG;
    a.table = static_cast<const uint4 *>(out);
    a.add = static_cast<const uint4 *>(residual);
    a.out = static_cast<uint4 *>(y);
    return launch_gather(a, static_cast<cudaStream_t>(stream));
}

extern "C" int ep_combine_backward(const ep_shape_t *shape, const void *dy, const void *out, int64_t out_rows, const int32_t *slot,
                                   const float *topk_weights, const ep_dropout_t *dropout, void *d_out, float *d_weights, int32_t *status,
                                   void *stream)
{
    using namespace ep;
    RowArgs a;
    int rc = row_args(shape, slot, topk_weights, out_rows, status, &a);
    if (rc == EP_OK) rc = dropout_args(dropout, &a.drop);
    if (rc != EP_OK || a.T == 0) return rc;
    if (!dy || !topk_weights || (d_weights && !out) || (!d_out && !d_weights)) return EP_ERR_NULL;
    if (!aligned16(dy) || !aligned16(out) || !aligned16(d_out)) return EP_ERR_INVALID_ARG;
    a.v = static_cast<const uint4 *>(dy);
    a.table = static_cast<const uint4 *>(out);
    a.out = static_cast<uint4 *>(d_out);
    a.dots = d_weights;
    return launch_spread(a, static_cast<cudaStream_t>(stream));
}

extern "C" int ep_dropout(const void *x, const void *residual, void *y, int64_t rows, int32_t cols, const int32_t *limit,
                          const ep_dropout_t *dropout, void *stream)
{
    using namespace ep;
    DropoutArgs d;
    const int rc = dropout_args(dropout, &d);
    if (rc != EP_OK) return rc;
    if (rows < 0 || rows >= (int64_t(1) << 31) || cols < 8 || cols % 8) return EP_ERR_INVALID_ARG;
    if (rows == 0) return EP_OK;
    if (!x || !y) return EP_ERR_NULL;
    if (!aligned16(x) || !aligned16(residual) || !aligned16(y)) return EP_ERR_INVALID_ARG;
    const int64_t vecs = rows * (cols / 8), blocks = (vecs + kDropThreads * kDropVecs - 1) / (kDropThreads * kDropVecs);
    if (blocks >= (int64_t(1) << 31)) return EP_ERR_INVALID_ARG;
    EP_CUDA_TRY(launch_pdl(dropout_kernel, dim3((unsigned)blocks), dim3(kDropThreads), 0, static_cast<cudaStream_t>(stream),
                           static_cast<const uint4 *>(x), static_cast<const uint4 *>(residual), static_cast<uint4 *>(y), limit, rows,
                           (int)(cols / 8), d));
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}
