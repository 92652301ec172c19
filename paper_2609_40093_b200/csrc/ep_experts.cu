// The experts' matrix products over the pair space, and their gradients.
//
//   forward   y[p] = act(x[p] W[e]^T + b[e]) (+ or *) operand[p]         rows p of expert e's segment
//   dx        dx[p] = dz[p] W[e]
//   dweight   dW[e] = sum_p dz[p]^T x[p]
//
// All three are one kernel. The accumulator's 128 lanes hold the axis that is contiguous in the result (features), its
// columns hold the other one (rows p, or the weight's out features), so a warp stores 32 neighbouring elements of a result
// row per column, and the ragged axis of a segment, the rows, is cut in steps of 16 columns: an expert that got one row
// costs a 16-column product, not one of 128 rows.
//
//   mode      lanes (M)       columns (N)     contracted (K)   lane operand             column operand
//   forward   out features    rows            in features      W, K-major               x, K-major
//   dx        in features     rows            out features     W, MN-major              dz, K-major
//   dweight   in features     out features    rows             x, MN-major              dz, MN-major
//
// One persistent CTA per SM. A warp keeps a ring of shared-memory stages full by TMA (64 of the contracted axis each), one
// thread issues the products, four warps empty the accumulators, of which there are two of 256 columns, so that a tile's
// epilogue runs under the next tile's products. Rows behind a segment's end that a box brings along only feed columns that
// are not stored; in the dweight mode, where the rows are contracted, the operands are read through tensor maps that end
// with the segment (one pair per expert, made on the device from the offsets), so that the rest of the last box is zero
// whatever the neighbouring rows hold.
#include "ep_tensor.cuh"

namespace ep {
namespace {

enum { kForward = 0, kDx = 1, kDweight = 2 };

constexpr int kThreads = 256;
constexpr int kTileM = 128;               // lanes of one CTA
constexpr int kTileK = 64;                // contracted elements per stage: one 128-byte line
constexpr int kAccColumns = 256;          // columns of one of the two accumulators
constexpr int kBytesA = kTileM * kTileK * 2;
constexpr int kMaxStages = 12;
constexpr int kSmemLimit = 227 * 1024;

struct ProductArgs {
    const int32_t *offsets;               // [E+1]
    int32_t *status;
    long long rows;
    int M, N, K;                          // extents of the three axes; the one that is `rows` long is 0
    int E;
    int columns;                          // columns per tile at most
    int stages;
    uint16_t *out;
    const CUtensorMap *segment_maps;      // dweight: [E][2]
    // forward epilogue
    const uint16_t *bias, *operand;
    uint16_t *pre;
    int activation, operand_op;
};

struct Tile {
    int e, m0;
    int c0, cols;                         // first column (row p, or out feature) and how many are real
    int n;                                // columns of the product: cols rounded up to what the tensor cores take
    int k0, nk;                           // first contracted index and stages
};

__device__ __forceinline__ int segment_bound(int32_t v, long long rows)
{
    return v < 0 ? 0 : (v > rows ? (int)rows : v);
}

__device__ __forceinline__ float act_value(int act, float z)
{
    switch (act) {
    case EP_ACT_RELU: return z <= 0.f ? 0.f : z;
    case EP_ACT_SILU: return __fdividef(z, 1.f + __expf(-z));
    case EP_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678f));
    default: return z;
    }
}

__device__ __forceinline__ float act_slope(int act, float z)
{
    switch (act) {
    case EP_ACT_RELU: return z <= 0.f ? 0.f : 1.f;
    case EP_ACT_SILU: {
        const float s = __fdividef(1.f, 1.f + __expf(-z));
        return s * (1.f + z * (1.f - s));
    }
    case EP_ACT_GELU: return 0.5f * (1.f + erff(z * 0.70710678f)) + z * __expf(-0.5f * z * z) * 0.39894228f;
    default: return 1.f;
    }
}

__device__ __forceinline__ float bf16_value(uint16_t u) { return __uint_as_float((uint32_t)u << 16); }
__device__ __forceinline__ uint16_t bf16_bits(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

// ---- the walk over tiles -----------------------------------------------------------------------------------------

template <int MODE, int CG>
struct Walk {
    const ProductArgs &a;
    const int *first_tile;   // [E+1] shared memory: tiles of the experts before e (forward, dx)
    const int *bound;        // [E+1] shared memory: the segments' bounds, clamped
    int m_tiles, n_tiles, total;

    __device__ Walk(const ProductArgs &args, const int *first, const int *b) : a(args), first_tile(first), bound(b)
    {
        m_tiles = (a.M + kTileM * CG - 1) / (kTileM * CG);
        n_tiles = MODE == kDweight ? (a.N + a.columns - 1) / a.columns : 0;
        total = MODE == kDweight ? a.E * m_tiles * n_tiles : first_tile[a.E];
    }

    __device__ bool get(int tile, Tile &t) const
    {
        if (tile >= total) return false;
        constexpr int kStep = 16 * CG;
        if (MODE == kDweight) {
            const int per = m_tiles * n_tiles;
            t.e = tile / per;
            const int r = tile - t.e * per;
            t.m0 = (r / n_tiles) * kTileM * CG;
            t.c0 = (r % n_tiles) * a.columns;
            t.cols = min(a.columns, a.N - t.c0);
            t.k0 = bound[t.e];
            t.nk = (max(0, bound[t.e + 1] - t.k0) + kTileK - 1) / kTileK;
        } else {
            int lo = 0, hi = a.E;                        // the expert e with first_tile[e] <= tile < first_tile[e+1]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first_tile[mid] <= tile) lo = mid; else hi = mid;
            }
            t.e = lo;
            const int r = tile - first_tile[lo], begin = bound[lo], count = bound[lo + 1] - begin;
            const int pieces = (count + a.columns - 1) / a.columns;
            const int width = ((count + pieces - 1) / pieces + kStep - 1) / kStep * kStep;   // equal pieces
            const int piece = r % pieces;
            t.m0 = (r / pieces) * kTileM * CG;
            t.c0 = begin + piece * width;
            t.cols = max(0, min(width, count - piece * width));
            t.k0 = 0;
            t.nk = (a.K + kTileK - 1) / kTileK;
        }
        t.n = max(kStep, (t.cols + kStep - 1) / kStep * kStep);
        return true;
    }
};

// ---- epilogues ---------------------------------------------------------------------------------------------------

// One block of up to 32 columns of the forward product: rows p, p+1, ... of feature n.
template <int ACT>
__device__ __forceinline__ void store_forward(const ProductArgs &a, const uint32_t (&acc)[32], const uint16_t (&r)[32], float b, size_t at,
                                              int cols)
{
#pragma unroll
    for (int c = 0; c < 32; ++c) {
        if (c < cols) {
            const float z = __uint_as_float(acc[c]) + b;
            float v = act_value(ACT, z);
            if (a.operand) v = a.operand_op == EP_OPERAND_MUL ? v * bf16_value(r[c]) : v + bf16_value(r[c]);
            if (a.pre) a.pre[at + (size_t)c * a.M] = bf16_bits(z);
            a.out[at + (size_t)c * a.M] = bf16_bits(v);
        }
    }
}

// ---- the kernel --------------------------------------------------------------------------------------------------

template <int MODE, int CG>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const ProductArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b)
{
    extern __shared__ char raw[];
    __shared__ uint64_t full_[kMaxStages], empty_[kMaxStages], acc_full_[2], acc_empty_[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_;
    __shared__ int warp_sum[kThreads / 32];
    volatile int *gave_up = &gave_up_;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int b_bytes = max(32, a.columns / CG) * kTileK * 2;
    const int stage_bytes = kBytesA + b_bytes;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
    char *tables = raw + (ring - smem_addr(raw)) + (size_t)a.stages * stage_bytes;
    int *first_tile = reinterpret_cast<int *>(tables), *bound = first_tile + a.E + 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            bar_init(smem_addr(&full_[s]), 1);
            bar_init(smem_addr(&empty_[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(smem_addr(&acc_full_[s]), 1);
            bar_init(smem_addr(&acc_empty_[s]), 4 * CG);
        }
        gave_up_ = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) tmem_alloc<CG>(smem_addr(&tmem_slot), 2 * kAccColumns);

    // the segments' bounds and, where tiles follow the segments, the experts' first tiles: each thread sums a run of experts
    for (int e = threadIdx.x; e <= a.E; e += kThreads) bound[e] = segment_bound(__ldg(a.offsets + e), a.rows);
    if (threadIdx.x == 0 && blockIdx.x == 0 && a.status && __ldg(a.offsets + a.E) > a.rows) atomicOr(a.status, EP_STATUS_CAPACITY);
    __syncthreads();
    if (MODE != kDweight) {
        const int m_tiles = (a.M + kTileM * CG - 1) / (kTileM * CG);
        const int per = (a.E + kThreads - 1) / kThreads, from = min(a.E, (int)threadIdx.x * per), to = min(a.E, from + per);
        int sum = 0;
        for (int e = from; e < to; ++e) sum += (max(0, bound[e + 1] - bound[e]) + a.columns - 1) / a.columns * m_tiles;
        int scan = sum;
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(kFullMask, scan, d);
            if (lane >= d) scan += v;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        int run = scan - sum;
        for (int w = 0; w < warp; ++w) run += warp_sum[w];
        for (int e = from; e < to; ++e) {
            first_tile[e] = run;
            run += (max(0, bound[e + 1] - bound[e]) + a.columns - 1) / a.columns * m_tiles;
        }
        if (threadIdx.x == kThreads - 1) first_tile[a.E] = run;
    }
    tmem_fence_before();
    if (CG == 2) cluster_sync();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_slot;
    const Walk<MODE, CG> walk(a, first_tile, bound);
    const int start = blockIdx.x / CG, stride = gridDim.x / CG;
    constexpr bool kAMn = MODE != kForward, kBMn = MODE == kDweight;
    Tile t;

    if (warp == 0 && lane == 0) {
        // ---- operands into the ring
        int it = 0;
        bool ok = true;
        for (int tile = start; ok && walk.get(tile, t); tile += stride) {
            const int half = t.n / CG;                                       // columns this CTA brings
            const int b_box = kBMn ? 64 : 32, boxes = (half + b_box - 1) / b_box;
            const uint32_t bytes = CG * (kBytesA + boxes * b_box * kTileK * 2);
            const int m = t.m0 + rank * kTileM, c = t.c0 + rank * half;
            const CUtensorMap *ma = &map_a, *mb = &map_b;
            if (MODE == kDweight && t.nk) {
                ma = a.segment_maps + 2 * (size_t)t.e, mb = ma + 1;
                asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(ma) : "memory");
                asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(mb) : "memory");
            }
            for (int kb = 0; kb < t.nk; ++kb, ++it) {
                const int s = it % a.stages;
                if (!(ok = bar_wait(smem_addr(&empty_[s]), ((it / a.stages) & 1) ^ 1, gave_up))) break;
                uint32_t full = smem_addr(&full_[s]);
                if (rank == 0) bar_expect(full, bytes);
                if (CG == 2) full = in_cta(full, 0);
                const uint32_t sa = ring + s * stage_bytes, sb = sa + kBytesA;
                const int k = t.k0 + kb * kTileK;
                if (MODE == kForward) {
                    tma_load<CG>(sa, ma, k, m, t.e, full);
                } else if (MODE == kDx) {
                    tma_load<CG>(sa, ma, m, k, t.e, full);
                    tma_load<CG>(sa + 8192, ma, m + 64, k, t.e, full);
                } else {
                    tma_load<CG>(sa, ma, m, k, 0, full);
                    tma_load<CG>(sa + 8192, ma, m + 64, k, 0, full);
                }
                for (int b = 0; b < boxes; ++b) {
                    if (kBMn) tma_load<CG>(sb + b * 8192, mb, c + b * 64, k, 0, full);
                    else tma_load<CG>(sb + b * 4096, mb, k, c + b * 32, 0, full);
                }
            }
        }
        if (!ok && rank == 0)                                                // gave up: let the copies in flight land
            for (int i = max(0, it - a.stages); i < it; ++i) {
                int none = 0;
                bar_wait(smem_addr(&full_[i % a.stages]), (i / a.stages) & 1, &none);
            }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---- products
        int it = 0, used = 0;
        bool ok = true;
        for (int tile = start; ok && walk.get(tile, t); tile += stride) {
            if (t.nk == 0) continue;
            const int acc = used & 1;
            if (!(ok = bar_wait(smem_addr(&acc_empty_[acc]), ((used >> 1) & 1) ^ 1, gave_up))) break;
            tmem_fence_after();
            const uint32_t d = tmem + acc * kAccColumns;
            const uint32_t idesc = instr_desc(kTileM * CG, t.n, kAMn, kBMn);
            for (int kb = 0; kb < t.nk; ++kb, ++it) {
                const int s = it % a.stages;
                if (!(ok = bar_wait(smem_addr(&full_[s]), (it / a.stages) & 1, gave_up))) break;
                tmem_fence_after();
                const uint32_t sa = ring + s * stage_bytes, sb = sa + kBytesA;
#pragma unroll
                for (int j = 0; j < kTileK / 16; ++j) {
                    const uint64_t da = kAMn ? desc_mn_major(sa + j * 2048) : desc_k_major(sa + j * 32);
                    const uint64_t db = kBMn ? desc_mn_major(sb + j * 2048) : desc_k_major(sb + j * 32);
                    mma_bf16<CG>(d, da, db, idesc, kb > 0 || j > 0);
                }
                mma_commit<CG>(smem_addr(&empty_[s]));
            }
            if (!ok) break;
            mma_commit<CG>(smem_addr(&acc_full_[acc]));
            ++used;
        }
    } else if (warp >= 4) {
        // ---- accumulators out
        const int q = warp - 4;                                              // this warp's quarter of the lanes
        int used = 0;
        for (int tile = start; walk.get(tile, t); tile += stride) {
            const int feature = t.m0 + rank * kTileM + q * 32 + lane;
            const bool live = feature < a.M;
            const int acc = used & 1;
            if (t.nk) {
                if (!bar_wait(smem_addr(&acc_full_[acc]), (used >> 1) & 1, gave_up)) break;
                tmem_fence_after();
            }
            const uint32_t from = tmem + (uint32_t(q * 32) << 16) + acc * kAccColumns;
            size_t at = MODE == kDweight ? ((size_t)t.e * a.N + t.c0) * a.M + feature : (size_t)t.c0 * a.M + feature;
            float b = 0.f;
            if (MODE == kForward && a.bias && live) b = bf16_value(__ldg(a.bias + (size_t)t.e * a.M + feature));
            for (int c0 = 0; c0 < t.cols; c0 += 32, at += (size_t)32 * a.M) {
                const int cols = live ? min(32, t.cols - c0) : 0;
                uint32_t v[32];
                uint16_t r[32];
                if (MODE == kForward && a.operand) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) r[c] = c < cols ? a.operand[at + (size_t)c * a.M] : (uint16_t)0;   // may be y: not through the read-only path
                }
                if (t.nk) {
                    tmem_load32(from + c0, v);
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] = 0u;
                }
                if (MODE == kForward) {
                    switch (a.activation) {
                    case EP_ACT_RELU: store_forward<EP_ACT_RELU>(a, v, r, b, at, cols); break;
                    case EP_ACT_SILU: store_forward<EP_ACT_SILU>(a, v, r, b, at, cols); break;
                    case EP_ACT_GELU: store_forward<EP_ACT_GELU>(a, v, r, b, at, cols); break;
                    default: store_forward<EP_ACT_NONE>(a, v, r, b, at, cols); break;
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (c < cols) a.out[at + (size_t)c * a.M] = bf16_bits(__uint_as_float(v[c]));
                }
            }
            if (t.nk) {
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(in_cta(smem_addr(&acc_empty_[acc]), 0));
                ++used;
            }
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();                                             // the peer's signals land in this CTA's memory
    tmem_fence_after();
    if (warp == 2) tmem_free<CG>(tmem, 2 * kAccColumns);
    if (threadIdx.x == 0 && gave_up_ && a.status) atomicOr(a.status, EP_STATUS_TIMEOUT);
}

// One pair of tensor maps per expert that end with its segment: {x, dz} of rows [0, bound[e+1]).
__global__ void __launch_bounds__(32)
segment_maps_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_dz, const int32_t *offsets,
                    long long rows, CUtensorMap *out)
{
    __shared__ alignas(128) uint32_t work[2][32];
    const int e = blockIdx.x, lane = threadIdx.x;
    work[0][lane] = reinterpret_cast<const uint32_t *>(&map_x)[lane];
    work[1][lane] = reinterpret_cast<const uint32_t *>(&map_dz)[lane];
    const uint32_t end = max(1, segment_bound(__ldg(offsets + e + 1), rows));
    __syncwarp();
    for (int i = 0; i < 2; ++i) {
        const uint32_t s = smem_addr(work[i]);
        if (lane == 0) asm volatile("tensormap.replace.tile.global_dim.shared::cta.b1024.b32 [%0], 1, %1;" ::"r"(s), "r"(end) : "memory");
        __syncwarp();
        asm volatile("tensormap.cp_fenceproxy.global.shared::cta.tensormap::generic.release.gpu.sync.aligned [%0], [%1], 128;" ::"l"(
                         out + 2 * (size_t)e + i),
                     "r"(s)
                     : "memory");
    }
}

// ---- dz = dy * (operand) * act'(pre), doperand = dy * act(pre), and the partial sums of dbias -------------------------
// A warp owns 256 columns (8 a lane) and a run of rows; three 16-byte loads and one or two 16-byte stores per row and lane,
// bound by memory. A run is cut where a segment ends: chunk c and expert e share at most one piece, and c + e grows along
// the rows, so it numbers the pieces; their sums go to partial[c + e] and the second kernel adds an expert's pieces in
// their order (no atomics: the same bits every time).

constexpr int kSlopeWarps = 4;

struct SlopeArgs {
    const uint4 *dy, *pre, *operand;
    uint4 *dz, *doperand;
    float *partial;
    const int32_t *offsets;
    long long rows;
    int vecs, E, chunk, activation;       // vecs: 16-byte vectors per row; chunk: rows per run
};

__device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8])
{
    f[0] = bf16_lo(v.x), f[1] = bf16_hi(v.x), f[2] = bf16_lo(v.y), f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z), f[5] = bf16_hi(v.z), f[6] = bf16_lo(v.w), f[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8])
{
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

template <int ACT>
__global__ void __launch_bounds__(kSlopeWarps * 32)
slope_kernel(const SlopeArgs a)
{
    const int lane = threadIdx.x & 31, vec = blockIdx.x * 32 + lane;
    const long long chunk = (long long)blockIdx.y * kSlopeWarps + (threadIdx.x >> 5);
    const int total = segment_bound(__ldg(a.offsets + a.E), a.rows);
    long long p = chunk * a.chunk;
    const long long end = min((long long)total, p + a.chunk);
    if (p >= end) return;
    int e = 0;
    if (a.partial) {                                     // the expert of row p: the last e with bound[e] <= p
        int lo = 0, hi = a.E;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (segment_bound(__ldg(a.offsets + mid), a.rows) <= p) lo = mid; else hi = mid;
        }
        e = lo;
    }
    const bool live = vec < a.vecs;
    constexpr int kRows = 4;
    while (p < end) {
        long long stop = end;
        if (a.partial) {
            int next;
            while ((next = segment_bound(__ldg(a.offsets + e + 1), a.rows)) <= p) ++e;   // ends: bound[E] = total > p
            stop = min(end, (long long)next);
        }
        float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (; p < stop; p += kRows) {
            uint4 g[kRows], z[kRows], r[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (live && p + i < stop) {
                    const size_t at = (size_t)(p + i) * a.vecs + vec;
                    g[i] = ld_stream(a.dy + at);
                    if (ACT != EP_ACT_NONE || a.doperand) z[i] = ld_stream(a.pre + at);
                    if (a.operand) r[i] = ld_stream(a.operand + at);
                }
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (live && p + i < stop) {
                    const size_t at = (size_t)(p + i) * a.vecs + vec;
                    float fg[8], fz[8], fr[8], o[8];
                    unpack8(g[i], fg);
                    if (ACT != EP_ACT_NONE || a.doperand) unpack8(z[i], fz);
                    if (a.doperand) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = fg[j] * act_value(ACT, fz[j]);
                        st_stream(a.doperand + at, pack8(o));
                    }
                    if (a.operand) {
                        unpack8(r[i], fr);
#pragma unroll
                        for (int j = 0; j < 8; ++j) fg[j] *= fr[j];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (ACT != EP_ACT_NONE) fg[j] *= act_slope(ACT, fz[j]);
                        sum[j] += fg[j];
                    }
                    if (a.dz) a.dz[at] = pack8(fg);
                }
        }
        p = stop;
        if (a.partial && live) {
            float4 *dst = reinterpret_cast<float4 *>(a.partial + ((size_t)(chunk + e) * a.vecs + vec) * 8);
            dst[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            dst[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        }
    }
}

// dbias[e][n] = sum of the expert's pieces in their order: eight runs of pieces at a time, then the eight sums.
__global__ void __launch_bounds__(256)
bias_grad_kernel(const float *__restrict__ partial, const int32_t *__restrict__ offsets, long long rows, int N, int chunk, float *dbias)
{
    __shared__ float part[8][32];
    const int e = blockIdx.y, lane = threadIdx.x & 31, w = threadIdx.x >> 5, n = blockIdx.x * 32 + lane;
    const int begin = segment_bound(__ldg(offsets + e), rows), end = segment_bound(__ldg(offsets + e + 1), rows);
    float s = 0.f;
    if (begin < end && n < N) {
        const int c0 = begin / chunk, count = (end - 1) / chunk - c0 + 1, per = (count + 7) / 8;
        const int from = c0 + min(count, w * per), to = c0 + min(count, w * per + per);
#pragma unroll 8
        for (int c = from; c < to; ++c) s += __ldg(partial + (size_t)(c + e) * N + n);
    }
    part[w][lane] = s;
    __syncthreads();
    if (w == 0 && n < N) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[i][lane];
        dbias[(size_t)e * N + n] = s;
    }
}

// ---- host side ---------------------------------------------------------------------------------------------------

int check_matmul(const ep_matmul_t *m)
{
    if (!m) return EP_ERR_NULL;
    if (m->rows < 0 || m->rows >= (int64_t(1) << 31) || m->in_features < 8 || m->in_features % 8 || m->out_features < 8 ||
        m->out_features % 8 || m->num_experts < 1 || m->num_experts > kMaxExperts || m->activation < EP_ACT_NONE ||
        m->activation > EP_ACT_GELU || m->operand_op < EP_OPERAND_ADD || m->operand_op > EP_OPERAND_MUL)
        return EP_ERR_INVALID_ARG;
    // an expert's weights are one TMA plane and all features of a tile row fit 31 bits
    if ((int64_t)m->in_features >= (1 << 24) || (int64_t)m->out_features >= (1 << 24)) return EP_ERR_INVALID_ARG;
    return EP_OK;
}

int sm_count(int *n)
{
    int dev = 0;
    EP_CUDA_TRY(cudaGetDevice(&dev));
    EP_CUDA_TRY(cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev));
    return EP_OK;
}

template <int MODE, int CG>
int launch_product(ProductArgs a, const CUtensorMap &map_a, const CUtensorMap &map_b, int64_t max_tiles, cudaStream_t stream)
{
    int sms = 0;
    const int rc = sm_count(&sms);
    if (rc != EP_OK) return rc;
    const int stage = kBytesA + (a.columns / CG < 32 ? 32 : a.columns / CG) * kTileK * 2;
    const int tables = 2 * (a.E + 1) * 4;
    a.stages = (kSmemLimit - 2048 - tables) / stage;                         // 2048: alignment of the ring, static words
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    int smem = 1024 + a.stages * stage + tables;
    if (smem < 120 * 1024) smem = 120 * 1024;                                // one CTA per SM: it holds all of the tensor memory
    EP_CUDA_TRY(cudaFuncSetAttribute(product_kernel<MODE, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    int64_t pairs = sms / CG;
    if (max_tiles < pairs) pairs = max_tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(pairs * CG));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = CG;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    EP_CUDA_TRY(cudaLaunchKernelEx(&cfg, product_kernel<MODE, CG>, a, map_a, map_b));
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

// Columns (rows p) per tile: as many as an expert has on average, in powers of two, so that most experts are one tile.
int row_columns(int64_t rows, int E)
{
    int c = 64;
    while (c < kAccColumns && (int64_t)c * E < rows + rows / 2) c *= 2;
    return c;
}

int64_t row_tiles(int64_t rows, int E, int columns, int features, int CG)
{
    const int64_t experts = rows < E ? rows : E;
    return (experts + rows / columns) * ((features + kTileM * CG - 1) / (kTileM * CG));
}

int slope_chunk(int64_t rows)   // rows per run: short runs fill the GPU, and at most 512 of them leave little to add up
{
    int64_t c = (rows + 511) / 512;
    c = (c + 3) / 4 * 4;
    return (int)(c < 32 ? 32 : c);
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

size_t maps_bytes(const ep_matmul_t &m) { return up256(sizeof(CUtensorMap) * 2 * (size_t)m.num_experts); }
size_t partial_bytes(const ep_matmul_t &m)
{
    const size_t chunks = (m.rows + slope_chunk(m.rows) - 1) / slope_chunk(m.rows);
    return up256((chunks + m.num_experts) * (size_t)m.out_features * 4);
}
size_t dz_bytes(const ep_matmul_t &m) { return up256((size_t)m.rows * m.out_features * 2); }

template <int ACT>
void launch_slope(const SlopeArgs &a, dim3 grid, cudaStream_t stream)
{
    slope_kernel<ACT><<<grid, kSlopeWarps * 32, 0, stream>>>(a);
}

}  // namespace

int tensor_map_encoder(TensorMapEncode *fn)
{
    static std::mutex mutex;
    static TensorMapEncode found = nullptr;
    std::lock_guard<std::mutex> hold(mutex);
    if (!found) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult state;
        EP_CUDA_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &state));
        if (state != cudaDriverEntryPointSuccess || !p) {
            note_cuda_error(cudaErrorNotSupported);
            return EP_ERR_CUDA;
        }
        found = reinterpret_cast<TensorMapEncode>(p);
    }
    *fn = found;
    return EP_OK;
}

}  // namespace ep

extern "C" int ep_expert_matmul(const ep_matmul_t *m, const void *x, const int32_t *expert_offsets, const void *weight, const void *bias,
                                const void *operand, void *y, void *pre, int32_t *status, void *stream_)
{
    using namespace ep;
    int rc = check_matmul(m);
    if (rc != EP_OK) return rc;
    if (m->rows == 0) return EP_OK;
    if (!x || !expert_offsets || !weight || !y) return EP_ERR_NULL;
    if (!aligned16(x) || !aligned16(weight) || !aligned16(bias) || !aligned16(operand) || !aligned16(y) || !aligned16(pre))
        return EP_ERR_INVALID_ARG;
    TensorMapEncode encode;
    rc = tensor_map_encoder(&encode);
    if (rc != EP_OK) return rc;
    CUtensorMap map_w, map_x;
    rc = make_map(encode, &map_w, weight, m->in_features, m->out_features, m->num_experts, kTileM);
    if (rc == EP_OK) rc = make_map(encode, &map_x, x, m->in_features, m->rows, 1, 32);
    if (rc != EP_OK) return rc;
    ProductArgs a = {};
    a.offsets = expert_offsets;
    a.status = status;
    a.rows = m->rows;
    a.M = m->out_features, a.K = m->in_features, a.E = m->num_experts;
    a.out = static_cast<uint16_t *>(y);
    a.bias = static_cast<const uint16_t *>(bias);
    a.operand = static_cast<const uint16_t *>(operand);
    a.pre = static_cast<uint16_t *>(pre);
    a.activation = m->activation, a.operand_op = m->operand_op;
    a.columns = row_columns(m->rows, m->num_experts);
    return launch_product<kForward, 1>(a, map_w, map_x, row_tiles(m->rows, a.E, a.columns, a.M, 1), static_cast<cudaStream_t>(stream_));
}

extern "C" size_t ep_expert_matmul_backward_workspace_bytes(const ep_matmul_t *m)
{
    using namespace ep;
    if (check_matmul(m) != EP_OK) return 0;
    return maps_bytes(*m) + partial_bytes(*m) + dz_bytes(*m);
}

extern "C" int ep_expert_matmul_backward(const ep_matmul_t *m, const void *dy, const void *x, const int32_t *expert_offsets,
                                         const void *weight, const void *pre, const void *operand, void *dx, void *dweight, float *dbias,
                                         void *doperand, int32_t *status, void *workspace, size_t workspace_bytes, void *stream_)
{
    using namespace ep;
    int rc = check_matmul(m);
    if (rc != EP_OK) return rc;
    const bool mul = operand && m->operand_op == EP_OPERAND_MUL;
    if (!expert_offsets || (m->rows && !dy)) return EP_ERR_NULL;
    if (m->rows && ((dx && !weight) || (dweight && !x))) return EP_ERR_NULL;
    if (m->rows && !pre && (m->activation != EP_ACT_NONE || doperand)) return EP_ERR_NULL;
    if (doperand && !mul) return EP_ERR_INVALID_ARG;                        // an added operand's gradient is dy itself
    if (!aligned16(dy) || !aligned16(x) || !aligned16(weight) || !aligned16(pre) || !aligned16(operand) || !aligned16(dx) ||
        !aligned16(dweight) || !aligned16(dbias) || !aligned16(doperand) || (reinterpret_cast<uintptr_t>(workspace) & 127u))
        return EP_ERR_INVALID_ARG;
    if (!workspace) return EP_ERR_NULL;
    if (workspace_bytes < ep_expert_matmul_backward_workspace_bytes(m)) return EP_ERR_CAPACITY;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const size_t E = m->num_experts, N = m->out_features, H = m->in_features;
    if (m->rows == 0) {
        if (dweight) EP_CUDA_TRY(cudaMemsetAsync(dweight, 0, E * N * H * 2, stream));
        if (dbias) EP_CUDA_TRY(cudaMemsetAsync(dbias, 0, E * N * 4, stream));
        return EP_OK;
    }
    char *ws = static_cast<char *>(workspace);
    CUtensorMap *maps = reinterpret_cast<CUtensorMap *>(ws);
    float *partial = reinterpret_cast<float *>(ws + maps_bytes(*m));
    void *dz_own = ws + maps_bytes(*m) + partial_bytes(*m);

    // ---- dz, unless it is dy itself
    const bool plain = m->activation == EP_ACT_NONE && !mul;
    const void *dz = plain ? dy : dz_own;
    if (dbias || doperand || (!plain && (dx || dweight))) {
        SlopeArgs s = {};
        s.dy = static_cast<const uint4 *>(dy);
        s.pre = static_cast<const uint4 *>(pre);
        s.operand = mul ? static_cast<const uint4 *>(operand) : nullptr;
        s.dz = plain || !(dx || dweight) ? nullptr : static_cast<uint4 *>(dz_own);
        s.doperand = static_cast<uint4 *>(doperand);
        s.partial = dbias ? partial : nullptr;
        s.offsets = expert_offsets;
        s.rows = m->rows;
        s.vecs = (int)(N / 8), s.E = (int)E, s.activation = m->activation;
        s.chunk = slope_chunk(m->rows);
        const int64_t chunks = (m->rows + s.chunk - 1) / s.chunk;
        const dim3 grid(ceil_div(s.vecs, 32), (unsigned)((chunks + kSlopeWarps - 1) / kSlopeWarps));
        switch (m->activation) {
        case EP_ACT_RELU: launch_slope<EP_ACT_RELU>(s, grid, stream); break;
        case EP_ACT_SILU: launch_slope<EP_ACT_SILU>(s, grid, stream); break;
        case EP_ACT_GELU: launch_slope<EP_ACT_GELU>(s, grid, stream); break;
        default: launch_slope<EP_ACT_NONE>(s, grid, stream); break;
        }
        EP_LAUNCH_CHECK(1);
        if (dbias) {
            bias_grad_kernel<<<dim3((unsigned)((N + 31) / 32), (unsigned)E), 256, 0, stream>>>(partial, expert_offsets, m->rows, (int)N,
                                                                                              s.chunk, dbias);
            EP_LAUNCH_CHECK(1);
        }
    }
    TensorMapEncode encode;
    rc = tensor_map_encoder(&encode);
    if (rc != EP_OK) return rc;
    ProductArgs a = {};
    a.offsets = expert_offsets;
    a.status = status;
    a.rows = m->rows;
    a.E = m->num_experts;
    CUtensorMap map_a, map_b;
    if (dx) {
        rc = make_map(encode, &map_a, weight, H, N, E, kTileK);
        if (rc == EP_OK) rc = make_map(encode, &map_b, dz, N, m->rows, 1, 32);
        if (rc != EP_OK) return rc;
        a.M = m->in_features, a.K = m->out_features, a.N = 0;
        a.out = static_cast<uint16_t *>(dx);
        a.columns = row_columns(m->rows, m->num_experts);
        rc = launch_product<kDx, 1>(a, map_a, map_b, row_tiles(m->rows, a.E, a.columns, a.M, 1), stream);
        if (rc != EP_OK) return rc;
    }
    if (dweight) {
        rc = make_map(encode, &map_a, x, H, m->rows, 1, kTileK);
        if (rc == EP_OK) rc = make_map(encode, &map_b, dz, N, m->rows, 1, kTileK);
        if (rc != EP_OK) return rc;
        segment_maps_kernel<<<(unsigned)E, 32, 0, stream>>>(map_a, map_b, expert_offsets, m->rows, maps);
        EP_LAUNCH_CHECK(1);
        a.M = m->in_features, a.N = m->out_features, a.K = 0;
        a.out = static_cast<uint16_t *>(dweight);
        a.segment_maps = maps;
        a.columns = kAccColumns;
        const int64_t tiles = (int64_t)E * ((a.M + kTileM - 1) / kTileM) * ((a.N + a.columns - 1) / a.columns);
        if (tiles >= (int64_t(1) << 31)) return EP_ERR_INVALID_ARG;
        rc = launch_product<kDweight, 1>(a, map_a, map_b, tiles, stream);
        if (rc != EP_OK) return rc;
    }
    return EP_OK;
}
