// The experts' matrix products over the pair space, and their gradients.
//
//   forward   y[p] = act(x[p] W[e]^T + b[e]) (+ or *) operand[p]         rows p of expert e's segment
//   dx        dx[p] = dz[p] W[e]
//   dweight   dW[e] = sum_p dz[p]^T x[p]
//
// All three are one kernel. The accumulator's 128 lanes hold the axis that is contiguous in the result (features), its
// columns hold the other one (rows p, or the weight's out features), so that a column is a run of neighbouring elements of a
// result row, and the ragged axis of a segment, the rows, is cut in steps of 16 columns: an expert that got one row costs a
// 16-column product, not one of 128 rows.
//
//   mode      lanes (M)       columns (N)     contracted (K)   lane operand             column operand
//   forward   out features    rows            in features      W, K-major               x, K-major
//   dx        in features     rows            out features     W, MN-major              dz, K-major
//   dweight   in features     out features    rows             x, MN-major              dz, MN-major
//
// Where there are fewer tiles than SMs, tiles get narrower (down to 64 columns), and then up to eight CTAs of a cluster share a
// tile, each with a part of the contracted axis, and add their accumulators through each other's shared memory in a fixed order.
//
// One persistent CTA per SM. A warp keeps a ring of shared-memory stages full by TMA (64 of the contracted axis each), one
// thread issues the products, eight warps empty the accumulators, of which there are two of 256 columns, so that a tile's
// epilogue runs under the next tile's products. Rows behind a segment's end that a box brings along only feed columns that
// are not stored; in the dweight mode, where the rows are contracted, the operands are read through tensor maps that end
// with the segment (one pair per expert, made on the device from the offsets), so that the rest of the last box is zero
// whatever the neighbouring rows hold.
#include <atomic>

#include "ep_tensor.cuh"

namespace ep {
namespace {

enum { kForward = 0, kDx = 1, kDweight = 2 };

constexpr int kEpilogueWarps = 8;         // two per quarter of the lanes, taking turns at blocks of 32 columns
constexpr int kThreads = 128 + 32 * kEpilogueWarps;
constexpr int kTileM = 128;               // lanes of one CTA
constexpr int kTileK = 64;                // contracted elements per stage: one 128-byte line
constexpr int kAccColumns = 256;          // columns of one of the two accumulators
constexpr int kBytesA = kTileM * kTileK * 2;
constexpr int kStageLd = 36, kStageWords = 16 * kStageLd;      // an epilogue warp's buffer: 16 columns of 32 lanes
constexpr int kStageBytes = kEpilogueWarps * kStageWords * 4;
constexpr int kSplitColumns = 64, kExchangeLd = kTileM + 4;    // a shared tile's accumulators as its CTAs exchange them
constexpr int kExchangeBytes = kSplitColumns * kExchangeLd * 4;
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
    int split;                            // CTAs that share a tile
    uint16_t *out;
    const CUtensorMap *segment_maps;      // dweight: [E][2]
    // forward epilogue
    const uint16_t *bias, *operand;
    uint16_t *pre;
    int activation, operand_op;
};

// The column operand's boxes: of 128, 64, 32 and 16 rows where it is K-major, so that a tile's columns (a multiple of 16) are
// fetched in at most five copies and no row more; box[0] alone (64 x 64) where it is MN-major.
struct ColumnMaps {
    CUtensorMap box[4];
};

struct Tile {
    int e, m0;
    int c0, cols;                         // first column (row p, or out feature) and how many are real
    int n;                                // columns of the product: cols rounded up to what the tensor cores take
    int k0, nk, all;                      // first contracted index, stages, and stages of all CTAs that share the tile (0: no rows)
};

__device__ __forceinline__ int segment_bound(int32_t v, long long rows)
{
    return v < 0 ? 0 : (v > rows ? (int)rows : v);
}

// a / b rounded up, for a up to 2^31 - 1
__device__ __forceinline__ int quotient_up(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) / (unsigned)b); }

// Activations by the fast exponential and division: errors of 2 + 1.16 |z| units in the last place of fp32 where the exponential
// decides (z < 0), some 2^-20 for |z| up to 8, far below the rounding to bf16 of y, dz and doperand; dbias, a sum in fp32, sees it. expf
// and an exact division cost: forward of 65536 rows through four experts of 512 x 512, silu, 100 us instead of 50; dz, doperand and dbias of
// 32768 rows of 1024 features, silu and a multiplied operand, 81 instead of 61. Phi as (1 + erf) / 2 is off by some 2^-25, absolute: a few per
// cent of itself at z = -5, all of it at -6. erfcf, which keeps its left tail, takes 167 us for the slopes of 32768 x 2048 instead of 123.
__device__ __forceinline__ float act_value(int act, float z)
{
    switch (act) {
    case EP_ACT_RELU: return z <= 0.f ? 0.f : z;
    case EP_ACT_SILU: return __fdividef(z, 1.f + __expf(-z));
    case EP_ACT_GELU: return 0.5f * z * (1.f + erff(z * 0.70710678f));
    default: return z;
    }
}

// act(z) and its derivative
__device__ __forceinline__ void act_both(int act, float z, float &value, float &slope)
{
    switch (act) {
    case EP_ACT_RELU: value = z <= 0.f ? 0.f : z, slope = z <= 0.f ? 0.f : 1.f; break;
    case EP_ACT_SILU: {
        const float s = __fdividef(1.f, 1.f + __expf(-z));
        value = z * s, slope = s * (1.f + z * (1.f - s));
        break;
    }
    case EP_ACT_GELU: {
        const float phi = 0.5f + 0.5f * erff(z * 0.70710678f);
        value = z * phi, slope = phi + z * __expf(-0.5f * z * z) * 0.39894228f;
        break;
    }
    default: value = z, slope = 1.f; break;
    }
}

// ---- the walk over tiles -----------------------------------------------------------------------------------------

// Tiles are dealt out to the CTAs (pairs) round by round, an expert's row pieces next to each other, then its feature tiles: what
// runs at the same time shares rows and weights in L2. Neither experts sorted by cost nor a shared counter was faster, with
// segments of even and of Zipf-distributed lengths (counter: 3 to 6 % slower; order: within 2 % either way).
template <int MODE, int CG, bool SPLIT>
struct Walk {
    const ProductArgs &a;
    const int *first_tile;   // [E+1] shared memory: tiles of the experts before e (forward, dx)
    const int *bound;        // [E+1] the segments' bounds, clamped
    int m_tiles, n_tiles, total, tile, step, part;

    __device__ Walk(const ProductArgs &args, const int *first, const int *b, int start, int stride, int which)
        : a(args), first_tile(first), bound(b), tile(start), step(stride), part(which)
    {
        m_tiles = (a.M + kTileM * CG - 1) / (kTileM * CG);
        n_tiles = MODE == kDweight ? (a.N + a.columns - 1) / a.columns : 0;
        total = MODE == kDweight ? a.E * m_tiles * n_tiles : first_tile[a.E];
    }

    // This CTA's next tile; false when there is none left.
    __device__ bool next(Tile &t)
    {
        if (tile >= total) return false;
        constexpr int kStep = 16 * CG;
        if (MODE == kDweight) {
            const int per = m_tiles * n_tiles;
            t.e = tile / per;
            const int r = tile - t.e * per, m = r / n_tiles;
            t.m0 = m * kTileM * CG;
            t.c0 = (r - m * n_tiles) * a.columns;
            t.cols = min(a.columns, a.N - t.c0);
            t.k0 = bound[t.e];
            t.nk = quotient_up(max(0, bound[t.e + 1] - t.k0), kTileK);
        } else {
            int lo = 0, hi = a.E;                        // the expert e with first_tile[e] <= tile < first_tile[e+1]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first_tile[mid] <= tile) lo = mid; else hi = mid;
            }
            t.e = lo;
            const int r = tile - first_tile[lo], begin = bound[lo], count = bound[lo + 1] - begin;
            const int pieces = quotient_up(count, a.columns), m = r / pieces, piece = r - m * pieces;
            const int width = (quotient_up(count, pieces) + kStep - 1) / kStep * kStep;   // equal pieces
            t.m0 = m * kTileM * CG;
            t.c0 = begin + piece * width;
            t.cols = max(0, min(width, count - piece * width));
            t.k0 = 0;
            t.nk = (a.K + kTileK - 1) / kTileK;
        }
        t.n = max(kStep, (t.cols + kStep - 1) / kStep * kStep);
        t.all = t.nk;
        if (SPLIT) {                                     // this CTA's part of the contracted axis (may be empty)
            const int from = t.nk * part / a.split, to = t.nk * (part + 1) / a.split;
            t.k0 += from * kTileK;
            t.nk = to - from;
        }
        tile += step;
        return true;
    }
};

// Where a role stands in the ring of stages. Counted up, not divided: one thread issues all copies, one all products, and
// a division by a run-time number of stages in either loop took longer than the products of a small tile.
struct Ring {
    uint32_t addr, base;
    int stage, phase, stages, bytes;
    __device__ Ring(uint32_t b, int stage_bytes, int n) : addr(b), base(b), stage(0), phase(0), stages(n), bytes(stage_bytes) {}
    __device__ void next()
    {
        ++stage, addr += bytes;
        if (stage == stages) stage = 0, phase ^= 1, addr = base;
    }
};

// ---- epilogues ---------------------------------------------------------------------------------------------------

// A warp's 32 lanes x 32 columns of accumulators pass through shared memory, so that afterwards a lane holds 8 neighbouring
// features of a column and reads and writes global memory 16 bytes at a time: the forward mode with an operand or `pre` 16 columns
// of fp32 at a time, the others, whose arithmetic is done before, all 32 columns as rounded pairs. The pairs matter where the contracted axis is
// short and a tile's epilogue takes as long as its products: shared memory feeds both, and with fp32 words the dweight mode
// took 220 us at 128 experts of 1024 x 2048 and 32768 rows, with pairs 195. (Stored straight from the accumulators' order,
// 2 bytes a lane, a column took ten instructions.) Rows are 36 words apart: 16-byte reads of eight lanes fall on all banks.
// z (8 features of one row) -> y, and pre if asked for.
template <int ACT>
__device__ __forceinline__ void finish8(const ProductArgs &a, float (&z)[8], const uint4 &operand, size_t at)
{
    if (a.pre) *reinterpret_cast<uint4 *>(a.pre + at) = pack8(z);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = act_value(ACT, z[i]);
    if (a.operand) {
        float r[8];
        unpack8(operand, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = a.operand_op == EP_OPERAND_MUL ? z[i] * r[i] : z[i] + r[i];
    }
    *reinterpret_cast<uint4 *>(a.out + at) = pack8(z);
}

// ---- the kernel --------------------------------------------------------------------------------------------------

// 32 accumulators of one feature: bias and activation, in place.
template <int ACT>
__device__ __forceinline__ void act_all(uint32_t (&v)[32], float bias)
{
#pragma unroll
    for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(act_value(ACT, __uint_as_float(v[c]) + bias));
}

// 8 features of a row: the mode's arithmetic and the store. operand: as loaded, if there is one.
template <int MODE>
__device__ __forceinline__ void finish_row(const ProductArgs &a, float (&z)[8], const float (&bias)[8], const uint4 &operand, size_t at)
{
    if (MODE == kForward) {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] += bias[j];
        switch (a.activation) {
        case EP_ACT_RELU: finish8<EP_ACT_RELU>(a, z, operand, at); break;
        case EP_ACT_SILU: finish8<EP_ACT_SILU>(a, z, operand, at); break;
        case EP_ACT_GELU: finish8<EP_ACT_GELU>(a, z, operand, at); break;
        default: finish8<EP_ACT_NONE>(a, z, operand, at); break;
        }
    } else {
        *reinterpret_cast<uint4 *>(a.out + at) = pack8(z);
    }
}

template <int MODE, int CG, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const ProductArgs a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ ColumnMaps map_b)
{
    extern __shared__ char raw[];
    __shared__ uint64_t full_[kMaxStages], empty_[kMaxStages], acc_full_[2], acc_empty_[2], ex_full_, done_;
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_;
    __shared__ int warp_sum[kThreads / 32];
    volatile int *gave_up = &gave_up_;

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // uniform in the warp, and seen to be
    const uint32_t rank = CG == 2 ? cluster_rank() : 0, part = SPLIT ? cluster_rank() : 0;
    const int split = SPLIT ? a.split : 1;
    const int b_bytes = max(32, a.columns / CG) * kTileK * 2;
    const int stage_bytes = kBytesA + b_bytes;
    const uint32_t ring_base = (smem_addr(raw) + 1023) & ~1023u;
    char *tables = raw + (ring_base - smem_addr(raw)) + (size_t)a.stages * stage_bytes;
    int *first_tile = reinterpret_cast<int *>(tables + (SPLIT ? kExchangeBytes : kStageBytes)), *bound = first_tile + a.E + 1;   // the epilogue's buffers first

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            bar_init(smem_addr(&full_[s]), 1);
            bar_init(smem_addr(&empty_[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(smem_addr(&acc_full_[s]), 1);
            bar_init(smem_addr(&acc_empty_[s]), kEpilogueWarps * CG);
        }
        if (SPLIT) bar_init(smem_addr(&ex_full_), split * kEpilogueWarps);
        bar_init(smem_addr(&done_), 1);
        gave_up_ = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < 5) {                                                   // the maps are arguments: theirs may be fetched already
        const CUtensorMap *map = threadIdx.x == 0 ? &map_a : &map_b.box[threadIdx.x - 1];
        if (MODE != kDweight) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    pdl_wait();                                                              // nothing is read or written before this
    // Tensor memory is taken after the kernels before are done and before the next one may come: a CTA that held it while it
    // waited, beside one that needs some, could wait for good.
    if (warp == 2) tmem_alloc<CG>(smem_addr(&tmem_slot), 2 * kAccColumns);
    // the segments' bounds and, where tiles follow the segments, the experts' first tiles
    for (int e = threadIdx.x; e <= a.E; e += kThreads) bound[e] = segment_bound(__ldg(a.offsets + e), a.rows);
    if (threadIdx.x == 0 && blockIdx.x == 0 && a.status && __ldg(a.offsets + a.E) > a.rows) atomicOr(a.status, EP_STATUS_CAPACITY);
    if (MODE == kDweight)                                                    // once for all maps: a fence in front of every tile stalled the copies
        for (int i = threadIdx.x; i < 2 * a.E; i += kThreads)
            asm volatile("fence.proxy.tensormap::generic.acquire.gpu [%0], 128;" ::"l"(a.segment_maps + i) : "memory");
    __syncthreads();
    if (MODE != kDweight) {                                                  // each thread sums a run of experts
        const int m_tiles = (a.M + kTileM * CG - 1) / (kTileM * CG);
        const int per = (a.E + kThreads - 1) / kThreads, from = min(a.E, (int)threadIdx.x * per), to = min(a.E, from + per);
        int sum = 0;
        for (int e = from; e < to; ++e) sum += quotient_up(max(0, bound[e + 1] - bound[e]), a.columns) * m_tiles;
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
            run += quotient_up(max(0, bound[e + 1] - bound[e]), a.columns) * m_tiles;
        }
        if (threadIdx.x == kThreads - 1) first_tile[a.E] = run;
    }
    tmem_fence_before();
    if (CG == 2 || SPLIT) cluster_sync();
    __syncthreads();
    tmem_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_slot;
    const int sharing = CG * split;
    Walk<MODE, CG, SPLIT> walk(a, first_tile, bound, blockIdx.x / sharing, gridDim.x / sharing, part);   // one per role
    const uint32_t full0 = smem_addr(full_), empty0 = smem_addr(empty_), full0_leader = CG == 2 ? in_cta(full0, 0) : full0;
    constexpr bool kAMn = MODE != kForward, kBMn = MODE == kDweight;
    Tile t;

    int in_flight = 0, next_stage = 0, next_phase = 0;                       // copies that may not have landed, and the ring's place behind them
    if (warp == 0 && elect_one()) {
        // ---- operands into the ring
        Ring ring(ring_base, stage_bytes, a.stages);
        bool ok = true;
        int sent = 0;
        while (ok && walk.next(t)) {
            const int half = t.n / CG;                                       // columns this CTA brings
            const int boxes = (half + 63) / 64;                              // MN-major
            const uint32_t bytes = CG * (kBytesA + (kBMn ? boxes * 8192 : half * 128));
            const int m = t.m0 + rank * kTileM, c = t.c0 + rank * half;
            const CUtensorMap *ma = &map_a, *mb = map_b.box;
            if (MODE == kDweight) ma = a.segment_maps + 2 * (size_t)t.e, mb = ma + 1;
            int k = t.k0;
            for (int kb = 0; kb < t.nk; ++kb, k += kTileK) {
                const int s = ring.stage;
                if (!(ok = bar_wait(empty0 + 8 * s, ring.phase ^ 1, gave_up))) break;
                const uint32_t full = full0_leader + 8 * s;
                if (rank == 0) bar_expect(full0 + 8 * s, bytes);
                const uint32_t sa = ring.addr, sb = sa + kBytesA;
                if (MODE == kForward) {
                    tma_load<CG>(sa, ma, k, m, t.e, full);
                } else if (MODE == kDx) {
                    tma_load<CG>(sa, ma, m, k, t.e, full);
                    tma_load<CG>(sa + 8192, ma, m + 64, k, t.e, full);
                } else {
                    tma_load<CG>(sa, ma, m, k, 0, full);
                    tma_load<CG>(sa + 8192, ma, m + 64, k, 0, full);
                }
                if (kBMn) {
#pragma unroll
                    for (int b = 0; b < kAccColumns / CG / 64; ++b)
                        if (b < boxes) tma_load<CG>(sb + b * 8192, mb, c + b * 64, k, 0, full);
                } else {
                    unsigned row = 0;                                        // c + row may pass 2^31 - 1 where no row is left
                    if (CG == 1 && half >= 256) tma_load<CG>(sb, mb, k, c, 0, full), row = 128;
                    if (half - row >= 128) tma_load<CG>(sb + row * 128, mb, k, c + row, 0, full), row += 128;
#pragma unroll
                    for (int b = 1; b < 4; ++b)
                        if (half & (128 >> b)) tma_load<CG>(sb + row * 128, mb + b, k, c + row, 0, full), row += 128 >> b;
                }
                ring.next();
                ++sent;
            }
        }
        if (rank == 0) in_flight = min(sent, a.stages), next_stage = ring.stage, next_phase = ring.phase;      // a pair's are counted there
    } else if (warp == 1 && rank == 0 && elect_one()) {
        // ---- products
        Ring ring(ring_base, stage_bytes, a.stages);
        int used = 0;
        bool ok = true;
        while (ok && walk.next(t)) {
            if (t.nk == 0) continue;
            const int acc = used & 1;
            if (!(ok = bar_wait(smem_addr(&acc_empty_[acc]), ((used >> 1) & 1) ^ 1, gave_up))) break;
            tmem_fence_after();
            const uint32_t d = tmem + acc * kAccColumns;
            const uint32_t idesc = instr_desc(kTileM * CG, t.n, kAMn, kBMn);
            for (int kb = 0; kb < t.nk; ++kb) {
                if (!(ok = bar_wait(full0 + 8 * ring.stage, ring.phase, gave_up))) break;
                tmem_fence_after();
                const uint64_t da = kAMn ? desc_mn_major(ring.addr) : desc_k_major(ring.addr);
                const uint64_t db = kBMn ? desc_mn_major(ring.addr + kBytesA) : desc_k_major(ring.addr + kBytesA);
#pragma unroll
                for (int j = 0; j < kTileK / 16; ++j)                        // the descriptors' addresses count 16 bytes
                    mma_bf16<CG>(d, da + j * (kAMn ? 128 : 2), db + j * (kBMn ? 128 : 2), idesc, kb > 0 || j > 0);
                mma_commit<CG>(empty0 + 8 * ring.stage);
                ring.next();
            }
            if (!ok) break;
            mma_commit<CG>(smem_addr(&acc_full_[acc]));
            ++used;
        }
    } else if (SPLIT && warp >= 4) {
        // ---- accumulators out, of a tile that `split` CTAs share: each writes its sums down, and finishes some of the columns
        const int q = warp & 3, first = (warp - 4) / 4 * 32, thread = threadIdx.x - 128;
        float *mine = reinterpret_cast<float *>(tables);
        const size_t ld = a.M;
        bool ok = walk.next(t) && t.all > 0;                                 // the grid has a cluster per tile: there is no second one
        if (ok && t.nk) {
            ok = warp_wait(smem_addr(&acc_full_[0]), 0, gave_up);
            tmem_fence_after();
        }
        if (ok) {
            if (first < t.cols) {
                uint32_t v[32];
                if (t.nk) {
                    tmem_load32(tmem + (uint32_t(q * 32) << 16) + first, v);
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] = 0u;
                }
#pragma unroll
                for (int c = 0; c < 32; ++c) mine[(first + c) * kExchangeLd + q * 32 + lane] = __uint_as_float(v[c]);
            }
            __syncwarp();
            if (lane < split) bar_arrive_cluster_release(in_cta(smem_addr(&ex_full_), lane));
            ok = warp_wait<true>(smem_addr(&ex_full_), 0, gave_up);
        }
        const int width = ok ? (t.cols + split - 1) / split : 0;
        for (int i = thread; i < width * (kTileM / 8); i += 32 * kEpilogueWarps) {
            const int c = part * width + i / (kTileM / 8), f = i % (kTileM / 8) * 8, feature = t.m0 + f;
            if (c >= t.cols || feature >= a.M) continue;
            const size_t at = ((MODE == kDweight ? (size_t)t.e * a.N + t.c0 : (size_t)t.c0) + c) * ld + feature;
            float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            uint4 operand = make_uint4(0u, 0u, 0u, 0u);
            if (MODE == kForward) {
                if (a.bias) unpack8(__ldg(reinterpret_cast<const uint4 *>(a.bias + (size_t)t.e * a.M + feature)), bias);
                if (a.operand) operand = *reinterpret_cast<const uint4 *>(a.operand + at);
            }
            const uint32_t from = smem_addr(mine + c * kExchangeLd + f);
            for (int s = 0; s < split; ++s) {
                const float4 lo = load_cluster(in_cta(from, s)), hi = load_cluster(in_cta(from, s) + 16);
                z[0] += lo.x, z[1] += lo.y, z[2] += lo.z, z[3] += lo.w, z[4] += hi.x, z[5] += hi.y, z[6] += hi.z, z[7] += hi.w;
            }
            finish_row<MODE>(a, z, bias, operand, at);
        }
    } else if (warp >= 4) {
        // ---- accumulators out
        const int q = warp & 3, first = (warp - 4) / 4 * 32;                 // a warp reaches the lanes 32 (warp mod 4) .. + 31
        constexpr int kStep = kEpilogueWarps / 4 * 32;
        uint32_t *stage = reinterpret_cast<uint32_t *>(tables) + (warp - 4) * kStageWords;
        const bool words = MODE == kForward && (a.operand || a.pre);         // fp32 through the buffer, or rounded pairs of columns
        const int my_col = (lane >> 2) * (words ? 1 : 2), my_seg = (lane & 3) * 8;
        const size_t ld = a.M;
        int used = 0;
        while (walk.next(t)) {
            if (t.nk == 0) continue;
            const int feature = t.m0 + rank * kTileM + q * 32 + my_seg;
            const bool live = feature < a.M;                                 // M is a multiple of 8
            const int acc = used & 1;
            const uint32_t from = tmem + (uint32_t(q * 32) << 16) + acc * kAccColumns;
            const size_t corner = ((MODE == kDweight ? (size_t)t.e * a.N + t.c0 : (size_t)t.c0) + my_col) * ld + feature;
            const int cols = live ? t.cols - my_col : 0;                     // column c + my_col of the tile is real iff c < cols
            uint4 r[4];                                                      // the operand of the lane's four columns of a block
            float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, lane_bias = 0.f;
            if (MODE == kForward && !words) {                                // the lane's own feature
                const int mine = t.m0 + rank * kTileM + q * 32 + lane;
                if (a.bias && mine < a.M) lane_bias = __uint_as_float((uint32_t)__ldg(a.bias + (size_t)t.e * a.M + mine) << 16);
            } else if (MODE == kForward) {
                if (a.bias && live) unpack8(__ldg(reinterpret_cast<const uint4 *>(a.bias + (size_t)t.e * a.M + feature)), bias);
                if (a.operand)                                               // under the products
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (first + 8 * i < cols) r[i] = *reinterpret_cast<const uint4 *>(a.operand + corner + (first + 8 * i) * ld);
            }
            if (!warp_wait(smem_addr(&acc_full_[acc]), (used >> 1) & 1, gave_up)) break;
            tmem_fence_after();
            const auto release = [&] {                                       // this warp has read its last column of the accumulator
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(in_cta(smem_addr(&acc_empty_[acc]), 0));
            };
            for (int c0 = first; c0 < t.cols; c0 += kStep) {
                uint32_t v[32];
                tmem_load32(from + c0, v);
                if (c0 + kStep >= t.cols) release();
                if (words) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (c0 + 16 * h >= t.cols) break;
                        __syncwarp();
#pragma unroll
                        for (int c = 0; c < 16; ++c) stage[c * kStageLd + lane] = v[16 * h + c];
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int c = c0 + 16 * h + 8 * i;
                            if (c < cols) {
                                const uint4 *src = reinterpret_cast<const uint4 *>(stage + (8 * i + my_col) * kStageLd + my_seg);
                                const uint4 lo = src[0], hi = src[1];
                                const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                                float z[8];
#pragma unroll
                                for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(w[j]);
                                const size_t at = corner + c * ld;
                                const uint4 mine = r[2 * h + i];
                                // the same columns of the warp's next block (the operand may be y itself: an ordinary load)
                                if (a.operand && c + kStep < cols)
                                    r[2 * h + i] = *reinterpret_cast<const uint4 *>(a.operand + at + kStep * ld);
                                finish_row<MODE>(a, z, bias, mine, at);
                            }
                        }
                    }
                } else {
                    // nothing else to read: a word carries two columns' results, rounded
                    if (MODE == kForward) {
                        switch (a.activation) {
                        case EP_ACT_RELU: act_all<EP_ACT_RELU>(v, lane_bias); break;
                        case EP_ACT_SILU: act_all<EP_ACT_SILU>(v, lane_bias); break;
                        case EP_ACT_GELU: act_all<EP_ACT_GELU>(v, lane_bias); break;
                        default: act_all<EP_ACT_NONE>(v, lane_bias); break;
                        }
                    }
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        stage[c * kStageLd + lane] = pack_bf16x2(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1]));
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int c = c0 + 16 * i;
                        if (c < cols) {
                            const uint4 *src = reinterpret_cast<const uint4 *>(stage + (8 * i + (lane >> 2)) * kStageLd + my_seg);
                            const uint4 lo = src[0], hi = src[1];
                            uint16_t *dst = a.out + corner + c * ld;
                            *reinterpret_cast<uint4 *>(dst) = make_uint4(__byte_perm(lo.x, lo.y, 0x5410), __byte_perm(lo.z, lo.w, 0x5410),
                                                                         __byte_perm(hi.x, hi.y, 0x5410), __byte_perm(hi.z, hi.w, 0x5410));
                            if (c + 1 < cols)
                                *reinterpret_cast<uint4 *>(dst + ld) =
                                    make_uint4(__byte_perm(lo.x, lo.y, 0x7632), __byte_perm(lo.z, lo.w, 0x7632),
                                               __byte_perm(hi.x, hi.y, 0x7632), __byte_perm(hi.z, hi.w, 0x7632));
                        }
                    }
                }
            }
            if (first >= t.cols) release();
            ++used;
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (gave_up_) {                                                          // whoever did: copies and products may be under way
        int none = 0;
        for (; in_flight > 0; --in_flight) {
            if (next_stage == 0) next_stage = a.stages, next_phase ^= 1;
            --next_stage;
            bar_wait(full0 + 8 * next_stage, next_phase, &none);
            none = 0;
        }
        if (warp == 1 && rank == 0 && elect_one()) {
            mma_commit<CG>(smem_addr(&done_));
            bar_wait(smem_addr(&done_), 0, &none);
        }
        __syncthreads();
    }
    if (CG == 2 || SPLIT) cluster_sync();                                    // the others' signals land in, and their reads come from, this CTA's memory
    tmem_fence_after();
    if (warp == 2) tmem_free<CG>(tmem, 2 * kAccColumns);
    if (threadIdx.x == 0 && gave_up_ && a.status) atomicOr(a.status, EP_STATUS_TIMEOUT);
}

// One pair of tensor maps per expert that end with its segment: {x, dz} of rows [0, bound[e+1]). An expert without rows gets its
// zeros here, from all blocks (e, *): the gradients of 240 experts of 5888 x 144, most of them without rows, take 161 us so, 211
// with one block per expert.
__global__ void __launch_bounds__(256)
segment_maps_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_dz, const int32_t *offsets,
                    long long rows, CUtensorMap *out, uint4 *dweight, long long vecs)
{
    __shared__ alignas(128) uint32_t work[2][32];
    const int e = blockIdx.x, lane = threadIdx.x & 31;
    pdl_trigger();
    pdl_wait();
    const int begin = segment_bound(__ldg(offsets + e), rows), end = segment_bound(__ldg(offsets + e + 1), rows);
    if (end <= begin) {
        uint4 *dst = dweight + (size_t)e * vecs;
        for (long long v = (long long)blockIdx.y * 256 + threadIdx.x; v < vecs; v += (long long)gridDim.y * 256)
            st_stream(dst + v, make_uint4(0u, 0u, 0u, 0u));
    }
    if (blockIdx.y || threadIdx.x >= 32) return;
    work[0][lane] = reinterpret_cast<const uint32_t *>(&map_x)[lane];
    work[1][lane] = reinterpret_cast<const uint32_t *>(&map_dz)[lane];
    __syncwarp();
    for (int i = 0; i < 2; ++i) {
        const uint32_t s = smem_addr(work[i]);
        if (lane == 0)
            asm volatile("tensormap.replace.tile.global_dim.shared::cta.b1024.b32 [%0], 1, %1;" ::"r"(s), "r"(max(1, end)) : "memory");
        __syncwarp();
        asm volatile("tensormap.cp_fenceproxy.global.shared::cta.tensormap::generic.release.gpu.sync.aligned [%0], [%1], 128;" ::"l"(
                         out + 2 * (size_t)e + i),
                     "r"(s)
                     : "memory");
    }
}

// ---- dz = dy * (operand) * act'(pre), doperand = dy * act(pre), and the partial sums of dbias -------------------------
// A warp owns 256 columns (8 a lane) and a run of rows; three 16-byte loads and one or two 16-byte stores per row and lane:
// bound by memory, with gelu by instruction issue (erff). 32768 rows of 1024 features, silu and a multiplied operand, doperand and dbias:
// 61 us with the sums' kernel, the bytes take 41; 32768 of 2048, gelu, dbias alone: 120 and 41. A run is cut where a segment ends: chunk c and expert e share at most one piece, and c + e grows along
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

template <int ACT>
__global__ void __launch_bounds__(kSlopeWarps * 32, 8)
slope_kernel(const SlopeArgs a)
{
    pdl_trigger();
    pdl_wait();
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
    while (p < end) {
        long long stop = end;
        if (a.partial) {
            int next;
            while ((next = segment_bound(__ldg(a.offsets + e + 1), a.rows)) <= p) ++e;   // ends: bound[E] = total > p
            stop = min(end, (long long)next);
        }
        float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (; live && p < stop; ++p) {
            const size_t at = (size_t)p * a.vecs + vec;
            uint4 z = make_uint4(0u, 0u, 0u, 0u), r = z;
            const uint4 g = ld_stream(a.dy + at);
            if (ACT != EP_ACT_NONE || a.doperand) z = ld_stream(a.pre + at);
            if (a.operand) r = ld_stream(a.operand + at);
            float fg[8], fz[8], fr[8], o[8];
            unpack8(g, fg);
            unpack8(z, fz);
            unpack8(r, fr);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float value = 0.f, slope = 1.f;
                if (ACT != EP_ACT_NONE || a.doperand) act_both(ACT, fz[j], value, slope);
                o[j] = fg[j] * value;
                if (a.operand) fg[j] *= fr[j];
                fg[j] *= slope;
                sum[j] += fg[j];
            }
            if (a.doperand) st_stream(a.doperand + at, pack8(o));
            if (a.dz) a.dz[at] = pack8(fg);
        }
        p = stop;
        if (a.partial && live) {
            float4 *dst = reinterpret_cast<float4 *>(a.partial + ((size_t)(chunk + e) * a.vecs + vec) * 8);
            dst[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            dst[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        }
    }
}

// dbias[e][n] = sum of the expert's pieces, a thread per column; with many pieces per expert eight threads per column take a run of
// them each, and the eight sums are added in order (SPLIT), in blocks of 32 columns instead of 256: 128 experts of 1024 columns and
// eight pieces each, unevenly, 437 us for all gradients with eight, 446 with one; 240 experts of 5888 columns and hardly a row, the
// other way round, 229 and 212.
template <int SPLIT>
__global__ void __launch_bounds__(256)
bias_grad_kernel(const float *__restrict__ partial, const int32_t *__restrict__ offsets, long long rows, int N, int chunk, float *dbias)
{
    constexpr int kColumns = 256 / SPLIT;
    __shared__ float part[SPLIT][kColumns];
    pdl_trigger();
    pdl_wait();
    const int e = blockIdx.y, col = threadIdx.x % kColumns, w = threadIdx.x / kColumns, n = blockIdx.x * kColumns + col;
    const int begin = segment_bound(__ldg(offsets + e), rows), end = segment_bound(__ldg(offsets + e + 1), rows);
    float s = 0.f;
    if (begin < end && n < N) {
        const int c0 = begin / chunk, count = (end - 1) / chunk - c0 + 1, per = (count + SPLIT - 1) / SPLIT;
        const int from = c0 + min(count, w * per), to = c0 + min(count, w * per + per);
#pragma unroll 8
        for (int c = from; c < to; ++c) s += __ldg(partial + (size_t)(c + e) * N + n);
    }
    if (SPLIT > 1) {
        part[w][col] = s;
        __syncthreads();
        if (w) return;
#pragma unroll
        for (int i = 1; i < SPLIT; ++i) s += part[i][col];
    }
    if (n < N) dbias[(size_t)e * N + n] = s;
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

template <int MODE, int CG, bool SPLIT>
int launch_product(ProductArgs a, const CUtensorMap &map_a, const ColumnMaps &map_b, int64_t max_tiles, cudaStream_t stream)
{
    static std::atomic<int> sm_counts[64] = {};                              // per device; set once the shared memory limit is raised
    int dev = 0;
    EP_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return EP_ERR_INVALID_ARG;
    int sms = sm_counts[dev].load();
    if (sms == 0) {
        EP_CUDA_TRY(cudaFuncSetAttribute(product_kernel<MODE, CG, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit - 1024));
        EP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        sm_counts[dev].store(sms);
    }
    const int stage = kBytesA + (a.columns / CG < 32 ? 32 : a.columns / CG) * kTileK * 2;
    const int tables = (SPLIT ? kExchangeBytes : kStageBytes) + 2 * (a.E + 1) * 4;
    a.stages = (kSmemLimit - 2048 - tables) / stage;                         // 2048: alignment of the ring, static words
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    int smem = 1024 + a.stages * stage + tables;
    if (smem < 120 * 1024) smem = 120 * 1024;                                // one CTA per SM: it holds all of the tensor memory
    const int sharing = SPLIT ? a.split : CG;
    int64_t groups = sms / sharing;
    if (max_tiles < groups || SPLIT) groups = max_tiles;                     // a shared tile has a cluster of its own
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * sharing));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = sharing;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    EP_CUDA_TRY(cudaLaunchKernelEx(&cfg, product_kernel<MODE, CG, SPLIT>, a, map_a, map_b));
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

// Picks the launch for tiles of at most a.columns columns. `pieces(columns)`: column tiles over all experts; `stages`: 64-element
// stages of the contracted axis of an average tile.
template <int MODE, class Pieces>
int launch_tiles(ProductArgs a, const CUtensorMap &map_a, const ColumnMaps &map_b, Pieces pieces, int64_t stages, cudaStream_t stream)
{
    const int64_t features = (a.M + kTileM - 1) / kTileM, pairs = (a.M + 2 * kTileM - 1) / (2 * kTileM);
    // Pairs of CTAs (256 features per tile, each operand row fetched once for both) wherever there is work for all pairs; with few
    // rows per expert the time is that of reading the weights and single CTAs spread it better. 128 experts of 1024 x 2048 on one
    // box: 16 rows each 86.9 us single, 88.9 paired; 256 experts of 2048 x 7168, 256 rows each: 1989 single, 1728 paired.
    if (a.columns >= 128 && pieces(a.columns) * pairs >= 74) return launch_product<MODE, 2, false>(a, map_a, map_b, pieces(a.columns) * pairs, stream);
    // Fewer tiles than SMs: narrower tiles, then CTAs that share a tile (at least four stages each).
    while (a.columns > kSplitColumns && pieces(a.columns) * features < 148) a.columns /= 2;
    const int64_t tiles = pieces(a.columns) * features;
    if (tiles >= (int64_t(1) << 31) - (1 << 20)) return EP_ERR_INVALID_ARG;
    a.split = 1;
    while (a.split < 8 && tiles * a.split * 2 <= 148 && stages >= 8 * a.split) a.split *= 2;
    if (a.split > 1) return launch_product<MODE, 1, true>(a, map_a, map_b, tiles, stream);
    return launch_product<MODE, 1, false>(a, map_a, map_b, tiles, stream);
}

int make_row_maps(TensorMapEncode encode, ColumnMaps *maps, const void *rows, int features, int64_t n)
{
    for (int b = 0; b < 4; ++b) {
        const int rc = make_map(encode, &maps->box[b], rows, features, n, 1, 128 >> b);
        if (rc != EP_OK) return rc;
    }
    return EP_OK;
}

// Columns (rows p) per tile: as many as an expert has on average, in powers of two, so that most experts are one tile.
int row_columns(int64_t rows, int E)
{
    int c = 64;
    while (c < kAccColumns && (int64_t)c * E < rows + rows / 2) c *= 2;
    return c;
}

template <int MODE>
int launch_rows(const ProductArgs &a, const CUtensorMap &map_a, const ColumnMaps &map_b, cudaStream_t stream)
{
    const auto pieces = [&](int columns) { return (a.rows < a.E ? a.rows : a.E) + a.rows / columns; };   // at most
    return launch_tiles<MODE>(a, map_a, map_b, pieces, (a.K + kTileK - 1) / kTileK, stream);
}

// Rows per run of the slope kernel: about 40 warps per SM (a warp is one run of 256 columns), runs of at least 8 rows, and no
// more than 1024 of them, which the second kernel adds up.
int slope_chunk(int64_t rows, int features)
{
    const int64_t strips = (features + 255) / 256, runs = 148 * 40 / strips + 1;
    int64_t c = (rows + runs - 1) / runs;
    if (c < (rows + 1023) / 1024) c = (rows + 1023) / 1024;
    return (int)(c < 8 ? 8 : (c + 1) / 2 * 2);
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

size_t maps_bytes(const ep_matmul_t &m) { return up256(sizeof(CUtensorMap) * 2 * (size_t)m.num_experts); }
size_t partial_bytes(const ep_matmul_t &m)
{
    const int chunk = slope_chunk(m.rows, m.out_features);
    const size_t chunks = (m.rows + chunk - 1) / chunk;
    return up256((chunks + m.num_experts) * (size_t)m.out_features * 4);
}
size_t dz_bytes(const ep_matmul_t &m) { return up256((size_t)m.rows * m.out_features * 2); }

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
    CUtensorMap map_w;
    ColumnMaps map_x;
    rc = make_map(encode, &map_w, weight, m->in_features, m->out_features, m->num_experts, kTileM);
    if (rc == EP_OK) rc = make_row_maps(encode, &map_x, x, m->in_features, m->rows);
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
    return launch_rows<kForward>(a, map_w, map_x, static_cast<cudaStream_t>(stream_));
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
        s.chunk = slope_chunk(m->rows, (int)N);
        const int64_t chunks = (m->rows + s.chunk - 1) / s.chunk;
        const dim3 grid(ceil_div(s.vecs, 32), (unsigned)((chunks + kSlopeWarps - 1) / kSlopeWarps));
        void (*kernel)(const SlopeArgs) = m->activation == EP_ACT_RELU   ? slope_kernel<EP_ACT_RELU>
                                          : m->activation == EP_ACT_SILU ? slope_kernel<EP_ACT_SILU>
                                          : m->activation == EP_ACT_GELU ? slope_kernel<EP_ACT_GELU>
                                                                         : slope_kernel<EP_ACT_NONE>;
        EP_CUDA_TRY(launch_pdl(kernel, grid, dim3(kSlopeWarps * 32), 0, stream, s));
        EP_LAUNCH_CHECK(1);
        if (dbias) {
            const bool many = chunks > (int64_t)E;
            EP_CUDA_TRY(launch_pdl(many ? bias_grad_kernel<8> : bias_grad_kernel<1>,
                                   dim3((unsigned)((N + (many ? 31 : 255)) / (many ? 32 : 256)), (unsigned)E), dim3(256), 0, stream,
                                   partial, expert_offsets, (long long)m->rows, (int)N, s.chunk, dbias));
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
    CUtensorMap map_a;
    ColumnMaps map_b;
    if (dx) {
        rc = make_map(encode, &map_a, weight, H, N, E, kTileK);
        if (rc == EP_OK) rc = make_row_maps(encode, &map_b, dz, N, m->rows);
        if (rc != EP_OK) return rc;
        a.M = m->in_features, a.K = m->out_features, a.N = 0;
        a.out = static_cast<uint16_t *>(dx);
        a.columns = row_columns(m->rows, m->num_experts);
        rc = launch_rows<kDx>(a, map_a, map_b, stream);
        if (rc != EP_OK) return rc;
    }
    if (dweight) {
        rc = make_map(encode, &map_a, x, H, m->rows, 1, kTileK);
        if (rc == EP_OK) rc = make_map(encode, &map_b.box[0], dz, N, m->rows, 1, kTileK);
        if (rc != EP_OK) return rc;
        const unsigned share = E >= 592 ? 2 : (unsigned)(1184 / E);           // blocks per expert: eight per SM, were all without rows
        EP_CUDA_TRY(launch_pdl(segment_maps_kernel, dim3((unsigned)E, share), dim3(256), 0, stream, map_a, map_b.box[0], expert_offsets,
                               (long long)m->rows, maps, static_cast<uint4 *>(dweight), (long long)(N * H / 8)));
        EP_LAUNCH_CHECK(1);
        a.M = m->in_features, a.N = m->out_features, a.K = 0;
        a.out = static_cast<uint16_t *>(dweight);
        a.segment_maps = maps;
        a.columns = kAccColumns;
        const auto pieces = [&](int columns) { return (int64_t)a.E * ((a.N + columns - 1) / columns); };
        rc = launch_tiles<kDweight>(a, map_a, map_b, pieces, m->rows / m->num_experts / kTileK, stream);
        if (rc != EP_OK) return rc;
    }
    return EP_OK;
}
