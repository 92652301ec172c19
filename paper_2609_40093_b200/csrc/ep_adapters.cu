// Low-rank adapters beside a shared projection, and their gradients.
//
//   forward   mid = x down[a]^T                   y[row]  = base[row] + scale[a] * mid up[a]^T          rows of adapter a
//   backward  dmid = scale[a] * dy up[a]          dx[row] = base[row] + dmid down[a]
//             ddown[a] = dmid^T x                 dup[a] = scale[a] * dy^T mid                          sums over the rows
//
// The first two lines are one kernel, the rank kernel: in -> (rank) -> out with the weights read along either axis. A tile is
// up to 128 rows of one adapter, the lanes of the accumulators; its rows may lie anywhere (tile::gather4 copies, four rows each).
// The first product contracts the features into at most 128 columns of tensor memory; they are rounded to bf16 (they are the operand of
// another product), laid out in shared memory as that product's row operand, and the output follows in blocks of 128 columns, whose
// epilogue adds to `base` in fp32 and rounds once. Nothing between the products goes through memory.
// Where there are few tiles, up to eight CTAs of a cluster share one: each contracts a part of the features, all add the parts through each
// other's shared memory in a fixed order, and each makes a part of the output's blocks. So a token that is generated alone has
// its adapter's weights read by eight SMs.
//
// The two sums over rows are the gradient kernel: 128 features are the lanes, the rank the columns, the rows are contracted. Entries behind
// the segment's end are read at a row that does not exist, which gives zeros for both operands whatever the memory holds.
#include <atomic>

#include "ep_tensor.cuh"

namespace ep {
namespace {

constexpr int kRows = 128;                // rows of a tile
constexpr int kTileK = 64;                // contracted elements per stage: one 128-byte line
constexpr int kLines = kRows * 128;       // bytes of 128 lines
constexpr int kBlockColumns = 128;        // output columns of one accumulator
constexpr int kMaxRank = 128;
constexpr int kMaxCluster = 8;

// a / b rounded up, for a up to 2^31 - 1
__device__ __forceinline__ int quotient_up(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) / (unsigned)b); }

__device__ __forceinline__ int segment_bound(int32_t v, long long entries) { return v < 0 ? 0 : (v > entries ? (int)entries : v); }

// 16 bytes from global to shared memory, in the background; zeros where `there` is false.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void copy_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All groups of this thread but the last N have landed.
template <int N>
__device__ __forceinline__ void copy_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Where 16-byte piece `piece` of line `line` lies in a tile with the 128-byte swizzle.
__device__ __forceinline__ uint32_t swizzled(int line, int piece) { return line * 128 + ((piece ^ (line & 7)) << 4); }

// What this thread wrote to shared memory is there for the tensor cores.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void store_cluster(uint32_t addr, const uint4 &v)
{
    asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// 16 accumulator columns of this warp's 32 lanes, and the wait for them: nothing reads v in between.
__device__ __forceinline__ void tmem_request16(uint32_t addr, uint32_t (&v)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void tmem_wait16(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                   "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}

// Bytes (a multiple of 16, from a 16-byte boundary) on their way into L2.
__device__ __forceinline__ void l2_prefetch(const void *p, uint32_t bytes)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

// ---- the rank kernel ----------------------------------------------------------------------------------------------

constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
// Shared memory. The stages of the first product take 96 KB (a stage: 128 lines of rows and 64 or 128 lines of weights); afterwards
// the same memory holds the row operand of the second (16 or 32 KB), the epilogue's buffers (16 KB for every 32 rows) and one to five
// blocks of the weights (16 KB each); barriers and tables follow. What the CTAs of a cluster exchange lies in the epilogue's buffers. Two CTAs
// fit on an SM, so that one reads while the other writes; 113 KB each also keep a CTA of the experts' products, which holds all of the
// tensor memory, from sharing an SM with one of a cluster: two clusters that each wait for the other's would wait for good.
constexpr int kRingBytes = 96 * 1024, kAreaBytes = 112 * 1024;
constexpr int kBufferBytes = 32 * 128;    // an epilogue warp's 32 rows x 64 columns of bf16; two of them
constexpr int kMaxStages = 4, kMaxUnits = 5;
constexpr int kLag = 2;                   // stages a loader has in flight behind the one it asks for

struct RankTables {
    uint64_t full[kMaxStages], empty[kMaxStages], unit_full[kMaxUnits], unit_empty[kMaxUnits], mid_full, mid_ready, acc_full[2], acc_empty[2],
        ex_full;
    uint32_t tmem_slot;
    int gave_up, warp_sum[kThreads / 32], where[3];
    int row_of[kRows];
};
constexpr int kRankSmem = kAreaBytes + 1024;
static_assert(sizeof(RankTables) <= 1024, "two CTAs per SM");

struct RankArgs {
    const int32_t *offsets;               // [A+1]
    const int32_t *index;                 // entry -> row, or NULL: entry i is row i
    int32_t *status;
    const float *scale;                   // [A] or NULL
    const uint16_t *base;                 // [rows][out], may be NULL or `out`
    uint16_t *out;                        // [rows][out], may be NULL: the first product alone
    uint16_t *mid;                        // [entries][rank], may be NULL
    long long rows, entries;
    const uint16_t *in_rows, *second;     // [rows][in]; the second product's weights
    int in, out_features, rank, A, split, width;      // width: rows of a tile at most
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

// BACK: the weights are read along the other axis (up for the first product, down for the second), and the scale goes to `mid`.
template <bool BACK>
__global__ void __launch_bounds__(kThreads, 2)
rank_kernel(const RankArgs a, const __grid_constant__ CUtensorMap map_first, const __grid_constant__ CUtensorMap map_second)
{
    extern __shared__ __align__(1024) char area[];                           // no static shared memory: it would push the area off its boundary
    RankTables &tab = *reinterpret_cast<RankTables *>(area + kAreaBytes);
    int *const warp_sum = tab.warp_sum, *const where = tab.where, *const row_of = tab.row_of;
    volatile int *gave_up = &tab.gave_up;

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int split = a.split, part = split > 1 ? (int)cluster_rank() : 0;
    const int tile = blockIdx.x / split;

    pdl_wait();                                                              // nothing is read or written before this
    // ---- this cluster's tile: each thread counts the tiles of a run of adapters
    if (threadIdx.x == 0) where[0] = -1;
    {
        const int per = (a.A + kThreads - 1) / kThreads, from = min(a.A, (int)threadIdx.x * per), to = min(a.A, from + per);
        int sum = 0, begin = from < to ? segment_bound(__ldg(a.offsets + from), a.entries) : 0;
        const int first = begin;
        for (int i = from; i < to; ++i) {
            const int end = segment_bound(__ldg(a.offsets + i + 1), a.entries);
            sum += quotient_up(max(0, end - begin), a.width);
            begin = end;
        }
        int scan = sum;
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(kFullMask, scan, d);
            if (lane >= d) scan += v;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        int run = scan - sum;
        for (int w = 0; w < warp; ++w) run += warp_sum[w];
        if (tile >= run && tile < run + sum) {                               // one thread: the tile is one of its adapters'
            begin = first;
            for (int i = from; i < to; ++i) {
                const int end = segment_bound(__ldg(a.offsets + i + 1), a.entries), count = max(0, end - begin);
                const int pieces = quotient_up(count, a.width);
                if (tile < run + pieces) {
                    const int width = (quotient_up(count, pieces) + 3) & ~3, piece = tile - run;
                    where[0] = i;
                    where[1] = begin + piece * width;
                    where[2] = max(0, min(width, count - piece * width));
                    break;
                }
                run += pieces;
                begin = end;
            }
        }
        if (threadIdx.x == 0 && blockIdx.x == 0 && a.status && __ldg(a.offsets + a.A) > a.entries) atomicOr(a.status, EP_STATUS_CAPACITY);
        __syncthreads();
    }
    const int adapter = where[0], entry0 = where[1], m = where[2];
    if (adapter < 0 || m == 0) return;                                       // all CTAs of the cluster

    const int chunks = (a.rank + 63) / 64, r16 = (a.rank + 15) & ~15;
    const int all_k = (a.in + kTileK - 1) / kTileK, k_from = all_k * part / split, k_to = all_k * (part + 1) / split;
    const int blocks = a.out ? (a.out_features + kBlockColumns - 1) / kBlockColumns : 0;
    const int b_from = (int)((long long)blocks * part / split), b_to = (int)((long long)blocks * (part + 1) / split);
    const int stage_bytes = kLines + chunks * 8192, stages = kRingBytes / stage_bytes;
    const int loaders = min(kEpilogueWarps, (m + 3) / 4), quarters = (m + 31) / 32;        // warps that bring rows; quarters of the lanes with rows
    const bool narrow = quarters == 1;                                       // each quarter of the lanes holds the same rows, see below
    const int units = kAreaBytes / kLines - chunks - quarters;
    const uint32_t ring = smem_addr(area), unit_base = ring + (chunks + quarters) * kLines;
    char *const buffers = area + chunks * kLines;
    float *const exchange = reinterpret_cast<float *>(buffers);              // [m][r16], 16-byte pieces turned so that neither axis meets a bank twice
    const int ex_turn = r16 % 32 == 0 ? 7 : 6;
    const auto ex_at = [&](int row, int piece) { return row * r16 + ((piece ^ (ex_turn == 7 ? row & 7 : (row & 6) >> 1)) << 2); };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) bar_init(smem_addr(&tab.full[s]), 1 + loaders), bar_init(smem_addr(&tab.empty[s]), 1);
        for (int s = 0; s < kMaxUnits; ++s) bar_init(smem_addr(&tab.unit_full[s]), 1), bar_init(smem_addr(&tab.unit_empty[s]), 1);
        for (int s = 0; s < 2; ++s) bar_init(smem_addr(&tab.acc_full[s]), 1), bar_init(smem_addr(&tab.acc_empty[s]), narrow ? kEpilogueWarps : 2 * quarters);
        bar_init(smem_addr(&tab.mid_full), 1);
        bar_init(smem_addr(&tab.mid_ready), split * kEpilogueWarps);
        bar_init(smem_addr(&tab.ex_full), split * kEpilogueWarps);
        tab.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_addr(&tab.tmem_slot), 2 * kBlockColumns);
    for (int i = threadIdx.x; i < kRows; i += kThreads) {
        int row = -1;
        if (i < m) {
            row = a.index ? __ldg(a.index + entry0 + i) : entry0 + i;
            if (row < 0 || row >= a.rows) {
                if (a.status) atomicOr(a.status, EP_STATUS_BAD_INDEX);
                row = -1;
            }
        }
        row_of[i] = row;
    }
    tmem_fence_before();
    if (split > 1) cluster_sync();
    __syncthreads();
    tmem_fence_after();
    pdl_trigger();
    const uint32_t tmem = tab.tmem_slot;
    const uint32_t full0 = smem_addr(tab.full), empty0 = smem_addr(tab.empty), unit_full0 = smem_addr(tab.unit_full), unit_empty0 = smem_addr(tab.unit_empty);

    if (warp == 0 && elect_one()) {
        // ---- weights
        const uint32_t bytes = (uint32_t)(BACK ? chunks * 8192 : r16 * 128);
        int s = 0, phase = 1, sent = 0;
        bool ok = true;
        for (int k = k_from; k < k_to; ++k) {
            if (!(ok = bar_wait(empty0 + 8 * s, phase, gave_up))) break;
            const uint32_t full = full0 + 8 * s, dst = ring + s * stage_bytes + kLines;
            bar_expect(full, bytes);
            if (BACK) {
                for (int u = 0; u < chunks; ++u) tma_load<1>(dst + u * 8192, &map_first, 64 * u, k * kTileK, adapter, full);
            } else {
                tma_load<1>(dst, &map_first, k * kTileK, 0, adapter, full);
            }
            ++sent;
            if (b_to > b_from && b_to - b_from <= 16 && sent == min(stages, k_to - k_from)) {
                // few blocks a CTA: nobody else has brought the second weights into L2
                const int col = b_from * kBlockColumns, cols = min(b_to * kBlockColumns, a.out_features) - col;
                if (BACK)
                    for (int j = 0; j < a.rank; ++j) l2_prefetch(a.second + ((size_t)adapter * a.rank + j) * a.out_features + col, cols * 2);
                else
                    l2_prefetch(a.second + ((size_t)adapter * a.out_features + col) * a.rank, cols * a.rank * 2);
            }
            if (++s == stages) s = 0, phase ^= 1;
        }
        if (!ok) {                                                           // gave up: let the copies in flight land
            for (int i = min(sent, stages); i > 0; --i) {
                int none = 0;
                if (s == 0) s = stages, phase ^= 1;
                --s;
                bar_wait(full0 + 8 * s, phase ^ 1, &none);
            }
        } else if (blocks) {
            // ---- the second weights, once the ring's memory is free
            ok = bar_wait(smem_addr(&tab.mid_full), 0, gave_up);
            int u = 0, uphase = 1, usent = 0;
            for (int b = b_from; ok && b < b_to; ++b)
                for (int c = 0; c < chunks; ++c) {
                    if (!(ok = bar_wait(unit_empty0 + 8 * u, uphase, gave_up))) break;
                    const uint32_t full = unit_full0 + 8 * u, dst = unit_base + u * kLines;
                    bar_expect(full, kLines);
                    if (BACK) {
                        tma_load<1>(dst, &map_second, b * kBlockColumns, 64 * c, adapter, full);
                        tma_load<1>(dst + 8192, &map_second, b * kBlockColumns + 64, 64 * c, adapter, full);
                    } else {
                        tma_load<1>(dst, &map_second, 64 * c, b * kBlockColumns, adapter, full);
                    }
                    ++usent;
                    if (++u == units) u = 0, uphase ^= 1;
                }
            if (!ok)
                for (int i = min(usent, units); i > 0; --i) {
                    int none = 0;
                    if (u == 0) u = units, uphase ^= 1;
                    --u;
                    bar_wait(unit_full0 + 8 * u, uphase ^ 1, &none);
                }
        }
    } else if (warp == 1 && elect_one()) {
        // ---- products
        int s = 0, phase = 0;
        bool ok = true;
        const uint32_t idesc = instr_desc(kRows, r16, false, BACK);
        for (int k = k_from; k < k_to; ++k) {
            if (!(ok = bar_wait(full0 + 8 * s, phase, gave_up))) break;
            tmem_fence_after();
            const uint32_t at = ring + s * stage_bytes;
            const uint64_t da = desc_k_major(at), db = BACK ? desc_mn_major(at + kLines) : desc_k_major(at + kLines);
#pragma unroll
            for (int j = 0; j < kTileK / 16; ++j) mma_bf16<1>(tmem, da + j * 2, db + j * (BACK ? 128 : 2), idesc, k > k_from || j > 0);
            mma_commit<1>(empty0 + 8 * s);
            if (++s == stages) s = 0, phase ^= 1;
        }
        if (ok) mma_commit<1>(smem_addr(&tab.mid_full));
        if (ok && blocks) {
            ok = bar_wait<true>(smem_addr(&tab.mid_ready), 0, gave_up);
            fence_async();                                                   // what the cluster's other CTAs wrote, too
            tmem_fence_after();
            const uint32_t idesc2 = instr_desc(kRows, kBlockColumns, false, BACK);
            int u = 0, uphase = 0, used = 0;
            for (int b = b_from; ok && b < b_to; ++b, ++used) {
                const int acc = used & 1;
                if (!(ok = bar_wait(smem_addr(&tab.acc_empty[acc]), ((used >> 1) & 1) ^ 1, gave_up))) break;
                tmem_fence_after();
                for (int c = 0; c < chunks; ++c) {
                    if (!(ok = bar_wait(unit_full0 + 8 * u, uphase, gave_up))) break;
                    tmem_fence_after();
                    const uint32_t at = unit_base + u * kLines;
                    const uint64_t da = desc_k_major(ring + c * kLines), db = BACK ? desc_mn_major(at) : desc_k_major(at);
                    const int steps = min(4, (r16 - 64 * c) / 16);
                    for (int j = 0; j < steps; ++j)
                        mma_bf16<1>(tmem + acc * kBlockColumns, da + j * 2, db + j * (BACK ? 128 : 2), idesc2, c > 0 || j > 0);
                    mma_commit<1>(unit_empty0 + 8 * u);
                    if (++u == units) u = 0, uphase ^= 1;
                }
                if (ok) mma_commit<1>(smem_addr(&tab.acc_full[acc]));
            }
        }
    } else if (warp >= 2) {
        const int q = warp & 3, half = (warp - 2) >> 2, thread = threadIdx.x - 64;
        const int my_row = q * 32 + lane;                                    // a warp reaches the lanes 32 (warp mod 4) .. + 31
        const float scale = a.scale ? __ldg(a.scale + adapter) : 1.f, mid_scale = BACK ? scale : 1.f, out_scale = BACK ? 1.f : scale;
        bool ok = true;
        if (a.base && narrow && thread < m && b_to > b_from && row_of[thread] >= 0)       // few rows: their base into L2, under the first product
            l2_prefetch(a.base + (size_t)row_of[thread] * a.out_features + b_from * kBlockColumns,
                        (min(b_to * kBlockColumns, a.out_features) - b_from * kBlockColumns) * 2);
        if (warp - 2 < loaders) {
            // ---- rows into the ring: eight lanes a row's line, four rows a warp, every 32 rows
            const int line = 4 * (warp - 2) + (lane >> 3), piece = lane & 7, n_k = k_to - k_from;
            const uint16_t *src[4];
            bool there[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = row_of[line + 32 * i];
                there[i] = row >= 0;
                src[i] = a.in_rows + (size_t)max(row, 0) * a.in;
            }
            int s = 0, phase = 1, done = 0;
            for (int i = 0; i < n_k + kLag; ++i) {
                if (i < n_k) {
                    if (!(ok = __all_sync(kFullMask, bar_wait(empty0 + 8 * s, phase, gave_up)))) break;
                    const int col = (k_from + i) * kTileK + piece * 8, at = col < a.in ? col : 0;
                    const uint32_t dst = ring + s * stage_bytes + swizzled(line, piece);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (line + 32 * j < m) copy16(dst + j * 32 * 128, src[j] + at, there[j] && col < a.in);
                    if (++s == stages) s = 0, phase ^= 1;
                }
                copy_group();
                if (i >= kLag) {
                    copy_wait<kLag>();
                    fence_async();
                    __syncwarp();
                    if (lane == 0) bar_arrive(full0 + 8 * done);
                    if (++done == stages) done = 0;
                }
            }
            copy_wait<0>();
        }
        ok = ok && bar_wait(smem_addr(&tab.mid_full), 0, gave_up);
        tmem_fence_after();
        // 8 columns of a row, rounded: the second product's operand, and `mid`
        const auto rounded = [&](int row, int col, float (&f)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= mid_scale;
            const uint4 v = pack8(f);
            if (a.mid && row < m && col < a.rank) *reinterpret_cast<uint4 *>(a.mid + (size_t)(entry0 + row) * a.rank + col) = v;
            return v;
        };
        const auto operand_at = [&](int row, int col) { return (col >> 6) * kLines + swizzled(row, (col & 63) >> 3); };
        if (ok) {
            for (int c0 = half * 32; c0 < r16; c0 += 64) {
                uint32_t v[32];
                tmem_load32(tmem + (uint32_t(q * 32) << 16) + c0, v);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (c0 + 8 * j < r16) {
                        if (split == 1) {
                            float f[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[8 * j + i]);
                            const uint4 w = rounded(my_row, c0 + 8 * j, f);
                            if (!narrow) {
                                *reinterpret_cast<uint4 *>(area + operand_at(my_row, c0 + 8 * j)) = w;
                            } else if (q == 0) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(area + operand_at(32 * i + lane, c0 + 8 * j)) = w;
                            }
                        } else if (my_row < m) {
                            const int piece = c0 / 4 + 2 * j;
                            *reinterpret_cast<uint4 *>(exchange + ex_at(my_row, piece)) = make_uint4(v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3]);
                            *reinterpret_cast<uint4 *>(exchange + ex_at(my_row, piece + 1)) =
                                make_uint4(v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]);
                        }
                    }
            }
        }
        if (split > 1 && ok) {
            // ---- the parts of all CTAs: each CTA adds a share of the elements, in the order of the CTAs, and tells all of them
            __syncwarp();
            if (lane < split) bar_arrive_cluster_release(in_cta(smem_addr(&tab.ex_full), lane));
            ok = bar_wait<true>(smem_addr(&tab.ex_full), 0, gave_up);
            const int groups = r16 / 8;
            for (int i = thread * split + part; ok && i < m * groups; i += 32 * kEpilogueWarps * split) {
                const int row = i / groups, col = i % groups * 8;
                const uint32_t lo = smem_addr(exchange + ex_at(row, col / 4)), hi = smem_addr(exchange + ex_at(row, col / 4 + 1));
                float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                for (int s = 0; s < split; s += 2) {                         // split is a power of two; four reads under way
                    const float4 l0 = load_cluster(in_cta(lo, s)), h0 = load_cluster(in_cta(hi, s));
                    const float4 l1 = load_cluster(in_cta(lo, s + 1)), h1 = load_cluster(in_cta(hi, s + 1));
                    f[0] += l0.x, f[1] += l0.y, f[2] += l0.z, f[3] += l0.w, f[4] += h0.x, f[5] += h0.y, f[6] += h0.z, f[7] += h0.w;
                    f[0] += l1.x, f[1] += l1.y, f[2] += l1.z, f[3] += l1.w, f[4] += h1.x, f[5] += h1.y, f[6] += h1.z, f[7] += h1.w;
                }
                const uint4 v = rounded(row, col, f);
                const uint32_t to = ring + operand_at(row, col);
                for (int s = 0; s < split; ++s) {
                    store_cluster(in_cta(to, s), v);
                    if (narrow)
#pragma unroll
                        for (int i = 1; i < 4; ++i) store_cluster(in_cta(to + i * 32 * 128, s), v);
                }
            }
        }
        fence_async();
        tmem_fence_before();
        __syncwarp();
        if (lane < split) bar_arrive_cluster_release(in_cta(smem_addr(&tab.mid_ready), lane));
        if (split > 1) ok = ok && bar_wait<true>(smem_addr(&tab.mid_ready), 0, gave_up);     // all have read: the buffers are free
        // ---- blocks of the output. A warp has 32 rows and 64 columns of one: whole lines of `base` come into its buffer in the
        // background, a block ahead; there each lane adds its row's accumulators and rounds, and whole lines go out.
        char *const buffer = buffers + (2 * q + half) * 2 * kBufferBytes;
        const uint32_t buffer_at = smem_addr(buffer);
        const int piece = lane & 7;
        long long line_at[8];                                                // eight lanes a row's line, four rows a pass; < 0: no row
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = row_of[q * 32 + 4 * i + (lane >> 3)];
            line_at[i] = row < 0 ? -1 : (long long)row * a.out_features + half * 64 + piece * 8;
        }
        const auto request = [&](int b, int which) {
            const int col = b * kBlockColumns;
            if (a.base && b < b_to && col + half * 64 + piece * 8 < a.out_features) {
                const uint32_t to = buffer_at + which * kBufferBytes;
#pragma unroll
                for (int i = 0; i < 8; ++i)                                  // `base` may be the output: not through the read-only path
                    if (line_at[i] >= 0) copy16(to + swizzled(4 * i + (lane >> 3), piece), a.base + line_at[i] + col, true);
            }
            copy_group();
        };
        int used = 0;
        if (q < quarters && !narrow) request(b_from, 0);
        for (int b = b_from; ok && q < quarters && !narrow && b < b_to; ++b, ++used) {
            const int acc = used & 1;
            request(b + 1, acc ^ 1);
            copy_wait<1>();
            __syncwarp();
            if (!(ok = bar_wait(smem_addr(&tab.acc_full[acc]), (used >> 1) & 1, gave_up))) break;
            tmem_fence_after();
            char *const mine = buffer + acc * kBufferBytes;
            // 16 columns at a time, the next ones on their way
            const uint32_t from = tmem + (uint32_t(q * 32) << 16) + acc * kBlockColumns + half * 64;
            uint32_t v[2][16];
            tmem_request16(from, v[0]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                tmem_wait16(v[c & 1]);
                if (c < 3) {
                    tmem_request16(from + 16 * (c + 1), v[(c + 1) & 1]);
                } else {
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_addr(&tab.acc_empty[acc]));
                }
                uint4 *at[2];
                float f[2][8];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    at[j] = reinterpret_cast<uint4 *>(mine + swizzled(lane, 2 * c + j));
                    unpack8(a.base ? *at[j] : make_uint4(0u, 0u, 0u, 0u), f[j]);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[j][k] = fmaf(out_scale, __uint_as_float(v[c & 1][8 * j + k]), f[j][k]);
                    *at[j] = pack8(f[j]);
                }
            }
            __syncwarp();
            const int col = b * kBlockColumns;
            if (col + half * 64 + piece * 8 < a.out_features) {
                uint4 line[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) line[i] = *reinterpret_cast<const uint4 *>(mine + swizzled(4 * i + (lane >> 3), piece));
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (line_at[i] >= 0) *reinterpret_cast<uint4 *>(a.out + line_at[i] + col) = line[i];
            }
            __syncwarp();                                                    // the buffer may be written again
        }
        copy_wait<0>();
        // ... of up to 32 rows: every quarter of the lanes has them, and each of the eight warps 16 of a block's columns, straight from
        // the accumulators: 256 rows on 64 adapters of 2048 x 8192 take 0.3 us a block so, with one quarter's two warps at work 0.9
        if (narrow) {
            const int row = row_of[lane], first = (q * 2 + half) * 16;
            const long long at = row < 0 ? -1 : (long long)row * a.out_features + first;
            uint4 r[2];
            const auto ask = [&](int b) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = b * kBlockColumns + 8 * j;
                    r[j] = make_uint4(0u, 0u, 0u, 0u);
                    if (a.base && at >= 0 && b < b_to && col + first < a.out_features) r[j] = *reinterpret_cast<const uint4 *>(a.base + at + col);
                }
            };
            ask(b_from);
            for (int b = b_from; ok && b < b_to; ++b, ++used) {
                const int acc = used & 1;
                if (!(ok = bar_wait(smem_addr(&tab.acc_full[acc]), (used >> 1) & 1, gave_up))) break;
                tmem_fence_after();
                uint32_t v[16];
                tmem_request16(tmem + (uint32_t(q * 32) << 16) + acc * kBlockColumns + first, v);
                tmem_wait16(v);
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_addr(&tab.acc_empty[acc]));
                float f[2][8];
#pragma unroll
                for (int j = 0; j < 2; ++j) unpack8(r[j], f[j]);
                ask(b + 1);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = b * kBlockColumns + 8 * j;
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[j][k] = fmaf(out_scale, __uint_as_float(v[8 * j + k]), f[j][k]);
                    if (at >= 0 && col + first < a.out_features) *reinterpret_cast<uint4 *>(a.out + at + col) = pack8(f[j]);
                }
            }
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (split > 1) cluster_sync();                                           // the others' reads come from this CTA's memory
    tmem_fence_after();
    if (warp == 1) tmem_free<1>(tmem, 2 * kBlockColumns);
    if (threadIdx.x == 0 && tab.gave_up && a.status) atomicOr(a.status, EP_STATUS_TIMEOUT);
}

// ---- the gradient kernel ------------------------------------------------------------------------------------------

// One warp issues the products, four bring entries, four empty the accumulators, of which there are two, so that an item's results
// leave under the next one's products. SPLIT: a cluster shares an item, one item per cluster.
constexpr int kGradLoaders = 8;
constexpr int kGradThreads = 32 * (5 + kGradLoaders);
constexpr int kGradLd = kRows + 4;        // accumulators on their way out: [rank][128 features]
constexpr int kGradColumns = 16;          // of them at a time
constexpr int kGradOutBytes = kGradColumns * kGradLd * 4;

struct GradArgs {
    const int32_t *offsets, *index;
    const float *scale;
    const uint16_t *x, *dmid, *dy, *mid;
    uint16_t *ddown, *dup;
    int32_t *status;
    long long rows, entries;
    int H, N, rank, A, split;
    int tiles_down, tiles_up;             // feature tiles of an adapter's ddown (0: not wanted) and dup
    int items;                            // A * (tiles_down + tiles_up)
    int columns;                          // of tensor memory, one accumulator
};

template <bool SPLIT, int STAGES>
__global__ void __launch_bounds__(kGradThreads, 2)
adapter_grad_kernel(const GradArgs a)
{
    extern __shared__ char raw[];
    __shared__ uint64_t full_[STAGES], empty_[STAGES], acc_full_[2], acc_empty_[2], ex_full_;
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_;
    volatile int *gave_up = &gave_up_;

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int split = SPLIT ? a.split : 1, part = SPLIT ? (int)cluster_rank() : 0;
    const int tiles = a.tiles_down + a.tiles_up;
    const int chunks = (a.rank + 63) / 64, r16 = (a.rank + 15) & ~15;
    constexpr int stages = STAGES, kLag = STAGES - 1;
    const int stage_bytes = kLines + chunks * 8192;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
    char *const ring_ptr = raw + (ring - smem_addr(raw));
    float *const out = reinterpret_cast<float *>(SPLIT ? ring_ptr : ring_ptr + stages * stage_bytes);    // SPLIT: all columns, where the stages were
    int *const bound = reinterpret_cast<int *>(ring_ptr + stages * stage_bytes + (SPLIT ? 0 : kGradOutBytes));

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) bar_init(smem_addr(&full_[s]), kGradLoaders), bar_init(smem_addr(&empty_[s]), 1);
        for (int s = 0; s < 2; ++s) bar_init(smem_addr(&acc_full_[s]), 1), bar_init(smem_addr(&acc_empty_[s]), 4);
        bar_init(smem_addr(&ex_full_), split * 4);
        gave_up_ = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    if (warp == 0) tmem_alloc<1>(smem_addr(&tmem_slot), 2 * a.columns);
    for (int i = threadIdx.x; i <= a.A; i += kGradThreads) bound[i] = segment_bound(__ldg(a.offsets + i), a.entries);
    tmem_fence_before();
    if (SPLIT) cluster_sync();
    __syncthreads();
    tmem_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_slot, full0 = smem_addr(full_), empty0 = smem_addr(empty_);
    const int first = blockIdx.x / split, step = gridDim.x / split;

    struct Item {
        int adapter, m0, begin, n, k_from, k_to;
        bool up;
    };
    const auto item_at = [&](int i) {
        Item t;
        t.adapter = i / tiles;
        const int f = i - t.adapter * tiles;
        t.up = f >= a.tiles_down;
        t.m0 = (t.up ? f - a.tiles_down : f) * kRows;
        t.begin = bound[t.adapter];
        t.n = max(0, bound[t.adapter + 1] - t.begin);
        const int all = quotient_up(t.n, kTileK);
        t.k_from = (int)((long long)all * part / split), t.k_to = (int)((long long)all * (part + 1) / split);
        return t;
    };

    if (warp >= 5) {
        // ---- entries into the ring: 16 lanes bring 128 features of one and its piece of the rank, every 16th entry. Pieces that no
        // result depends on (features and ranks behind the last) are not brought; entries behind the segment's end are zeros.
        const int thread = threadIdx.x - 32 * 5, piece = thread & 15, line = thread >> 4;
        const uint32_t at = (piece >> 3) * 8192 + swizzled(line, piece & 7);
        int s = 0, phase = 1, done = 0, waiting = 0;
        bool ok = true;
        const auto arrive = [&] {
            fence_async();
            __syncwarp();
            if (lane == 0) bar_arrive(full0 + 8 * done);
            if (++done == stages) done = 0;
        };
        for (int i = first; ok && i < a.items; i += step) {
            const Item t = item_at(i);
            const int features = t.up ? a.N : a.H;
            const bool live = t.m0 + piece * 8 < features, real = piece * 8 < a.rank;
            const uint16_t *const rows = (t.up ? a.dy : a.x) + (live ? t.m0 + piece * 8 : 0);
            const uint16_t *const ranks = (t.up ? a.mid : a.dmid) + (real ? piece * 8 : 0) + (size_t)t.begin * a.rank;
            const bool plain = a.index == nullptr;
            const size_t row_step = (size_t)16 * features, rank_step = (size_t)16 * a.rank;
            // indexed rows are looked up two stages ahead; -1 behind the end
            int next[2][4];
            const auto look = [&](int k, int (&row)[4]) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int e = k * kTileK + line + 16 * j;
                    row[j] = k < t.k_to && e < t.n ? (plain ? t.begin + e : __ldg(a.index + t.begin + e)) : -1;
                }
            };
            if (!plain) look(t.k_from, next[0]), look(t.k_from + 1, next[1]);
            for (int k = t.k_from; k < t.k_to; ++k) {
                if (!(ok = __all_sync(kFullMask, bar_wait(empty0 + 8 * s, phase, gave_up)))) break;
                const uint32_t dst = ring + s * stage_bytes + at;
                const int e = k * kTileK + line;
                const uint16_t *rank = ranks + (size_t)e * a.rank;
                if (plain && (k + 1) * (long long)kTileK <= t.n) {           // a whole stage of rows one behind the other
                    const uint16_t *row = rows + (size_t)(t.begin + e) * features;
#pragma unroll
                    for (int j = 0; j < 4; ++j, row += row_step, rank += rank_step) {
                        if (live) copy16(dst + j * 2048, row, true);
                        if (real) copy16(dst + kLines + j * 2048, rank, true);
                    }
                } else {
                    if (plain) look(k, next[0]);
                    bool bad = false;
#pragma unroll
                    for (int j = 0; j < 4; ++j, rank += rank_step) {
                        const unsigned row = (unsigned)next[0][j];
                        const bool there = row < (unsigned)a.rows;           // others are zeros, in both operands
                        bad |= !there && e + 16 * j < t.n;
                        if (live) copy16(dst + j * 2048, rows + (there ? (size_t)row * (unsigned)features : 0), there);
                        if (real) copy16(dst + kLines + j * 2048, there ? rank : ranks, there);
                        next[0][j] = next[1][j];
                    }
                    if (bad && a.status && piece == 0) atomicOr(a.status, EP_STATUS_BAD_INDEX);
                    if (!plain) look(k + 2, next[1]);
                }
                copy_group();
                if (++s == stages) s = 0, phase ^= 1;
                if (waiting == kLag) copy_wait<kLag>(), arrive(); else ++waiting;
            }
        }
        copy_wait<0>();
        for (; ok && waiting > 0; --waiting) arrive();
    } else if (warp == 0 && elect_one()) {
        // ---- products
        int s = 0, phase = 0, used = 0;
        bool ok = true;
        const uint32_t idesc = instr_desc(kRows, r16, true, true);
        for (int i = first; ok && i < a.items; i += step) {
            const Item t = item_at(i);
            if (t.k_from == t.k_to) continue;
            const int acc = used & 1;
            if (!(ok = bar_wait(smem_addr(&acc_empty_[acc]), ((used >> 1) & 1) ^ 1, gave_up))) break;
            tmem_fence_after();
            for (int k = t.k_from; k < t.k_to; ++k) {
                if (!(ok = bar_wait(full0 + 8 * s, phase, gave_up))) break;
                tmem_fence_after();
                const uint32_t at = ring + s * stage_bytes;
                const uint64_t da = desc_mn_major(at), db = desc_mn_major(at + kLines);
#pragma unroll
                for (int j = 0; j < kTileK / 16; ++j) mma_bf16<1>(tmem + acc * a.columns, da + j * 128, db + j * 128, idesc, k > t.k_from || j > 0);
                mma_commit<1>(empty0 + 8 * s);
                if (++s == stages) s = 0, phase ^= 1;
            }
            if (ok) mma_commit<1>(smem_addr(&acc_full_[acc]));
            ++used;
        }
    } else if (warp >= 1) {
        // ---- accumulators out, through shared memory; SPLIT: added up over the CTAs that share them
        const int q = warp & 3, thread = threadIdx.x - 32;
        int used = 0;
        bool ok = true;
        for (int i = first; ok && i < a.items; i += step) {
            const Item t = item_at(i);
            const bool some = t.k_from < t.k_to;
            const int acc = used & 1, features = t.up ? a.N : a.H;
            const float scale = t.up && a.scale ? __ldg(a.scale + t.adapter) : 1.f;
            if (some) {
                ok = bar_wait(smem_addr(&acc_full_[acc]), (used >> 1) & 1, gave_up);
                tmem_fence_after();
                ++used;
            }
            uint32_t v[32];
            // columns [c0, c0 + 32) of the accumulator, or zeros
            const auto load = [&](int c0) {
                if (some) {
                    tmem_load32(tmem + (uint32_t(q * 32) << 16) + acc * a.columns + c0, v);
                } else {
#pragma unroll
                    for (int c = 0; c < 32; ++c) v[c] = 0u;
                }
            };
            // 8 results: ddown, 8 features of a rank; dup, 8 ranks of a feature
            const auto store = [&](float (&z)[8], int feature, int rank) {
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] *= scale;
                uint16_t *dst = t.up ? a.dup + ((size_t)t.adapter * a.N + t.m0 + feature) * a.rank + rank
                                     : a.ddown + ((size_t)t.adapter * a.rank + rank) * a.H + t.m0 + feature;
                *reinterpret_cast<uint4 *>(dst) = pack8(z);
            };
            if (SPLIT) {
                for (int c0 = 0; ok && c0 < r16; c0 += 32) {
                    load(c0);
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (c0 + c < r16) out[(c0 + c) * kGradLd + q * 32 + lane] = __uint_as_float(v[c]);
                }
                __syncwarp();
                if (ok && lane < split) bar_arrive_cluster_release(in_cta(smem_addr(&ex_full_), lane));
                ok = ok && bar_wait<true>(smem_addr(&ex_full_), 0, gave_up);
                const int total = t.up ? kRows * (a.rank / 8) : a.rank * (kRows / 8);
                const int from = total * part / split, to = total * (part + 1) / split;
                for (int j = from + thread; ok && j < to; j += 128) {
                    const int feature = t.up ? j % kRows : j % (kRows / 8) * 8, rank = t.up ? j / kRows * 8 : j / (kRows / 8);
                    if (t.m0 + feature >= features) continue;
                    float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    const uint32_t src = smem_addr(out + rank * kGradLd + feature);
                    for (int s = 0; s < split; ++s) {
                        const uint32_t at = in_cta(src, s);
                        if (t.up) {
#pragma unroll
                            for (int l = 0; l < 8; ++l) {
                                float w;
                                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w) : "r"(at + l * kGradLd * 4) : "memory");
                                z[l] += w;
                            }
                        } else {
                            const float4 lo = load_cluster(at), hi = load_cluster(at + 16);
                            z[0] += lo.x, z[1] += lo.y, z[2] += lo.z, z[3] += lo.w, z[4] += hi.x, z[5] += hi.y, z[6] += hi.z, z[7] += hi.w;
                        }
                    }
                    store(z, feature, rank);
                }
            } else {
                for (int c0 = 0; ok && c0 < r16; c0 += 32) {
                    load(c0);
                    if (some && c0 + 32 >= r16) {                            // this warp has read its last column
                        tmem_fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_addr(&acc_empty_[acc]));
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (c0 + kGradColumns * h >= a.rank) break;
#pragma unroll
                        for (int c = 0; c < kGradColumns; ++c) out[c * kGradLd + q * 32 + lane] = __uint_as_float(v[kGradColumns * h + c]);
                        asm volatile("bar.sync 1, 128;" ::: "memory");       // the four warps
                        const int ranks = min(kGradColumns, a.rank - c0 - kGradColumns * h), total = t.up ? kRows * (ranks / 8) : ranks * (kRows / 8);
                        for (int j = thread; j < total; j += 128) {
                            const int feature = t.up ? j % kRows : j % (kRows / 8) * 8, rank = t.up ? j / kRows * 8 : j / (kRows / 8);
                            if (t.m0 + feature >= features) continue;
                            const float *src = out + rank * kGradLd + feature;
                            float z[8];
                            if (t.up) {
#pragma unroll
                                for (int l = 0; l < 8; ++l) z[l] = src[l * kGradLd];
                            } else {
                                const float4 lo = *reinterpret_cast<const float4 *>(src), hi = *reinterpret_cast<const float4 *>(src + 4);
                                z[0] = lo.x, z[1] = lo.y, z[2] = lo.z, z[3] = lo.w, z[4] = hi.x, z[5] = hi.y, z[6] = hi.z, z[7] = hi.w;
                            }
                            store(z, feature, c0 + kGradColumns * h + rank);
                        }
                        asm volatile("bar.sync 1, 128;" ::: "memory");       // `out` may be written again
                    }
                }
            }
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (SPLIT) cluster_sync();                                               // the others' reads come from this CTA's memory
    tmem_fence_after();
    if (warp == 0) tmem_free<1>(tmem, 2 * a.columns);
    if (threadIdx.x == 0 && gave_up_ && a.status) atomicOr(a.status, EP_STATUS_TIMEOUT);
}

// ---- host side ---------------------------------------------------------------------------------------------------

int check_adapter(const ep_adapter_t *m)
{
    if (!m) return EP_ERR_NULL;
    const int64_t limit = int64_t(1) << 31;
    if (m->rows < 0 || m->rows >= limit || m->entries < 0 || m->entries >= limit) return EP_ERR_INVALID_ARG;
    if (m->in_features < 8 || m->in_features % 8 || m->out_features < 8 || m->out_features % 8 || m->in_features >= (1 << 24) ||
        m->out_features >= (1 << 24))
        return EP_ERR_INVALID_ARG;
    if (m->rank < 8 || m->rank % 8 || m->rank > kMaxRank || m->num_adapters < 1 || m->num_adapters > kMaxExperts) return EP_ERR_INVALID_ARG;
    return EP_OK;
}

template <class Kernel, class... Args>
int launch_cluster(Kernel kernel, std::atomic<uint64_t> &ready, int64_t groups, int split, int threads, int smem, int smem_most, cudaStream_t stream,
                   const Args &...args)
{
    int dev = 0;
    EP_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return EP_ERR_INVALID_ARG;
    if (!(ready.load() >> dev & 1)) {                                        // once per device
        EP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_most));
        ready.fetch_or(uint64_t(1) << dev);
    }
    if (groups * split >= (int64_t(1) << 31)) return EP_ERR_INVALID_ARG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(groups * split));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 2 : 1;
    EP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, args...));
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

// One launch of the rank kernel: `in` [rows][in], weights down [A][rank][*], up [A][*][rank].
template <bool BACK>
int launch_rank(const ep_adapter_t &m, TensorMapEncode encode, RankArgs a, const void *in, const void *down, const void *up, cudaStream_t stream)
{
    static std::atomic<uint64_t> ready{0};
    const uint64_t H = m.in_features, N = m.out_features, r = m.rank, A = m.num_adapters;
    a.rows = m.rows, a.entries = m.entries, a.rank = m.rank, a.A = m.num_adapters;
    a.in = BACK ? m.out_features : m.in_features, a.out_features = BACK ? m.in_features : m.out_features;
    a.in_rows = static_cast<const uint16_t *>(in), a.second = static_cast<const uint16_t *>(BACK ? down : up);
    CUtensorMap map_first, map_second;
    int rc = BACK ? make_map(encode, &map_first, up, r, N, A, 64) : make_map(encode, &map_first, down, H, r, A, (uint32_t)((r + 15) & ~15));
    if (rc == EP_OK) {
        if (!a.out) map_second = map_first;
        else rc = BACK ? make_map(encode, &map_second, down, H, r, A, 64) : make_map(encode, &map_second, up, r, N, A, 128);
    }
    if (rc != EP_OK) return rc;
    // At most this many tiles of `width` rows; two CTAs per SM. Clusters while they fit at once, then narrower tiles up to that number.
    const int64_t adapters = m.entries < m.num_adapters ? m.entries : m.num_adapters, slots = 2 * 148;
    int64_t tiles = m.entries / kRows + adapters;
    const int stages = (a.in + kTileK - 1) / kTileK;
    a.split = 1;
    while (a.split < kMaxCluster && tiles * a.split * 2 <= slots && stages >= 4 * a.split) a.split *= 2;
    a.width = kRows;
    if (slots / a.split > adapters) {
        const int64_t even = (m.entries + slots / a.split - adapters - 1) / (slots / a.split - adapters);
        if (even > 64 && even < kRows) a.width = (int)(even + 3) / 4 * 4;
    }
    tiles = m.entries / a.width + adapters;
    return launch_cluster(rank_kernel<BACK>, ready, tiles, a.split, kThreads, kRankSmem, kRankSmem, stream, a, map_first, map_second);
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace
}  // namespace ep

extern "C" int ep_adapter_matmul(const ep_adapter_t *m, const void *x, const int32_t *adapter_offsets, const int32_t *row_index, const void *down,
                                 const void *up, const float *scale, const void *base, void *y, void *mid, int32_t *status, void *stream)
{
    using namespace ep;
    int rc = check_adapter(m);
    if (rc != EP_OK) return rc;
    if (!row_index && m->entries > m->rows) return EP_ERR_INVALID_ARG;
    if (m->entries == 0 || m->rows == 0) return EP_OK;
    if (!x || !adapter_offsets || !down || (y && !up) || (!y && !mid)) return EP_ERR_NULL;
    if (!aligned16(x) || !aligned16(down) || !aligned16(up) || !aligned16(base) || !aligned16(y) || !aligned16(mid)) return EP_ERR_INVALID_ARG;
    TensorMapEncode encode;
    rc = tensor_map_encoder(&encode);
    if (rc != EP_OK) return rc;
    RankArgs a = {};
    a.offsets = adapter_offsets, a.index = row_index, a.status = status, a.scale = scale;
    a.base = static_cast<const uint16_t *>(base);
    a.out = static_cast<uint16_t *>(y), a.mid = static_cast<uint16_t *>(mid);
    return launch_rank<false>(*m, encode, a, x, down, up, static_cast<cudaStream_t>(stream));
}

extern "C" size_t ep_adapter_matmul_backward_workspace_bytes(const ep_adapter_t *m)
{
    using namespace ep;
    if (check_adapter(m) != EP_OK) return 0;
    return up256((size_t)m->entries * m->rank * 2) + 256;
}

extern "C" int ep_adapter_matmul_backward(const ep_adapter_t *m, const void *dy, const void *x, const int32_t *adapter_offsets, const int32_t *row_index,
                                          const void *down, const void *up, const float *scale, const void *mid, const void *base, void *dx, void *ddown,
                                          void *dup, int32_t *status, void *workspace, size_t workspace_bytes, void *stream_)
{
    using namespace ep;
    int rc = check_adapter(m);
    if (rc != EP_OK) return rc;
    if (!row_index && m->entries > m->rows) return EP_ERR_INVALID_ARG;
    if (!dx && !ddown && !dup) return EP_ERR_NULL;
    const size_t A = m->num_adapters, r = m->rank, H = m->in_features, N = m->out_features;
    if (!aligned16(dy) || !aligned16(x) || !aligned16(down) || !aligned16(up) || !aligned16(mid) || !aligned16(base) || !aligned16(dx) ||
        !aligned16(ddown) || !aligned16(dup) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return EP_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (m->entries == 0 || m->rows == 0) {
        if (ddown) EP_CUDA_TRY(cudaMemsetAsync(ddown, 0, A * r * H * 2, stream));
        if (dup) EP_CUDA_TRY(cudaMemsetAsync(dup, 0, A * N * r * 2, stream));
        return EP_OK;
    }
    if (!dy || !adapter_offsets || ((dx || ddown) && !up) || (dx && !down) || (ddown && !x) || (dup && !mid)) return EP_ERR_NULL;
    void *dmid = workspace;
    if (ddown && !workspace) return EP_ERR_NULL;
    if (ddown && workspace_bytes < ep_adapter_matmul_backward_workspace_bytes(m)) return EP_ERR_CAPACITY;
    TensorMapEncode encode;
    rc = tensor_map_encoder(&encode);
    if (rc != EP_OK) return rc;
    if (dx || ddown) {
        RankArgs a = {};
        a.offsets = adapter_offsets, a.index = row_index, a.status = status, a.scale = scale;
        a.base = static_cast<const uint16_t *>(base);
        a.out = static_cast<uint16_t *>(dx);
        a.mid = ddown ? static_cast<uint16_t *>(dmid) : nullptr;
        rc = launch_rank<true>(*m, encode, a, dy, down, up, stream);
        if (rc != EP_OK) return rc;
    }
    if (!ddown && !dup) return EP_OK;
    GradArgs g = {};
    g.offsets = adapter_offsets, g.index = row_index, g.scale = scale, g.status = status;
    g.x = static_cast<const uint16_t *>(x), g.dmid = static_cast<const uint16_t *>(dmid);
    g.dy = static_cast<const uint16_t *>(dy), g.mid = static_cast<const uint16_t *>(mid);
    g.ddown = static_cast<uint16_t *>(ddown), g.dup = static_cast<uint16_t *>(dup);
    g.rows = m->rows, g.entries = m->entries, g.H = m->in_features, g.N = m->out_features, g.rank = m->rank, g.A = m->num_adapters;
    g.tiles_down = ddown ? (m->in_features + kRows - 1) / kRows : 0;
    g.tiles_up = dup ? (m->out_features + kRows - 1) / kRows : 0;
    const int64_t items = (int64_t)g.A * (g.tiles_down + g.tiles_up), average = m->entries / m->num_adapters / kTileK;
    if (items * kMaxCluster >= (int64_t(1) << 31)) return EP_ERR_INVALID_ARG;
    g.items = (int)items;
    g.split = 1;
    while (g.split < kMaxCluster && items * g.split * 2 <= 2 * 148 && average >= 4 * g.split) g.split *= 2;
    const int r16 = (m->rank + 15) & ~15, chunks = (m->rank + 63) / 64, stage = kLines + chunks * 8192, table = (g.A + 1) * 4;
    g.columns = r16 <= 32 ? 32 : r16 <= 64 ? 64 : 128;
    static std::atomic<uint64_t> ready[4];
    const int fixed = 1024 + kGradOutBytes + table;                          // beside the stages
    if (g.split > 1) {                                                       // over half of an SM's memory each: see the rank kernel
        if (chunks == 1) return launch_cluster(adapter_grad_kernel<true, 4>, ready[0], items, g.split, kGradThreads, kRankSmem, kRankSmem, stream, g);
        return launch_cluster(adapter_grad_kernel<true, 6>, ready[1], items, g.split, kGradThreads, fixed + 6 * stage, 222 * 1024, stream, g);
    }
    if (chunks == 1 && fixed + 4 * stage <= kRankSmem - 1024)                // two on an SM
        return launch_cluster(adapter_grad_kernel<false, 4>, ready[2], items < 296 ? items : 296, 1, kGradThreads, fixed + 4 * stage, kRankSmem, stream, g);
    return launch_cluster(adapter_grad_kernel<false, 6>, ready[3], items < 148 ? items : 148, 1, kGradThreads, fixed + 6 * stage, 222 * 1024, stream, g);
}
