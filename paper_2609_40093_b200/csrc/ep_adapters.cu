// Low-rank adapters beside a shared projection, and their gradients.
//
//   forward   mid = x down[a]^T                   y[row]  = base[row] + scale[a] * mid up[a]^T          rows of adapter a
//   backward  dmid = scale[a] * dy up[a]          dx[row] = base[row] + dmid down[a]
//             ddown[a] = dmid^T x                 dup[a] = scale[a] * dy^T mid                          sums over the rows
//
// The first two lines are one kernel, the rank kernel: in -> (rank) -> out with the weights read along either axis. A tile is
// up to 128 rows of one adapter, the lanes of the accumulators; its rows may lie anywhere.
// The first product contracts the features into at most 128 columns of tensor memory; they are rounded to bf16 (they are the operand of
// another product), laid out in shared memory as that product's row operand, and the output follows in blocks of 128 columns, whose
// epilogue adds to `base` in fp32 and rounds once. Nothing between the products goes through memory.
// Where there are few tiles, up to eight CTAs of a cluster share one: each contracts a part of the features, all add the parts through each
// other's shared memory in a fixed order, and each makes a part of the output's blocks. So a token that is generated alone has
// its adapter's weights read by eight SMs.
//
// The two sums over rows are the gradient kernel: 128 features are the lanes, the rank the columns, the rows are contracted. Entries behind
// a segment's end are zeros in both operands, whatever the memory holds.
//
// All of it is bound by memory where there are rows enough: a row's 2 (in + 2 out) bytes carry 2 rank (in + out) operations, a
// tenth of what the tensor cores do meanwhile (rank 64: pipe 11 % active). 16384 rows, 4096 -> 8192 features, rank 64, four adapters: 126 to 129 us
// for 0.67 GB, 5.3 TB/s; what is missing to the copy's 6.5 is the time between the two products, when a CTA has nothing in flight. With few rows it
// is latency. By the GPU's clock, medians over the CTAs: a row of 4096 -> 4096 (9 us) takes 1.0 for the tables, 1.2 for tensor memory and the list of
// rows, 1.9 for rows and weights, 1.5 for the exchange and 0.6 for its sums, 0.5 for the first block and 0.35 for the second, 1.0 to leave; 256 rows on 64
// adapters, 2048 -> 8192 (24 us), 1.0, 1.3, 2.3, 1.5, 0.7, 0.6 and 0.39 for each of 15 more blocks, 1.8 to leave: 15 for a CTA. Two in five start 2.7 later,
// in the places that the kernel before leaves last, nine in ten are done after 19.6, and the slowest is 5 behind them.
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
constexpr int kPartStages = 8;            // of the contracted features, for every CTA but one that shares them
constexpr int kGradMost = 2 * 148;        // CTAs of the gradient kernel
constexpr int kGradFeatures = kRows;      // of an item: an accumulator's lanes

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

// The two halves of a barrier of the cluster.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

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

struct RankTables {
    uint64_t full[kMaxStages], empty[kMaxStages], unit_full[kMaxUnits], unit_empty[kMaxUnits], mid_full, mid_ready, mid_ready_all, acc_full[2], acc_empty[2],
        ex_full, done;
    uint32_t tmem_slot;
    int gave_up, warp_sum[kThreads / 32], where[3];
    int row_of[kRows];
};
constexpr int kRankSmem = kAreaBytes + 1024;
static_assert(sizeof(RankTables) <= 1024, "two CTAs per SM");

// ---- the pieces of the gradient kernel's work -----------------------------------------------------------------------

// Made by one CTA, in front of the rank kernel's or by itself: a list of pieces (a run of an adapter's stages of 64 entries each), the
// longest first, and behind them the adapters without entries, whose gradients are zeros. The same list every time.
constexpr int kGradBins = 16;             // lengths that are told apart
constexpr int kGradCuts = 8;              // cuts of the longest adapter that are tried
__device__ __forceinline__ int cut_of(int d) { return d == 0 ? 1 : (d & 1 ? 2 : 3) << ((d - 1) >> 1); }        // 1, 2, 3, 4, 6, 8, 12, 16

struct GradPiece {
    int adapter, begin, n;                // its first entry and how many it has
    int of;                               // its pieces
    int k_from, k_to;                     // the piece's stages
    int number, part;                     // which piece; the adapter's first part in the workspace, if there are several
};

struct PlanArgs {
    const int32_t *offsets;
    long long entries;
    int A, piece, tiles, ctas;            // piece: stages of a piece at least, where an adapter has more
    int counters;
    int *arrived;                         // [counters], to be zeroed
    int *pieces;                          // how many there are
    GradPiece *list;                      // NULL: no plan
    int32_t *status;
};

struct PlanTables {
    unsigned long long entries;
    int most, sum, parts[kGradCuts], warp_sum[2][kThreads / 32];
    int bins[(kGradBins + 1) * kThreads]; // [bin][thread] pieces, then where they start
    int stages[kMaxExperts];
};

// The exclusive sum of v over the block's threads.
__device__ __forceinline__ int block_scan(int v, int *warp_sum)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int scan = v;
    for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(kFullMask, scan, d);
        if (lane >= d) scan += u;
    }
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    scan -= v;
    for (int w = 0; w < warp; ++w) scan += warp_sum[w];
    return scan;
}

__device__ void plan_pieces(const PlanArgs &a, PlanTables &tab)
{
    const int per = (a.A + kThreads - 1) / kThreads, from = min(a.A, (int)threadIdx.x * per), to = min(a.A, from + per), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) tab.most = 0, tab.sum = 0, tab.entries = 0;
    if (threadIdx.x < kGradCuts) tab.parts[threadIdx.x] = 0;
    for (int i = threadIdx.x; i < a.counters; i += kThreads) a.arrived[i] = 0;
    for (int b = 0; b <= kGradBins; ++b) tab.bins[b * kThreads + threadIdx.x] = 0;
    __syncthreads();
    const auto begin_of = [&](int e) { return segment_bound(__ldg(a.offsets + e), a.entries); };
    int most = 0, sum = 0;
    unsigned long long entries = 0;
    for (int e = from; e < to; ++e) {
        const int count = max(0, begin_of(e + 1) - begin_of(e)), n = quotient_up(count, kTileK);
        tab.stages[e] = n;
        entries += count;
        most = max(most, n), sum += n;
    }
    atomicAdd(&tab.entries, entries);
    __syncthreads();
    if (threadIdx.x == 0 && a.status && (tab.entries > (unsigned long long)a.entries || __ldg(a.offsets + a.A) > a.entries))
        atomicOr(a.status, EP_STATUS_CAPACITY);
    if (tab.entries > (unsigned long long)a.entries) {                       // offsets that decrease: the list has no room for what they name
        if (threadIdx.x == 0) *a.pieces = 0;
        return;
    }
    most = __reduce_max_sync(kFullMask, most), sum = __reduce_add_sync(kFullMask, sum);
    if (lane == 0 && sum) atomicMax(&tab.most, most), atomicAdd(&tab.sum, sum);
    __syncthreads();
    // How long a piece may be: the longest adapter's stages over 1, 2, 3, 4, 6, 8, 12 or 16, whichever should end first: with the
    // longest piece, whose stages take some 0.6 of the usual time while others are done already, or with a CTA's share of all. A part costs
    // about five stages, and adding parts some eight at the end.
    for (int d = 0; d < kGradCuts; ++d) {
        const int piece = max(a.piece, quotient_up(tab.most, cut_of(d)));
        int split = 0;
        for (int e = from; e < to; ++e) {
            const int of = quotient_up(tab.stages[e], piece);
            split += of > 1 ? of : 0;
        }
        split = __reduce_add_sync(kFullMask, split);
        if (lane == 0 && split) atomicAdd(&tab.parts[d], split);
    }
    __syncthreads();
    int piece = 1;
    float best = 3.4e38f;
    for (int d = 0; d < kGradCuts; ++d) {
        const int longest = max(a.piece, quotient_up(tab.most, cut_of(d)));
        const float share = ((float)tab.sum + 5.f * tab.parts[d]) * a.tiles / a.ctas;
        const float cost = fmaxf(0.6f * min(longest, tab.most), share) + (tab.parts[d] ? 8.f : 0.f);
        if (cost < best) best = cost, piece = longest;
    }
    // ---- a counting sort, the adapters of a bin in their order
    const auto bin_of = [&](int n, int of) { return n ? kGradBins - 1 - min(kGradBins - 1, (int)((float)n * kGradBins / ((float)of * (piece + 1)))) : kGradBins; };
    int split = 0;
    for (int e = from; e < to; ++e) {
        const int n = tab.stages[e], of = quotient_up(n, piece);
        tab.bins[bin_of(n, of) * kThreads + threadIdx.x] += n ? of : 1;
        split += of > 1 ? of : 0;
    }
    __syncthreads();
    int *const run = tab.bins + threadIdx.x * (kGradBins + 1);
    int total = 0;
    for (int i = 0; i <= kGradBins; ++i) total += run[i];
    int start = block_scan(total, tab.warp_sum[0]), part = block_scan(split, tab.warp_sum[1]);
    for (int i = 0; i <= kGradBins; ++i) {
        const int v = run[i];
        run[i] = start;
        start += v;
    }
    if (threadIdx.x == kThreads - 1) *a.pieces = start;
    __syncthreads();
    for (int e = from; e < to; ++e) {
        const int n = tab.stages[e], of = quotient_up(n, piece), begin = begin_of(e), count = max(0, begin_of(e + 1) - begin);
        int &at = tab.bins[bin_of(n, of) * kThreads + threadIdx.x];
        for (int i = 0; i < max(1, of); ++i)
            a.list[at++] = GradPiece{e, begin, count, of, of > 1 ? (int)((long long)n * i / of) : 0, of > 1 ? (int)((long long)n * (i + 1) / of) : n, i, part};
        part += of > 1 ? of : 0;
    }
}

__global__ void __launch_bounds__(kThreads)
plan_kernel(const PlanArgs a)
{
    extern __shared__ __align__(1024) char area[];
    pdl_trigger();
    pdl_wait();
    plan_pieces(a, *reinterpret_cast<PlanTables *>(area));
}

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
    int in, out_features, rank, A, width; // width: rows of a tile at most
    int split, copies;                    // CTAs of a cluster, that share the contracted features; clusters that share the output's blocks
};

// BACK: the weights are read along the other axis (up for the first product, down for the second), and the scale goes to `mid`.
template <bool BACK>
__global__ void __launch_bounds__(kThreads, 2)
rank_kernel(const RankArgs a, const PlanArgs plan, const __grid_constant__ CUtensorMap map_in, const __grid_constant__ CUtensorMap map_first, const __grid_constant__ CUtensorMap map_second)
{
    extern __shared__ __align__(1024) char area[];                           // no static shared memory: it would push the area off its boundary
    RankTables &tab = *reinterpret_cast<RankTables *>(area + kAreaBytes);
    int *const warp_sum = tab.warp_sum, *const where = tab.where, *const row_of = tab.row_of;
    volatile int *gave_up = &tab.gave_up;

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int split = a.split, part = split > 1 ? (int)cluster_rank() : 0;
    const int cluster = (int)blockIdx.x / split - (plan.list != nullptr), tile = cluster < 0 ? -1 : cluster / a.copies, copy = cluster - tile * a.copies;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) bar_init(smem_addr(&tab.full[s]), a.index ? 3 : 1), bar_init(smem_addr(&tab.empty[s]), 1);
        for (int s = 0; s < kMaxUnits; ++s) bar_init(smem_addr(&tab.unit_full[s]), 1), bar_init(smem_addr(&tab.unit_empty[s]), 1);
        for (int s = 0; s < 2; ++s) bar_init(smem_addr(&tab.acc_full[s]), 1), bar_init(smem_addr(&tab.acc_empty[s]), kEpilogueWarps);
        bar_init(smem_addr(&tab.mid_full), 1);
        bar_init(smem_addr(&tab.done), 1);
        bar_init(smem_addr(&tab.mid_ready), kEpilogueWarps);
        bar_init(smem_addr(&tab.mid_ready_all), split * kEpilogueWarps);
        bar_init(smem_addr(&tab.ex_full), split * kEpilogueWarps);
        tab.gave_up = 0;
        where[0] = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();                                                              // nothing is read or written before this
    // ---- this cluster's tile: each thread counts the tiles of a run of adapters
    if (tile < 0) {                                                          // the first cluster plans what the gradient kernel does
        if (part == 0) plan_pieces(plan, *reinterpret_cast<PlanTables *>(area));
        return;
    }
    {
        const int per = (a.A + kThreads - 1) / kThreads, from = min(a.A, (int)threadIdx.x * per), to = min(a.A, from + per);
        int sum = 0, begin = from < to ? segment_bound(__ldg(a.offsets + from), a.entries) : 0;
        const int first = begin;
        for (int i = from; i < to; ++i) {
            const int end = segment_bound(__ldg(a.offsets + i + 1), a.entries);
            sum += quotient_up(max(0, end - begin), a.width);
            begin = end;
        }
        int run = block_scan(sum, warp_sum);
        if (tile >= run && tile < run + sum) {                               // one thread: the tile is one of its adapters'
            begin = first;
            for (int i = from; i < to; ++i) {
                const int end = segment_bound(__ldg(a.offsets + i + 1), a.entries), count = max(0, end - begin);
                const int pieces = quotient_up(count, a.width);
                if (tile >= run && tile < run + pieces) {
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
        if (threadIdx.x == 0 && cluster == 0 && part == 0 && a.status && __ldg(a.offsets + a.A) > a.entries) atomicOr(a.status, EP_STATUS_CAPACITY);
        __syncthreads();
    }
    const int adapter = where[0], entry0 = where[1], m = where[2];
    if (adapter < 0 || m == 0) return;                                       // all CTAs of the cluster

    const int chunks = (a.rank + 63) / 64, r16 = (a.rank + 15) & ~15;
    const int all_k = (a.in + kTileK - 1) / kTileK, k_from = all_k * part / split, k_to = all_k * (part + 1) / split;
    const int blocks = a.out ? (a.out_features + kBlockColumns - 1) / kBlockColumns : 0;
    const int sharing = split * a.copies, share = copy * split + part;
    const int b_from = (int)((long long)blocks * share / sharing), b_to = (int)((long long)blocks * (share + 1) / sharing);
    const int stage_bytes = kLines + chunks * 8192, stages = kRingBytes / stage_bytes;
    const int quarters = (m + 31) / 32;                                      // of the lanes, with rows
    const bool boxes = a.index == nullptr;                                   // rows one behind the other
    const bool narrow = quarters == 1;                                       // each quarter of the lanes holds the same rows, see below
    // The parts that a cluster's CTAs have of the first product are sent to all of them where there is room for all of all beside the
    // ring; more of it is added up by shares (see below).
    const bool send = split > 1 && narrow && split * m * r16 * 4 <= kAreaBytes - kRingBytes;
    const int units = kAreaBytes / kLines - chunks - quarters - (send ? 1 : 0);
    const uint32_t ring = smem_addr(area), unit_base = ring + (chunks + quarters) * kLines;
    char *const buffers = area + chunks * kLines;
    float *const exchange = reinterpret_cast<float *>(buffers);              // [m][r16], 16-byte pieces turned so that neither axis meets a bank twice
    const int ex_turn = r16 % 32 == 0 ? 7 : 6;
    const auto ex_at = [&](int row, int piece) { return row * r16 + ((piece ^ (ex_turn == 7 ? row & 7 : (row & 6) >> 1)) << 2); };

    // From here on the weights' warp does not wait for the others. A cluster's CTAs write to each other's memory only after cluster_wait().
    if (split > 1) cluster_arrive();
    if (warp > 0) {
        if (warp == 1) tmem_alloc<1>(smem_addr(&tab.tmem_slot), 2 * kBlockColumns);
        const int i = (int)threadIdx.x - 64;
        if (i >= 0 && i < kRows) {
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
        asm volatile("bar.sync 1, %0;" ::"n"(kThreads - 32) : "memory");
        tmem_fence_after();
        if (warp == 1) pdl_trigger();
    }
    const uint32_t tmem = warp > 0 ? tab.tmem_slot : 0u;
    const uint32_t full0 = smem_addr(tab.full), empty0 = smem_addr(tab.empty), unit_full0 = smem_addr(tab.unit_full), unit_empty0 = smem_addr(tab.unit_empty);

    int s = 0, phase = 1, sent = 0, u = 0, uphase = 1, usent = 0;            // copies: the next places of the two rings, and how many were sent
    if (warp == 0 && elect_one()) {
        // ---- weights
        const uint32_t bytes = (uint32_t)((BACK ? chunks * 8192 : r16 * 128) + (boxes ? quarters * 4096 : 0));
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
            if (boxes)                                                       // rows behind the tile's last are lanes that nobody looks at
                for (int i = 0; i < quarters; ++i) tma_load<1>(dst - kLines + i * 4096, &map_in, k * kTileK, entry0 + 32 * i, 0, full);
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
        if (ok && blocks) {
            // ---- the second weights, once the ring's memory is free
            ok = bar_wait(smem_addr(&tab.mid_full), 0, gave_up);
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
            ok = bar_wait<true>(smem_addr(split > 1 && !send ? &tab.mid_ready_all : &tab.mid_ready), 0, gave_up);
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
        if (!boxes && (warp - 2) >> 1 < stages) {
            // ---- rows by index into the ring: two warps for each of its places, eight lanes a row's line. A thread waits for its own
            // copies before it hands them to the tensor cores; the other places' are under way meanwhile.
            const int place = (warp - 2) >> 1, line = (thread & 63) >> 3, piece = lane & 7;
            const uint32_t full = full0 + 8 * place, empty = empty0 + 8 * place, dst = ring + place * stage_bytes + swizzled(line, piece);
            int phase = 1;
            for (int k = k_from + place; k < k_to; k += stages, phase ^= 1) {
                if (!(ok = warp_wait(empty, phase, gave_up))) break;
                const int col = k * kTileK + piece * 8;
                const bool real = col < a.in;
                const uint16_t *const src = a.in_rows + (real ? col : 0);
#pragma unroll 4
                for (int j = line; j < m; j += 8) {
                    const int row = row_of[j];
                    copy16(dst + (j - line) * 128, src + (size_t)max(row, 0) * a.in, real && row >= 0);
                }
                copy_group();
                copy_wait<0>();
                fence_async();
                __syncwarp();
                if (lane == 0) bar_arrive(full);
            }
        }
        ok = ok && warp_wait(smem_addr(&tab.mid_full), 0, gave_up);
        tmem_fence_after();
        // 8 columns of a row, rounded: the second product's operand, and `mid`. Columns from the rank on, up to the step of 16, are zeros whatever
        // the row holds: an infinite element times the first weights' padding is NaN, which the second's would not take away.
        const auto rounded = [&](int row, int col, float (&f)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= mid_scale;
            const uint4 v = col < a.rank ? pack8(f) : make_uint4(0u, 0u, 0u, 0u);
            if (a.mid && copy == 0 && row < m && col < a.rank && (!send || part == 0)) *reinterpret_cast<uint4 *>(a.mid + (size_t)(entry0 + row) * a.rank + col) = v;
            return v;
        };
        const auto operand_at = [&](int row, int col) { return (col >> 6) * kLines + swizzled(row, (col & 63) >> 3); };
        __syncwarp();
        if (split > 1) cluster_wait();                                       // all are there
        float *const sent = reinterpret_cast<float *>(area + kRingBytes);    // [CTA][m][r16]
        if (ok && (!narrow || q == 0)) {
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
                            } else {
#pragma unroll
                                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(area + operand_at(32 * i + lane, c0 + 8 * j)) = w;
                            }
                        } else if (send && my_row < m) {
                            const uint32_t to = smem_addr(sent + (part * m + my_row) * r16 + c0 + 8 * j);
                            const uint4 lo = make_uint4(v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3]);
                            const uint4 hi = make_uint4(v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]);
                            for (int s = 0; s < split; ++s) store_cluster(in_cta(to, s), lo), store_cluster(in_cta(to, s) + 16, hi);
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
            ok = warp_wait<true>(smem_addr(&tab.ex_full), 0, gave_up);
            const int groups = r16 / 8;
            for (int i = thread; ok && send && i < m * groups; i += 32 * kEpilogueWarps) {
                const int row = i / groups, col = i % groups * 8;
                float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                for (int s = 0; s < split; ++s) {
                    const float4 *from = reinterpret_cast<const float4 *>(sent + (s * m + row) * r16 + col);
                    const float4 l = from[0], h = from[1];
                    f[0] += l.x, f[1] += l.y, f[2] += l.z, f[3] += l.w, f[4] += h.x, f[5] += h.y, f[6] += h.z, f[7] += h.w;
                }
                const uint4 v = rounded(row, col, f);
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) *reinterpret_cast<uint4 *>(area + operand_at(32 * i4 + row, col)) = v;
            }
            for (int i = thread * split + part; ok && !send && i < m * groups; i += 32 * kEpilogueWarps * split) {
                const int row = i / groups, col = i % groups * 8;
                const uint32_t lo = smem_addr(exchange + ex_at(row, col / 4)), hi = smem_addr(exchange + ex_at(row, col / 4 + 1));
                float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                for (int s = 0; s < split; s += 4) {                         // split is 2, 4 or 8; eight reads under way
                    float4 l[4], h[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        if (p < split) l[p] = load_cluster(in_cta(lo, s + p)), h[p] = load_cluster(in_cta(hi, s + p));
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        if (p < split) {
                            f[0] += l[p].x, f[1] += l[p].y, f[2] += l[p].z, f[3] += l[p].w;
                            f[4] += h[p].x, f[5] += h[p].y, f[6] += h[p].z, f[7] += h[p].w;
                        }
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
        if (split == 1 || send) {
            if (lane == 0) bar_arrive(smem_addr(&tab.mid_ready));
        } else {
            if (lane < split) bar_arrive_cluster_release(in_cta(smem_addr(&tab.mid_ready_all), lane));
            ok = ok && warp_wait<true>(smem_addr(&tab.mid_ready_all), 0, gave_up);           // all have read: the buffers are free
        }
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
            if (!(ok = warp_wait(smem_addr(&tab.acc_full[acc]), (used >> 1) & 1, gave_up))) break;
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
        for (int b = b_from; q >= quarters && !narrow && b < b_to; ++b, ++used) {                // lanes without rows
            if (!(ok = ok && warp_wait(smem_addr(&tab.acc_full[used & 1]), (used >> 1) & 1, gave_up))) break;
            if (lane == 0) bar_arrive(smem_addr(&tab.acc_empty[used & 1]));
        }
        // ... of up to 32 rows: every quarter of the lanes has them, and each of the eight warps 16 of a block's columns, straight from
        // the accumulators: 256 rows on 64 adapters of 2048 x 8192 take 0.4 us a block so, with one quarter's two warps at work 0.95
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
                if (!(ok = warp_wait(smem_addr(&tab.acc_full[acc]), (used >> 1) & 1, gave_up))) break;
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
    if (split > 1 && warp < 2) cluster_wait();
    tmem_fence_before();
    __syncthreads();
    if (tab.gave_up) {
        // Whoever gave up: copies may be on their way into this CTA's memory, and products may read it.
        const auto land = [](uint32_t bars, int places, int at, int parity, int n) {
            for (n = min(n, places); n > 0; --n) {
                int none = 0;
                if (at == 0) at = places, parity ^= 1;
                --at;
                bar_wait(bars + 8 * at, parity ^ 1, &none);
            }
        };
        land(full0, stages, s, phase, sent);
        land(unit_full0, units, u, uphase, usent);
        if (warp == 1 && elect_one()) {
            int none = 0;
            mma_commit<1>(smem_addr(&tab.done));
            bar_wait(smem_addr(&tab.done), 0, &none);
        }
        __syncthreads();
    }
    if (split > 1) cluster_sync();                                           // the others read from this CTA's memory and, where it gave up, may still write to it
    tmem_fence_after();
    if (warp == 1) tmem_free<1>(tmem, 2 * kBlockColumns);
    if (threadIdx.x == 0 && tab.gave_up && a.status) atomicOr(a.status, EP_STATUS_TIMEOUT);
}

// ---- the gradient kernel ------------------------------------------------------------------------------------------

// An adapter's entries are cut into pieces of about the same length, at most `piece` stages of 64; an item is a piece and 128 features of
// ddown or dup. Items are dealt out round by round, the longest pieces first, a piece's feature tiles next to each other: what runs at
// the same time reads the same rows (equal runs of work that end inside items balance better, but take the rows apart: dup of 32768 rows
// on 128 adapters alike 33 us instead of 15) and has the same length. The parts of an adapter with several pieces go to the workspace in
// fp32, and who comes last adds them in their order, so that the bits are the same every time. One warp issues the products, two
// for each stage bring entries, four empty the accumulators, of which there are two, so that an item's results leave under the next one's products.
constexpr int kGradEpilogueWarps = 4;
constexpr int grad_threads(int stages) { return 32 * (2 + kGradEpilogueWarps + 2 * stages); }     // one each for the products and the items, two for each stage
constexpr int kGradAhead = 4;             // items that are known ahead
constexpr int kGradLd = kRows + 4;        // accumulators on their way out: [rank][128 features]
constexpr int kGradColumns = 16;          // of them at a time
constexpr int kGradOutBytes = kGradColumns * kGradLd * 4;

struct GradArgs {
    const int32_t *index;
    const float *scale;
    const uint16_t *x, *dmid, *dy, *mid;
    uint16_t *ddown, *dup;
    int32_t *status;
    float *parts;                         // [parts of split adapters][feature tile][r16][128]
    int *arrived;                         // [parts of split adapters][feature tile] zeros: how many parts are there, at an adapter's first
    long long rows;
    int H, N, rank;
    int tiles_down, tiles_up;             // feature tiles of an adapter's ddown (0: not wanted) and dup
    int *counter;                         // 0: items handed out beyond the CTAs' first
    const int *pieces;                    // the plan
    const GradPiece *list;
    int columns;                          // of tensor memory, one accumulator
};

struct GradMaps {
    CUtensorMap x, dmid, dy, mid;         // in boxes of 64 rows
};

// An item: a piece, and which features of which product.
struct GradItem {
    GradPiece p;
    int f, m0, up, more;                  // more: 0 behind the last item
};

template <int STAGES>
__global__ void __launch_bounds__(grad_threads(STAGES), STAGES == 4 ? 2 : 1)
adapter_grad_kernel(const GradArgs a, const __grid_constant__ GradMaps maps)
{
    extern __shared__ char raw[];
    __shared__ uint64_t full_[STAGES], empty_[STAGES], acc_full_[2], acc_empty_[2], item_full_[kGradAhead], item_empty_[kGradAhead], done_;
    __shared__ GradItem items_[kGradAhead];
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_, last_;
    volatile int *gave_up = &gave_up_;

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int chunks = (a.rank + 63) / 64, r16 = (a.rank + 15) & ~15;
    constexpr int stages = STAGES;
    const int stage_bytes = kLines + chunks * 8192;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
    char *const ring_ptr = raw + (ring - smem_addr(raw));
    float *const out = reinterpret_cast<float *>(ring_ptr + stages * stage_bytes);

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) bar_init(smem_addr(&full_[s]), 2), bar_init(smem_addr(&empty_[s]), 1);
        for (int s = 0; s < 2; ++s) bar_init(smem_addr(&acc_full_[s]), 1), bar_init(smem_addr(&acc_empty_[s]), kGradEpilogueWarps);
        for (int s = 0; s < kGradAhead; ++s)
            bar_init(smem_addr(&item_full_[s]), 1), bar_init(smem_addr(&item_empty_[s]), 1 + kGradEpilogueWarps + 2 * STAGES);
        bar_init(smem_addr(&done_), 1);
        gave_up_ = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    if (warp == 0) tmem_alloc<1>(smem_addr(&tmem_slot), 2 * a.columns);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_slot, full0 = smem_addr(full_), empty0 = smem_addr(empty_);
    // The next item, in every warp (or thread) that works on it.
    GradItem t;
    int slot = 0, slot_phase = 0;
    const auto next = [&](bool warp_wide) {
        const uint32_t full = smem_addr(&item_full_[slot]);
        if (!(warp_wide ? warp_wait(full, slot_phase, gave_up) : bar_wait(full, slot_phase, gave_up))) return false;
        t = items_[slot];
        if (warp_wide) __syncwarp();
        if (!warp_wide || lane == 0) bar_arrive(smem_addr(&item_empty_[slot]));
        if (++slot == kGradAhead) slot = 0, slot_phase ^= 1;
        return t.more != 0;
    };

    uint32_t boxes = 0, boxes_phase = 0;                                     // where this thread's last boxes arrive; 0: it sent none
    if (warp == 1 + kGradEpilogueWarps) {
        // ---- items: the first is the CTA's own, the others who comes first gets
        if (elect_one()) {
            const int tiles = a.tiles_down + a.tiles_up, all = __ldcg(a.pieces) * tiles;
            for (int i = blockIdx.x;;) {
                GradItem it = {};
                if (i < all) {
                    const int4 *from = reinterpret_cast<const int4 *>(a.list + i / tiles);
                    const int4 lo = __ldcg(from), hi = __ldcg(from + 1);
                    it.p = GradPiece{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                    it.f = i % tiles;
                    it.up = it.f >= a.tiles_down;
                    it.m0 = (it.up ? it.f - a.tiles_down : it.f) * kGradFeatures;
                    it.more = 1;
                }
                if (!bar_wait(smem_addr(&item_empty_[slot]), slot_phase ^ 1, gave_up)) break;
                items_[slot] = it;
                bar_arrive(smem_addr(&item_full_[slot]));
                if (++slot == kGradAhead) slot = 0, slot_phase ^= 1;
                if (!it.more) break;
                i = atomicAdd(a.counter, 1) + gridDim.x;
            }
        }
    } else if (warp >= 2 + kGradEpilogueWarps) {
        // ---- entries into the ring: two warps for each of its places. A whole stage of rows one behind the other comes in boxes. Rows by
        // index, and a segment's last ones, are copied 16 bytes a thread, zeros where there is none (in both operands); a thread waits
        // for its own before it hands them to the tensor cores, and other warps' stages are under way meanwhile. (With all warps on every
        // stage that hand-over waits for the later stages, too: dup of 16384 x 8192 rows on four adapters of unequal length 80 us, so 58;
        // by index, with gather4 copies, 148, so 75.)
        const int s = (warp - 2 - kGradEpilogueWarps) >> 1, thread = (threadIdx.x - 32 * (2 + kGradEpilogueWarps)) & 63, piece = thread & 15, line = thread >> 4;
        const bool first = (thread >> 5) == 0;                               // of the two warps
        const uint32_t full = full0 + 8 * s, dst = ring + s * stage_bytes, at = dst + (piece >> 3) * 8192;
        const uint32_t at_even = at + swizzled(line, piece & 7), at_odd = at + swizzled(line + 4, piece & 7);
        int phase = 1, skip = s;                                             // stages until this place's next one
        bool ok = true;
        while (ok && next(true)) {
            const int features = t.up ? a.N : a.H;
            const bool live = t.m0 + piece * 8 < features, real = piece * 8 < a.rank, plain = a.index == nullptr;
            const uint16_t *const rows = (t.up ? a.dy : a.x) + (live ? t.m0 + piece * 8 : 0);
            const uint16_t *const ranks = (t.up ? a.mid : a.dmid) + (real ? piece * 8 : 0);
            int k = t.p.k_from + skip;
            for (; k < t.p.k_to; k += stages) {
                if (!(ok = warp_wait(empty0 + 8 * s, phase, gave_up))) break;
                phase ^= 1;
                if (plain && (k + 1) * (long long)kTileK <= t.p.n) {
                    if (lane == 0) {
                        if (first) {
                            const int row = t.p.begin + k * kTileK;
                            bar_expect(full, stage_bytes);
                            tma_load<1>(dst, t.up ? &maps.dy : &maps.x, t.m0, row, 0, full);
                            tma_load<1>(dst + 8192, t.up ? &maps.dy : &maps.x, t.m0 + 64, row, 0, full);
                            for (int c = 0; c < chunks; ++c) tma_load<1>(dst + kLines + c * 8192, t.up ? &maps.mid : &maps.dmid, 64 * c, row, 0, full);
                            boxes = full;
                        } else {
                            bar_arrive(full);
                        }
                    }
                    continue;
                }
                bool bad = false;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    int row[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int e = k * kTileK + line + 4 * (8 * h + j);
                        row[j] = e < t.p.n ? (plain ? t.p.begin + e : __ldg(a.index + t.p.begin + e)) : -1;
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int e = k * kTileK + line + 4 * (8 * h + j);
                        const bool there = (unsigned)row[j] < (unsigned)a.rows;
                        const uint32_t to = (j & 1 ? at_odd : at_even) + (4 * h + (j >> 1)) * 1024;
                        bad |= !there && e < t.p.n;
                        if (live) copy16(to, rows + (there ? (size_t)(unsigned)row[j] * (unsigned)features : 0), there);
                        if (real) copy16(to + kLines, ranks + (there ? (size_t)(unsigned)(t.p.begin + e) * (unsigned)a.rank : 0), there);
                    }
                }
                if (bad && a.status && piece == 0) atomicOr(a.status, EP_STATUS_BAD_INDEX);
                copy_group();
                copy_wait<0>();
                fence_async();
                __syncwarp();
                if (lane == 0) bar_arrive(full);
            }
            skip = k - t.p.k_to;
        }
        copy_wait<0>();
        boxes_phase = phase;
    } else if (warp == 0 && elect_one()) {
        // ---- products
        int s = 0, phase = 0, used = 0;
        bool ok = true;
        const uint32_t idesc = instr_desc(kRows, r16, true, true);
        while (ok && next(false)) {
            if (t.p.n == 0) continue;
            const int acc = used & 1;
            if (!(ok = bar_wait(smem_addr(&acc_empty_[acc]), ((used >> 1) & 1) ^ 1, gave_up))) break;
            tmem_fence_after();
            for (int k = t.p.k_from; k < t.p.k_to; ++k) {
                if (!(ok = bar_wait(full0 + 8 * s, phase, gave_up))) break;
                tmem_fence_after();
                const uint32_t at = ring + s * stage_bytes;
                const uint64_t da = desc_mn_major(at), db = desc_mn_major(at + kLines);
#pragma unroll
                for (int j = 0; j < kTileK / 16; ++j) mma_bf16<1>(tmem + acc * a.columns, da + j * 128, db + j * 128, idesc, k > t.p.k_from || j > 0);
                mma_commit<1>(empty0 + 8 * s);
                if (++s == stages) s = 0, phase ^= 1;
            }
            if (ok) mma_commit<1>(smem_addr(&acc_full_[acc]));
            ++used;
        }
    } else if (warp >= 1) {
        // ---- accumulators out, through shared memory, or as a part of an item's sums
        const int q = warp & 3, thread = threadIdx.x - 32;
        const auto together = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };        // the four warps
        // together(), and whether all of them go on: each may have given up by itself, and none must wait there for one that has left
        const auto agreed = [](bool go) {
            uint32_t all;
            asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.and.pred p, 1, 128, q;\n selp.u32 %0, 1, 0, p;\n}"
                         : "=r"(all)
                         : "r"(uint32_t(go))
                         : "memory");
            return all != 0;
        };
        int used = 0;
        for (;;) {
            bool go = next(true);
            const float scale = go && t.up && a.scale ? __ldg(a.scale + t.p.adapter) : 1.f;
            if (go && t.p.n) go = warp_wait(smem_addr(&acc_full_[used & 1]), (used >> 1) & 1, gave_up);
            if (!agreed(go)) break;                                          // no wait that may run out from here to the next item
            const int acc = used & 1, features = t.up ? a.N : a.H, m0 = t.m0, tiles = a.tiles_down + a.tiles_up;
            const bool whole = t.p.of == 1;
            float *const mine = a.parts + (((size_t)(t.p.part + t.p.number) * tiles + t.f)) * r16 * kRows;
            // 8 results: ddown, 8 features of a rank; dup, 8 ranks of a feature
            const auto store = [&](float (&z)[8], int feature, int rank) {
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] *= scale;
                uint16_t *dst = t.up ? a.dup + ((size_t)t.p.adapter * a.N + m0 + feature) * a.rank + rank
                                     : a.ddown + ((size_t)t.p.adapter * a.rank + rank) * a.H + m0 + feature;
                *reinterpret_cast<uint4 *>(dst) = pack8(z);
            };
            if (t.p.n == 0) {
                const int real = min(kRows, features - m0);
                for (int j = thread; j < real * a.rank / 8; j += 128) {
                    uint16_t *dst = t.up ? a.dup + ((size_t)t.p.adapter * a.N + m0) * a.rank + j * 8
                                         : a.ddown + ((size_t)t.p.adapter * a.rank + j / (real / 8)) * a.H + m0 + j % (real / 8) * 8;
                    *reinterpret_cast<uint4 *>(dst) = make_uint4(0u, 0u, 0u, 0u);
                }
                continue;
            }
            tmem_fence_after();
            ++used;
            for (int c0 = 0; c0 < r16; c0 += 32) {
                uint32_t v[32];
                tmem_load32(tmem + (uint32_t(q * 32) << 16) + acc * a.columns + c0, v);
                if (c0 + 32 >= r16) {                                        // this warp has read its last column
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_addr(&acc_empty_[acc]));
                }
                if (!whole) {
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (c0 + c < r16) mine[(c0 + c) * kRows + q * 32 + lane] = __uint_as_float(v[c]);
                    continue;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (c0 + kGradColumns * h >= a.rank) break;
#pragma unroll
                    for (int c = 0; c < kGradColumns; ++c) out[c * kGradLd + q * 32 + lane] = __uint_as_float(v[kGradColumns * h + c]);
                    together();
                    const int ranks = min(kGradColumns, a.rank - c0 - kGradColumns * h), total = t.up ? kRows * (ranks / 8) : ranks * (kRows / 8);
                    for (int j = thread; j < total; j += 128) {
                        const int feature = t.up ? j % kRows : j % (kRows / 8) * 8, rank = t.up ? j / kRows * 8 : j / (kRows / 8);
                        if (m0 + feature >= features) continue;
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
                    together();                                              // `out` may be written again
                }
            }
            if (whole) continue;
            // who comes last adds the parts
            __threadfence();
            together();
            if (thread == 0) last_ = atomicAdd(a.arrived + ((size_t)t.p.part * tiles + t.f), 1) == t.p.of - 1;
            together();
            if (last_) {
                __threadfence();
                for (int j = thread; j < (t.up ? kRows * (a.rank / 8) : a.rank * (kRows / 8)); j += 128) {
                    const int feature = t.up ? j % kRows : j % (kRows / 8) * 8, rank = t.up ? j / kRows * 8 : j / (kRows / 8);
                    if (m0 + feature >= features) continue;
                    float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
                    for (int p = 0; p < t.p.of; ++p) {
                        const float *src = a.parts + ((((size_t)(t.p.part + p) * tiles + t.f)) * r16 + rank) * kRows + feature;
                        if (t.up) {
#pragma unroll
                            for (int l = 0; l < 8; ++l) z[l] += __ldcg(src + l * kRows);
                        } else {
                            const float4 lo = __ldcg(reinterpret_cast<const float4 *>(src)), hi = __ldcg(reinterpret_cast<const float4 *>(src + 4));
                            z[0] += lo.x, z[1] += lo.y, z[2] += lo.z, z[3] += lo.w, z[4] += hi.x, z[5] += hi.y, z[6] += hi.z, z[7] += hi.w;
                        }
                    }
                    store(z, feature, rank);
                }
            }
            together();                                                      // `last_` may be written again
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (gave_up_) {                                                          // whoever did: copies and products may be under way
        int none = 0;
        if (boxes) bar_wait(boxes, boxes_phase, &none);
        if (warp == 0 && elect_one()) {
            mma_commit<1>(smem_addr(&done_));
            bar_wait(smem_addr(&done_), 0, &none);
        }
        __syncthreads();
    }
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
int launch_rank(const ep_adapter_t &m, TensorMapEncode encode, RankArgs a, const PlanArgs &plan, const void *in, const void *down, const void *up, cudaStream_t stream)
{
    static std::atomic<uint64_t> ready{0};
    const uint64_t H = m.in_features, N = m.out_features, r = m.rank, A = m.num_adapters;
    a.rows = m.rows, a.entries = m.entries, a.rank = m.rank, a.A = m.num_adapters;
    a.in = BACK ? m.out_features : m.in_features, a.out_features = BACK ? m.in_features : m.out_features;
    a.in_rows = static_cast<const uint16_t *>(in), a.second = static_cast<const uint16_t *>(BACK ? down : up);
    CUtensorMap map_in = {}, map_first, map_second;
    int rc = a.index ? EP_OK : make_map(encode, &map_in, in, a.in, m.rows, 1, 32);
    if (rc == EP_OK) rc = BACK ? make_map(encode, &map_first, up, r, N, A, 64) : make_map(encode, &map_first, down, H, r, A, (uint32_t)((r + 15) & ~15));
    if (rc == EP_OK) {
        if (!a.out) map_second = map_first;
        else rc = BACK ? make_map(encode, &map_second, down, H, r, A, 64) : make_map(encode, &map_second, up, r, N, A, 128);
    }
    if (rc != EP_OK) return rc;
    // At most this many tiles of `width` rows; two CTAs per SM. While they fit at once: clusters that share a tile's contracted features (at
    // least eight stages a CTA: the exchange takes as long as that many), then clusters that share its output's blocks, each with a first
    // product of its own (at least two blocks a CTA); then narrower tiles up to that number.
    const int64_t adapters = m.entries < m.num_adapters ? m.entries : m.num_adapters, slots = 2 * 148;
    int64_t tiles = m.entries / kRows + adapters;
    const int stages = (a.in + kTileK - 1) / kTileK, blocks = a.out ? (a.out_features + kBlockColumns - 1) / kBlockColumns : 0;
    a.split = 1;
    while (a.split < kMaxCluster && tiles * a.split * 2 <= slots && stages >= kPartStages * a.split) a.split *= 2;
    a.copies = (int)(slots / (tiles * a.split));
    if (a.copies > blocks / (2 * a.split)) a.copies = blocks / (2 * a.split);
    if (a.copies < 1) a.copies = 1;
    a.width = kRows;
    if (a.copies == 1 && slots / a.split > adapters) {
        const int64_t even = (m.entries + slots / a.split - adapters - 1) / (slots / a.split - adapters);
        if (even > 64 && even < kRows) a.width = (int)(even + 3) / 4 * 4;
    }
    // A few more tiles (an adapter's last is half empty, on average) than fit at once would run by themselves at the end: then about
    // two rounds of narrower ones (32768 rows, 128 adapters of 2048 x 1024: 70 us with 128 rows, 66 with 64).
    const int64_t likely = m.entries / kRows + adapters / 2;
    if (likely > slots && 2 * likely < 3 * slots) {
        const int64_t even = m.entries / (2 * slots - slots / 16 - adapters / 2) + 1;
        a.width = (int)((even < 64 ? 64 : even) + 3) / 4 * 4;
    }
    tiles = m.entries / a.width + adapters;
    return launch_cluster(rank_kernel<BACK>, ready, tiles * a.copies + (plan.list ? 1 : 0), a.split, kThreads, kRankSmem, kRankSmem, stream, a, plan, map_in, map_first, map_second);
}

// A call without rows: each entry that an adapter has names one that does not exist, and its mid is 0. One without entries, too: the offsets
// may still name some.
__global__ void __launch_bounds__(kThreads)
no_rows_kernel(const int32_t *offsets, int A, long long entries, int rank, uint16_t *mid, int32_t *status)
{
    pdl_trigger();
    pdl_wait();
    const int32_t end = __ldg(offsets + A);
    const int named = segment_bound(end, entries), first = blockIdx.x * kThreads + threadIdx.x;
    const int found = (end > entries ? EP_STATUS_CAPACITY : 0) | (named > 0 ? EP_STATUS_BAD_INDEX : 0);
    if (first == 0 && status && found) atomicOr(status, found);
    const long long vectors = mid ? (long long)named * (rank / 8) : 0;
    for (long long i = first; i < vectors; i += (long long)gridDim.x * kThreads) reinterpret_cast<uint4 *>(mid)[i] = make_uint4(0u, 0u, 0u, 0u);
}
int without_rows(const ep_adapter_t &m, const int32_t *offsets, void *mid, int32_t *status, cudaStream_t stream)
{
    if (m.entries == 0 && (!status || !offsets)) return EP_OK;               // nothing to write, nobody to tell
    if (!offsets) return EP_ERR_NULL;
    if (m.entries > 0 && !aligned16(mid)) return EP_ERR_INVALID_ARG;
    const int64_t blocks = mid ? (m.entries * (m.rank / 8) + kThreads - 1) / kThreads : 1, most = 8 * 148;
    EP_CUDA_TRY(launch_pdl(no_rows_kernel, dim3((unsigned)(blocks < 1 ? 1 : blocks < most ? blocks : most)), dim3(kThreads), 0, stream, offsets,
                           m.num_adapters, (long long)m.entries, m.rank, static_cast<uint16_t *>(mid), status));
    EP_LAUNCH_CHECK(1);
    return EP_OK;
}

size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

// The gradient kernel's launch and workspace.
struct GradPlan {
    int ctas, stages, smem, piece;
    int64_t counters;
    size_t counter_bytes, list_bytes, dmid_bytes, parts_bytes;
};
int feature_tiles(int features) { return (features + kGradFeatures - 1) / kGradFeatures; }
GradPlan plan_grads(const ep_adapter_t &m)
{
    GradPlan p;
    const int r16 = (m.rank + 15) & ~15, chunks = (m.rank + 63) / 64, stage = kLines + chunks * 8192;
    const int64_t tiles = feature_tiles(m.in_features) + feature_tiles(m.out_features), all = m.entries / kTileK;
    // Pieces of at least eight stages, and not so short that there are more than some three a CTA and feature tile.
    const int64_t even = (all * tiles + 3 * kGradMost - 1) / (3 * kGradMost);
    p.piece = (int)(even < 8 ? 8 : even);
    // An adapter with more stages than that has more than 64 * piece entries: there are at most `cuts` of those, and their pieces are at
    // most that many more.
    const int64_t cuts = all / p.piece, split = cuts + (m.num_adapters < cuts ? m.num_adapters : cuts);
    const int64_t pieces = m.num_adapters + cuts;
    p.stages = chunks == 1 ? 4 : 6;                                          // two CTAs on an SM, or one
    p.smem = 1024 + kGradOutBytes + p.stages * stage;
    const int64_t most = chunks == 1 ? kGradMost : kGradMost / 2, items = pieces * tiles;
    p.ctas = (int)(items < most ? items : most);                             // below 2^31: 4096 adapters x 2^18 tiles at most, and some 900 for the cuts
    p.counters = 1 + split * tiles;
    p.counter_bytes = up256((size_t)p.counters * 4 + 4);
    p.list_bytes = up256((size_t)pieces * sizeof(GradPiece));
    p.dmid_bytes = up256((size_t)m.entries * m.rank * 2);
    p.parts_bytes = (size_t)(split * tiles) * r16 * kGradFeatures * 4;
    return p;
}

}  // namespace
}  // namespace ep

extern "C" int ep_adapter_matmul(const ep_adapter_t *m, const void *x, const int32_t *adapter_offsets, const int32_t *row_index, const void *down,
                                 const void *up, const float *scale, const void *base, void *y, void *mid, int32_t *status, void *stream)
{
    using namespace ep;
    int rc = check_adapter(m);
    if (rc != EP_OK) return rc;
    if (!row_index && m->entries > m->rows) return EP_ERR_INVALID_ARG;
    if (m->entries == 0 || m->rows == 0) return without_rows(*m, adapter_offsets, mid, status, static_cast<cudaStream_t>(stream));
    if (!x || !adapter_offsets || !down || (y && !up) || (!y && !mid)) return EP_ERR_NULL;
    if (!aligned16(x) || !aligned16(down) || !aligned16(up) || !aligned16(base) || !aligned16(y) || !aligned16(mid)) return EP_ERR_INVALID_ARG;
    TensorMapEncode encode;
    rc = tensor_map_encoder(&encode);
    if (rc != EP_OK) return rc;
    RankArgs a = {};
    a.offsets = adapter_offsets, a.index = row_index, a.status = status, a.scale = scale;
    a.base = static_cast<const uint16_t *>(base);
    a.out = static_cast<uint16_t *>(y), a.mid = static_cast<uint16_t *>(mid);
    return launch_rank<false>(*m, encode, a, PlanArgs{}, x, down, up, static_cast<cudaStream_t>(stream));
}

extern "C" size_t ep_adapter_matmul_backward_workspace_bytes(const ep_adapter_t *m)
{
    using namespace ep;
    if (check_adapter(m) != EP_OK) return 0;
    const GradPlan p = plan_grads(*m);
    return p.counter_bytes + p.list_bytes + p.dmid_bytes + p.parts_bytes;
}

extern "C" int ep_adapter_matmul_backward(const ep_adapter_t *m, const void *dy, const void *x, const int32_t *adapter_offsets, const int32_t *row_index,
                                          const void *down, const void *up, const float *scale, const void *mid, const void *base, void *dx, void *ddown,
                                          void *dup, int32_t *status, void *workspace, size_t workspace_bytes, void *stream_)
{
    using namespace ep;
    int rc = check_adapter(m);
    if (rc != EP_OK) return rc;
    if (!row_index && m->entries > m->rows) return EP_ERR_INVALID_ARG;
    if (!dx && !ddown && !dup && m->rows > 0) return EP_ERR_NULL;            // a dx without rows has no address
    const size_t A = m->num_adapters, r = m->rank, H = m->in_features, N = m->out_features;
    if (!aligned16(dy) || !aligned16(x) || !aligned16(down) || !aligned16(up) || !aligned16(mid) || !aligned16(base) || !aligned16(dx) ||
        !aligned16(ddown) || !aligned16(dup) || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return EP_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (m->entries == 0 || m->rows == 0) {
        if (ddown) EP_CUDA_TRY(cudaMemsetAsync(ddown, 0, A * r * H * 2, stream));
        if (dup) EP_CUDA_TRY(cudaMemsetAsync(dup, 0, A * N * r * 2, stream));
        return without_rows(*m, adapter_offsets, nullptr, status, stream);
    }
    if (!dy || !adapter_offsets || ((dx || ddown) && !up) || (dx && !down) || (ddown && !x) || (dup && !mid)) return EP_ERR_NULL;
    if ((ddown || dup) && !workspace) return EP_ERR_NULL;
    if ((ddown || dup) && workspace_bytes < ep_adapter_matmul_backward_workspace_bytes(m)) return EP_ERR_CAPACITY;
    const GradPlan plan = plan_grads(*m);
    char *const ws = static_cast<char *>(workspace);
    void *dmid = ws + plan.counter_bytes + plan.list_bytes;
    PlanArgs pieces = {};
    if (ddown || dup) {
        const int64_t tiles = (ddown ? feature_tiles(m->in_features) : 0) + (dup ? feature_tiles(m->out_features) : 0);
        pieces.offsets = adapter_offsets, pieces.entries = m->entries;
        pieces.A = m->num_adapters, pieces.piece = plan.piece, pieces.tiles = (int)tiles, pieces.ctas = plan.ctas;
        pieces.counters = (int)plan.counters;
        pieces.pieces = reinterpret_cast<int *>(ws), pieces.arrived = pieces.pieces + 1;
        pieces.list = reinterpret_cast<GradPiece *>(ws + plan.counter_bytes);
        pieces.status = status;
    }
    TensorMapEncode encode;
    rc = tensor_map_encoder(&encode);
    if (rc != EP_OK) return rc;
    if (dx || ddown) {
        RankArgs a = {};
        a.offsets = adapter_offsets, a.index = row_index, a.status = status, a.scale = scale;
        a.base = static_cast<const uint16_t *>(base);
        a.out = static_cast<uint16_t *>(dx);
        a.mid = ddown ? static_cast<uint16_t *>(dmid) : nullptr;
        rc = launch_rank<true>(*m, encode, a, pieces, dy, down, up, stream);
        if (rc != EP_OK) return rc;
    }
    if (!ddown && !dup) return EP_OK;
    if (!dx && !ddown) {
        static std::atomic<uint64_t> planned{0};
        rc = launch_cluster(plan_kernel, planned, 1, 1, kThreads, (int)sizeof(PlanTables), (int)sizeof(PlanTables), stream, pieces);
        if (rc != EP_OK) return rc;
    }
    GradArgs g = {};
    g.index = row_index, g.scale = scale, g.status = status;
    g.x = static_cast<const uint16_t *>(x), g.dmid = static_cast<const uint16_t *>(dmid);
    g.dy = static_cast<const uint16_t *>(dy), g.mid = static_cast<const uint16_t *>(mid);
    GradMaps maps = {};
    if (ddown) {
        rc = make_map(encode, &maps.x, x, H, m->rows, 1, kTileK);
        if (rc == EP_OK) rc = make_map(encode, &maps.dmid, dmid, r, m->entries, 1, kTileK);
        if (rc != EP_OK) return rc;
    }
    if (dup) {
        rc = make_map(encode, &maps.dy, dy, N, m->rows, 1, kTileK);
        if (rc == EP_OK) rc = make_map(encode, &maps.mid, mid, r, m->entries, 1, kTileK);
        if (rc != EP_OK) return rc;
    }
    g.ddown = static_cast<uint16_t *>(ddown), g.dup = static_cast<uint16_t *>(dup);
    g.pieces = pieces.pieces, g.list = pieces.list, g.counter = pieces.arrived, g.arrived = pieces.arrived + 1;
    g.parts = reinterpret_cast<float *>(static_cast<char *>(dmid) + plan.dmid_bytes);
    g.rows = m->rows, g.H = m->in_features, g.N = m->out_features, g.rank = m->rank;
    g.tiles_down = ddown ? feature_tiles(m->in_features) : 0;
    g.tiles_up = dup ? feature_tiles(m->out_features) : 0;
    const int r16 = (m->rank + 15) & ~15;
    g.columns = r16 <= 32 ? 32 : r16 <= 64 ? 64 : 128;
    static std::atomic<uint64_t> ready[2];
    if (plan.stages == 4) return launch_cluster(adapter_grad_kernel<4>, ready[0], plan.ctas, 1, grad_threads(4), plan.smem, kRankSmem, stream, g, maps);
    return launch_cluster(adapter_grad_kernel<6>, ready[1], plan.ctas, 1, grad_threads(6), plan.smem, 222 * 1024, stream, g, maps);
}
