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

// Four rows' 64 elements from column x on, as four 128-byte lines. A row that does not exist gives zeros.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap *map, int x, const int (&row)[4], uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(map), "r"(x), "r"(row[0]), "r"(row[1]), "r"(row[2]), "r"(row[3]), "r"(bar)
        : "memory");
}

// What this thread wrote to shared memory is there for the tensor cores.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- the rank kernel ----------------------------------------------------------------------------------------------

constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 64 + 32 * kEpilogueWarps;
// Shared memory, from a 1024-byte boundary. The stages of the first product take 96 KB (a stage: 128 lines of rows and 64 or 128 lines
// of weights); afterwards the same memory holds the row operand of the second (16 or 32 KB), the epilogue's buffers (32 KB) and the
// weights' blocks (16 KB each). 15 KB behind them are for what the CTAs of a cluster exchange, if it fits there. Two CTAs
// fit on an SM, so that one reads while the other writes; 113 KB each also keep a CTA of the experts' products, which holds all of the
// tensor memory, from sharing an SM with one of a cluster: two clusters that each wait for the other's would wait for good.
constexpr int kRingBytes = 96 * 1024, kTailBytes = 15 * 1024 - 512;
constexpr int kStageWords = 32 * 32, kStageBytes = kEpilogueWarps * kStageWords * 4;      // an epilogue warp's 32 rows x 32 columns
constexpr int kRankSmem = 1024 + kRingBytes + kTailBytes;
constexpr int kMaxStages = 4, kMaxUnits = 3;

struct RankArgs {
    const int32_t *offsets;               // [A+1]
    const int32_t *index;                 // entry -> row, or NULL: entry i is row i
    int32_t *status;
    const float *scale;                   // [A] or NULL
    const uint16_t *base;                 // [rows][out], may be NULL or `out`
    uint16_t *out;                        // [rows][out], may be NULL: the first product alone
    uint16_t *mid;                        // [entries][rank], may be NULL
    long long rows, entries;
    int in, out_features, rank, A, split;
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
rank_kernel(const RankArgs a, const __grid_constant__ CUtensorMap map_in, const __grid_constant__ CUtensorMap map_first,
            const __grid_constant__ CUtensorMap map_second)
{
    extern __shared__ char raw[];
    __shared__ uint64_t full_[kMaxStages], empty_[kMaxStages], unit_full_[kMaxUnits], unit_empty_[kMaxUnits], mid_full_, mid_ready_, acc_full_[2],
        acc_empty_[2], ex_full_, ex_read_;
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_, warp_sum[kThreads / 32], where[3];
    __shared__ int row_of[kRows];
    volatile int *gave_up = &gave_up_;

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
            sum += quotient_up(max(0, end - begin), kRows);
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
                const int pieces = quotient_up(count, kRows);
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
    const int stage_bytes = kLines + chunks * 8192, stages = kRingBytes / stage_bytes;
    const int units = (kRingBytes - kStageBytes) / kLines - chunks;
    const int ex_ld = r16 + 4;
    const bool ex_small = m * ex_ld * 4 <= kTailBytes;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
    char *const ring_ptr = raw + (ring - smem_addr(raw));
    const uint32_t s_base = ring, unit_base = ring + chunks * kLines + kStageBytes;
    char *const stage_ptr = ring_ptr + chunks * kLines;
    float *const exchange = reinterpret_cast<float *>(ex_small ? ring_ptr + kRingBytes : stage_ptr);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) bar_init(smem_addr(&full_[s]), 1), bar_init(smem_addr(&empty_[s]), 1);
        for (int s = 0; s < kMaxUnits; ++s) bar_init(smem_addr(&unit_full_[s]), 1), bar_init(smem_addr(&unit_empty_[s]), 1);
        for (int s = 0; s < 2; ++s) bar_init(smem_addr(&acc_full_[s]), 1), bar_init(smem_addr(&acc_empty_[s]), kEpilogueWarps);
        bar_init(smem_addr(&mid_full_), 1);
        bar_init(smem_addr(&mid_ready_), kEpilogueWarps);
        bar_init(smem_addr(&ex_full_), split * kEpilogueWarps);
        bar_init(smem_addr(&ex_read_), split * kEpilogueWarps);
        gave_up_ = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_addr(&tmem_slot), 2 * kBlockColumns);
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
    const uint32_t tmem = tmem_slot;
    const uint32_t full0 = smem_addr(full_), empty0 = smem_addr(empty_), unit_full0 = smem_addr(unit_full_), unit_empty0 = smem_addr(unit_empty_);

    if (warp == 0) {
        // ---- rows and the first weights into the ring: lane l brings rows 4 l .. 4 l + 3
        int row[4];
        const bool mine = 4 * lane < m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            row[i] = mine ? row_of[4 * lane + i] : -1;
            if (row[i] < 0) row[i] = (int)a.rows;                            // does not exist: zeros
        }
        const uint32_t bytes = (uint32_t)((m + 3) / 4 * 512 + (BACK ? chunks * 8192 : r16 * 128));
        int s = 0, phase = 1, sent = 0;
        bool ok = true;
        for (int k = k_from; k < k_to; ++k) {
            ok = __all_sync(kFullMask, bar_wait(empty0 + 8 * s, phase, gave_up));
            if (!ok) break;
            const uint32_t full = full0 + 8 * s, dst = ring + s * stage_bytes;
            if (lane == 0) {
                bar_expect(full, bytes);
                if (BACK) {
                    for (int u = 0; u < chunks; ++u) tma_load<1>(dst + kLines + u * 8192, &map_first, 64 * u, k * kTileK, adapter, full);
                } else {
                    tma_load<1>(dst + kLines, &map_first, k * kTileK, 0, adapter, full);
                }
            }
            __syncwarp();
            if (mine) tma_gather4(dst + lane * 512, &map_in, k * kTileK, row, full);
            ++sent;
            if (++s == stages) s = 0, phase ^= 1;
        }
        if (!ok) {                                                           // gave up: let the copies in flight land
            for (int i = min(sent, stages); i > 0; --i) {
                int none = 0;
                if (s == 0) s = stages, phase ^= 1;
                --s;
                bar_wait(full0 + 8 * s, phase ^ 1, &none);
            }
        } else if (lane == 0 && blocks) {
            // ---- the second weights, once the ring's memory is free
            ok = bar_wait(smem_addr(&mid_full_), 0, gave_up);
            if (ok && split > 1 && !ex_small) ok = bar_wait<true>(smem_addr(&ex_read_), 0, gave_up);
            int u = 0, uphase = 1, usent = 0;
            for (int b = part; ok && b < blocks; b += split)
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
        if (ok) mma_commit<1>(smem_addr(&mid_full_));
        if (ok && blocks) {
            ok = bar_wait(smem_addr(&mid_ready_), 0, gave_up);
            tmem_fence_after();
            const uint32_t idesc2 = instr_desc(kRows, kBlockColumns, false, BACK);
            int u = 0, uphase = 0, used = 0;
            for (int b = part; ok && b < blocks; b += split, ++used) {
                const int acc = used & 1;
                if (!(ok = bar_wait(smem_addr(&acc_empty_[acc]), ((used >> 1) & 1) ^ 1, gave_up))) break;
                tmem_fence_after();
                for (int c = 0; c < chunks; ++c) {
                    if (!(ok = bar_wait(unit_full0 + 8 * u, uphase, gave_up))) break;
                    tmem_fence_after();
                    const uint32_t at = unit_base + u * kLines;
                    const uint64_t da = desc_k_major(s_base + c * kLines), db = BACK ? desc_mn_major(at) : desc_k_major(at);
                    const int steps = min(4, (r16 - 64 * c) / 16);
                    for (int j = 0; j < steps; ++j)
                        mma_bf16<1>(tmem + acc * kBlockColumns, da + j * 2, db + j * (BACK ? 128 : 2), idesc2, c > 0 || j > 0);
                    mma_commit<1>(unit_empty0 + 8 * u);
                    if (++u == units) u = 0, uphase ^= 1;
                }
                if (ok) mma_commit<1>(smem_addr(&acc_full_[acc]));
            }
        }
    } else if (warp >= 2) {
        const int q = warp & 3, half = (warp - 2) >> 2, thread = threadIdx.x - 64;
        const int my_row = q * 32 + lane;                                    // a warp reaches the lanes 32 (warp mod 4) .. + 31
        const float scale = a.scale ? __ldg(a.scale + adapter) : 1.f, mid_scale = BACK ? scale : 1.f, out_scale = BACK ? 1.f : scale;
        bool ok = bar_wait(smem_addr(&mid_full_), 0, gave_up);
        tmem_fence_after();
        // 8 columns of a row, rounded: the second product's operand, and `mid`
        const auto put = [&](int row, int col, float (&f)[8], bool store) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= mid_scale;
            const uint4 v = pack8(f);
            *reinterpret_cast<uint4 *>(ring_ptr + (col >> 6) * kLines + row * 128 + ((((col & 63) >> 3) ^ (row & 7)) << 4)) = v;
            if (store && a.mid && row < m && col < a.rank)
                *reinterpret_cast<uint4 *>(a.mid + (size_t)(entry0 + row) * a.rank + col) = v;
        };
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
                            put(my_row, c0 + 8 * j, f, true);
                        } else if (my_row < m) {
                            uint4 *dst = reinterpret_cast<uint4 *>(exchange + my_row * ex_ld + c0 + 8 * j);
                            dst[0] = make_uint4(v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3]);
                            dst[1] = make_uint4(v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]);
                        }
                    }
            }
        }
        if (split > 1 && ok) {
            // ---- the parts of all CTAs, added in their order by each of them
            __syncwarp();
            if (lane < split) bar_arrive_cluster_release(in_cta(smem_addr(&ex_full_), lane));
            ok = bar_wait<true>(smem_addr(&ex_full_), 0, gave_up);
            const int groups = r16 / 8;
            for (int i = thread; ok && i < m * groups; i += 32 * kEpilogueWarps) {
                const int row = i / groups, col = i % groups * 8;
                const uint32_t from = smem_addr(exchange + row * ex_ld + col);
                float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                for (int s = 0; s < split; ++s) {
                    const float4 lo = load_cluster(in_cta(from, s)), hi = load_cluster(in_cta(from, s) + 16);
                    f[0] += lo.x, f[1] += lo.y, f[2] += lo.z, f[3] += lo.w, f[4] += hi.x, f[5] += hi.y, f[6] += hi.z, f[7] += hi.w;
                }
                put(row, col, f, part == 0);
            }
            __syncwarp();
            if (!ex_small) {
                if (lane < split) bar_arrive_cluster_release(in_cta(smem_addr(&ex_read_), lane));
                ok = ok && bar_wait<true>(smem_addr(&ex_read_), 0, gave_up);
            }
        }
        fence_async();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_cluster_release(smem_addr(&mid_ready_));
        // ---- blocks of the output: lane l of a pass holds 8 columns of row 8 i + l / 4
        float *stage = reinterpret_cast<float *>(stage_ptr) + (warp - 2) * kStageWords;
        int rows[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) rows[i] = row_of[q * 32 + 8 * i + (lane >> 2)];
        int used = 0;
        for (int b = part; ok && b < blocks; b += split, ++used) {
            const int acc = used & 1;
            uint4 r[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col = b * kBlockColumns + half * 64 + h * 32 + (lane & 3) * 8;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    r[h][i] = make_uint4(0u, 0u, 0u, 0u);
                    if (a.base && rows[i] >= 0 && col < a.out_features)       // `base` may be the output: an ordinary load
                        r[h][i] = *reinterpret_cast<const uint4 *>(a.base + (size_t)rows[i] * a.out_features + col);
                }
            }
            if (!(ok = bar_wait(smem_addr(&acc_full_[acc]), (used >> 1) & 1, gave_up))) break;
            tmem_fence_after();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t v[32];
                tmem_load32(tmem + (uint32_t(q * 32) << 16) + acc * kBlockColumns + half * 64 + h * 32, v);
                if (h == 1) {
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_cluster(smem_addr(&acc_empty_[acc]));
                }
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<uint4 *>(stage + lane * 32 + ((j ^ (lane & 7)) << 2)) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                __syncwarp();
                const int col = b * kBlockColumns + half * 64 + h * 32 + (lane & 3) * 8;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 8 * i + (lane >> 2), j = (lane & 3) * 2;
                    const float4 lo = *reinterpret_cast<const float4 *>(stage + row * 32 + ((j ^ (row & 7)) << 2));
                    const float4 hi = *reinterpret_cast<const float4 *>(stage + row * 32 + (((j + 1) ^ (row & 7)) << 2));
                    const float z[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
                    float f[8];
                    unpack8(r[h][i], f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] = fmaf(out_scale, z[k], f[k]);
                    if (rows[i] >= 0 && col < a.out_features)
                        *reinterpret_cast<uint4 *>(a.out + (size_t)rows[i] * a.out_features + col) = pack8(f);
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
    if (threadIdx.x == 0 && gave_up_ && a.status) atomicOr(a.status, EP_STATUS_TIMEOUT);
}

// ---- the gradient kernel ------------------------------------------------------------------------------------------

constexpr int kGradThreads = 64 + 128;
constexpr int kGradLd = kRows + 4;        // accumulators on their way out: [rank][128 features]
constexpr int kGradStages = 4;

struct GradArgs {
    const int32_t *offsets, *index;
    const float *scale;
    int32_t *status;
    uint16_t *ddown, *dup;
    long long rows, entries;
    int H, N, rank, A, split;
    int tiles_down, tiles_up;             // feature tiles of an adapter's ddown (0: not wanted) and dup
    int stages, columns;                  // columns of tensor memory
};

__global__ void __launch_bounds__(kGradThreads)
adapter_grad_kernel(const GradArgs a, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_dmid,
                    const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_mid)
{
    extern __shared__ char raw[];
    __shared__ uint64_t full_[kGradStages], empty_[kGradStages], acc_full_, ex_full_;
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_;
    volatile int *gave_up = &gave_up_;

    const int warp = __shfl_sync(kFullMask, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int split = a.split, part = split > 1 ? (int)cluster_rank() : 0;
    const int item = blockIdx.x / split, tiles = a.tiles_down + a.tiles_up, adapter = item / tiles, f = item - adapter * tiles;
    const bool up = f >= a.tiles_down;
    const int m0 = (up ? f - a.tiles_down : f) * kRows, features = up ? a.N : a.H;
    const int chunks = (a.rank + 63) / 64, r16 = (a.rank + 15) & ~15;

    pdl_wait();
    const int begin = segment_bound(__ldg(a.offsets + adapter), a.entries), end = segment_bound(__ldg(a.offsets + adapter + 1), a.entries);
    const int n = max(0, end - begin), all_k = quotient_up(n, kTileK);
    const int k_from = (int)((long long)all_k * part / split), k_to = (int)((long long)all_k * (part + 1) / split);
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
    float *const out = reinterpret_cast<float *>(raw + (ring - smem_addr(raw)));
    const int stage_bytes = kLines + chunks * 8192, stages = a.stages;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kGradStages; ++s) bar_init(smem_addr(&full_[s]), 1), bar_init(smem_addr(&empty_[s]), 1);
        bar_init(smem_addr(&acc_full_), 1);
        bar_init(smem_addr(&ex_full_), split * 4);
        gave_up_ = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<1>(smem_addr(&tmem_slot), a.columns);
    tmem_fence_before();
    if (split > 1) cluster_sync();
    __syncthreads();
    tmem_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_slot, full0 = smem_addr(full_), empty0 = smem_addr(empty_);

    if (warp == 0) {
        // ---- entries into the ring: lane l brings entries 4 (l mod 16) .. + 3 of a stage, one half of the features each
        const CUtensorMap *rows_map = up ? &map_dy : &map_x, *rank_map = up ? &map_mid : &map_dmid;
        const int quad = lane & 15, side = lane >> 4;
        const uint32_t bytes = (uint32_t)stage_bytes;
        int s = 0, phase = 1, sent = 0;
        bool ok = true;
        for (int k = k_from; k < k_to; ++k) {
            int row[4], entry[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = k * kTileK + 4 * quad + i;
                entry[i] = (int)a.entries, row[i] = (int)a.rows;             // does not exist: zeros
                if (e < n) {
                    const int r = a.index ? __ldg(a.index + begin + e) : begin + e;
                    if (r >= 0 && r < a.rows) row[i] = r, entry[i] = begin + e;
                    else if (a.status) atomicOr(a.status, EP_STATUS_BAD_INDEX);
                }
            }
            ok = __all_sync(kFullMask, bar_wait(empty0 + 8 * s, phase, gave_up));
            if (!ok) break;
            const uint32_t full = full0 + 8 * s, dst = ring + s * stage_bytes;
            if (lane == 0) bar_expect(full, bytes);
            __syncwarp();
            tma_gather4(dst + side * 8192 + quad * 512, rows_map, m0 + side * 64, row, full);
            if (side < chunks) tma_gather4(dst + kLines + side * 8192 + quad * 512, rank_map, side * 64, entry, full);
            ++sent;
            if (++s == stages) s = 0, phase ^= 1;
        }
        if (!ok)
            for (int i = min(sent, stages); i > 0; --i) {
                int none = 0;
                if (s == 0) s = stages, phase ^= 1;
                --s;
                bar_wait(full0 + 8 * s, phase ^ 1, &none);
            }
    } else if (warp == 1 && elect_one()) {
        int s = 0, phase = 0;
        bool ok = true;
        const uint32_t idesc = instr_desc(kRows, r16, true, true);
        for (int k = k_from; k < k_to; ++k) {
            if (!(ok = bar_wait(full0 + 8 * s, phase, gave_up))) break;
            tmem_fence_after();
            const uint32_t at = ring + s * stage_bytes;
            const uint64_t da = desc_mn_major(at), db = desc_mn_major(at + kLines);
#pragma unroll
            for (int j = 0; j < kTileK / 16; ++j) mma_bf16<1>(tmem, da + j * 128, db + j * 128, idesc, k > k_from || j > 0);
            mma_commit<1>(empty0 + 8 * s);
            if (++s == stages) s = 0, phase ^= 1;
        }
        if (ok && k_to > k_from) mma_commit<1>(smem_addr(&acc_full_));
    } else if (warp >= 2) {
        // ---- accumulators out: through shared memory, added up over the CTAs that share them
        const int q = warp & 3, thread = threadIdx.x - 64;
        bool ok = true;
        if (k_to > k_from) ok = bar_wait(smem_addr(&acc_full_), 0, gave_up);
        tmem_fence_after();
        for (int c0 = 0; ok && c0 < r16; c0 += 32) {
            uint32_t v[32];
            if (k_to > k_from) {
                tmem_load32(tmem + (uint32_t(q * 32) << 16) + c0, v);
            } else {
#pragma unroll
                for (int c = 0; c < 32; ++c) v[c] = 0u;
            }
#pragma unroll
            for (int c = 0; c < 32; ++c)
                if (c0 + c < r16) out[(c0 + c) * kGradLd + q * 32 + lane] = __uint_as_float(v[c]);
        }
        if (split > 1) {
            __syncwarp();
            if (ok && lane < split) bar_arrive_cluster_release(in_cta(smem_addr(&ex_full_), lane));
            ok = ok && bar_wait<true>(smem_addr(&ex_full_), 0, gave_up);
        } else {
            asm volatile("bar.sync 1, 128;" ::: "memory");                   // the four warps
        }
        const float scale = up && a.scale ? __ldg(a.scale + adapter) : 1.f;
        // ddown: 8 features of a rank; dup: 8 ranks of a feature
        const int total = up ? kRows * (a.rank / 8) : a.rank * (kRows / 8);
        const int from = total * part / split, to = total * (part + 1) / split;
        for (int i = from + thread; ok && i < to; i += 128) {
            const int feature = up ? i % kRows : i % (kRows / 8) * 8, rank = up ? i / kRows * 8 : i / (kRows / 8);
            if (m0 + feature >= features) continue;
            float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            const float *src = out + rank * kGradLd + feature;
            for (int s = 0; s < split; ++s) {
                if (split == 1 && up) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = src[j * kGradLd];
                } else if (split == 1) {
                    const float4 lo = *reinterpret_cast<const float4 *>(src), hi = *reinterpret_cast<const float4 *>(src + 4);
                    z[0] = lo.x, z[1] = lo.y, z[2] = lo.z, z[3] = lo.w, z[4] = hi.x, z[5] = hi.y, z[6] = hi.z, z[7] = hi.w;
                } else if (up) {
                    const uint32_t at = in_cta(smem_addr(src), s);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float w;
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w) : "r"(at + j * kGradLd * 4) : "memory");
                        z[j] += w;
                    }
                } else {
                    const uint32_t at = in_cta(smem_addr(src), s);
                    const float4 lo = load_cluster(at), hi = load_cluster(at + 16);
                    z[0] += lo.x, z[1] += lo.y, z[2] += lo.z, z[3] += lo.w, z[4] += hi.x, z[5] += hi.y, z[6] += hi.z, z[7] += hi.w;
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] *= scale;
            uint16_t *dst = up ? a.dup + ((size_t)adapter * a.N + m0 + feature) * a.rank + rank : a.ddown + ((size_t)adapter * a.rank + rank) * a.H + m0 + feature;
            *reinterpret_cast<uint4 *>(dst) = pack8(z);
        }
    }
    __syncwarp();
    tmem_fence_before();
    __syncthreads();
    if (split > 1) cluster_sync();
    tmem_fence_after();
    if (warp == 1) tmem_free<1>(tmem, a.columns);
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

// A bf16 array [rows][inner], read four single rows at a time.
int make_gather_map(TensorMapEncode encode, CUtensorMap *map, const void *base, uint64_t inner, uint64_t rows)
{
    const cuuint64_t dim[2] = {inner, rows}, stride[1] = {inner * 2};
    const cuuint32_t box[2] = {64, 1}, step[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dim, stride, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        note_cuda_error(cudaErrorInvalidValue);
        return EP_ERR_CUDA;
    }
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
    CUtensorMap map_in, map_first, map_second;
    int rc = make_gather_map(encode, &map_in, in, a.in, m.rows);
    if (rc == EP_OK)
        rc = BACK ? make_map(encode, &map_first, up, r, N, A, 64) : make_map(encode, &map_first, down, H, r, A, (uint32_t)((r + 15) & ~15));
    if (rc == EP_OK) {
        if (!a.out) map_second = map_first;
        else rc = BACK ? make_map(encode, &map_second, down, H, r, A, 64) : make_map(encode, &map_second, up, r, N, A, 128);
    }
    if (rc != EP_OK) return rc;
    const int64_t tiles = m.entries / kRows + (m.entries < m.num_adapters ? m.entries : m.num_adapters);      // at most
    const int stages = (a.in + kTileK - 1) / kTileK;
    a.split = 1;
    while (a.split < kMaxCluster && tiles * a.split * 2 <= 2 * 148 && stages >= 4 * a.split) a.split *= 2;
    return launch_cluster(rank_kernel<BACK>, ready, tiles, a.split, kThreads, kRankSmem, kRankSmem, stream, a, map_in, map_first, map_second);
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
    CUtensorMap map_x, map_dmid, map_dy, map_mid;
    if (ddown) {
        rc = make_gather_map(encode, &map_x, x, H, m->rows);
        if (rc == EP_OK) rc = make_gather_map(encode, &map_dmid, dmid, r, m->entries);
        if (rc != EP_OK) return rc;
    }
    if (dup) {
        rc = make_gather_map(encode, &map_dy, dy, N, m->rows);
        if (rc == EP_OK) rc = make_gather_map(encode, &map_mid, mid, r, m->entries);
        if (rc != EP_OK) return rc;
    }
    if (!ddown) map_x = map_dy, map_dmid = map_mid;
    if (!dup) map_dy = map_x, map_mid = map_dmid;
    GradArgs g = {};
    g.offsets = adapter_offsets, g.index = row_index, g.scale = scale, g.status = status;
    g.ddown = static_cast<uint16_t *>(ddown), g.dup = static_cast<uint16_t *>(dup);
    g.rows = m->rows, g.entries = m->entries, g.H = m->in_features, g.N = m->out_features, g.rank = m->rank, g.A = m->num_adapters;
    g.tiles_down = ddown ? (m->in_features + kRows - 1) / kRows : 0;
    g.tiles_up = dup ? (m->out_features + kRows - 1) / kRows : 0;
    const int64_t items = (int64_t)g.A * (g.tiles_down + g.tiles_up), average = m->entries / m->num_adapters / kTileK;
    g.split = 1;
    while (g.split < kMaxCluster && items * g.split * 2 <= 2 * 148 && average >= 4 * g.split) g.split *= 2;
    const int r16 = (m->rank + 15) & ~15, chunks = (m->rank + 63) / 64, stage = kLines + chunks * 8192;
    g.columns = r16 <= 32 ? 32 : r16 <= 64 ? 64 : 128;
    // three or four CTAs on an SM; those of a cluster take over half of it (see the rank kernel)
    g.stages = chunks == 1 ? 3 : 3;
    int smem = 1024 + g.stages * stage;
    if (g.split > 1) smem = kRankSmem, g.stages = (smem - 1024) / stage < kGradStages ? (smem - 1024) / stage : kGradStages;
    static std::atomic<uint64_t> ready{0};
    return launch_cluster(adapter_grad_kernel, ready, items, g.split, kGradThreads, smem, kRankSmem, stream, g, map_x, map_dmid, map_dy, map_mid);
}
