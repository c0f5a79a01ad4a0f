// Matrix products of two 16-bit matrices for many tokens: the codes have been turned into 16-bit floats once, by a
// kernel before this one, since every 256 rows of the result would otherwise convert them anew.
#pragma once

#include "linear_gemm.cuh"

namespace sq {

constexpr int kPairRows = 256;    // rows of a tile: two thread blocks with 128 each
constexpr int kDenseEpilogueWarps = 8;
constexpr int kDenseThreads = 32 * (kDenseEpilogueWarps + 2);

template <int kCols>
struct DenseShape {
    static constexpr int kBytesA = 128 * 128;            // of one thread block: 128 rows
    static constexpr int kBytesB = kCols / 2 * 128;      // and half of the columns
    static constexpr int kStages = kCols == 256 ? 6 : 8;
    static constexpr int kTmemCols = 2 * kCols;
    static constexpr int kSmem = 1024 + kStages * (kBytesA + kBytesB) + kDenseEpilogueWarps * kTurnBytes + 8 * (2 * kStages + 4);
    static_assert(kSmem + 1024 + 128 <= 228 << 10, "fits a multiprocessor");
    static_assert(kSmem + kFusedSmem > 228 << 10 && 2 * kSmem > 228 << 10 && kTmemCols <= 512,
                  "alone among the kernels that use tensor memory, so that what it asks for is always there");
};

__device__ __forceinline__ void remote_arrive(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// bar_wait_warp() for arrivals of the other block too.
__device__ __forceinline__ bool pair_wait(uint32_t bar, uint32_t parity, volatile int *gave_up)
{
    if (!bar_wait_warp(bar, parity, gave_up)) return false;
    asm volatile("fence.acq_rel.cluster;" ::: "memory");
    return true;
}
// A copy into this thread block's shared memory whose bytes count at a barrier of the pair's first block.
__device__ __forceinline__ void pair_tma_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t cluster_bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void pair_tmem_alloc(uint32_t where, uint32_t columns)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void pair_tmem_free(uint32_t addr, uint32_t columns)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
// The products issued so far have been taken: arrives at the barrier of this place in both thread blocks.
__device__ __forceinline__ void pair_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void pair_mma_f16(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)), "n"(kDescHigh) : "memory");
}

// Clusters of two thread blocks, persistent, one block a multiprocessor.  A tile of 256 rows belongs to a pair: each
// block copies its 128 rows of the one operand and its half of the columns of the other into its own shared memory, the
// first block's matrix instructions read both, and each block's tensor memory receives its own 128 rows.  Per product
// the shared memory is so read and written half as often as by one block alone (a tile of 128 x 256 by one block, converting the
// codes itself: 600 TFLOP/s; this 1,480 to 1,520, tensor pipe 76 % busy, bound by board power in long runs).  Warps 0-7 epilogue (two per quarter of the
// tensor memory's lanes, half of the columns each), 8 copies, 9 issues the matrix instructions (first block only).
template <int kMode, bool kHalf, int kCols>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kDenseThreads, 1)
dense_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ GemmArgs p)
{
    using S = DenseShape<kCols>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t smem_a = base, smem_b = base + S::kStages * S::kBytesA;
    const uint32_t turns = smem_b + S::kStages * S::kBytesB, bars = turns + kDenseEpilogueWarps * kTurnBytes;
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (S::kStages + s); };
    auto acc_full = [&](int a) { return bars + 8 * (2 * S::kStages + a); };
    auto acc_empty = [&](int a) { return bars + 8 * (2 * S::kStages + 2 + a); };
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up_word;
    volatile int *gave_up = &gave_up_word;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();

    if (threadIdx.x == 0) {
        gave_up_word = 0;
        for (int s = 0; s < S::kStages; ++s) {
            bar_init(full(s), 1);
            bar_init(empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            bar_init(acc_full(a), 1);
            bar_init(acc_empty(a), 2 * kDenseEpilogueWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kDenseEpilogueWarps + 1) pair_tmem_alloc(smem_addr(&tmem_base), S::kTmemCols);
    tc_fence_before();
    __syncthreads();
    cluster_arrive_wait();   // the other block's barriers are there
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    const int steps = p.steps;
    const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    SQ_LINEAR_CHECK(bars + 8 * (2 * S::kStages + 4) <= smem_end(smem_raw) && (turns & 3) == 0, 1040);
    SQ_LINEAR_CHECK(steps >= 1 && static_cast<int64_t>(steps) * kTileDepth <= kLongestSum && p.first_step >= 0 &&
                    static_cast<int64_t>(p.first_step + steps - 1) * kTileDepth < p.depth, 1041);

    if (warp < kDenseEpilogueWarps) {
        const int quarter = warp & 3, part = warp >> 2;
        int n = 0;
        for (int64_t t = pair; t < p.tiles; t += pairs, ++n) {
            const int a = n & 1;
            if (!bar_wait_warp(acc_full(a), (n >> 1) & 1, gave_up)) break;
            tc_fence_after();
            const int64_t row = (t % p.row_tiles) * kPairRows + rank * 128 + quarter * 32;
            const int64_t col0 = t / p.row_tiles * kCols;
            for (int c = part * (kCols / 2); c < (part + 1) * (kCols / 2); c += 32) {
                if (col0 + c >= p.cols) break;
                SQ_LINEAR_CHECK(a * kCols + c + 32 <= S::kTmemCols, 1042);
                uint32_t acc[32];
                __syncwarp();
                tmem_ld32(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + a * kCols + c, acc);
                finish32<kMode, kHalf>(p, row, static_cast<int>(col0) + c, acc, turns + warp * kTurnBytes);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) remote_arrive(cluster_addr(acc_empty(a), 0));
        }
    } else if (warp == kDenseEpilogueWarps) {
        bool ok = true;
        int s = 0, issued = 0;
        uint32_t parity = 1;
        for (int64_t t = pair; t < p.tiles && ok; t += pairs) {
            const int row0 = static_cast<int>(t % p.row_tiles) * kPairRows + static_cast<int>(rank) * 128;
            const int col0 = static_cast<int>(t / p.row_tiles * kCols) + static_cast<int>(rank) * (kCols / 2);
            for (int k = 0; k < steps; ++k) {
                ok = bar_wait_warp(empty(s), parity, gave_up);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = cluster_addr(full(s), 0);
                    if (rank == 0) bar_expect(full(s), 2 * (S::kBytesA + S::kBytesB));
                    const uint32_t at = smem_a + s * S::kBytesA, bt = smem_b + s * S::kBytesB;
                    const int from = (p.first_step + k) * kTileDepth;
                    SQ_LINEAR_CHECK(s >= 0 && s < S::kStages && row0 >= 0 && col0 >= 0 && from >= 0 && from < p.depth, 1043);
                    if (kMode == kWeightGrad) {
                        pair_tma_2d(at, &map_a, row0, from, bar);
                        pair_tma_2d(at + 8192, &map_a, row0 + 64, from, bar);
                    } else {
                        pair_tma_2d(at, &map_a, from, row0, bar);
                    }
                    if (kMode == kForward) {
                        pair_tma_2d(bt, &map_b, from, col0, bar);
                    } else {
#pragma unroll
                        for (int j = 0; j < kCols / 128; ++j) pair_tma_2d(bt + 8192 * j, &map_b, col0 + 64 * j, from, bar);
                    }
                }
                __syncwarp();
                if (issued < S::kStages) ++issued;
                if (++s == S::kStages) { s = 0; parity ^= 1; }
            }
        }
        // the last copies have landed and the matrix instructions have read them before the block may end
        for (int i = 0; i < issued; ++i) {
            if (--s < 0) { s = S::kStages - 1; parity ^= 1; }
            if (rank == 0) bar_drain(full(s), parity ^ 1);
            bar_drain(empty(s), parity ^ 1);
        }
    } else if (rank == 0) {
        constexpr uint32_t kIdesc = (1u << 4) | (kHalf ? 0u : 1u << 7) | (kHalf ? 0u : 1u << 10) |
                                    (kMode == kWeightGrad ? 1u << 15 : 0u) | (kMode != kForward ? 1u << 16 : 0u) |
                                    (static_cast<uint32_t>(kCols >> 3) << 17) | (static_cast<uint32_t>(kPairRows >> 4) << 24);
        constexpr uint32_t kStepA = kMode == kWeightGrad ? 2048 : 32, kStepB = kMode == kForward ? 32 : 2048;
        bool ok = true;
        int s = 0, n = 0;
        uint32_t parity = 0;
        for (int64_t t = pair; t < p.tiles && ok; t += pairs, ++n) {
            const int a = n & 1;
            ok = pair_wait(acc_empty(a), ((n >> 1) & 1) ^ 1, gave_up);
            if (!ok) break;
            tc_fence_after();
            for (int k = 0; k < steps; ++k) {
                ok = bar_wait_warp(full(s), parity, gave_up);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = desc_low(smem_a + s * S::kBytesA, kMode == kWeightGrad ? 8192 : 16);
                const uint32_t bt = desc_low(smem_b + s * S::kBytesB, kMode == kForward ? 16 : 8192);
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < kTileDepth / 16; ++i)
                        pair_mma_f16(tmem + a * kCols, at + i * (kStepA >> 4), bt + i * (kStepB >> 4), kIdesc, k > 0 || i > 0);
                    pair_commit(empty(s));
                    if (k + 1 == steps) pair_commit(acc_full(a));
                }
                __syncwarp();
                if (++s == S::kStages) { s = 0; parity ^= 1; }
            }
        }
    }
    __syncwarp();
    if (*gave_up) __nanosleep(100000);   // nobody has waited for the last signal of a tile's sums: it is here by then
    tc_fence_before();
    __syncthreads();
    cluster_arrive_wait();   // the other block reads this one's shared memory and signals its barriers until here
    if (warp == kDenseEpilogueWarps + 1) {
        tc_fence_after();
        pair_tmem_free(tmem, S::kTmemCols);
    }
}

}  // namespace sq
