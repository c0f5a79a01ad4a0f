// Attention over the cache for few rows: decoding steps and the check of drafted tokens.
//
//   s_ij = scale q_i k_j,   p_ij = exp(s_ij - max_j s_ij),   out_i = sum_j p_ij v_j / sum_j p_ij,   lse_i = log sum_j exp(s_ij)
//
// A tile is 8 (or 16) rows of one sequence and kv head: tokens times the query heads of the group.  What bounds it is the cache's bytes, and next to them the instructions that turn
// codes into floats: at the copy bandwidth a multiprocessor gets 23 bytes a clock, a position of 128 channels (144 bytes) every 6.2 clocks or 25 issue slots,
// of which the conversion takes 12 and softmax and matrix instructions 7.
//
// Work is cut by what there is, not by sequence: the units (32 positions of a tile) of all sequences stand in one row, and each thread block takes an equal stretch of
// it, which may hold the end of one tile, whole ones and the beginning of another.  A tile that several blocks have a part of is put together by the block that ends
// last, in the order of the blocks, so that results repeat to the bit.
#pragma once

#include "cache_device.cuh"

namespace sq {

struct AttendArgs {
    const uint8_t *cache;
    CacheRows r;
    const uint16_t *q;
    int64_t q_stride, q_head;      // elements from row to row and from head to head
    uint16_t *out;
    int64_t out_stride, out_head;
    float *lse;                    // [rows][q heads], or null
    int32_t group;
    int32_t q_vector, out_vector;  // rows of q start on 16 bytes, of out on 16
    float scale_log2;              // the scale over log 2
    unsigned long long *tickets;   // workspace, see arrive()
    float *parts;
    unsigned long long nonce;
};

constexpr int kStepWarps = 8, kStepThreads = 32 * kStepWarps;
constexpr int kStepStages = 2;                 // of a warp: one being read, one in flight
constexpr int kStepPositions = 2 * kGranule;   // of a unit
constexpr int kMergeRows = 8;
constexpr float kGrowth = 8.0f;                // the running maximum is replaced when a new one is 2^8 as large: sums stay far inside fp32 and bf16

template <int D>
struct StepShape {
    static constexpr int kBlocks = D > 128 ? 1 : 2;   // on a multiprocessor
    static constexpr int kStage = kStepPositions / kGranule * CacheFormat<D>::kBytes;
    static constexpr int kRing = kStepWarps * kStepStages * kStage;
    static constexpr int kPitch = D + 4;              // floats of a row's sums
    static constexpr int kMerge = kStepWarps * kMergeRows * kPitch * 4, kSums = kStepWarps * kMergeRows * 8;
    static constexpr int kSmem = kRing + kMerge + kSums + 8 * kStepWarps * kStepStages;
};
// Floats of a tile's part in the workspace: its rows' sums, then maximum and sum of each row.
template <int D>
__host__ __device__ constexpr int part_floats(int rows) { return rows * (D + 2); }

// True in the last of `n` blocks of this call to say so.  The word may hold anything before the call but for its nonce, which no other call has: the first block to come puts
// nonce and count in, the last one takes them away, so that a replayed graph starts as the call did.
__device__ __forceinline__ bool arrive(unsigned long long *word, unsigned long long nonce, unsigned n)
{
    unsigned long long old = *const_cast<volatile unsigned long long *>(word);
    unsigned count;
    for (;;) {
        if ((old >> 16) == nonce) {
            count = static_cast<unsigned>(atomicAdd(word, 1ull) & 0xffffu) + 1;
            break;
        }
        const unsigned long long found = atomicCAS(word, old, nonce << 16 | 1ull);   // fails only where another block has been quicker
        if (found == old) {
            count = 1;
            break;
        }
        old = found;
    }
    if (count != n) return false;
    atomicExch(word, 0ull);
    return true;
}

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, bool half_type)
{
    if (half_type)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A walk over the row of units, the same in all threads of a block.
struct Walk {
    int64_t x, end;       // next unit, and where the block's stretch ends
    int64_t base;         // first unit of sequence b
    int64_t tiles, row0;  // tiles of sequence b and kv head; its first row
    int64_t item0, item1; // units of the piece's tile
    int b, n, len, units; // sequence, its rows and positions, units of a tile
    int head, first, last;   // of the piece: kv head, units [first, last)
    int64_t tile;

    __device__ __forceinline__ int64_t work(const CacheRows &r) const { return tiles * r.kv_heads * units; }
    __device__ __forceinline__ void load(const CacheRows &r, int group, int rows)
    {
        row0 = row_start(r, b);
        n = static_cast<int>(max(static_cast<int64_t>(0), (r.starts ? row_start(r, b + 1) : row0 + 1) - row0));
        len = length_of(r, b);
        units = max(1, (len + kStepPositions - 1) / kStepPositions);
        tiles = (static_cast<int64_t>(n) * group + rows - 1) / rows;
    }
    // The next piece; false at the end.
    __device__ __forceinline__ bool next(const CacheRows &r, int group, int rows)
    {
        if (x >= end) return false;
        for (int64_t w; x >= base + (w = work(r));) {
            base += w;
            ++b;
            load(r, group, rows);
        }
        const int64_t item = (x - base) / units;
        item0 = base + item * units;
        item1 = item0 + units;
        head = static_cast<int>(item / tiles);
        tile = item % tiles;
        first = static_cast<int>(x - item0);
        x = min(end, item1);
        last = static_cast<int>(x - item0);
        return true;
    }
    // The last position that row `at` of the sequence's rows times heads sees; below 0: none.
    __device__ __forceinline__ int limit(int64_t at, int group) const { return len - n + static_cast<int>(at / group); }
};

// rows of a tile: 8 * kHalves.  With 8 rows, the other eight of the matrix instructions' 16 hold what the rounding of the first eight's probabilities left over,
// so that the products with the values are as good as fp32's; with 16 rows probabilities are rounded to the values' type (2^-9 or 2^-12 of each).
template <int D, bool kHalf, int kHalves>
__global__ void __launch_bounds__(kStepThreads, StepShape<D>::kBlocks)
cache_step_kernel(const __grid_constant__ AttendArgs p)
{
    using F = CacheFormat<D>;
    using S = StepShape<D>;
    constexpr int kRows = 8 * kHalves, kGroupsAll = D / kGroup;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t warp_sums[kStepWarps];
    __shared__ int64_t start_base;
    __shared__ int start_b, gave_up_word, is_last;
    volatile int *gave_up = &gave_up_word;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    float *const merge = reinterpret_cast<float *>(smem + S::kRing);
    float2 *const sums = reinterpret_cast<float2 *>(smem + S::kRing + S::kMerge);
    const uint32_t ring = smem_addr(smem) + warp * kStepStages * S::kStage;
    const uint32_t bars = smem_addr(smem) + S::kRing + S::kMerge + S::kSums + 8 * warp * kStepStages;
    SQ_LINEAR_CHECK(smem_addr(smem) + S::kSmem <= smem_end(smem) && (smem_addr(smem) & 15) == 0, 2010);
    if (threadIdx.x == 0) gave_up_word = 0;
    if (lane == 0) {
        for (int s = 0; s < kStepStages; ++s) bar_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }

    // the block's stretch of the units of all sequences
    Walk walk;
    const auto work_of = [&](int b) {
        if (b >= p.r.batch) return static_cast<int64_t>(0);
        Walk w;
        w.b = b;
        w.load(p.r, p.group, kRows);
        return w.work(p.r);
    };
    int64_t sum = 0;
    for (int b = threadIdx.x; b < p.r.batch; b += kStepThreads) sum += work_of(b);
#pragma unroll
    for (int s = 16; s; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if (lane == 0) warp_sums[warp] = sum;
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < kStepWarps; ++w) total += warp_sums[w];
    const int64_t share = max(static_cast<int64_t>(kStepWarps), (total + gridDim.x - 1) / gridDim.x);
    walk.x = share * blockIdx.x;
    walk.end = min(total, walk.x + share);
    if (walk.x >= total) return;
    int64_t before = 0;
    for (int b0 = 0; b0 < p.r.batch; b0 += kStepThreads) {
        const int64_t mine = work_of(b0 + threadIdx.x);
        int64_t upto = mine;
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, upto, s);
            if (lane >= s) upto += v;
        }
        __syncthreads();
        if (lane == 31) warp_sums[warp] = upto;
        __syncthreads();
        int64_t all = 0;
#pragma unroll
        for (int w = 0; w < kStepWarps; ++w) {
            if (w == warp) upto += before + all;
            all += warp_sums[w];
        }
        if (walk.x >= upto - mine && walk.x < upto) {   // one thread of all chunks
            start_b = b0 + static_cast<int>(threadIdx.x);
            start_base = upto - mine;
        }
        before += all;
        if (before > walk.x) break;
    }
    __syncthreads();
    walk.b = start_b;
    walk.base = start_base;
    walk.load(p.r, p.group, kRows);

    // copies of the warp's units, ahead of what it computes
    Walk ahead = walk;
    int ahead_unit = 0, fetched = 0, consumed = 0;
    uint32_t there = 0;   // two bits a stage: which of its granules have been copied
    bool more = ahead.next(p.r, p.group, kRows), dead = false;
    ahead_unit = ahead.first + warp;
    const auto fetch = [&]() {
        while (more && ahead_unit >= ahead.last) {
            more = ahead.next(p.r, p.group, kRows);
            ahead_unit = ahead.first + warp;
        }
        if (!more) return;
        const int stage = fetched % kStepStages, position = ahead_unit * kStepPositions;
        const int seen = ahead.limit(min(static_cast<int64_t>(ahead.n) * p.group, (ahead.tile + 1) * kRows) - 1, p.group);   // by the tile's last row
        const int granules = p.r.page_size / kGranule;
        const uint8_t *from[2];
        uint32_t have = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = position + i * kGranule;
            if (at > seen) continue;
            const int column = at / p.r.page_size;
            const int64_t page = page_of(p.r, ahead.b, column);
            if (page < 0) continue;
            have |= 1u << i;
            from[i] = p.cache + ((page * p.r.kv_heads + ahead.head) * granules + (at - column * p.r.page_size) / kGranule) * F::kBytes;
            SQ_LINEAR_CHECK(column < p.r.width && from[i] >= p.cache && from[i] + F::kBytes <= p.cache + p.r.page_count * p.r.kv_heads * granules * F::kBytes, 2011);
        }
        if (elect_one()) {
            const uint32_t to = ring + stage * S::kStage;
            bar_expect(bars + 8 * stage, __popc(have) * F::kBytes);
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (have >> i & 1) bulk_load(to + i * F::kBytes, from[i], F::kBytes, bars + 8 * stage);
        }
        __syncwarp();
        there = (there & ~(3u << (2 * stage))) | have << (2 * stage);
        ++fetched;
        ahead_unit += kStepWarps;
    };
#pragma unroll
    for (int s = 0; s < kStepStages; ++s) fetch();

    const CodePairs<kHalf> pairs;
    const int heads = p.r.kv_heads * p.group;
    while (walk.next(p.r, p.group, kRows)) {
        const int64_t at0 = walk.tile * kRows, rows_all = static_cast<int64_t>(walk.n) * p.group;   // of the sequence's rows times heads
        uint32_t q[kGroupsAll][kHalves][4];
        int limit[kHalves];
#pragma unroll
        for (int r = 0; r < kHalves; ++r) {
            const int64_t at = at0 + 8 * r + g;
            limit[r] = walk.limit(min(at, rows_all - 1), p.group);
            const uint16_t *from = p.q + (walk.row0 + at / p.group) * p.q_stride + (static_cast<int64_t>(walk.head) * p.group + at % p.group) * p.q_head;
#pragma unroll
            for (int n = 0; n < kGroupsAll; ++n) {
                const uint4 v = at < rows_all ? load8(from + kGroup * n + 8 * c, p.q_vector) : make_uint4(0, 0, 0, 0);
                q[n][r][0] = v.x; q[n][r][1] = v.y; q[n][r][2] = v.z; q[n][r][3] = v.w;
            }
        }
        const int seen_least = walk.limit(at0, p.group), seen_most = walk.limit(min(rows_all, at0 + kRows) - 1, p.group);
        float o[D / 8][4], most[kHalves], total_p[kHalves];
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
#pragma unroll
        for (int r = 0; r < kHalves; ++r) {
            most[r] = -INFINITY;
            total_p[r] = 0.0f;
        }

        for (int unit = walk.first + warp; unit < walk.last; unit += kStepWarps) {
            if (dead) break;
            const int stage = consumed % kStepStages;
            if (!bar_wait_warp(bars + 8 * stage, consumed / kStepStages & 1, gave_up)) {
                dead = true;
                break;
            }
            SQ_LINEAR_CHECK(consumed < fetched, 2012);
            const uint32_t have = there >> (2 * stage) & 3u, data = ring + stage * S::kStage;
            const int position = unit * kStepPositions;
            if (have) {
                // scores of 32 positions, 8 at a time; the lane has positions 8 i + 2 c and the next of row g (and g + 8)
                float s[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
                    if (!(have >> (i >> 1) & 1)) continue;
                    const uint32_t granule = data + (i >> 1) * F::kBytes;
                    const int t = 8 * (i & 1) + g;
                    uint32_t scales[kGroupsAll / 2];
                    if constexpr (kGroupsAll == 2) {
                        scales[0] = lds32(granule + F::key_scale(0, 0) + t * 4);
                    } else {
#pragma unroll
                        for (int n = 0; n < kGroupsAll / 4; ++n) {
                            const uint2 v = lds64(granule + F::key_scale(0, 0) + t * (2 * kGroupsAll) + 8 * n);
                            scales[2 * n] = v.x;
                            scales[2 * n + 1] = v.y;
                        }
                    }
#pragma unroll
                    for (int a = 0; a < F::kSlabs; ++a) {
                        uint32_t w[4];
                        if constexpr (F::kGroups == 2) {
                            const uint2 v = lds64(granule + t * (4 * F::kWords) + 8 * c);
                            w[0] = v.x; w[1] = v.y;
                        } else {
                            const uint4 v = lds128(granule + a * (64 * F::kWords) + t * (4 * F::kWords) + 16 * c);
                            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                        }
#pragma unroll
                        for (int j = 0; j < F::kGroups; ++j) {
                            const int n = a * F::kGroups + j;
                            const uint32_t scale = scale_twice<kHalf>(scales[n / 2], n & 1);
                            uint32_t k[4];
                            pairs(w[j], scale, pairs.offset(scale), k);
                            const uint32_t (&x)[4] = q[n][0], (&y)[4] = q[n][kHalves - 1];
                            mma_16816(s[i], x[0], kHalves > 1 ? y[0] : 0u, x[1], kHalves > 1 ? y[1] : 0u, k[0], k[1], kHalf);
                            mma_16816(s[i], x[2], kHalves > 1 ? y[2] : 0u, x[3], kHalves > 1 ? y[3] : 0u, k[2], k[3], kHalf);
                        }
                    }
                }
                const bool masked = position + kStepPositions - 1 > seen_least || have != 3;   // some row does not see all
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 2 * kHalves; ++e) {
                        s[i][e] *= p.scale_log2;
                        if (masked && (position + 8 * i + 2 * c + (e & 1) > limit[e >> 1] || !(have >> (i >> 1) & 1))) s[i][e] = -INFINITY;
                    }
                float reached[kHalves];
                bool grows = false;
#pragma unroll
                for (int r = 0; r < kHalves; ++r) {
                    float v = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v = fmaxf(v, fmaxf(s[i][2 * r], s[i][2 * r + 1]));
                    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
                    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
                    reached[r] = v;
                    grows |= v > most[r] + kGrowth;
                }
                if (__any_sync(0xffffffffu, grows)) {
                    float factor[kHalves];
#pragma unroll
                    for (int r = 0; r < kHalves; ++r) {
                        const float next = fmaxf(most[r], reached[r]);
                        factor[r] = next == most[r] ? 1.0f : exp2_fast(most[r] - next);
                        most[r] = next;
                        total_p[r] *= factor[r];
                    }
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        o[i][0] *= factor[0];
                        o[i][1] *= factor[0];
                        o[i][2] *= factor[kHalves - 1];
                        o[i][3] *= factor[kHalves - 1];
                    }
                }
                // probabilities as the first operand of the product with the values
                uint32_t hi[4][kHalves], lo[4];
#pragma unroll
                for (int r = 0; r < kHalves; ++r) {
                    const float from = most[r] == -INFINITY ? 0.0f : most[r];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float a = exp2_fast(s[i][2 * r] - from), b = exp2_fast(s[i][2 * r + 1] - from);
                        total_p[r] += a + b;
                        hi[i][r] = to_16x2<kHalf>(a, b);
                        if (kHalves == 1) lo[i] = to_16x2<kHalf>(a - to_float<kHalf>(static_cast<uint16_t>(hi[i][r])), b - to_float<kHalf>(static_cast<uint16_t>(hi[i][r] >> 16)));
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (!(have >> i & 1)) continue;
                    const uint32_t granule = data + i * F::kBytes;
                    const int left = seen_most + 1 - (position + i * kGranule);   // positions of the granule that any row sees
                    // scales of positions 2 c, 2 c + 1 and 2 c + 8, 2 c + 9 for the groups of the lane's words
                    uint32_t scales[2][D / 64];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int a = 0; a < F::kSlabs; ++a) {
                            const uint32_t at = granule + F::kValueScales + a * (32 * F::kGroups) + (c + 4 * h) * (4 * F::kGroups) + (g >> 2) * (2 * F::kGroups);
                            if constexpr (F::kGroups == 2) {
                                scales[h][0] = lds32(at);
                            } else {
                                const uint2 v = lds64(at);
                                scales[h][2 * a] = v.x;
                                scales[h][2 * a + 1] = v.y;
                            }
                        }
                    }
                    if (masked) {
                        // positions behind the last one may hold anything
                        bool odd = false;
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int n = 0; n < D / 64; ++n) {
                                if (2 * c + 8 * h >= left) scales[h][n] &= 0xffff0000u;
                                if (2 * c + 8 * h + 1 >= left) scales[h][n] &= 0x0000ffffu;
                                odd |= (scales[h][n] & 0x7f80u) == 0x7f80u || (scales[h][n] & 0x7f800000u) == 0x7f800000u;
                            }
                        if (__any_sync(0xffffffffu, odd)) {
                            // a group without a number, which some row may not see: it makes NaN of the rows that do and no product
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int n = 0; n < D / 64; ++n) {
                                    if ((scales[h][n] & 0x7f80u) == 0x7f80u) scales[h][n] &= 0xffff0000u;
                                    if ((scales[h][n] & 0x7f800000u) == 0x7f800000u) scales[h][n] &= 0x0000ffffu;
                                }
                            for (int t = 0; t < min(left, kGranule); ++t)
#pragma unroll
                                for (int n = 0; n < kGroupsAll; ++n) {
                                    uint16_t v;
                                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(granule + F::value_scale(0, n) + (t >> 1) * (4 * F::kGroups) + 2 * (t & 1)) : "memory");
                                    if ((v & 0x7f80u) != 0x7f80u || (c >> 1) != (n & 1)) continue;
#pragma unroll
                                    for (int r = 0; r < kHalves; ++r)
                                        if (position + i * kGranule + t <= limit[r])
#pragma unroll
                                            for (int e = 0; e < 8; ++e) o[n / 2 * 8 + e][2 * r] = o[n / 2 * 8 + e][2 * r + 1] = __uint_as_float(0x7fffffffu);
                                }
                        }
                    }
#pragma unroll
                    for (int a = 0; a < F::kSlabs; ++a) {
                        uint32_t w[2][4];   // [pair of positions][position % 2, word / 8]
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if constexpr (F::kGroups == 2) {
                                const uint2 v = lds64(granule + F::kValues + ((c + 4 * h) * 8 + g) * 8);
                                w[h][0] = v.x; w[h][1] = v.y;
                            } else {
                                const uint4 v = lds128(granule + F::kValues + a * (64 * F::kWords) + ((c + 4 * h) * 8 + g) * 16);
                                w[h][0] = v.x; w[h][1] = v.y; w[h][2] = v.z; w[h][3] = v.w;
                            }
                        }
                        constexpr int kLaneWords = F::kWords / 8;
#pragma unroll
                        for (int m = 0; m < kLaneWords; ++m) {
                            const int n = a * kLaneWords + m;
                            uint32_t v[2][2][4];   // [pair of positions][channel % 2][channel / 2]
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t scale = scale_pair<kHalf>(scales[h][n]), off = pairs.offset(scale);
                                pairs(__byte_perm(w[h][m], w[h][kLaneWords + m], 0x5410), scale, off, v[h][0]);
                                pairs(__byte_perm(w[h][m], w[h][kLaneWords + m], 0x7632), scale, off, v[h][1]);
                            }
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                mma_16816(o[n * 8 + e], hi[2 * i][0], kHalves > 1 ? hi[2 * i][kHalves - 1] : lo[2 * i], hi[2 * i + 1][0],
                                          kHalves > 1 ? hi[2 * i + 1][kHalves - 1] : lo[2 * i + 1], v[0][e & 1][e >> 1], v[1][e & 1][e >> 1], kHalf);
                        }
                    }
                }
            }
            ++consumed;
            __syncwarp();   // all lanes have read the stage
            if (!*gave_up) fetch();
        }

        // the warps' sums, then those of the other blocks that have a part of the tile
        const int64_t block0 = walk.item0 / share, block1 = (walk.item1 - 1) / share;
        const unsigned blocks = static_cast<unsigned>(block1 - block0 + 1);
        const int64_t slot = 2 * static_cast<int64_t>(blockIdx.x) + (blockIdx.x == block0 && walk.item0 % share != 0);
        float *const part = p.parts + slot * part_floats<D>(kRows);
#pragma unroll
        for (int r = 0; r < kHalves; ++r) {
            float l = total_p[r];
            l += __shfl_xor_sync(0xffffffffu, l, 1);
            l += __shfl_xor_sync(0xffffffffu, l, 2);
            __syncthreads();   // the sums before have been read
            if (c == 0) sums[warp * kMergeRows + g] = make_float2(most[r], l);
            float *to = merge + (warp * kMergeRows + g) * S::kPitch;
#pragma unroll
            for (int n = 0; n < D / 64; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {   // channels 64 n + 16 c + 8 h + e
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = kHalves == 1 ? o[n * 8 + e][h] + o[n * 8 + e][2 + h] : o[n * 8 + e][2 * r + h];
                    *reinterpret_cast<float4 *>(to + 64 * n + 16 * c + 8 * h) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float4 *>(to + 64 * n + 16 * c + 8 * h + 4) = make_float4(v[4], v[5], v[6], v[7]);
                }
            __syncthreads();
            for (int i = threadIdx.x; i < kMergeRows * (D / 4); i += kStepThreads) {
                const int row = i / (D / 4), column = i % (D / 4) * 4;
                float top = -INFINITY, l_all = 0.0f;
                float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
                for (int w = 0; w < kStepWarps; ++w) top = fmaxf(top, sums[w * kMergeRows + row].x);
#pragma unroll
                for (int w = 0; w < kStepWarps; ++w) {
                    const float2 ml = sums[w * kMergeRows + row];
                    const float factor = exp2_fast(ml.x - top);
                    const float4 x = *reinterpret_cast<const float4 *>(merge + (w * kMergeRows + row) * S::kPitch + column);
                    if (ml.y == 0.0f) continue;   // such a row has seen nothing
                    l_all = fmaf(ml.y, factor, l_all);
                    v.x = fmaf(x.x, factor, v.x); v.y = fmaf(x.y, factor, v.y); v.z = fmaf(x.z, factor, v.z); v.w = fmaf(x.w, factor, v.w);
                }
                if (blocks > 1) {
                    __stcg(reinterpret_cast<float4 *>(part + (8 * r + row) * D + column), v);
                    if (column == 0) __stcg(reinterpret_cast<float2 *>(part + kRows * D) + 8 * r + row, make_float2(top, l_all));
                    continue;
                }
                const int64_t at = at0 + 8 * r + row;
                if (at >= rows_all || *gave_up) continue;
                const int64_t q_row = walk.row0 + at / p.group, q_head = static_cast<int64_t>(walk.head) * p.group + at % p.group;
                const float inverse = l_all == 0.0f ? 0.0f : 1.0f / l_all;
                SQ_LINEAR_CHECK(q_row < p.r.rows && q_head < heads, 2013);
                uint16_t *out = p.out + q_row * p.out_stride + q_head * p.out_head + column;
                const uint32_t w0 = to_16x2<kHalf>(v.x * inverse, v.y * inverse), w1 = to_16x2<kHalf>(v.z * inverse, v.w * inverse);
                if (p.out_vector) {
                    *reinterpret_cast<uint2 *>(out) = make_uint2(w0, w1);
                } else {
                    out[0] = static_cast<uint16_t>(w0); out[1] = static_cast<uint16_t>(w0 >> 16);
                    out[2] = static_cast<uint16_t>(w1); out[3] = static_cast<uint16_t>(w1 >> 16);
                }
                if (p.lse && column == 0) p.lse[q_row * heads + q_head] = l_all == 0.0f ? -INFINITY : (top + log2f(l_all)) * 0.69314718055994531f;
            }
        }
        if (blocks > 1) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) is_last = arrive(p.tickets + block0, p.nonce, blocks);
            __syncthreads();
            if (is_last) {
                __threadfence();
                for (int i = threadIdx.x; i < kRows * (D / 4); i += kStepThreads) {
                    const int row = i / (D / 4), column = i % (D / 4) * 4;
                    const int64_t at = at0 + row;
                    if (at >= rows_all || *gave_up) continue;
                    const float *from = p.parts + (2 * block0 + (walk.item0 % share != 0)) * part_floats<D>(kRows);
                    float top = -INFINITY, l_all = 0.0f;
                    float4 v = make_float4(0, 0, 0, 0);
#pragma unroll 4
                    for (int64_t b = block0; b <= block1; ++b) {
                        const float *mine = b == block0 ? from : p.parts + 2 * b * part_floats<D>(kRows);
                        const float4 x = __ldcg(reinterpret_cast<const float4 *>(mine + row * D + column));
                        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(mine + kRows * D) + row);
                        if (ml.y == 0.0f) continue;
                        const float next = fmaxf(top, ml.x), old = l_all == 0.0f ? 0.0f : exp2_fast(top - next), factor = exp2_fast(ml.x - next);
                        l_all = fmaf(ml.y, factor, l_all * old);
                        v.x = fmaf(x.x, factor, v.x * old); v.y = fmaf(x.y, factor, v.y * old); v.z = fmaf(x.z, factor, v.z * old); v.w = fmaf(x.w, factor, v.w * old);
                        top = next;
                    }
                    const int64_t q_row = walk.row0 + at / p.group, q_head = static_cast<int64_t>(walk.head) * p.group + at % p.group;
                    const float inverse = l_all == 0.0f ? 0.0f : 1.0f / l_all;
                    SQ_LINEAR_CHECK(q_row < p.r.rows && q_head < heads, 2014);
                    uint16_t *out = p.out + q_row * p.out_stride + q_head * p.out_head + column;
                    const uint32_t w0 = to_16x2<kHalf>(v.x * inverse, v.y * inverse), w1 = to_16x2<kHalf>(v.z * inverse, v.w * inverse);
                    if (p.out_vector) {
                        *reinterpret_cast<uint2 *>(out) = make_uint2(w0, w1);
                    } else {
                        out[0] = static_cast<uint16_t>(w0); out[1] = static_cast<uint16_t>(w0 >> 16);
                        out[2] = static_cast<uint16_t>(w1); out[3] = static_cast<uint16_t>(w1 >> 16);
                    }
                    if (p.lse && column == 0) p.lse[q_row * heads + q_head] = l_all == 0.0f ? -INFINITY : (top + log2f(l_all)) * 0.69314718055994531f;
                }
            }
        }
    }
    // no copy of a block that has given up may land after its end
    for (; consumed < fetched; ++consumed) bar_drain(bars + 8 * (consumed % kStepStages), consumed / kStepStages & 1);
}

}  // namespace sq
