// Attention over the cache for few rows: decoding steps and the check of drafted tokens.
//
//   s_ij = scale q_i k_j,   p_ij = exp(s_ij - max_j s_ij),   out_i = sum_j p_ij v_j / sum_j p_ij,   lse_i = log sum_j exp(s_ij)
//
// A tile is 8 (or 16) rows of one sequence and kv head: tokens times the query heads of the group.  What bounds it is the cache's bytes, and next to them the instructions that turn
// codes into floats: at the copy bandwidth a multiprocessor gets 23 bytes a clock, a position of 128 channels (144 bytes) every 6.2 clocks or 25 issue slots.
//
// Work is cut by what there is, not by sequence: the units (32 positions of a tile) of all sequences stand in one row, and each warp takes an equal stretch of
// it, which may hold the end of one tile, whole ones and the beginning of another.  Whole tiles a warp finishes by itself.  Parts of tiles are put together at the end of the block, and
// where several blocks have a part, by the block that ends last, always in the order of the stretches, so that results repeat to the bit.
#pragma once

#include <type_traits>

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
constexpr float kNoScore = -3.0e38f;           // the maximum of no scores
constexpr float kGrowth = 8.0f;                // the running maximum is replaced when a score is 2^8 beyond it: sums stay far inside fp32 and bf16

// A tile has 8 * kTiles rows.
template <int D, int kTiles>
struct StepShape {
    static constexpr int kRows = 8 * kTiles;
    static constexpr int kBlocks = D * kTiles > 256 ? 1 : 2;             // on a multiprocessor
    static constexpr int kGranules = D * kTiles == 256 ? 1 : 2;          // of a unit: as many as registers and shared memory allow
    static constexpr int kStages = 2;                                    // of a warp: one being read, one in flight
    static constexpr int kPositions = kGranules * kGranule;              // of a unit
    static constexpr int kStage = kGranules * CacheFormat<D>::kBytes;
    static constexpr int kWarpBytes = kStages * kStage;
    static constexpr int kRing = kStepWarps * kWarpBytes;
    static constexpr bool kHeld = kTiles * D <= 128;                     // queries stay in registers
    static constexpr int kQueries = kHeld ? 0 : kRows * D * 2;           // of a warp
    static constexpr int kSmem = kRing + kStepWarps * kQueries + 8 * kStepWarps * kStages;
    static constexpr int kPitch = D + 4;                                 // floats of a row's sums in shared memory
    static constexpr int kPart = kRows * (D + 2);                        // floats of a tile's part in the workspace: sums, then maximum and sum of exponentials of each row
    static constexpr int kParts = 2 + kStepWarps;                        // of a block: its own two, and each warp's end of a tile that began before
    static_assert(kBlocks * (kSmem + 1024 + 512) <= 228 << 10, "blocks on a multiprocessor");
    static_assert(kRows * kPitch * 4 + kRows * 8 <= kWarpBytes, "a warp's part of a tile takes the place of its copies");
};

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

// c += a b: a 16 x 16, b 16 x 8
template <bool kHalf>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (kHalf)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit values turned round; a lane has two neighbours of row lane / 4.
__device__ __forceinline__ uint32_t turned(uint32_t v)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// A walk over the row of units, the same in all threads of a warp; sequences are looked up 32 at a time.
struct Walk {
    int64_t x, end;            // next unit, and where the stretch ends
    int64_t base, item0;       // first unit of sequence b, and of the piece's tile
    int chunk, row0s, ns, lens;   // sequences chunk + lane: first row, rows, positions
    int b, row0, n, len;
    int units, tiles;          // of a tile; of a sequence and kv head
    int head, tile, first, last;   // of the piece: kv head, tile, units [first, last)

    __device__ __forceinline__ void look_up(const CacheRows &r, int from)
    {
        chunk = from;
        const int at = from + static_cast<int>(threadIdx.x & 31);
        row0s = ns = lens = 0;
        if (at < r.batch) {
            const int64_t start = row_start(r, at);
            row0s = static_cast<int>(start);
            ns = static_cast<int>(max(static_cast<int64_t>(0), (r.starts ? row_start(r, at + 1) : start + 1) - start));
            lens = length_of(r, at);
        }
    }
    template <typename S>
    static __device__ __forceinline__ int units_of(int len) { return max(1, (len + S::kPositions - 1) / S::kPositions); }
    template <typename S>
    static __device__ __forceinline__ int tiles_of(int n, int group) { return static_cast<int>((static_cast<int64_t>(n) * group + S::kRows - 1) / S::kRows); }
    template <typename S>
    __device__ __forceinline__ int64_t lane_work(const CacheRows &r, int group) const
    {
        return static_cast<int64_t>(tiles_of<S>(ns, group)) * r.kv_heads * units_of<S>(lens);
    }
    template <typename S>
    __device__ __forceinline__ void enter(const CacheRows &r, int group)
    {
        if (b - chunk >= 32) look_up(r, b);
        row0 = __shfl_sync(0xffffffffu, row0s, b - chunk);
        n = __shfl_sync(0xffffffffu, ns, b - chunk);
        len = __shfl_sync(0xffffffffu, lens, b - chunk);
        units = units_of<S>(len);
        tiles = tiles_of<S>(n, group);
    }
    // The next piece; false at the end.
    template <typename S>
    __device__ __forceinline__ bool next(const CacheRows &r, int group)
    {
        if (x >= end) return false;
        for (int64_t w; x >= base + (w = static_cast<int64_t>(tiles) * r.kv_heads * units);) {
            base += w;
            ++b;
            enter<S>(r, group);
        }
        const int64_t in = x - base;
        const int64_t item = in >> 31 ? in / units : static_cast<int64_t>(static_cast<uint32_t>(in) / static_cast<uint32_t>(units));
        item0 = base + item * units;
        head = static_cast<int>(tiles == 1 ? item : item / tiles);
        tile = static_cast<int>(item - static_cast<int64_t>(head) * tiles);
        first = static_cast<int>(x - item0);
        x = min(end, item0 + units);
        last = static_cast<int>(x - item0);
        return true;
    }
    __device__ __forceinline__ int rows_all(int group) const { return n * group; }   // below 2^31
    // The last position that row `at` of the sequence's rows times heads sees; below 0: none.
    __device__ __forceinline__ int limit(int at, int group) const { return len - n + static_cast<int>(static_cast<uint32_t>(at) / static_cast<uint32_t>(group)); }
};

// The warp's stretch and its block's [x0, x1); false: the block has none.
template <typename S>
__device__ __forceinline__ bool begin(Walk &walk, const CacheRows &r, int group, int64_t &share, int64_t &x0, int64_t &x1)
{
    const int lane = threadIdx.x & 31;
    int64_t total = 0, upto = 0, mine = 0;
    const auto scan = [&](int from) {   // 32 sequences
        walk.look_up(r, from);
        upto = mine = walk.lane_work<S>(r, group);
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, upto, s);
            if (lane >= s) upto += v;
        }
        return __shfl_sync(0xffffffffu, upto, 31);
    };
    for (int from = 0; from < r.batch; from += 32) total += scan(from);
    share = kStepWarps * max(static_cast<int64_t>(1), (total + kStepWarps * gridDim.x - 1) / (kStepWarps * gridDim.x));
    x0 = share * blockIdx.x;
    x1 = min(total, x0 + share);
    if (x0 >= total) return false;
    const int64_t sub = share / kStepWarps, x = min(x1, x0 + (threadIdx.x >> 5) * sub);
    walk.x = x;
    walk.end = min(x1, x + sub);
    if (x >= total) return true;   // the last block's last warps
    int64_t before = 0;
    if (r.batch > 32) {
        for (int from = 0;; from += 32) {   // ends, since x is below the sum of all
            const int64_t all = scan(from);
            if (before + all > x) break;
            before += all;
        }
    }
    const int at = __ffs(__ballot_sync(0xffffffffu, before + upto > x)) - 1;
    walk.base = before + __shfl_sync(0xffffffffu, upto - mine, at);
    walk.b = walk.chunk + at;
    walk.enter<S>(r, group);
    return true;
}

// Where row `at` of a tile's sequence goes.
struct Target {
    int64_t row, head;
    __device__ __forceinline__ Target(const AttendArgs &p, int row0, int kv_head, int at)
    {
        row = row0 + static_cast<uint32_t>(at) / static_cast<uint32_t>(p.group);
        head = static_cast<int64_t>(kv_head) * p.group + static_cast<uint32_t>(at) % static_cast<uint32_t>(p.group);
        SQ_LINEAR_CHECK(row < p.r.rows && head < static_cast<int64_t>(p.r.kv_heads) * p.group, 2013);
    }
};
__device__ __forceinline__ void store_lse(const AttendArgs &p, const Target &to, float top, float l)
{
    p.lse[to.row * p.r.kv_heads * p.group + to.head] = l == 0.0f ? -INFINITY : (top + log2f(l)) * 0.69314718055994531f;
}
template <bool kHalf>
__device__ __forceinline__ void finish4(const AttendArgs &p, const Target &to, int column, float4 v, float top, float l)
{
    const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t *out = p.out + to.row * p.out_stride + to.head * p.out_head + column;
    const uint32_t w0 = to_16x2<kHalf>(v.x * inverse, v.y * inverse), w1 = to_16x2<kHalf>(v.z * inverse, v.w * inverse);
    if (p.out_vector) {
        *reinterpret_cast<uint2 *>(out) = make_uint2(w0, w1);
    } else {
        out[0] = static_cast<uint16_t>(w0); out[1] = static_cast<uint16_t>(w0 >> 16);
        out[2] = static_cast<uint16_t>(w1); out[3] = static_cast<uint16_t>(w1 >> 16);
    }
    if (p.lse && column == 0) store_lse(p, to, top, l);
}
// Sums of parts of a tile, one part after the other; the maximum is taken ahead of the sums it scales.
struct Joined {
    float top = kNoScore, l = 0.0f;
    float4 v = make_float4(0, 0, 0, 0);
    template <int kCount>
    __device__ __forceinline__ void add(const float4 (&x)[kCount], const float2 (&ml)[kCount])   // ml: maximum and sum; a row that has seen nothing has sum 0
    {
        float next = top;
#pragma unroll
        for (int j = 0; j < kCount; ++j)
            if (ml[j].y != 0.0f) next = fmaxf(next, ml[j].x);
        const float old = l == 0.0f ? 0.0f : exp2_fast(top - next);
        l *= old;
        v.x *= old; v.y *= old; v.z *= old; v.w *= old;
        top = next;
#pragma unroll
        for (int j = 0; j < kCount; ++j) {
            if (ml[j].y == 0.0f) continue;
            const float factor = exp2_fast(ml[j].x - top);
            l = fmaf(ml[j].y, factor, l);
            v.x = fmaf(x[j].x, factor, v.x); v.y = fmaf(x[j].y, factor, v.y); v.z = fmaf(x[j].z, factor, v.z); v.w = fmaf(x[j].w, factor, v.w);
        }
    }
    // What warps [w, until) of the block have left in shared memory.
    template <typename S>
    __device__ __forceinline__ void add_warps(const uint8_t *smem, int w, int until, int row, int column)
    {
        float4 x[kStepWarps];
        float2 ml[kStepWarps];
#pragma unroll
        for (int j = 0; j < kStepWarps; ++j) {
            const float *at = reinterpret_cast<const float *>(smem + min(w + j, until - 1) * S::kWarpBytes);
            x[j] = *reinterpret_cast<const float4 *>(at + row * S::kPitch + column);
            ml[j] = reinterpret_cast<const float2 *>(at + S::kRows * S::kPitch)[row];
            if (w + j >= until) ml[j].y = 0.0f;
        }
        add(x, ml);
    }
};

// What a warp leaves for the end of the block: the tile that its stretch ends in.
struct Left {
    int64_t item0;      // first unit, -1: none
    int64_t item1;
    int row0, rows_all, head, tile;
};

// Keys and values are the first operands of the matrix instructions, 16 positions (16 channels) high, and rows of queries (of weights) are the second ones'
// columns, so that none of the instructions' work goes to rows that do not exist, and sums take few registers (queries first and codes second: 120 us for 131,072 positions of 8
// heads, 54 % more instructions and twice the sums' registers).  What the rounding of a weight to 16 bits leaves over goes through a second instruction: products with the values
// are as good as fp32's.  62 us now, 38 % of the copy bandwidth: 810 instructions a unit and warp, 52 % of the issue slots (the copies alone take 21 us, 7.3 TB/s), 3 us until the
// first copies are under way and 12 us for the last blocks to join the parts of 37.
// Units without a hidden position have code of their own, without masks (931 to 810 instructions).
template <int D, bool kHalf, int kTiles>
__global__ void __launch_bounds__(kStepThreads, (StepShape<D, kTiles>::kBlocks))
cache_step_kernel(const __grid_constant__ AttendArgs p)
{
    using F = CacheFormat<D>;
    using S = StepShape<D, kTiles>;
    constexpr int kRows = S::kRows, kGroupsAll = D / kGroup;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ Left left_over[kStepWarps], first_end;   // first_end: of a tile that begins before the block and ends in the first warp's stretch
    __shared__ int gave_up_word, is_last[2];
    volatile int *gave_up = &gave_up_word;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    uint8_t *const ring = smem + warp * S::kWarpBytes;
    uint4 *const held_q = reinterpret_cast<uint4 *>(smem + S::kRing + warp * S::kQueries);
    const uint32_t bars = smem_addr(smem) + S::kRing + kStepWarps * S::kQueries + 8 * warp * S::kStages;
    SQ_LINEAR_CHECK(smem_addr(smem) + S::kSmem <= smem_end(smem) && (smem_addr(smem) & 15) == 0, 2010);
    if (threadIdx.x == 0) {
        gave_up_word = 0;
        first_end.item0 = -1;
    }
    if (lane == 0) {
        left_over[warp].item0 = -1;
        for (int s = 0; s < S::kStages; ++s) bar_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    Walk walk;
    int64_t share, x0, x1;
    if (!begin<S>(walk, p.r, p.group, share, x0, x1)) return;   // all threads of the block
    __syncthreads();

    // Copies of the warp's units, ahead of what it computes: the numbers of the next granules lie in the warp's lanes, looked up together.
    Walk ahead = walk;
    constexpr int kBatch = 32 / S::kGranules;   // units
    int ahead_unit = 0, listed = 0, taken = 0, granule = -1;
    unsigned fetched = 0, consumed = 0;
    uint32_t there = 0;   // which granules of a stage have been copied: two bits a stage
    bool more = ahead.next<S>(p.r, p.group), dead = false;
    ahead_unit = ahead.first;
    const auto fetch = [&]() {
        if (taken == listed) {
            if (more && ahead_unit == ahead.last) {
                more = ahead.next<S>(p.r, p.group);
                ahead_unit = ahead.first;
            }
            if (!more) return;
            listed = min(kBatch, ahead.last - ahead_unit);
            taken = 0;
            const int at = (ahead_unit + lane / S::kGranules) * S::kPositions + lane % S::kGranules * kGranule;
            const int seen = ahead.limit(min(ahead.rows_all(p.group) - ahead.tile * kRows, kRows) - 1 + ahead.tile * kRows, p.group);   // by the tile's last row
            granule = -1;
            if (lane / S::kGranules < listed && at <= seen) {
                const int column = at / p.r.page_size;
                const int64_t page = page_of(p.r, ahead.b, column);
                const int granules = p.r.page_size / kGranule;
                SQ_LINEAR_CHECK(column < p.r.width, 2011);
                if (page >= 0) granule = static_cast<int>((page * p.r.kv_heads + ahead.head) * granules + (at - column * p.r.page_size) / kGranule);
            }
            ahead_unit += listed;
        }
        const unsigned stage = fetched % S::kStages;
        int from[S::kGranules];
        uint32_t have = 0;
#pragma unroll
        for (int i = 0; i < S::kGranules; ++i) {
            from[i] = __shfl_sync(0xffffffffu, granule, taken * S::kGranules + i);
            have |= from[i] >= 0 ? 1u << i : 0u;
        }
        if (elect_one()) {
            const uint32_t to = smem_addr(ring) + stage * S::kStage, bar = bars + 8 * stage;
            bar_expect(bar, __popc(have) * F::kBytes);
            if (S::kGranules == 2 && have == 3 && from[S::kGranules - 1] == from[0] + 1) {
                bulk_load(to, p.cache + static_cast<int64_t>(from[0]) * F::kBytes, S::kStage, bar);
            } else {
#pragma unroll
                for (int i = 0; i < S::kGranules; ++i)
                    if (have >> i & 1) bulk_load(to + i * F::kBytes, p.cache + static_cast<int64_t>(from[i]) * F::kBytes, F::kBytes, bar);
            }
        }
        __syncwarp();
        there = (there & ~(3u << (2 * stage))) | have << (2 * stage);
        ++fetched;
        ++taken;
    };
#pragma unroll
    for (int s = 0; s < S::kStages; ++s) fetch();

    const CodePairs<kHalf> pairs;
    while (walk.next<S>(p.r, p.group)) {
        const int at0 = walk.tile * kRows, rows_all = walk.rows_all(p.group);   // of the sequence's rows times heads
        // queries: lane (g, c) has 8 channels of each group of row g
        uint4 q[S::kHeld ? kTiles * kGroupsAll : 1];
        const auto queries = [&](auto on_vectors) {   // tile i / kGroupsAll, group i % kGroupsAll
            constexpr int kBatch = kGroupsAll;         // loads in flight
#pragma unroll
            for (int r = 0; r < kTiles; ++r) {
                uint4 v[kBatch];
                const int at = at0 + 8 * r + g;
                const Target to(p, walk.row0, walk.head, min(at, rows_all - 1));
                const uint16_t *const from = p.q + to.row * p.q_stride + to.head * p.q_head + 8 * c;
#pragma unroll
                for (int n = 0; n < kBatch; ++n) v[n] = at < rows_all ? load8(from + kGroup * n, decltype(on_vectors)::value) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int n = 0; n < kBatch; ++n) {
                    if constexpr (S::kHeld) q[r * kGroupsAll + n] = v[n];
                    else held_q[(r * kGroupsAll + n) * 32 + lane] = v[n];   // read back by the lane itself
                }
            }
        };
        if (p.q_vector) queries(std::true_type{});
        else queries(std::false_type{});
        // the lane's rows: 8 r + 2 c and the next
        int limit[kTiles][2];
#pragma unroll
        for (int r = 0; r < kTiles; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) limit[r][e] = walk.limit(min(at0 + 8 * r + 2 * c + e, rows_all - 1), p.group);
        const int seen_least = walk.limit(at0, p.group), seen_most = walk.limit(min(rows_all - at0, kRows) - 1 + at0, p.group);
        float o[kTiles][D / 16][4], most[kTiles][2], total_p[kTiles][2];
#pragma unroll
        for (int r = 0; r < kTiles; ++r) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[r][i][0] = o[r][i][1] = o[r][i][2] = o[r][i][3] = 0.0f;
            most[r][0] = most[r][1] = kNoScore;
            total_p[r][0] = total_p[r][1] = 0.0f;
        }

        for (int unit = dead ? walk.last : walk.first; unit < walk.last; ++unit) {
            const unsigned stage = consumed % S::kStages;
            if (!bar_wait_warp(bars + 8 * stage, consumed / S::kStages & 1, gave_up)) {
                dead = true;
                break;
            }
            SQ_LINEAR_CHECK(consumed < fetched, 2012);
            const uint32_t have = there >> (2 * stage) & 3u;
            const uint8_t *const data = ring + stage * S::kStage;
            const int position = unit * S::kPositions;
            const auto attend = [&](auto some_hidden) {
                constexpr bool kMasked = decltype(some_hidden)::value;
                // scores: the lane has positions g and g + 8 of a granule for its two rows
                float s[kTiles][S::kGranules][4];
#pragma unroll
                for (int i = 0; i < S::kGranules; ++i) {
#pragma unroll
                    for (int r = 0; r < kTiles; ++r) s[r][i][0] = s[r][i][1] = s[r][i][2] = s[r][i][3] = 0.0f;
                    if (kMasked && !(have >> i & 1)) continue;
                    const uint8_t *const at = data + i * F::kBytes;
                    uint32_t scales[2][kGroupsAll / 2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint8_t *const from = at + F::kKeyScales + (g + 8 * h) * (2 * kGroupsAll);
                        if constexpr (kGroupsAll == 2) {
                            scales[h][0] = *reinterpret_cast<const uint32_t *>(from);
                        } else {
#pragma unroll
                            for (int n = 0; n < kGroupsAll / 4; ++n) {
                                const uint2 v = *reinterpret_cast<const uint2 *>(from + 8 * n);
                                scales[h][2 * n] = v.x;
                                scales[h][2 * n + 1] = v.y;
                            }
                        }
                    }
#pragma unroll
                    for (int a = 0; a < F::kSlabs; ++a) {
                        uint32_t w[2][4];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint8_t *const from = at + a * (64 * F::kWords) + (g + 8 * h) * (4 * F::kWords) + c * F::kWords;
                            if constexpr (F::kGroups == 2) {
                                const uint2 v = *reinterpret_cast<const uint2 *>(from);
                                w[h][0] = v.x; w[h][1] = v.y;
                            } else {
                                const uint4 v = *reinterpret_cast<const uint4 *>(from);
                                w[h][0] = v.x; w[h][1] = v.y; w[h][2] = v.z; w[h][3] = v.w;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < F::kGroups; ++j) {
                            const int n = a * F::kGroups + j;
                            uint32_t k[2][4];
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                pairs(w[h][j], pairs.scales(scale_twice<kHalf>(scales[h][n / 2], n & 1)), k[h]);
                            }
#pragma unroll
                            for (int r = 0; r < kTiles; ++r) {
                                const uint4 x = S::kHeld ? q[r * kGroupsAll + n] : held_q[(r * kGroupsAll + n) * 32 + lane];
                                mma_16816<kHalf>(s[r][i], k[0][0], k[1][0], k[0][1], k[1][1], x.x, x.y);
                                mma_16816<kHalf>(s[r][i], k[0][2], k[1][2], k[0][3], k[1][3], x.z, x.w);
                            }
                        }
                    }
                }
                const auto hidden = [&](int r, int i, int e) {
                    return kMasked && (position + i * kGranule + g + 8 * (e >> 1) > limit[r][e & 1] || !(have >> i & 1));
                };
                // exponents against the maximum so far
                float x[kTiles][S::kGranules][4];
                bool grows = false;
#pragma unroll
                for (int r = 0; r < kTiles; ++r)
#pragma unroll
                    for (int i = 0; i < S::kGranules; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[r][i][e] = hidden(r, i, e) ? -INFINITY : fmaf(s[r][i][e], p.scale_log2, -most[r][e & 1]);
                            grows |= x[r][i][e] > kGrowth;
                        }
                if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
                    for (int r = 0; r < kTiles; ++r) {
                        float factor[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float next = most[r][e];
#pragma unroll
                            for (int i = 0; i < S::kGranules; ++i)
#pragma unroll
                                for (int h = 0; h < 2; ++h) next = fmaxf(next, hidden(r, i, 2 * h + e) ? kNoScore : s[r][i][2 * h + e] * p.scale_log2);
#pragma unroll
                            for (int j = 4; j < 32; j <<= 1) next = fmaxf(next, __shfl_xor_sync(0xffffffffu, next, j));
                            factor[e] = exp2_fast(most[r][e] - next);
                            most[r][e] = next;
                            total_p[r][e] *= factor[e];
#pragma unroll
                            for (int i = 0; i < S::kGranules; ++i)
#pragma unroll
                                for (int h = 0; h < 2; ++h) x[r][i][2 * h + e] = hidden(r, i, 2 * h + e) ? -INFINITY : fmaf(s[r][i][2 * h + e], p.scale_log2, -next);
                        }
#pragma unroll
                        for (int i = 0; i < D / 16; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[r][i][e] *= factor[e & 1];
                    }
                }
                // weights, turned round: the lane has positions 2 c and the next (and 8 on) for row g
                uint32_t hi[kTiles][S::kGranules][2], lo[kTiles][S::kGranules][2];
#pragma unroll
                for (int r = 0; r < kTiles; ++r)
#pragma unroll
                    for (int i = 0; i < S::kGranules; ++i)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float a = exp2_fast(x[r][i][2 * h]), b = exp2_fast(x[r][i][2 * h + 1]);
                            total_p[r][0] += a;
                            total_p[r][1] += b;
                            const uint32_t v = to_16x2<kHalf>(a, b);
                            hi[r][i][h] = turned(v);
                            lo[r][i][h] = turned(to_16x2<kHalf>(a - to_float<kHalf>(static_cast<uint16_t>(v)), b - to_float<kHalf>(static_cast<uint16_t>(v >> 16))));
                        }
#pragma unroll
                for (int i = 0; i < S::kGranules; ++i) {
                    if (kMasked && !(have >> i & 1)) continue;
                    const uint8_t *const at = data + i * F::kBytes;
                    [[maybe_unused]] const int left = seen_most + 1 - (position + i * kGranule);   // positions of the granule that any row sees
                    // scales of positions 2 c, 2 c + 1 and 2 c + 8, 2 c + 9 for the groups of the lane's words
                    uint32_t scales[2][D / 64];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int a = 0; a < F::kSlabs; ++a) {
                            const uint8_t *const from = at + F::kValueScales + a * (32 * F::kGroups) + (c + 4 * h) * (4 * F::kGroups) + (g >> 2) * (2 * F::kGroups);
                            if constexpr (F::kGroups == 2) {
                                scales[h][0] = *reinterpret_cast<const uint32_t *>(from);
                            } else {
                                const uint2 v = *reinterpret_cast<const uint2 *>(from);
                                scales[h][2 * a] = v.x;
                                scales[h][2 * a + 1] = v.y;
                            }
                        }
                    }
                    if constexpr (kMasked) {
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
                                    const uint16_t v = *reinterpret_cast<const uint16_t *>(at + F::value_scale(0, n) + (t >> 1) * (4 * F::kGroups) + 2 * (t & 1));
                                    if ((v & 0x7f80u) != 0x7f80u || (g >> 2) != (n & 1)) continue;   // channels 64 (n / 2) + 8 g and on
#pragma unroll
                                    for (int r = 0; r < kTiles; ++r)
#pragma unroll
                                        for (int j = 0; j < 4; ++j)
#pragma unroll
                                            for (int e = 0; e < 4; ++e)
                                                if (position + i * kGranule + t <= limit[r][e & 1]) o[r][n / 2 * 4 + j][e] = __uint_as_float(0x7fffffffu);
                                }
                        }
                    }
#pragma unroll
                    for (int a = 0; a < F::kSlabs; ++a) {
                        constexpr int kLaneWords = F::kWords / 8;
                        uint32_t w[2][4];   // [pair of positions][position % 2, word / 8]
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if constexpr (F::kGroups == 2) {
                                const uint2 v = *reinterpret_cast<const uint2 *>(at + F::kValues + ((c + 4 * h) * 8 + g) * 8);
                                w[h][0] = v.x; w[h][1] = v.y;
                            } else {
                                const uint4 v = *reinterpret_cast<const uint4 *>(at + F::kValues + a * (64 * F::kWords) + ((c + 4 * h) * 8 + g) * 16);
                                w[h][0] = v.x; w[h][1] = v.y; w[h][2] = v.z; w[h][3] = v.w;
                            }
                        }
#pragma unroll
                        for (int m = 0; m < kLaneWords; ++m) {
                            const int n = a * kLaneWords + m;
                            uint32_t v[2][2][4];   // [pair of positions][channel % 2][channel / 2]
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const PairScales<kHalf> scale = pairs.scales(scale_pair<kHalf>(scales[h][n]));
                                pairs(__byte_perm(w[h][m], w[h][kLaneWords + m], 0x5410), scale, v[h][0]);
                                pairs(__byte_perm(w[h][m], w[h][kLaneWords + m], 0x7632), scale, v[h][1]);
                            }
                            // rows of the first operand: channels 64 n + 8 g + 2 j, and from 8 on 64 n + 8 g + 2 j + 1
#pragma unroll
                            for (int r = 0; r < kTiles; ++r)
#pragma unroll
                                for (int j = 0; j < 4; ++j) mma_16816<kHalf>(o[r][n * 4 + j], v[0][0][j], v[0][1][j], v[1][0][j], v[1][1][j], hi[r][i][0], hi[r][i][1]);
#pragma unroll
                            for (int r = 0; r < kTiles; ++r)
#pragma unroll
                                for (int j = 0; j < 4; ++j) mma_16816<kHalf>(o[r][n * 4 + j], v[0][0][j], v[0][1][j], v[1][0][j], v[1][1][j], lo[r][i][0], lo[r][i][1]);
                        }
                    }
                }
            };
            // few units have positions that some row does not see, or pages that are not there
            if (have == (1u << S::kGranules) - 1 && position + S::kPositions - 1 <= seen_least) attend(std::false_type{});
            else if (have) attend(std::true_type{});
            ++consumed;
            // all lanes have read the stage, and a copy into it comes behind what they have read: nothing else keeps one, which is not theirs, from overtaking their loads
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            fetch();
        }

        float l[kTiles][2];
#pragma unroll
        for (int r = 0; r < kTiles; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[r][e] = total_p[r][e];
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[r][e] += __shfl_xor_sync(0xffffffffu, l[r][e], x);
            }
        // 8 neighbouring channels, 64 n + 8 g and on, of the lane's row e of 8 r
        const auto sums8 = [&](int r, int e, int n, float (&v)[8]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] = o[r][4 * n + j][e];
                v[2 * j + 1] = o[r][4 * n + j][2 + e];
            }
        };
        if (walk.first == 0 && walk.last == walk.units) {   // the whole tile
            if (dead) continue;
#pragma unroll
            for (int r = 0; r < kTiles; ++r)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = at0 + 8 * r + 2 * c + e;
                    if (at >= rows_all) continue;
                    const Target to(p, walk.row0, walk.head, at);
                    const float inverse = l[r][e] == 0.0f ? 0.0f : 1.0f / l[r][e];
                    uint16_t *out = p.out + to.row * p.out_stride + to.head * p.out_head + 8 * g;
#pragma unroll
                    for (int n = 0; n < D / 64; ++n) {
                        float v[8];
                        uint32_t w[4];
                        sums8(r, e, n, v);
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = to_16x2<kHalf>(v[2 * j] * inverse, v[2 * j + 1] * inverse);
                        if (p.out_vector) {
                            *reinterpret_cast<uint4 *>(out + 64 * n) = make_uint4(w[0], w[1], w[2], w[3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) out[64 * n + j] = static_cast<uint16_t>(w[j / 2] >> (16 * (j & 1)));
                        }
                    }
                    if (p.lse && g == 0) store_lse(p, to, most[r][e], l[r][e]);
                }
            continue;
        }
        const bool ends_here = walk.x == walk.end;   // the last piece of the warp's stretch: nothing is being copied any more
        // otherwise the end of a tile that began before: what the block has of it if the block's stretch begins in it too
        float *const global = p.parts + (static_cast<int64_t>(blockIdx.x) * S::kParts + (warp == 0 ? 0 : 2 + warp)) * S::kPart;
        float *const local = reinterpret_cast<float *>(ring);
        SQ_LINEAR_CHECK(ends_here || (walk.first > 0 && walk.last == walk.units), 2015);
        __syncwarp();
#pragma unroll
        for (int r = 0; r < kTiles; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = 8 * r + 2 * c + e;
#pragma unroll
                for (int n = 0; n < D / 64; ++n) {
                    float v[8];
                    sums8(r, e, n, v);
                    const float4 a = make_float4(v[0], v[1], v[2], v[3]), b = make_float4(v[4], v[5], v[6], v[7]);
                    if (ends_here) {
                        float4 *to = reinterpret_cast<float4 *>(local + row * S::kPitch + 64 * n + 8 * g);
                        to[0] = a;
                        to[1] = b;
                    } else {
                        float4 *to = reinterpret_cast<float4 *>(global + row * D + 64 * n + 8 * g);
                        __stcg(to, a);
                        __stcg(to + 1, b);
                    }
                }
                if (g == 0) {
                    if (ends_here) reinterpret_cast<float2 *>(local + kRows * S::kPitch)[row] = make_float2(most[r][e], l[r][e]);
                    else __stcg(reinterpret_cast<float2 *>(global + kRows * D) + row, make_float2(most[r][e], l[r][e]));
                }
            }
        if (lane == 0 && (ends_here || warp == 0)) (ends_here ? left_over[warp] : first_end) = Left{walk.item0, walk.item0 + walk.units, walk.row0, rows_all, walk.head, walk.tile};
    }
    // no copy of a block that has given up may land after its end, or in a part of a tile
    for (; consumed < fetched; ++consumed) bar_drain(bars + 8 * (consumed % S::kStages), consumed / S::kStages & 1);
    __syncthreads();

    // parts of tiles that the block has, each begun by a warp's end, with those of the warps that follow it
    Left mine[2];               // the block's own parts of tiles that others have parts of, too: the one that begins before it, the one that ends after it
    mine[0].item0 = mine[1].item0 = -1;
    const int64_t sub = share / kStepWarps;
    for (int w = 0; w < kStepWarps; ++w) {
        const Left t = left_over[w];
        if (t.item0 < 0 || (w > 0 && left_over[w - 1].item0 == t.item0)) continue;
        int until = w + 1;      // warps [w, until) end in the tile, and the end of it may be the beginning of the next one's stretch
        while (until < kStepWarps && left_over[until].item0 == t.item0) ++until;
        const bool further = t.item1 > x0 + until * sub && x0 + until * sub < x1;
        const bool alone = t.item0 >= x0 && t.item1 <= x1;
        float *const part = p.parts + (static_cast<int64_t>(blockIdx.x) * S::kParts + (t.item0 >= x0)) * S::kPart;
        for (int i = threadIdx.x; i < kRows * (D / 4); i += kStepThreads) {
            const int row = i / (D / 4), column = i % (D / 4) * 4;
            Joined sum;
            sum.add_warps<S>(smem, w, until, row, column);
            if (further) {
                const float *at = p.parts + (static_cast<int64_t>(blockIdx.x) * S::kParts + 2 + until) * S::kPart;
                const float4 x1[1] = {__ldcg(reinterpret_cast<const float4 *>(at + row * D + column))};
                const float2 ml1[1] = {__ldcg(reinterpret_cast<const float2 *>(at + kRows * D) + row)};
                sum.add(x1, ml1);
            }
            if (!alone) {
                __stcg(reinterpret_cast<float4 *>(part + row * D + column), sum.v);
                if (column == 0) __stcg(reinterpret_cast<float2 *>(part + kRows * D) + row, make_float2(sum.top, sum.l));
            } else if (t.tile * kRows + row < t.rows_all && !*gave_up) {
                finish4<kHalf>(p, Target(p, t.row0, t.head, t.tile * kRows + row), column, sum.v, sum.top, sum.l);
            }
        }
        if (!alone) mine[t.item0 >= x0] = t;
    }
    if (first_end.item0 >= 0) mine[0] = first_end;
    // tiles that other blocks have parts of: who comes last puts them together
    if (mine[0].item0 < 0 && mine[1].item0 < 0) return;
    __threadfence();
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const Left &t = mine[k];
        if (threadIdx.x == 32 * k && t.item0 >= 0) {
            const int64_t block0 = t.item0 / share, block1 = (t.item1 - 1) / share;
            is_last[k] = arrive(p.tickets + block0, p.nonce, static_cast<unsigned>(block1 - block0 + 1));
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const Left &t = mine[k];
        if (t.item0 < 0 || !is_last[k]) continue;
        __threadfence();
        const int64_t block0 = t.item0 / share;
        const int blocks = static_cast<int>((t.item1 - 1) / share - block0 + 1);
        const float *const from = p.parts + block0 * S::kParts * S::kPart;
        // each warp joins every eighth part, row by row, then the block the warps'
        constexpr int kPieces = kRows * (D / 4) / 32, kAtOnce = kPieces < 8 ? kPieces : 8;
        float *const local = reinterpret_cast<float *>(ring);
        __syncthreads();   // what was there has been read
        for (int i0 = 0; i0 < kPieces; i0 += kAtOnce) {
            Joined sum[kAtOnce];
            for (int b = warp; b < blocks; b += kStepWarps) {
                const float *at = from + (static_cast<int64_t>(b) * S::kParts + (b == 0)) * S::kPart;
                float4 x[kAtOnce][1];
                float2 ml[kAtOnce][1];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const int i = (i0 + j) * 32 + lane;
                    x[j][0] = __ldcg(reinterpret_cast<const float4 *>(at) + i);
                    ml[j][0] = __ldcg(reinterpret_cast<const float2 *>(at + kRows * D) + i / (D / 4));
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) sum[j].add(x[j], ml[j]);
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int i = (i0 + j) * 32 + lane, row = i / (D / 4), column = i % (D / 4) * 4;
                *reinterpret_cast<float4 *>(local + row * S::kPitch + column) = sum[j].v;
                if (column == 0) reinterpret_cast<float2 *>(local + kRows * S::kPitch)[row] = make_float2(sum[j].top, sum[j].l);
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < kRows * (D / 4); i += kStepThreads) {
            const int row = i / (D / 4), column = i % (D / 4) * 4;
            if (t.tile * kRows + row >= t.rows_all || *gave_up) continue;
            Joined sum;
            sum.add_warps<S>(smem, 0, kStepWarps, row, column);
            finish4<kHalf>(p, Target(p, t.row0, t.head, t.tile * kRows + row), column, sum.v, sum.top, sum.l);
        }
    }
}

}  // namespace sq
