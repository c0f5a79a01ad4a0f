// Attention over the cache for many rows: prompts, parts of prompts, many drafted tokens (formulas in cache_step.cuh).
//
// A tile is 256 rows (128 with 256 channels) of one sequence and kv head, tokens times the query heads of the group, in two slots of 128.  Its queries stay in shared memory; for 128
// positions at a time (64) converter warps turn keys and values into 16-bit floats for the tensor cores, which both slots use:
//
//   S = Q K^T   [128 x 128] in tensor memory, a row a lane: softmax warps own a row a thread
//   P = exp2(scale S - m) over S's place, 16 bits;  O += P V, P from tensor memory
//
// Weights are rounded to 16 bits for the product.  In sequences of up to kWholeRows rows what that leaves of them goes through a second one, as in cache_step.cuh: such
// sequences come to either kernel, by what the caller says of the others, and are as exact in both (drafted tokens 0.00166 off, which is all the output's own rounding, and 80
// us; with one product 0.0020 and 75 us).  In longer ones 16 bits are all there is: prompts are 0.0021 off instead of 0.0016 in bf16 and 0.0003 instead of 0.0002 in fp16, in
// 434 us instead of 513 and 349 instead of 432.
//
// m is the maximum of the row's first tile.  It is replaced when a later tile has reached 2^8 beyond it, before the next one: then O is scaled, between two products.  Within a
// tile weights may be as large as 2^kRoom, so that a row's scores are read once.  Per 128 positions the tensor cores work 2,048 clocks for both slots, and
// the exponentials take as long: one slot's products run while the other one's exponentials do.  A tile of up to 128 rows has its positions shared by the slots, every other tile
// of scores each, and their sums are joined at the end.
//
// Measured (4 prompts of 423 to 4,096 tokens, 32 query and 8 kv heads of 128 channels): 433 us, 450 TFLOP/s, 27 % of the matrix rate; tensor pipe 24 % busy, a score tile
// takes 5,000 clocks instead of 2,048.  Without exponentials 342 us, without conversion 440, without both 333: what is left is the chain from scores over weights to sums, whose
// links (barriers, loads of tensor memory, the next product's issue) wait for one another, and 20,000 clocks a tile for queries and results.  What was tried: blocks of 128 rows, two a
// multiprocessor (757 us: everything is converted twice); eight softmax warps of half a row a thread (857; 72 registers); eight converter warps (646; 96 registers); loads of the
// next scores during the exponentials, in straight-line code (467) or a loop (473), against 433 for a loop of load, weigh, store: instructions are fetched faster than they
// are needed only where loops are short.
//
// Work is cut as in cache_step.cuh: the units (256 positions that a tile sees, so that a causal prompt's later tiles have more) of all tiles stand in one row, each block
// takes an equal stretch, and a tile that several blocks have parts of is put together, in order, by the one that ends last.
#pragma once

#include "cache_step.cuh"

namespace sq {

constexpr int kSlotRows = 128;           // the tensor memory's lanes
constexpr int kPromptConverters = 4;     // warps
constexpr int kWholeRows = 128;          // more than any sequence has that the host leaves to cache_step_kernel
// Of a weight's exponent.  fp16 holds weights up to 2^16; in bf16 a sum of 2^30 of them times values of 2^80 is inside fp32 (with 64, which bf16 would hold, values from 2^50 on
// were not, where scores grow).
constexpr float kRoom = 14.0f;
constexpr int kTilesAhead = 8;           // score tiles that are being copied, converted or weighed at the same time, at most

template <int D>
struct PromptShape {
    static constexpr int kSlots = D > 128 ? 1 : 2, kRows = kSlots * kSlotRows;
    static constexpr int kSoftmax = 4 * kSlots, kThreads = 32 * (kSoftmax + kPromptConverters + 2);   // warps; one for the copies, one for the tensor cores
    static constexpr int kPositions = D > 128 ? 64 : 128;            // of a score tile
    static constexpr int kGranules = kPositions / kGranule;
    static constexpr int kQueries = kSlotRows * D * 2, kOperand = kPositions * D * 2, kPanel = kPositions * 128, kQueryPanel = kSlotRows * 128;
    // stages of granules as they are, ahead of the converters
    static constexpr int kRawGranules = D > 128 ? 2 : 4, kRaw = kRawGranules * CacheFormat<D>::kBytes, kRawStages = D > 64 ? 3 : 6;
    static constexpr int kParts = kGranules / kRawGranules;          // stages of a score tile
    static constexpr int kBars = 2 * kRawStages + 18;
    static constexpr int kSmem = 1024 + kSlots * kQueries + 4 * kOperand + kRawStages * kRaw + 8 * kBars;
    // tensor memory: columns of a slot's scores, sums and weights, which take the scores' place where there is no other
    static constexpr int kScores = 128, kSums = D, kFirstSums = 256, kColumns = 512;
    static constexpr bool kApart = kFirstSums + kSlots * (kSums + kPositions / 2) <= kColumns;
    static constexpr int kFirstWeights = kApart ? kFirstSums + kSlots * kSums : 0, kWeights = kApart ? kPositions / 2 : kScores;
    static constexpr int kPart = kRows * (D + 2);                    // floats of a tile's part in the workspace
    static_assert(kSmem + 2048 <= 227 << 10 && 2 * kSmem > 228 << 10, "one block a multiprocessor, so that all of its tensor memory is there");
    static_assert(kSlots * kScores <= kFirstSums && kFirstSums + kSlots * kSums <= kColumns, "tensor memory");
};

// The walk over units of as many positions as a tile has rows, R.  The tile t of a sequence sees its first tokens, and those of its rows up to the tile's last:
//   units(t) = ceil((len - n + floor((R t + R - 1) / group) + 1) / R) = floor((t + q) / group),   q = floor((group (len - n + R) + R - 1) / R),
// and kExtra more, with q + kExtra group.  It is one too many at most, for the last tile.  Sums of floor(i / group) have a closed form, and so does the row of all sequences' units.
template <int kRows>
struct PromptWalk {
    static constexpr int kUnit = kRows;
    // A tile's first units stand for what it costs besides its positions: its queries, its first scores, its results (20,000 clocks; a unit takes 10,000).  Without them a
    // block whose stretch was made of short prompts worked twice as long as the others.
    static constexpr int kExtra = 2;
    int64_t x, end, base, item0;
    int chunk, row0s, ns, lens;   // sequences chunk + lane
    int b, row0, n, len, tiles;
    int head, tile, first, last;  // of the piece: kv head, tile, units [first, last) of the tile's positions
    bool whole;                   // the piece is all of the tile
    int units, over;              // floor and remainder of (tile + q) / group: the tile's units, with the extra ones
    int64_t q, span;              // span: units of a kv head of sequence b

    static __device__ __forceinline__ int64_t floors(int64_t n, int group)   // sum of floor(i / group) below n
    {
        const int64_t k = n >> 31 ? n / group : static_cast<int64_t>(static_cast<uint32_t>(n) / static_cast<uint32_t>(group));
        return k * (k - 1) / 2 * group + k * (n - k * group);
    }
    static __device__ __forceinline__ int64_t offset_of(int n, int len, int group)
    {
        return (static_cast<int64_t>(group) * (max(0, len - n) + kUnit) + kRows - 1) / kRows + static_cast<int64_t>(kExtra) * group;
    }
    static __device__ __forceinline__ int tiles_of(int n, int group) { return static_cast<int>((static_cast<int64_t>(n) * group + kRows - 1) / kRows); }
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
    __device__ __forceinline__ int64_t lane_work(const CacheRows &r, int group) const
    {
        const int64_t o = offset_of(ns, lens, group);
        return (floors(o + tiles_of(ns, group), group) - floors(o, group)) * r.kv_heads;
    }
    __device__ __forceinline__ void enter(const CacheRows &r, int group)
    {
        if (b - chunk >= 32) look_up(r, b);
        row0 = __shfl_sync(0xffffffffu, row0s, b - chunk);
        n = __shfl_sync(0xffffffffu, ns, b - chunk);
        len = __shfl_sync(0xffffffffu, lens, b - chunk);
        tiles = tiles_of(n, group);
        q = offset_of(n, len, group);
        span = floors(q + tiles, group) - floors(q, group);
    }
    // The tile that unit x is in; the walk is in its sequence.
    __device__ __forceinline__ void find(const CacheRows &r, int group)
    {
        const int64_t in = x - base;
        head = static_cast<int>(in / span);
        const int64_t at = in - head * span, before = floors(q, group);
        int lo = 0, hi = tiles;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (floors(q + mid, group) - before <= at) lo = mid;
            else hi = mid;
        }
        tile = lo;
        item0 = base + head * span + (floors(q + lo, group) - before);
        units = static_cast<int>((lo + q) / group);
        over = static_cast<int>(lo + q - static_cast<int64_t>(units) * group);
    }
    // The next piece; false at the end.  Of the tile that was found, then of the ones that follow it.
    __device__ __forceinline__ bool next(const CacheRows &r, int group)
    {
        if (x >= end) return false;
        if (x >= item0 + units) {
            item0 += units;
            ++tile;
            if (++over == group) {
                over = 0;
                ++units;
            }
            if (tile == tiles) {
                tile = 0;
                if (++head == r.kv_heads) {
                    head = 0;
                    do {
                        ++b;
                        enter(r, group);
                    } while (tiles == 0);   // ends, since there are units left
                }
                units = static_cast<int>(static_cast<uint32_t>(q) / static_cast<uint32_t>(group));   // q is below 2^31: (positions + R) * group / R, rounded up
                over = static_cast<int>(static_cast<uint32_t>(q) % static_cast<uint32_t>(group));
            }
        }
        whole = x == item0 && end >= item0 + units;
        first = max(0, static_cast<int>(x - item0) - kExtra);
        x = min(end, item0 + units);
        last = max(0, static_cast<int>(x - item0) - kExtra);
        return true;
    }
    __device__ __forceinline__ int rows_all(int group) const { return n * group; }
    __device__ __forceinline__ int limit(int at, int group) const { return len - n + static_cast<int>(static_cast<uint32_t>(at) / static_cast<uint32_t>(group)); }
    __device__ __forceinline__ int seen_least(int group) const { return limit(tile * kRows, group); }
    __device__ __forceinline__ int seen_most(int group) const { return limit(min(rows_all(group) - tile * kRows, kRows) - 1 + tile * kRows, group); }
    // Score tiles of the piece that any row sees.
    template <int kPositions>
    __device__ __forceinline__ int steps(int group) const
    {
        const int seen = seen_most(group) + 1 - first * kUnit;
        return seen <= 0 ? 0 : min((last - first) * (kUnit / kPositions), (seen + kPositions - 1) / kPositions);
    }
};
// The block's stretch; false: it has none.  Each warp for itself.
template <int kRows>
__device__ __forceinline__ bool begin(PromptWalk<kRows> &walk, const CacheRows &r, int group, int64_t &share)
{
    const int lane = threadIdx.x & 31;
    int64_t total = 0, upto = 0, mine = 0;
    const auto scan = [&](int from) {
        walk.look_up(r, from);
        upto = mine = walk.lane_work(r, group);
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const int64_t v = __shfl_up_sync(0xffffffffu, upto, s);
            if (lane >= s) upto += v;
        }
        return __shfl_sync(0xffffffffu, upto, 31);
    };
    for (int from = 0; from < r.batch; from += 32) total += scan(from);
    share = max(static_cast<int64_t>(1), (total + gridDim.x - 1) / gridDim.x);
    walk.x = share * blockIdx.x;
    walk.end = min(total, walk.x + share);
    if (walk.x >= total) return false;
    int64_t before = 0;
    if (r.batch > 32) {
        for (int from = 0;; from += 32) {   // ends, since x is below the sum of all
            const int64_t all = scan(from);
            if (before + all > walk.x) break;
            before += all;
        }
    }
    const int at = __ffs(__ballot_sync(0xffffffffu, before + upto > walk.x)) - 1;
    walk.base = before + __shfl_sync(0xffffffffu, upto - mine, at);
    walk.b = walk.chunk + at;
    walk.enter(r, group);
    walk.find(r, group);
    return true;
}

// A block that has given up still counts for the tiles it shares with others, but for the first `counted`, which it has said are there: what the others have counted would be left in the
// workspace, and a replay of a captured call, whose number is the same, would go on counting from there.  One warp; not inlined, so that the walk that this takes costs the
// regular way nothing (part of a prompt 345 us; 357 where the kernel's own walk goes on).
template <int kRows>
__device__ __noinline__ void count_what_is_left(const AttendArgs &p, int counted)
{
    PromptWalk<kRows> walk;
    int64_t share;
    if (!begin(walk, p.r, p.group, share)) return;
    while (walk.next(p.r, p.group)) {
        if (walk.whole || counted-- > 0) continue;
        const int64_t block0 = walk.item0 / share;
        if ((threadIdx.x & 31) == 0) arrive(p.tickets + block0, p.nonce, static_cast<unsigned>((walk.item0 + walk.units - 1) / share - block0 + 1));
    }
}

// The first operand in tensor memory.
__device__ __forceinline__ void mma_f16_tmem(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tmov.b64 db, {%2, %5};\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)), "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
          "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
          "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t addr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// Before another thread, a product or a load of the thread's own may see what it has stored: stores are asynchronous, and loads of the same columns do not wait for them.
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Two weights in 16 bits, and what that leaves of them, in 16 bits too.
template <bool kHalf>
__device__ __forceinline__ void split(float a, float b, uint32_t &w, uint32_t &rest)
{
    w = to_16x2<kHalf>(a, b);
    float c, d;
    fma(Two(to_float<kHalf>(static_cast<uint16_t>(w)), to_float<kHalf>(static_cast<uint16_t>(w >> 16))), Two(-1.0f, -1.0f), Two(a, b)).get(c, d);
    rest = to_16x2<kHalf>(c, d);
}
// Scores of 32 positions from `position` on that the row does not see, or whose granules are not there.
__device__ __forceinline__ void hide(uint32_t (&s)[32], int position, int limit, uint32_t have)
{
#pragma unroll
    for (int e = 0; e < 32; ++e)
        if (position + e > limit || !(have >> (e / kGranule) & 1)) s[e] = 0xff800000u;
}

// Two slots work on a tile's score tiles in turn.  Events are products of queries and keys (and of weights and values): with more than 128 rows both slots' for each score tile, else the
// slots take every other one.
template <int kSlots>
struct Events {
    bool shared;   // by both slots
    int count;
    __device__ __forceinline__ Events(int steps, bool both) : shared(kSlots == 2 && both), count(shared ? 2 * steps : steps) {}
    __device__ __forceinline__ int tile(int e) const { return shared ? e >> 1 : e; }
    __device__ __forceinline__ int of_slot(int slot) const { return kSlots == 1 ? count : (count + 1 - slot) >> 1; }
};

// Calls f with constants.  The operands of matrix instructions are uniform registers: addresses that the compiler cannot see to be the same in all lanes cost it a move each, and
// an instruction its 64 clocks' worth of issue time.
template <typename F>
__device__ __forceinline__ void with_flags(uint32_t a, bool b, const F &f)
{
    const auto second = [&](auto x) {
        if (b) f(x, std::true_type{});
        else f(x, std::false_type{});
    };
    if (a) second(std::true_type{});
    else second(std::false_type{});
}
// Whether the phase is over, without a wait.
__device__ __forceinline__ bool bar_test_warp(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return __all_sync(0xffffffffu, ok != 0);
}

template <int D, bool kHalf>
__global__ void __launch_bounds__(PromptShape<D>::kThreads, 1)
cache_prompt_kernel(const __grid_constant__ AttendArgs p)
{
    using F = CacheFormat<D>;
    using S = PromptShape<D>;
    constexpr int kGroupsAll = D / kGroup;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *const smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_addr(smem);
    const uint32_t smem_q = base, smem_k = base + S::kSlots * S::kQueries, smem_v = smem_k + 2 * S::kOperand, smem_c = smem_v + 2 * S::kOperand;
    const uint32_t bars = smem_c + S::kRawStages * S::kRaw;
    SQ_LINEAR_CHECK(bars + 8 * S::kBars <= smem_end(smem_raw) && (bars & 7) == 0, 2020);
    const auto raw_full = [&](int s) { return bars + 8 * s; };
    const auto raw_empty = [&](int s) { return bars + 8 * (S::kRawStages + s); };
    const uint32_t queries_full = bars + 16 * S::kRawStages, together = queries_full + 8;
    // of the two places of keys and values, and of the slots
    const auto keys_full = [&](int i) { return queries_full + 16 + 8 * i; };
    const auto keys_empty = [&](int i) { return queries_full + 32 + 8 * i; };
    const auto values_full = [&](int i) { return queries_full + 48 + 8 * i; };
    const auto values_empty = [&](int i) { return queries_full + 64 + 8 * i; };
    const auto scores_full = [&](int slot) { return queries_full + 80 + 8 * slot; };
    const auto weights_full = [&](int slot) { return queries_full + 96 + 8 * slot; };
    const auto weights_empty = [&](int slot) { return queries_full + 112 + 8 * slot; };
    const auto sums_full = [&](int slot) { return queries_full + 128 + 8 * slot; };
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up_word, is_last;
    __shared__ uint32_t granules_there[kTilesAhead];   // of the last score tiles, by their number
    __shared__ int no_number[4][kGroupsAll];     // of the last pieces: the first position whose value group has no number
    __shared__ float2 slot_sums[kSlotRows];      // maximum and sum of the second slot's rows
    volatile int *gave_up = &gave_up_word;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    PromptWalk<S::kRows> walk;
    int64_t share;
    if (!begin(walk, p.r, p.group, share)) return;   // all threads of the block

    if (threadIdx.x == 0) {
        gave_up_word = 0;
        for (int s = 0; s < S::kRawStages; ++s) {
            bar_init(raw_full(s), 1);
            bar_init(raw_empty(s), kPromptConverters);
        }
        bar_init(queries_full, S::kSoftmax);
        bar_init(together, S::kSoftmax);
        for (int i = 0; i < 2; ++i) {
            bar_init(keys_full(i), kPromptConverters);
            bar_init(keys_empty(i), 1);
            bar_init(values_full(i), kPromptConverters);
            bar_init(values_empty(i), 1);
            bar_init(scores_full(i), 1);
            bar_init(weights_full(i), 4);
            bar_init(weights_empty(i), 1);
            bar_init(sums_full(i), 1);
        }
        for (int i = 0; i < 4 * kGroupsAll; ++i) no_number[i / kGroupsAll][i % kGroupsAll] = 0x7fffffff;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == S::kSoftmax + kPromptConverters + 1) tmem_alloc(smem_addr(&tmem_base), S::kColumns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    constexpr uint32_t tmem = 0;   // where the columns begin, since all have been asked for
    SQ_LINEAR_CHECK(tmem_base == tmem, 2023);

    if (warp < S::kSoftmax) {
        const int quarter = warp & 3, slot = warp >> 2;
        const uint32_t mine = tmem + (static_cast<uint32_t>(32 * quarter) << 16);   // the warp's lanes of tensor memory
        const uint32_t scores = mine + slot * S::kScores, weights = mine + S::kFirstWeights + slot * S::kWeights, sums = mine + S::kFirstSums + slot * S::kSums;
        const float scale = fmaxf(fabsf(p.scale_log2), 1.17549435e-38f);   // 0: no score is hidden by a product with infinity; scores of 2^126 make exponents of 1
        uint32_t tiles_before = 0, weighed = 0, summed = 0, pieces = 0, joins = 0;
        int counted = 0;   // tiles shared with other blocks that the block has counted for
        bool ok = true;
        const auto join = [&]() {
            __syncwarp();
            if (lane == 0) bar_arrive(together);
            ok = bar_wait_warp(together, joins++ & 1, gave_up);
        };
        while (ok && walk.next(p.r, p.group)) {
            const int rows_all = walk.rows_all(p.group), tile_row = walk.tile * S::kRows, steps = walk.template steps<S::kPositions>(p.group);
            const Events<S::kSlots> events(steps, rows_all - tile_row > kSlotRows);
            const bool alone = S::kSlots == 1 || events.shared;   // the slot has rows of its own
            const int row = (alone ? slot * kSlotRows : 0) + 32 * quarter + lane, at = tile_row + row;
            const bool valid = at < rows_all;
            const Target to(p, walk.row0, walk.head, min(at, rows_all - 1));
            const int limit = walk.limit(min(at, rows_all - 1), p.group), seen_least = walk.seen_least(p.group);
            const bool idle = at - lane >= rows_all;   // all rows of the warp
            float most = kNoScore, total = 0.0f, beyond = 0.0f;   // beyond: how far the tile before reached beyond the maximum
            if (steps > 0) {
                // a row's pieces by neighbouring lanes; with a negative scale the queries change their signs, so that larger scores are larger exponents
                const int64_t offset = to.row * p.q_stride + to.head * p.q_head;
                const uint32_t flip = p.scale_log2 < 0.0f ? 0x80008000u : 0u;
                constexpr int kPieces = D / 8, kAtOnce = 32 / kPieces;   // rows at once
                const auto queries = [&](auto on_vectors) {
                    constexpr bool kVector = decltype(on_vectors)::value;
                    constexpr int kBatch = kVector ? 8 : 1;   // pieces in flight
#pragma unroll 1
                    for (int j0 = 0; j0 < 32; j0 += kAtOnce * kBatch) {
                        uint4 v[kBatch];
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) {
                            const int r = j0 + i * kAtOnce + lane / kPieces;
                            const int64_t from = __shfl_sync(0xffffffffu, offset, r);
                            v[i] = make_uint4(0, 0, 0, 0);
                            if (row - lane + r + tile_row < rows_all) v[i] = load8(p.q + from + 8 * (lane % kPieces), kVector);
                        }
#pragma unroll
                        for (int i = 0; i < kBatch; ++i) {
                            const int local = 32 * quarter + j0 + i * kAtOnce + lane / kPieces, piece = lane % kPieces;
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(smem_q + slot * S::kQueries + piece / 8 * S::kQueryPanel + local * 128 + ((piece ^ local) & 7) * 16),
                                         "r"(v[i].x ^ flip), "r"(v[i].y ^ flip), "r"(v[i].z ^ flip), "r"(v[i].w ^ flip));
                        }
                    }
                };
                if (alone || slot == 0) {
                    if (p.q_vector) queries(std::true_type{});
                    else queries(std::false_type{});
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive(queries_full);
            }
            const int mine_of = events.of_slot(slot);
            // Weights of 32 positions take 16 columns, with what rounding leaves of them the place of their scores, which is 32.  Each way has a loop of its own, here and where the products are
            // made, and this one comes first: a choice in the loop costs part of a prompt 7 % (376 us instead of 350), the other order 1 % (356).
            const auto weigh_tiles = [&](auto in_two_c) {
                constexpr bool kTwo = decltype(in_two_c)::value;
                for (int i = 0; i < mine_of; ++i, ++weighed) {
                    ok = bar_wait_warp(scores_full(slot), weighed & 1, gave_up);
                    if (!ok) break;
                    tc_fence_after();
                    const int step = alone ? i : 2 * i + slot, position = walk.first * S::kRows + step * S::kPositions;
                    const uint32_t have = *const_cast<volatile uint32_t *>(&granules_there[(tiles_before + step) % kTilesAhead]);
                    const bool masked = position + S::kPositions - 1 > seen_least || have != (1u << S::kGranules) - 1;
                    const auto scale_sums = [&](float factor) {   // the products with the values of the tiles before have been made
                        total *= factor;
                        if (i == 0) return;
#pragma unroll 1
                        for (int j = 0; j < D; j += 32) {
                            uint32_t o[32];
                            tmem_ld32(sums + j, o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                            tmem_st32(sums + j, o);
                        }
                    };
                    const auto weigh = [&](auto some_hidden) {
                        constexpr bool kMasked = decltype(some_hidden)::value;
                        if (__any_sync(0xffffffffu, most == kNoScore)) {   // the first scores that a row sees: their maximum
                            float top = -INFINITY;
#pragma unroll 1
                            for (int j = 0; j < S::kPositions; j += 32) {
                                uint32_t s[32];
                                tmem_ld32(scores + j, s);
                                if constexpr (kMasked) hide(s, position + j, limit, have >> (j / kGranule));
#pragma unroll
                                for (int e = 0; e < 32; e += 2) top = max3(top, __uint_as_float(s[e]), __uint_as_float(s[e + 1]));
                            }
                            const float next = fmaxf(fmaxf(top * scale, most), kNoScore);
                            scale_sums(exp2_fast(most - next));
                            most = next;
                        } else if (__any_sync(0xffffffffu, beyond > kGrowth)) {
                            scale_sums(exp2_fast(-beyond));
                            most += beyond;
                        }
                        beyond = 0.0f;
                        const Two by(scale, scale);
                        Two sum(total, 0.0f);
#pragma unroll 1
                        for (int j = 0; j < S::kPositions; j += 32) {
                            uint32_t s[32];
                            tmem_ld32(scores + j, s);
                            if constexpr (kMasked) hide(s, position + j, limit, have >> (j / kGranule));
                            const Two less(-most, -most);
                            float x[32], tops[4];
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                fma(Two(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), by, less).get(x[e], x[e + 1]);
                                tops[e / 2 % 4] = e < 8 ? fmaxf(x[e], x[e + 1]) : max3(tops[e / 2 % 4], x[e], x[e + 1]);
                            }
                            float top = max3(max3(tops[0], tops[1], tops[2]), tops[3], beyond);
                            if (__any_sync(0xffffffffu, top > kRoom)) {
                                // too far beyond the maximum: what there is of the row is scaled at once, this tile's weights so far among it, by a power of two, which
                                // rounds none of them again
                                tmem_st_wait();   // weights and sums that this tile has stored are about to be loaded
                                const float down = floorf(top), factor = exp2_fast(-down);   // the row's largest weight stays 1 at least
                                float a, b;
                                sum.get(a, b);
                                total = a + b;
                                scale_sums(factor);
                                sum = Two(total, 0.0f);
                                most += down;
#pragma unroll 1
                                for (int k = 0; k < (kTwo ? j : j / 2); k += 8) {
                                    uint32_t w[8];
                                    tmem_ld8((kTwo ? scores : weights) + k, w);
#pragma unroll
                                    for (int e = 0; e < 8; ++e)
                                        w[e] = to_16x2<kHalf>(to_float<kHalf>(static_cast<uint16_t>(w[e])) * factor, to_float<kHalf>(static_cast<uint16_t>(w[e] >> 16)) * factor);
                                    tmem_st8((kTwo ? scores : weights) + k, w);
                                }
#pragma unroll
                                for (int e = 0; e < 32; ++e) x[e] -= down;
                                top -= down;
                            }
                            beyond = top;
                            uint32_t w[16];
                            if constexpr (kTwo) {
                                uint32_t rest[16];
#pragma unroll
                                for (int e = 0; e < 32; e += 2) {
                                    const float a = exp2_fast(x[e]), b = exp2_fast(x[e + 1]);
                                    sum = add(sum, Two(a, b));
                                    split<kHalf>(a, b, w[e / 2], rest[e / 2]);
                                }
                                tmem_st16(scores + j, w);
                                tmem_st16(scores + j + 16, rest);
                            } else {
#pragma unroll
                                for (int e = 0; e < 32; e += 2) {
                                    const float a = exp2_fast(x[e]), b = exp2_fast(x[e + 1]);
                                    sum = add(sum, Two(a, b));
                                    w[e / 2] = to_16x2<kHalf>(a, b);
                                }
                                tmem_st16(weights + j / 2, w);   // the scores there have been read
                            }
                        }
                        float a, b;
                        sum.get(a, b);
                        total = a + b;
                        tmem_st_wait();
                    };
                    if (!idle) {
                        if (masked) weigh(std::true_type{});
                        else weigh(std::false_type{});
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(weights_full(slot));
                }
            };
            if (rows_all > kWholeRows) weigh_tiles(std::false_type{});
            else weigh_tiles(std::true_type{});
            tiles_before += steps;
            if (!ok) break;
            if (mine_of > 0) {
                ok = bar_wait_warp(sums_full(slot), summed++ & 1, gave_up);
                if (!ok) break;
            }
            const bool whole = walk.whole;
            float factor = 1.0f, other = 0.0f;   // of the slots' sums
            if (!alone) {
                if (slot == 1) slot_sums[32 * quarter + lane] = make_float2(most, total);
                tc_fence_before();
                join();
                if (!ok) break;
                if (slot == 0) {
                    const float2 ml = slot_sums[row];
                    const float next = fmaxf(most, ml.x);
                    factor = exp2_fast(most - next);
                    other = exp2_fast(ml.x - next);   // no score: 0, unless neither has one
                    total = total * factor + ml.y * other;
                    most = next;
                }
            }
            tc_fence_after();
            const bool both = !alone && events.count > 1;   // the other slot has sums
            const int64_t block0 = walk.item0 / share;
            float *const part = p.parts + (2 * static_cast<int64_t>(blockIdx.x) + (walk.item0 >= share * blockIdx.x)) * S::kPart;
            const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
            if (alone || slot == 0) {
#pragma unroll 1
                for (int j = 0; j < D; j += 32) {
                    uint32_t o[32];
                    if (steps > 0) {
                        tmem_ld32(sums + j, o);
                        if (both) {
                            uint32_t more[32];
                            tmem_ld32(sums + S::kSums + j, more);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(fmaf(__uint_as_float(more[e]), other, __uint_as_float(o[e]) * factor));
                        }
                        const bool none = *const_cast<volatile int *>(&no_number[pieces & 3][j / kGroup]) <= limit;
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = none ? 0x7fffffffu : o[e];
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = 0;
                    }
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            __stcg(reinterpret_cast<float4 *>(part + row * D + j + e), make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]),
                                                                                                     __uint_as_float(o[e + 2]), __uint_as_float(o[e + 3])));
                    } else if (valid) {
                        uint16_t *out = p.out + to.row * p.out_stride + to.head * p.out_head + j;
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int h = 0; h < 4; ++h) w[h] = to_16x2<kHalf>(__uint_as_float(o[e + 2 * h]) * inverse, __uint_as_float(o[e + 2 * h + 1]) * inverse);
                            if (p.out_vector) {
                                *reinterpret_cast<uint4 *>(out + e) = make_uint4(w[0], w[1], w[2], w[3]);
                            } else {
#pragma unroll
                                for (int h = 0; h < 8; ++h) out[e + h] = static_cast<uint16_t>(w[h / 2] >> (16 * (h & 1)));
                            }
                        }
                    }
                }
                if (whole && valid && p.lse) store_lse(p, to, most, total);
                if (!whole) __stcg(reinterpret_cast<float2 *>(part + S::kRows * D) + row, make_float2(most, total));
            }
            tc_fence_before();
            // all have read the sums and what goes with them, and written their part
            if (!whole) __threadfence();
            join();
            if (!ok) break;
            if (steps > 0) {
                if (threadIdx.x < kGroupsAll) no_number[pieces & 3][threadIdx.x] = 0x7fffffff;
                ++pieces;
            }
            if (whole) continue;
            const int blocks = static_cast<int>((walk.item0 + walk.units - 1) / share - block0 + 1);
            if (threadIdx.x == 0) is_last = arrive(p.tickets + block0, p.nonce, blocks);
            ++counted;
            join();
            if (!ok) break;
            if (!*const_cast<volatile int *>(&is_last)) continue;
            __threadfence();
            const float *const parts = p.parts + 2 * block0 * S::kPart;
            constexpr int kAtOnce = 4;   // rows in flight, with two parts of each
            for (int i0 = threadIdx.x; i0 < S::kRows * (D / 4); i0 += kAtOnce * 32 * S::kSoftmax) {
                if (walk.tile * S::kRows + i0 / (D / 4) >= rows_all) break;
                Joined sum[kAtOnce];
                for (int b0 = 0; b0 < blocks; b0 += 2) {
                    float4 x[kAtOnce][2];
                    float2 ml[kAtOnce][2];
#pragma unroll
                    for (int k = 0; k < 2 * kAtOnce; ++k) {
                        const int b = min(b0 + k % 2, blocks - 1), i = i0 + k / 2 * 32 * S::kSoftmax;
                        const float *from = parts + (2 * static_cast<int64_t>(b) + (b == 0)) * S::kPart;
                        x[k / 2][k % 2] = __ldcg(reinterpret_cast<const float4 *>(from) + i);
                        ml[k / 2][k % 2] = __ldcg(reinterpret_cast<const float2 *>(from + S::kRows * D) + i / (D / 4));
                        if (b0 + k % 2 >= blocks) ml[k / 2][k % 2].y = 0.0f;
                    }
#pragma unroll
                    for (int k = 0; k < kAtOnce; ++k) sum[k].add(x[k], ml[k]);
                }
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int i = i0 + k * 32 * S::kSoftmax, r = i / (D / 4), column = i % (D / 4) * 4;
                    if (walk.tile * S::kRows + r < rows_all)
                        finish4<kHalf>(p, Target(p, walk.row0, walk.head, walk.tile * S::kRows + r), column, sum[k].v, sum[k].top, sum[k].l);
                }
            }
        }
        if (!ok && warp == 0) count_what_is_left<S::kRows>(p, counted);
    } else if (warp < S::kSoftmax + kPromptConverters) {
        // keys and values of two granules: 128 pieces of 16 bytes (8) and slab of each
        static_assert(kPromptConverters == 4, "one of each a thread and two granules");
        const int unit = threadIdx.x - 32 * S::kSoftmax;
        const CodePairs<kHalf> pairs;
        uint32_t stage = 0, turn = 0, tiles_done = 0, pieces = 0;
        bool ok = true;
        while (ok && walk.next(p.r, p.group)) {
            const int steps = walk.template steps<S::kPositions>(p.group), seen_most = walk.seen_most(p.group);
            for (int i = 0; ok && i < steps; ++i, ++tiles_done) {
                const int position = walk.first * S::kRows + i * S::kPositions;
                if (tiles_done > 1)   // the products with what is there have been made
                    ok = bar_wait_warp(keys_empty(tiles_done & 1), (tiles_done / 2 - 1) & 1, gave_up) &&
                         bar_wait_warp(values_empty(tiles_done & 1), (tiles_done / 2 - 1) & 1, gave_up);
#pragma unroll 1
                for (int part = 0; ok && part < S::kParts; ++part) {
                    ok = bar_wait_warp(raw_full(stage), turn, gave_up);
                    if (!ok) break;
#pragma unroll 1
                    for (int two = 0; two < S::kRawGranules; two += 2) {
                        const uint8_t *const raw = smem + (smem_c - base) + stage * S::kRaw + two * F::kBytes;
                        const int first_row = (part * S::kRawGranules + two) * kGranule;
                        {
                            const uint32_t to = smem_k + (tiles_done & 1) * S::kOperand;
                            // (position, word % 4): neighbouring lanes have the words % 4 of positions t and t + 4, whose 16-byte pieces are in different banks
                            const int c = unit & 3, t = (unit >> 2 & 1) * 4 | (unit >> 3 & 3) | (unit >> 5) * 8, row = first_row + t;   // t: 0 .. 31
                            const uint8_t *const granule = raw + t / kGranule * F::kBytes;
                            uint32_t scales[kGroupsAll / 2], w[F::kSlabs][4];
#pragma unroll
                            for (int j = 0; j < kGroupsAll / 2; ++j) scales[j] = *reinterpret_cast<const uint32_t *>(granule + F::kKeyScales + t % kGranule * (2 * kGroupsAll) + 4 * j);
#pragma unroll
                            for (int a = 0; a < F::kSlabs; ++a) {
                                const uint8_t *const from = granule + a * (64 * F::kWords) + t % kGranule * (4 * F::kWords) + c * F::kWords;
                                if constexpr (F::kGroups == 2) {
                                    const uint2 v = *reinterpret_cast<const uint2 *>(from);
                                    w[a][0] = v.x; w[a][1] = v.y;
                                } else {
                                    const uint4 v = *reinterpret_cast<const uint4 *>(from);
                                    w[a][0] = v.x; w[a][1] = v.y; w[a][2] = v.z; w[a][3] = v.w;
                                }
                            }
#pragma unroll
                            for (int g = 0; g < kGroupsAll; ++g) {
                                const int word = 4 * g + c;
                                uint32_t o[4];
                                pairs(w[g / F::kGroups][g % F::kGroups], pairs.scales(scale_twice<kHalf>(scales[g / 2], g & 1)), o);
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + word / 8 * S::kPanel + row * 128 + ((word ^ row) & 7) * 16),
                                             "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                            }
                        }
                        {
                            const uint32_t to = smem_v + (tiles_done & 1) * S::kOperand;
                            // (pair of positions, word % 8)
                            constexpr int kLaneWords = F::kWords / 8;
                            const int g = unit & 7, pair = unit >> 3, row = first_row + 2 * pair;   // pair: 0 .. 15
                            const uint8_t *const granule = raw + pair / 8 * F::kBytes;
                            const bool there = *const_cast<volatile uint32_t *>(&granules_there[tiles_done % kTilesAhead]) >> (first_row / kGranule + pair / 8) & 1;
                            // positions behind the last one that any row sees, and granules that are not there, may hold anything
                            const uint32_t seen = (there && position + row <= seen_most ? 0xffffu : 0u) | (there && position + row + 1 <= seen_most ? 0xffff0000u : 0u);
                            uint32_t scales[F::kSlabs][kLaneWords], w[F::kSlabs][4];
                            bool odd = false;
#pragma unroll
                            for (int a = 0; a < F::kSlabs; ++a) {
                                const uint8_t *const from = granule + F::kValues + a * (64 * F::kWords) + (pair % 8 * 8 + g) * (8 * kLaneWords);
                                if constexpr (kLaneWords == 1) {
                                    const uint2 v = *reinterpret_cast<const uint2 *>(from);
                                    w[a][0] = v.x; w[a][1] = v.y;
                                } else {
                                    const uint4 v = *reinterpret_cast<const uint4 *>(from);
                                    w[a][0] = v.x; w[a][1] = v.y; w[a][2] = v.z; w[a][3] = v.w;
                                }
#pragma unroll
                                for (int m = 0; m < kLaneWords; ++m) {
                                    scales[a][m] = seen & *reinterpret_cast<const uint32_t *>(granule + F::kValueScales + a * (32 * F::kGroups) + pair % 8 * (4 * F::kGroups) + (g >> 2) * (2 * F::kGroups) + 4 * m);
                                    odd |= (scales[a][m] & 0x7f80u) == 0x7f80u || (scales[a][m] & 0x7f800000u) == 0x7f800000u;
                                }
                            }
                            if (odd) {   // no number: for rows that see the position only, see the end of the tile
#pragma unroll
                                for (int a = 0; a < F::kSlabs; ++a)
#pragma unroll
                                    for (int m = 0; m < kLaneWords; ++m)
#pragma unroll
                                        for (int h = 0; h < 2; ++h)
                                            if ((scales[a][m] >> (16 * h) & 0x7f80u) == 0x7f80u) {
                                                scales[a][m] &= h ? 0x0000ffffu : 0xffff0000u;
                                                atomicMin(&no_number[pieces & 3][a * F::kGroups + 2 * m + (g >> 2)], position + row + h);
                                            }
                            }
#pragma unroll
                            for (int a = 0; a < F::kSlabs; ++a)
#pragma unroll
                                for (int m = 0; m < kLaneWords; ++m)
#pragma unroll
                                    for (int h = 0; h < 2; ++h) {
                                        uint32_t o[4];
                                        pairs(w[a][h * kLaneWords + m], pairs.scales(scale_twice<kHalf>(scales[a][m], h)), o);
                                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (a * kLaneWords + m) * S::kPanel + (row + h) * 128 + ((g ^ (row + h)) & 7) * 16),
                                                     "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                                    }
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        bar_arrive(raw_empty(stage));
                        if (part == S::kParts - 1) {
                            bar_arrive(keys_full(tiles_done & 1));
                            bar_arrive(values_full(tiles_done & 1));
                        }
                    }
                    if (++stage == S::kRawStages) {
                        stage = 0;
                        turn ^= 1;
                    }
                }
            }
            if (steps > 0) ++pieces;
        }
    } else if (warp == S::kSoftmax + kPromptConverters) {
        uint32_t stage = 0, turn = 1, issued = 0, tiles_done = 0;
        int granule = -1;   // the lane's, of the score tiles to come
        bool ok = true;
        const int granules = p.r.page_size / kGranule;
        while (ok && walk.next(p.r, p.group)) {
            const int steps = walk.template steps<S::kPositions>(p.group), seen_most = walk.seen_most(p.group);
            for (int i = 0; ok && i < steps; ++i, ++tiles_done) {
                constexpr int kBatch = 32 / S::kGranules;   // score tiles whose granules are looked up together
                if (i % kBatch == 0) {
                    const int at = walk.first * S::kRows + i * S::kPositions + lane * kGranule;
                    granule = -1;
                    if (at <= seen_most) {
                        const int column = at / p.r.page_size;
                        const int64_t page = page_of(p.r, walk.b, column);
                        SQ_LINEAR_CHECK(column < p.r.width, 2022);
                        if (page >= 0) granule = static_cast<int>((page * p.r.kv_heads + walk.head) * granules + (at - column * p.r.page_size) / kGranule);
                    }
                }
                const int from_lane = i % kBatch * S::kGranules;
                const uint32_t have = __ballot_sync(0xffffffffu, granule >= 0) >> from_lane & ((1u << S::kGranules) - 1);
#pragma unroll 1
                for (int part = 0; part < S::kParts; ++part) {
                    ok = bar_wait_warp(raw_empty(stage), turn, gave_up);
                    if (!ok) break;
                    int from[S::kRawGranules];
                    bool run = true;   // one behind the other
#pragma unroll
                    for (int j = 0; j < S::kRawGranules; ++j) {
                        from[j] = __shfl_sync(0xffffffffu, granule, from_lane + part * S::kRawGranules + j);
                        run = run && from[j] >= 0 && from[j] == from[0] + j;
                    }
                    if (elect_one()) {
                        const uint32_t dst = smem_c + stage * S::kRaw, bar = raw_full(stage);
                        if (part == 0) *const_cast<volatile uint32_t *>(&granules_there[tiles_done % kTilesAhead]) = have;
                        bar_expect(bar, __popc(have >> (part * S::kRawGranules) & ((1u << S::kRawGranules) - 1)) * F::kBytes);
                        if (run) {
                            bulk_load(dst, p.cache + static_cast<int64_t>(from[0]) * F::kBytes, S::kRaw, bar);
                        } else {
#pragma unroll
                            for (int j = 0; j < S::kRawGranules; ++j)
                                if (from[j] >= 0) bulk_load(dst + j * F::kBytes, p.cache + static_cast<int64_t>(from[j]) * F::kBytes, F::kBytes, bar);
                        }
                    }
                    __syncwarp();
                    if (issued < S::kRawStages) ++issued;
                    if (++stage == S::kRawStages) {
                        stage = 0;
                        turn ^= 1;
                    }
                }
            }
        }
        // the last copies have landed before the block may end
        for (uint32_t i = 0; i < issued; ++i) {
            if (stage-- == 0) {
                stage = S::kRawStages - 1;
                turn ^= 1;
            }
            bar_drain(raw_full(stage), turn ^ 1);
        }
    } else {
        constexpr uint32_t kType = (1u << 4) | (kHalf ? 0u : 1u << 7) | (kHalf ? 0u : 1u << 10) | (static_cast<uint32_t>(kSlotRows >> 4) << 24);
        constexpr uint32_t kScoresDesc = kType | (static_cast<uint32_t>(S::kPositions >> 3) << 17);
        constexpr uint32_t kSumsDesc = kType | 1u << 16 | (static_cast<uint32_t>(D >> 3) << 17);   // values with their channels next to each other
        uint32_t tiles_before = 0, pieces = 0, scored[2] = {}, summed[2] = {};   // products of each slot
        int keys_used[2] = {}, values_used[2] = {}, tries = 0;   // by how many slots, of the tile in a place
        bool ok = true;
        while (ok && walk.next(p.r, p.group)) {
            const int steps = walk.template steps<S::kPositions>(p.group);
            if (steps == 0) continue;
            const Events<S::kSlots> events(steps, walk.rows_all(p.group) - walk.tile * S::kRows > kSlotRows);
            const bool in_two = walk.rows_all(p.group) <= kWholeRows;
            ok = bar_wait_warp(queries_full, pieces & 1, gave_up);
            // each slot's next product, as soon as what it takes is there: the scores of event at[], or, if they have been asked for, the sums of it
            int at[2] = {0, 1};
            bool asked[2] = {false, false};
            const int used_by = events.shared ? 2 : 1;
            const auto turn = [&](auto slot_c, auto two_c) {
                constexpr int kSlot = decltype(slot_c)::value;
                constexpr bool kTwo = decltype(two_c)::value;
                const int e = at[kSlot];
                if (e >= events.count) return;
                const uint32_t tile = tiles_before + events.tile(e), place = tile & 1;
                if (!asked[kSlot]) {
                    // keys; the scores' place, if the weights of the slot's product before have it, when that has been made
                    if (!bar_test_warp(keys_full(place), tile >> 1 & 1)) return;
                    if ((!S::kApart || kTwo) && summed[kSlot] > 0 && !bar_test_warp(weights_empty(kSlot), (summed[kSlot] - 1) & 1)) return;
                    tc_fence_after();
                    const bool last = ++keys_used[place] == used_by;
                    if (last) keys_used[place] = 0;
                    with_flags(place, !kTwo && events.shared, [&](auto place_c, auto shared_c) {
                        constexpr int kPlace = decltype(place_c)::value, kOwn = decltype(shared_c)::value ? kSlot : 0;
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < D / 16; ++k)
                                mma_f16(kSlot * S::kScores, desc_low(smem_q + kOwn * S::kQueries + k / 4 * S::kQueryPanel + k % 4 * 32, 16),
                                        desc_low(smem_k + kPlace * S::kOperand + k / 4 * S::kPanel + k % 4 * 32, 16), kScoresDesc, k > 0);
                            mma_commit(scores_full(kSlot));
                            if (last) mma_commit(keys_empty(kPlace));
                        }
                    });
                    __syncwarp();
                    ++scored[kSlot];
                    asked[kSlot] = true;
                } else {
                    if (!bar_test_warp(weights_full(kSlot), (scored[kSlot] - 1) & 1) || !bar_test_warp(values_full(place), tile >> 1 & 1)) return;
                    tc_fence_after();
                    const bool last = ++values_used[place] == used_by, begins = e < S::kSlots, ends = e + S::kSlots >= events.count;
                    if (last) values_used[place] = 0;
                    with_flags(place, false, [&](auto place_c, auto) {
                        constexpr int kPlace = decltype(place_c)::value;
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < S::kPositions / 16; ++k)
#pragma unroll
                                for (int rest = 0; rest < (kTwo ? 2 : 1); ++rest)
                                    mma_f16_tmem(S::kFirstSums + kSlot * S::kSums, kTwo ? kSlot * S::kScores + k / 2 * 32 + k % 2 * 8 + 16 * rest : S::kFirstWeights + kSlot * S::kWeights + 8 * k,
                                                 desc_low(smem_v + kPlace * S::kOperand + k * 2048, S::kPanel), kSumsDesc, k > 0 || rest > 0 || !begins);
                            mma_commit(weights_empty(kSlot));
                            if (last) mma_commit(values_empty(kPlace));
                            if (ends) mma_commit(sums_full(kSlot));
                        }
                    });
                    __syncwarp();
                    ++summed[kSlot];
                    asked[kSlot] = false;
                    at[kSlot] = e + S::kSlots;
                    tries = 0;
                }
            };
            const auto products = [&](auto two_c) {
                while (ok && (at[0] < events.count || (S::kSlots > 1 && at[1] < events.count))) {
                    turn(std::integral_constant<int, 0>{}, two_c);
                    if constexpr (S::kSlots > 1) turn(std::integral_constant<int, 1>{}, two_c);
                    // no try waits: a second's worth of them
                    if (__any_sync(0xffffffffu, ++tries > (wait_limit() << 6 | 63) || *gave_up)) {
                        if (lane == 0) {
                            *gave_up = 1;
                            atomicExch(&g_linear_status, 1);
                        }
                        ok = false;
                    }
                }
            };
            if (!in_two) products(std::false_type{});
            else products(std::true_type{});
            tiles_before += steps;
            ++pieces;
        }
        // the tensor cores have done their last products, and said so, before the block may end
#pragma unroll
        for (int slot = 0; slot < S::kSlots; ++slot) {
            if (scored[slot] > 0) bar_drain(scores_full(slot), (scored[slot] - 1) & 1);
            if (summed[slot] > 0) bar_drain(weights_empty(slot), (summed[slot] - 1) & 1);
        }
        if (ok && tiles_before > 0) bar_drain(values_empty((tiles_before - 1) & 1), (tiles_before - 1) >> 1 & 1);
    }
    __syncwarp();
    if (*gave_up) __nanosleep(100000);
    tc_fence_before();
    __syncthreads();
    if (warp == S::kSoftmax + kPromptConverters + 1) {
        tc_fence_after();
        tmem_free(tmem, S::kColumns);
    }
}

}  // namespace sq
