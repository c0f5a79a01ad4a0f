// Matrix products of the linear operators on the tensor cores (tcgen05), and the epilogue they share.  Here: up to 256
// tokens, one operand a 16-bit matrix that TMA brings into shared memory, the other one 8- or 4-bit codes that converter warps
// turn into 16-bit floats.
//
//   forward          u[t][m]  = sum_k x[t][k]    codes[m][k]     y = act(s_m u + b_m) + r     (both "K-major")
//   input gradient   dx[t][k] = sum_m dzs[t][m]  codes[m][k]     dzs = dz * s                 (codes "MN-major")
//   weight gradient  dw[m][k] = sum_t dz[t][m]   xhat[t][k]      xhat: 8-bit checkpoint       (both "MN-major")
//
// A code is exact in bf16 and fp16 and so is a checkpoint's value in bf16: every product the tensor cores form is exact and
// summed in fp32; scales and biases are applied to the fp32 sums.
#pragma once

#include "linear_device.cuh"

namespace sq {

enum GemmMode { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

struct GemmArgs {
    const uint8_t *codes;    // coded operand, rows of code_pitch bytes
    int64_t code_pitch;
    int32_t code_rows;
    int32_t rows, cols;      // of the result
    int32_t depth;           // of the contraction
    // dense_kernel only: the launch's part of a long contraction, in steps of kTileDepth, and the fp32 sums that its parts hand on
    int32_t first_step, steps;
    float *sums;             // [rows][sums_pitch], or null: one part
    int64_t sums_pitch;      // a multiple of 32
    int32_t sums_in, sums_out;   // add what the parts before left; leave the sums and no result
    int32_t row_tiles;
    int32_t box_rows;        // of a copy of the 16-bit operand
    int64_t tiles;
    uint16_t *out;           // 16-bit result
    int64_t out_stride;
    int32_t out_vector;      // rows of the result start on 16 bytes
    // forward only
    const float *scales, *bias;
    int32_t param_vector;    // scales and bias start on 16 bytes
    const uint16_t *residual;
    int64_t residual_stride;
    int32_t residual_vector;
    int32_t act;
    uint8_t *z_codes, *z_exps;   // checkpoint of the pre-activation, or null
    int64_t z_pitch, z_exps_pitch;
};

constexpr int kTileDepth = 64;        // of the contraction per stage: 128 bytes

// Terms of a contraction that one accumulator of a matrix instruction takes, at most.  The tensor cores cut off what does not fit when they add
// up: sums of values of one sign lose 5.6e-9 of themselves a term (dweight of 2^21 tokens 1.2 %, 2^16 tokens 4e-4, an eighth of bf16's half step).
// Longer contractions are shared by warps and thread blocks where they are shared anyhow, or go through dense_kernel in parts whose sums are added
// in fp32, to the nearest.  A part also bounds what a wait for a tile's sums has to cover: 1,024 steps, below a millisecond.
// Parts cost little: dweight of 131,072 tokens 4096 x 4096 3.76 ms in two and 3.78 in one, of 262,144 tokens 512 x 512 701 us in four and 665 in one.
constexpr int64_t kLongestSum = 1 << 16;

// Places where a warp turns 32 rows by 32 columns of 16-bit values round, for rows that a thread cannot read or write in vectors: a
// thread's row lies in 17 words, so that rows and columns hit all banks.
constexpr int kTurnWords = 17, kTurnBytes = 4 * 32 * kTurnWords;

// `out`: the warp's first row and column of the matrix; rows, n: of them inside it.
__device__ __forceinline__ void turn_store(uint32_t turn, const uint32_t (&packed)[16], uint16_t *out, int64_t stride, int rows, int n)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(turn + 4 * (lane * kTurnWords + i)), "r"(packed[i]) : "memory");
    __syncwarp();
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
        uint16_t v;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(turn + 4 * r * kTurnWords + 2 * lane) : "memory");
        if (lane < n) out[r * stride + lane] = v;
    }
}
__device__ __forceinline__ void turn_load(uint32_t turn, uint32_t (&packed)[16], const uint16_t *in, int64_t stride, int rows, int n)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll 8
    for (int r = 0; r < rows; ++r) {
        const uint16_t v = lane < n ? in[r * stride + lane] : static_cast<uint16_t>(0);
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(turn + 4 * r * kTurnWords + 2 * lane), "h"(v) : "memory");
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(packed[i]) : "r"(turn + 4 * (lane * kTurnWords + i)) : "memory");
}

// 32 columns of 32 rows of the result from `row0` on; a lane owns a row, so the 32 channels that share a checkpoint's exponent are
// all its own.  All lanes of a warp call it; `turn` is the warp's place in shared memory.
template <int kMode, bool kHalf>
__device__ __forceinline__ void finish32(const GemmArgs &p, int64_t row0, int col, const uint32_t (&acc)[32], uint32_t turn)
{
    const int n = min(32, p.cols - col), rows = static_cast<int>(min(static_cast<int64_t>(32), p.rows - row0));   // rows may be negative
    if (rows <= 0) return;
    SQ_LINEAR_CHECK(n > 0 && row0 >= 0 && col >= 0, 1020);
    const int64_t row = row0 + (threadIdx.x & 31);
    const bool valid = static_cast<int>(threadIdx.x & 31) < rows;
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(acc[i]);
    if (p.sums) {
        SQ_LINEAR_CHECK(col + 32 <= p.sums_pitch && (!valid || row < p.rows), 1021);
        float4 *sums = reinterpret_cast<float4 *>(p.sums + row * p.sums_pitch + col);   // 32 columns: the pitch is a multiple of that
        if (valid && p.sums_in)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float4 s = get(sums + j);
                v[4 * j] += s.x;
                v[4 * j + 1] += s.y;
                v[4 * j + 2] += s.z;
                v[4 * j + 3] += s.w;
            }
        if (p.sums_out) {
            if (valid)
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            return;
        }
    }
    if constexpr (kMode == kForward) {
        if (p.param_vector && n == 32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float4 s = get(reinterpret_cast<const float4 *>(p.scales + col) + j);
                const float4 b = p.bias ? get(reinterpret_cast<const float4 *>(p.bias + col) + j) : make_float4(0, 0, 0, 0);
                v[4 * j] = fmaf(v[4 * j], s.x, b.x);
                v[4 * j + 1] = fmaf(v[4 * j + 1], s.y, b.y);
                v[4 * j + 2] = fmaf(v[4 * j + 2], s.z, b.z);
                v[4 * j + 3] = fmaf(v[4 * j + 3], s.w, b.w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                v[i] = i < n ? fmaf(v[i], get(p.scales + col + i), p.bias ? get(p.bias + col + i) : 0.0f) : 0.0f;
        }
        if (p.z_codes) {
            float a = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i) a = max_nan(a, fabsf(v[i]));
            const uint32_t e = ckpt_exponent(a);
            const float inverse = ckpt_inverse(e);
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = ckpt_codes(v + 4 * i, inverse);
            if (valid) {
                SQ_LINEAR_CHECK(row < p.rows && col + 32 <= p.z_pitch && (col >> 5) < p.z_exps_pitch, 1022);
                uint4 *zc = reinterpret_cast<uint4 *>(p.z_codes + row * p.z_pitch + col);
                zc[0] = make_uint4(w[0], w[1], w[2], w[3]);
                zc[1] = make_uint4(w[4], w[5], w[6], w[7]);
                p.z_exps[row * p.z_exps_pitch + (col >> 5)] = static_cast<uint8_t>(e);
            }
        }
        act_values(v, p.act);
        if (p.residual) {
            uint32_t w[16];
            if (p.residual_vector && n == 32) {
                const uint16_t *r = p.residual + (valid ? row : row0) * p.residual_stride + col;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 q = get(reinterpret_cast<const uint4 *>(r) + j);
                    w[4 * j] = q.x; w[4 * j + 1] = q.y; w[4 * j + 2] = q.z; w[4 * j + 3] = q.w;
                }
            } else {
                turn_load(turn, w, p.residual + row0 * p.residual_stride + col, p.residual_stride, rows, n);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                v[2 * i] += to_float<kHalf>(static_cast<uint16_t>(w[i]));
                v[2 * i + 1] += to_float<kHalf>(static_cast<uint16_t>(w[i] >> 16));
            }
        }
    }
    uint32_t packed[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) packed[i] = to_16x2<kHalf>(v[2 * i], v[2 * i + 1]);
    if (p.out_vector && n == 32) {
        if (valid) {
            SQ_LINEAR_CHECK(row < p.rows && col + 32 <= p.cols && (reinterpret_cast<uintptr_t>(p.out + row * p.out_stride + col) & 15) == 0, 1023);
            uint4 *out = reinterpret_cast<uint4 *>(p.out + row * p.out_stride + col);
#pragma unroll
            for (int j = 0; j < 4; ++j) out[j] = make_uint4(packed[4 * j], packed[4 * j + 1], packed[4 * j + 2], packed[4 * j + 3]);
        }
    } else {
        turn_store(turn, packed, p.out + row0 * p.out_stride + col, p.out_stride, rows, n);
    }
}

// The same for four columns a thread: eight neighbouring lanes hold the 32 channels of an exponent, all lanes of a warp call it.
template <int kMode, bool kHalf>
__device__ __forceinline__ void finish4(const GemmArgs &p, int64_t row, int col, const float (&scale)[4], const float (&bias)[4], float (&v)[4])
{
    const int n = p.cols - col;   // columns of this thread, if below four
    SQ_LINEAR_CHECK(row >= 0 && row < p.rows, 1024);
    if constexpr (kMode == kForward) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf(v[i], scale[i], bias[i]);   // 0 behind the last channel
        if (p.z_codes) {
            float a = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) a = max_nan(a, fabsf(v[i]));
#pragma unroll
            for (int s = 1; s <= 4; s <<= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, s));
            const uint32_t e = ckpt_exponent(a);
            const float inverse = ckpt_inverse(e);
            const uint32_t w = ckpt_codes(v, inverse);
            if ((col & ~31) < p.cols) {   // rows end on 32
                SQ_LINEAR_CHECK(col + 4 <= p.z_pitch && (col >> 5) < p.z_exps_pitch, 1025);
                *reinterpret_cast<uint32_t *>(p.z_codes + row * p.z_pitch + col) = w;
                if ((col & 31) == 0) p.z_exps[row * p.z_exps_pitch + (col >> 5)] = static_cast<uint8_t>(e);
            }
        }
        act_values(v, p.act);
        if (p.residual) {
            const uint16_t *r = p.residual + row * p.residual_stride + col;
            if (p.residual_vector && n >= 4) {
                const uint2 q = get(reinterpret_cast<const uint2 *>(r));
                v[0] += to_float<kHalf>(static_cast<uint16_t>(q.x));
                v[1] += to_float<kHalf>(static_cast<uint16_t>(q.x >> 16));
                v[2] += to_float<kHalf>(static_cast<uint16_t>(q.y));
                v[3] += to_float<kHalf>(static_cast<uint16_t>(q.y >> 16));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < n) v[i] += to_float<kHalf>(get(r + i));
            }
        }
    }
    uint16_t *out = p.out + row * p.out_stride + col;
    if (p.out_vector && n >= 4) {
        *reinterpret_cast<uint2 *>(out) = make_uint2(to_16x2<kHalf>(v[0], v[1]), to_16x2<kHalf>(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) out[i] = to_16<kHalf>(v[i]);
    }
}

constexpr int kFusedCols = 128;       // columns of the result a tile: the tensor memory's lanes
constexpr int kFusedTokens = 128;     // rows of the result a tile, at most
constexpr int kConverterGroups = 2, kGroupWarps = 4, kConverterWarps = kConverterGroups * kGroupWarps;
constexpr int kFusedThreads = 32 * (kConverterWarps + 3);   // converters (four of them read the result), copies of either operand, tensor cores
constexpr int kFusedBytesA = kFusedCols * 128;              // of a stage: 64 codes of 128 columns as 16-bit floats
constexpr int kFusedMemory = 110 << 10;                     // stages, then codes as they are, ahead of the converters
constexpr int kFusedMostStages = 3, kFusedMostRaw = 13;
constexpr int kFusedPartPitch = kFusedCols + 4;             // floats of a token's partial sums
constexpr int kFusedSmem = 1024 + kFusedMemory + 8 * (4 * kFusedMostStages + 4 * kFusedMostRaw + 1);
constexpr int kFusedMostRanks = 8;    // thread blocks of a cluster, which share a tile's contraction
static_assert(4 * (kFusedTokens + kFusedMostRanks - 1) * kFusedPartPitch <= kFusedMemory, "all ranks' sums of a share of the tokens take the stages' place");
static_assert(2 * (kFusedSmem + 128 + 1024) <= 228 << 10, "two blocks a multiprocessor");
static_assert(3 * kFusedSmem > 228 << 10 && 2 * kFusedTokens <= 512, "and no more, so that the tensor memory they ask for is always there");
static_assert(2 * (kFusedBytesA + 128 * kFusedTokens) + 2 * (8 << 10) <= kFusedMemory, "two stages and two of codes fit always");

// One 16-byte piece of a coded row: 32 int4 codes or 16 8-bit codes.  Neighbouring converter lanes take the pieces of a row's 64
// codes, then the next rows': eight lanes hold all chunks j of 2 or 4 rows, whose 16-byte stores, permuted by the row, cover
// all banks.
template <int kMode, int kKind>
struct Pieces {
    static constexpr int kPerRow = kKind == kInt4 ? 2 : 4;                       // pieces of a panel row
    static constexpr int kChunks = kKind == kInt4 ? 4 : 2;                       // 16-byte chunks of 16-bit floats a piece becomes
    static constexpr int kCount = kFusedCols * kPerRow / (32 * kGroupWarps); // of a converter thread and stage
    static constexpr int kRawBytes = kFusedCols * kPerRow * 16;                  // of a stage

    int row, panel, sub;
    // forward: one panel of 128 rows (columns of the result) by 64 codes of the contraction; gradient: two panels of 64 rows (of the
    // contraction) by 64 columns
    __device__ __forceinline__ explicit Pieces(int i)
    {
        const int piece = static_cast<int>(threadIdx.x) % (32 * kGroupWarps) + i * 32 * kGroupWarps, r = piece / kPerRow;
        sub = piece % kPerRow;
        row = kMode == kForward ? r : r & 63;
        panel = kMode == kForward ? 0 : r >> 6;
    }
};

template <int kMode, int kKind>
__device__ __forceinline__ uint4 read_codes(uint32_t raw, const Pieces<kMode, kKind> &at)
{
    const uint32_t from = raw + ((kMode == kForward ? at.row : 2 * at.row + at.panel) * at.kPerRow + at.sub) * 16;
    uint4 c;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(c.x), "=r"(c.y), "=r"(c.z), "=r"(c.w) : "r"(from) : "memory");
    return c;
}

template <int kMode, int kKind, bool kHalf>
__device__ __forceinline__ void store_codes(uint32_t stage, const Pieces<kMode, kKind> &at, const uint4 &c, const Int4To16<kHalf> &int4)
{
    const uint32_t w[4] = {c.x, c.y, c.z, c.w}, to = stage + at.panel * 8192 + at.row * 128;
#pragma unroll
    for (int j = 0; j < at.kChunks; ++j) {
        uint32_t o[4];
        if constexpr (kKind == kInt4) {
            int4(w[j], o);
        } else {
            int8_to_16<kHalf>(w[2 * j], o);
            int8_to_16<kHalf>(w[2 * j + 1], o + 2);
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (((at.sub * at.kChunks + j) ^ (at.row & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                     "r"(o[2]), "r"(o[3]) : "memory");
    }
}

// Step k of a ring of n places: place k mod n, barriers k mod 2n.  Two barriers a place, since the steps of a place fall to both
// groups of converters when n is odd, and a waiter must not be more than one phase ahead of its barrier: with two, the next
// phase of the barrier that step k waits for (of step k - n) is that of step k + n, which cannot be before step k.
struct Turn {
    int n, bar;
    uint32_t parity = 0;   // of the barriers' phase for this step
    __device__ __forceinline__ Turn(int places, int k) : n(places), bar(k) {}   // k < 2n
    __device__ __forceinline__ int place() const { return bar >= n ? bar - n : bar; }
    __device__ __forceinline__ int before() const { return bar >= n ? bar - n : bar + n; }
    __device__ __forceinline__ uint32_t before_parity() const { return bar >= n ? parity : parity ^ 1; }
    __device__ __forceinline__ void next(int by)
    {
        bar += by;
        if (bar >= 2 * n) { bar -= 2 * n; parity ^= 1; }
    }
};

// A cluster of `ranks` thread blocks a tile of 128 columns and up to 128 tokens; each takes a share of the contraction, and
// two blocks share a multiprocessor.  The codes are the matrix instructions' first operand, whose 128 rows they always fill, so
// that a step of the contraction (64) does as much as it can: the issuing warp's chain of one wait, four matrix instructions and one
// commit is among the longest (0.2 us; with the tokens as first operand and 64 columns a tile 0.33 us for half the codes).  16
// tokens int4 4096 -> 11008 14.5 us, 11008 -> 32768 70 us (2.6 TB/s at 58 % issue), 64 tokens 4096 -> 4096 12.5, 256 tokens 17.  TMA
// brings the codes as they are ahead, two groups of converter warps turn the stages into 16-bit floats in turn.  Codes loaded by the converters
// themselves cost more: the fence between their stores and the tensor cores' reads waits for a warp's loads in flight, too (so rows
// that start anywhere are copied first).  The ranks' sums meet in shared memory, added in the order of the ranks, and each rank
// finishes a share of the tokens.
template <int kMode, int kKind, bool kHalf>
__global__ void __launch_bounds__(kFusedThreads, 2)
fused_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap code_map, const __grid_constant__ GemmArgs p)
{
    using P = Pieces<kMode, kKind>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    // three stages where that leaves room for two of codes, else two (8-bit codes, more than 64 tokens)
    const int bytes_b = p.box_rows * 128, stages = kFusedMemory - 3 * (kFusedBytesA + bytes_b) >= 2 * P::kRawBytes ? 3 : 2;
    const uint32_t smem_a = base, smem_b = base + stages * kFusedBytesA, smem_c = smem_b + stages * bytes_b;
    const int raws = min(kFusedMostRaw, (kFusedMemory - stages * (kFusedBytesA + bytes_b)) / P::kRawBytes);   // at least two
    const uint32_t bars = base + kFusedMemory;
    SQ_LINEAR_CHECK(stages >= 2 && raws >= 2 && smem_c + raws * P::kRawBytes <= bars && p.box_rows <= kFusedTokens && p.box_rows % 16 == 0, 1030);
    SQ_LINEAR_CHECK(bars + 8 * (4 * kFusedMostStages + 4 * kFusedMostRaw + 1) <= smem_end(smem_raw), 1031);
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (2 * kFusedMostStages + s); };
    auto raw_full = [&](int s) { return bars + 8 * (4 * kFusedMostStages + s); };
    auto raw_empty = [&](int s) { return bars + 8 * (4 * kFusedMostStages + 2 * kFusedMostRaw + s); };
    const uint32_t done = bars + 8 * (4 * kFusedMostStages + 4 * kFusedMostRaw);
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up_word;
    volatile int *gave_up = &gave_up_word;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank(), ranks = cluster_ranks();
    const int64_t tile = blockIdx.x / ranks;
    const int64_t row0 = tile % p.row_tiles * kFusedTokens;
    const int col0 = static_cast<int>(tile / p.row_tiles) * kFusedCols;
    const int all = (p.depth + kTileDepth - 1) / kTileDepth;
    const int first = static_cast<int>(static_cast<int64_t>(all) * rank / ranks);
    const int steps = static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / ranks) - first;   // at least one
    const int here = static_cast<int>(min(static_cast<int64_t>(kFusedTokens), p.rows - row0));
    SQ_LINEAR_CHECK(ranks >= 1 && ranks <= kFusedMostRanks && tile < p.tiles && here > 0 && here <= p.box_rows && col0 < p.cols, 1032);
    SQ_LINEAR_CHECK(steps >= 1 && static_cast<int64_t>(steps) * kTileDepth <= kLongestSum && first + steps <= all, 1033);

    if (threadIdx.x == 0) {
        gave_up_word = 0;
        for (int s = 0; s < 2 * stages; ++s) {
            bar_init(full(s), 1 + kGroupWarps);
            bar_init(empty(s), 1);
        }
        for (int s = 0; s < 2 * raws; ++s) {
            bar_init(raw_full(s), 1);
            bar_init(raw_empty(s), kGroupWarps);
        }
        bar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kConverterWarps + 1) tmem_alloc(smem_addr(&tmem_base), kFusedTokens);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;

    if (warp < kConverterWarps) {
        const Int4To16<kHalf> int4;
        Turn stage(stages, warp / kGroupWarps), raw(raws, warp / kGroupWarps);
        for (int k = warp / kGroupWarps; k < steps; k += kConverterGroups) {
            uint4 codes[P::kCount];
            if (!bar_wait_warp(raw_full(raw.bar), raw.parity, gave_up)) break;
#pragma unroll
            for (int i = 0; i < P::kCount; ++i) codes[i] = read_codes<kMode, kKind>(smem_c + raw.place() * P::kRawBytes, P(i));
            if (k >= stages && !bar_wait_warp(empty(stage.before()), stage.before_parity(), gave_up)) break;
            SQ_LINEAR_CHECK(raw.place() == k % raws && raw.bar == k % (2 * raws) && stage.place() == k % stages && stage.bar == k % (2 * stages), 1034);
#pragma unroll
            for (int i = 0; i < P::kCount; ++i) SQ_LINEAR_CHECK(P(i).row * 128 + P(i).panel * 8192 + 128 <= kFusedBytesA, 1035);
#pragma unroll
            for (int i = 0; i < P::kCount; ++i) store_codes<kMode, kKind, kHalf>(smem_a + stage.place() * kFusedBytesA, P(i), codes[i], int4);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(full(stage.bar));
            stage.next(kConverterGroups);
            if (lane == 0) bar_arrive(raw_empty(raw.bar));   // not before: the codes have been read for certain once their floats are stored
            raw.next(kConverterGroups);
        }
        if (bar_wait_warp(done, 0, gave_up)) {
            tc_fence_after();
            const int quarter = warp & 3;
            const uint32_t part = base + 4 * (quarter * 32 + lane);
            for (int t = warp / 4 * 32; t < here; t += 64) {
                SQ_LINEAR_CHECK(t + 32 <= kFusedTokens && part + (min(t + 31, here - 1) * kFusedPartPitch + 1) * 4 <= base + kFusedMemory, 1036);
                uint32_t acc[32];
                tmem_ld32(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + t, acc);
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (t + i < here) asm volatile("st.shared.b32 [%0], %1;" ::"r"(part + (t + i) * (4 * kFusedPartPitch)), "r"(acc[i]) : "memory");
            }
            tc_fence_before();
        }
    } else if (warp == kConverterWarps) {
        Turn stage(stages, 0);
        int k = 0;
        for (; k < steps; ++k) {
            if (k >= stages && !bar_wait_warp(empty(stage.before()), stage.before_parity(), gave_up)) break;
            if (elect_one()) {
                bar_expect(full(stage.bar), bytes_b);
                tma_2d(smem_b + stage.place() * bytes_b, &map, (first + k) * kTileDepth, static_cast<int>(row0), full(stage.bar));
            }
            __syncwarp();
            stage.next(1);
        }
        // the last copies have landed before the block may end
        for (int i = max(0, k - stages); i < k; ++i) bar_drain(full(i % (2 * stages)), i / (2 * stages) & 1);
    } else if (warp == kConverterWarps + 2) {
        constexpr int along = kKind == kInt4 ? kTileDepth / 2 : kTileDepth;   // bytes of 64 codes
        Turn raw(raws, 0);
        int k = 0;
        for (; k < steps; ++k) {
            if (k >= raws && !bar_wait_warp(raw_empty(raw.before()), raw.before_parity(), gave_up)) break;
            if (elect_one()) {
                const uint32_t to = smem_c + raw.place() * P::kRawBytes;
                bar_expect(raw_full(raw.bar), P::kRawBytes);
                if (kMode == kForward) tma_2d(to, &code_map, (first + k) * along, col0, raw_full(raw.bar));
                else tma_2d(to, &code_map, col0 / 64 * along, (first + k) * kTileDepth, raw_full(raw.bar));
            }
            __syncwarp();
            raw.next(1);
        }
        for (int i = max(0, k - raws); i < k; ++i) bar_drain(raw_full(i % (2 * raws)), i / (2 * raws) & 1);
    } else {
        const uint32_t idesc = (1u << 4) | (kHalf ? 0u : 1u << 7) | (kHalf ? 0u : 1u << 10) | (kMode != kForward ? 1u << 15 : 0u) |
                               (static_cast<uint32_t>(p.box_rows >> 3) << 17) | (static_cast<uint32_t>(kFusedCols >> 4) << 24);
        constexpr uint32_t kStepA = kMode == kForward ? 32 : 2048;
        Turn stage(stages, 0);
        int k = 0;
        for (; k < steps; ++k) {
            if (!bar_wait_warp(full(stage.bar), stage.parity, gave_up)) break;
            tc_fence_after();
            const uint32_t at = desc_low(smem_a + stage.place() * kFusedBytesA, kMode == kForward ? 16 : 8192);
            const uint32_t bt = desc_low(smem_b + stage.place() * bytes_b, 16);
            if (elect_one()) {
#pragma unroll
                for (int i = 0; i < kTileDepth / 16; ++i) mma_f16(tmem, at + i * (kStepA >> 4), bt + i * 2, idesc, k > 0 || i > 0);
                mma_commit(k + 1 == steps ? done : empty(stage.bar));
            }
            __syncwarp();
            stage.next(1);
        }
        // the tensor cores have read their last stage before the block may end
        if (k == steps) bar_drain(done, 0);
        else if (k > 0) bar_drain(empty((k - 1) % (2 * stages)), (k - 1) / (2 * stages) & 1);
    }
    __syncwarp();
    const int col = col0 + 4 * lane;   // a warp finishes tokens, a lane four channels of each
    float scale[4] = {}, bias[4] = {};
    if (kMode == kForward && warp < kConverterWarps) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < p.cols) {
                scale[i] = get(p.scales + col + i);
                if (p.bias) bias[i] = get(p.bias + col + i);
            }
    }
    const int share = (here + static_cast<int>(ranks) - 1) / static_cast<int>(ranks);   // of the tokens a rank finishes
    cluster_arrive_wait();   // all ranks' sums are in shared memory
    if (warp < kConverterWarps && !*gave_up) {   // a warp a token
        const int end = min(here, (static_cast<int>(rank) + 1) * share);
        for (int r = static_cast<int>(rank) * share + warp; r < end; r += kConverterWarps) {
            const uint32_t mine = base + 4 * (r * kFusedPartPitch + 4 * lane);
            SQ_LINEAR_CHECK(mine + 16 <= base + kFusedMemory, 1037);
            float v[4] = {}, part[kFusedMostRanks][4];
#pragma unroll
            for (uint32_t q = 0; q < kFusedMostRanks; ++q)
                if (q < ranks)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(part[q][0]), "=f"(part[q][1]), "=f"(part[q][2]), "=f"(part[q][3])
                                 : "r"(cluster_addr(mine, q)));
#pragma unroll
            for (uint32_t q = 0; q < kFusedMostRanks; ++q)
                if (q < ranks)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += part[q][i];
            finish4<kMode, kHalf>(p, row0 + r, col, scale, bias, v);
        }
    }
    __syncwarp();
    cluster_arrive_wait();   // the others' sums stay until they have been read
    if (warp == kConverterWarps + 1) {
        tc_fence_after();
        tmem_free(tmem, kFusedTokens);
    }
}

}  // namespace sq
