// Matrix products of the linear operators on the tensor cores (tcgen05), and the epilogue they share.  Here: up to 128
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
    int64_t code_bytes;      // of the whole operand
    int32_t code_rows;       // rows of the coded operand
    int32_t code_row_bytes;  // bytes of a row that may be read
    int32_t rows, cols;      // of the result
    int32_t depth;           // of the contraction
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

// Up to eight 16-bit values of one row from fp32, as one 16-byte store where it is possible.
template <bool kHalf>
__device__ __forceinline__ void store8(uint16_t *out, const float *v, int n, bool vector)
{
    if (vector && n >= 8) {
        *reinterpret_cast<uint4 *>(out) = make_uint4(to_16x2<kHalf>(v[0], v[1]), to_16x2<kHalf>(v[2], v[3]),
                                                     to_16x2<kHalf>(v[4], v[5]), to_16x2<kHalf>(v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) out[i] = to_16<kHalf>(v[i]);
    }
}

// 32 columns of one row of the result.  A thread of the epilogue owns a row, so the 32 channels that share a
// checkpoint's exponent are all its own.
template <int kMode, bool kHalf>
__device__ __forceinline__ void finish32(const GemmArgs &p, int64_t row, int col, const uint32_t (&acc)[32])
{
    const int n = min(32, p.cols - col);
    uint16_t *out = p.out + row * p.out_stride + col;
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(acc[i]);
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
            for (int i = 0; i < 32; ++i) {
                const int c = i < n ? col + i : col;
                v[i] = fmaf(v[i], get(p.scales + c), p.bias ? get(p.bias + c) : 0.0f);
            }
        }
        if (p.z_codes) {
            float a = 0.0f;
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < n) a = max_nan(a, fabsf(v[i]));
            const uint32_t e = ckpt_exponent(a);
            const float inverse = ckpt_inverse(e);
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (4 * i + b < n) w[i] |= static_cast<uint32_t>(ckpt_code(v[4 * i + b], inverse) & 255) << (8 * b);
            }
            uint4 *zc = reinterpret_cast<uint4 *>(p.z_codes + row * p.z_pitch + col);
            zc[0] = make_uint4(w[0], w[1], w[2], w[3]);
            zc[1] = make_uint4(w[4], w[5], w[6], w[7]);
            p.z_exps[row * p.z_exps_pitch + (col >> 5)] = static_cast<uint8_t>(e);
        }
        if (p.act == kActRelu) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = act_value(v[i], kActRelu);
        } else if (p.act == kActGelu) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = act_value(v[i], kActGelu);
        } else if (p.act == kActSilu) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = act_value(v[i], kActSilu);
        }
        if (p.residual) {
            const uint16_t *r = p.residual + row * p.residual_stride + col;
            if (p.residual_vector && n == 32) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint4 q = get(reinterpret_cast<const uint4 *>(r) + j);
                    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[8 * j + 2 * i] += to_float<kHalf>(static_cast<uint16_t>(w[i]));
                        v[8 * j + 2 * i + 1] += to_float<kHalf>(static_cast<uint16_t>(w[i] >> 16));
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i < n) v[i] += to_float<kHalf>(get(r + i));
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (8 * j < n) store8<kHalf>(out + 8 * j, v + 8 * j, n - 8 * j, p.out_vector);
}

// The same for four columns a thread: eight neighbouring lanes hold the 32 channels of an exponent.  All lanes of a warp call
// it; `valid`: this lane's row is there.
template <int kMode, bool kHalf>
__device__ __forceinline__ void finish4(const GemmArgs &p, int64_t row, int col, float (&v)[4], bool valid)
{
    const int n = valid ? p.cols - col : 0;   // columns of this thread, if below four
    if constexpr (kMode == kForward) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = i < n ? fmaf(v[i], get(p.scales + col + i), p.bias ? get(p.bias + col + i) : 0.0f) : 0.0f;
        if (p.z_codes) {
            float a = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) a = max_nan(a, fabsf(v[i]));
#pragma unroll
            for (int s = 1; s <= 4; s <<= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, s));
            const uint32_t e = ckpt_exponent(a);
            const float inverse = ckpt_inverse(e);
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) w |= static_cast<uint32_t>(ckpt_code(v[i], inverse) & 255) << (8 * i);
            if (valid && (col & ~31) < p.cols) {   // rows end on 32
                *reinterpret_cast<uint32_t *>(p.z_codes + row * p.z_pitch + col) = w;
                if ((col & 31) == 0) p.z_exps[row * p.z_exps_pitch + (col >> 5)] = static_cast<uint8_t>(e);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = act_value(v[i], p.act);
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

constexpr int kFusedRows = 128;       // rows of a tile: the tensor memory's lanes
constexpr int kFusedCols = 64;
constexpr int kConverterGroups = 2, kGroupWarps = 4, kConverterWarps = kConverterGroups * kGroupWarps;
constexpr int kFusedThreads = 32 * (kConverterWarps + 3);   // converters (four of them read the result), copies of either operand, tensor cores
constexpr int kFusedBytesB = kFusedCols * 128;
constexpr int kFusedStageBytes = 96 << 10;                  // 4 stages of 128 rows, 6 of up to 64, 8 of up to 32
constexpr int kFusedMostStages = 8;
constexpr int kFusedRawBytes = 12 << 10;                    // codes as they are, ahead of the converters
constexpr int kFusedRawBars = 6;                           // even and a multiple of the stages of codes: one group waits for each
constexpr int kFusedPartPitch = kFusedCols + 4;             // floats of a row of partial sums: 16-byte accesses hit all banks
constexpr int kFusedSmem = 1024 + kFusedStageBytes + kFusedRawBytes + 8 * (2 * kFusedMostStages + 2 * kFusedRawBars + 1);
constexpr int kFusedMostRanks = 8;    // thread blocks of a cluster, which share a tile's contraction
static_assert(4 * kFusedRows * kFusedPartPitch <= kFusedStageBytes, "partial sums take the stages' place");
// Even: a stage belongs to one group of converters (a waiter must not be more than one phase ahead of its barrier).
__host__ __device__ constexpr int fused_stages(int box_rows) { return box_rows > 64 ? 4 : box_rows > 32 ? 6 : 8; }
static_assert(4 * (128 * 128 + kFusedBytesB) <= kFusedStageBytes && 6 * (64 * 128 + kFusedBytesB) <= kFusedStageBytes &&
              8 * (32 * 128 + kFusedBytesB) <= kFusedStageBytes && 4 * kFusedBytesB >= 128 * 128,
              "the stages fit, and 128 rows from any stage of the 16-bit operand on are inside them");

// One 16-byte piece of a coded row: 32 int4 codes or 16 8-bit codes.  A converter warp takes 16 of a stage's 64 rows of 64
// codes, neighbouring lanes neighbouring pieces.  Eight lanes then hold all chunks j of 2 or 4 rows whose 16-byte stores, permuted by the
// row, cover all banks.
template <int kKind>
struct Pieces {
    static constexpr int kPerRow = kKind == kInt4 ? 2 : 4;       // pieces of a panel row
    static constexpr int kChunks = kKind == kInt4 ? 4 : 2;       // 16-byte chunks of 16-bit floats a piece becomes
    static constexpr int kRows = 32 / kPerRow;                   // rows of a warp's load
    static constexpr int kCount = 64 / kGroupWarps / kRows;      // loads of a stage
    static constexpr int kRawBytes = kFusedCols * 16 * kPerRow;  // of a stage
    static constexpr int kRaw = kFusedRawBytes / kRawBytes;      // stages of codes ahead
};

// Rows that start anywhere: straight from global memory.
template <int kMode, int kKind>
__device__ __forceinline__ void load_codes(const GemmArgs &p, int col0, int step, int part, uint4 (&c)[Pieces<kKind>::kCount])
{
    using P = Pieces<kKind>;
    const int lane = threadIdx.x & 31;
    // forward: rows are the tile's columns; gradient: rows are the contraction's
    const int row = (kMode == kForward ? col0 : step * kTileDepth) + 64 / kGroupWarps * part + lane / P::kPerRow;
    const int first = (kMode == kForward ? step * kTileDepth : col0) + lane % P::kPerRow * (64 / P::kPerRow);
    const int off = kKind == kInt4 ? first >> 1 : first;
    const uint8_t *q = p.codes + static_cast<int64_t>(row) * p.code_pitch + off;
#pragma unroll
    for (int i = 0; i < P::kCount; ++i) {
        c[i] = make_uint4(0, 0, 0, 0);
        if (row + i * P::kRows < p.code_rows && off < p.code_row_bytes) c[i] = load_bytes16(q, p.codes, p.codes + p.code_bytes);
        q += P::kRows * p.code_pitch;
    }
}

template <int kKind>
__device__ __forceinline__ void read_codes(uint32_t raw, int part, uint4 (&c)[Pieces<kKind>::kCount])
{
    using P = Pieces<kKind>;
    const uint32_t at = raw + part * (P::kRawBytes / kGroupWarps) + (threadIdx.x & 31) * 16;
#pragma unroll
    for (int i = 0; i < P::kCount; ++i)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(c[i].x), "=r"(c[i].y), "=r"(c[i].z), "=r"(c[i].w) : "r"(at + 512 * i) : "memory");
}

template <int kKind, bool kHalf>
__device__ __forceinline__ void store_codes(uint32_t panel, int part, const uint4 (&c)[Pieces<kKind>::kCount])
{
    using P = Pieces<kKind>;
    const int lane = threadIdx.x & 31, sub = lane % P::kPerRow;
#pragma unroll
    for (int i = 0; i < P::kCount; ++i) {
        const int row = 64 / kGroupWarps * part + i * P::kRows + lane / P::kPerRow;
        const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
        for (int j = 0; j < P::kChunks; ++j) {
            uint32_t o[4];
            if constexpr (kKind == kInt4) {
                int4_to_16<kHalf>(w[j], o);
            } else {
                int8_to_16<kHalf>(w[2 * j], o);
                int8_to_16<kHalf>(w[2 * j + 1], o + 2);
            }
            const uint32_t chunk = sub * P::kChunks + j;
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(panel + row * 128 + ((chunk ^ (row & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                         "r"(o[2]), "r"(o[3]) : "memory");
        }
    }
}

// A cluster of `ranks` thread blocks a tile of 128 rows and 64 columns; each takes a share of the contraction.  Reading the
// codes is most of the work, so the tile is narrow and two blocks share a multiprocessor.  TMA brings the codes as they are
// ahead; two groups of converter warps turn those of a stage into 16-bit floats in turn.  The issuing warp's loop of one wait, four
// matrix instructions and one commit is the longest chain: with a barrier for either operand and six converter warps a step of 64
// took 0.45 us.  Codes loaded by the converters themselves, as rows that start anywhere are (kVector false), cost more: the fence
// between their stores and the tensor cores' reads waits for a warp's loads in flight, too.  The ranks' sums meet in shared
// memory, added in the order of the ranks, and each rank finishes a share of the rows.
template <int kMode, int kKind, bool kHalf, bool kVector>
__global__ void __launch_bounds__(kFusedThreads, 2)
fused_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap code_map, const __grid_constant__ GemmArgs p)
{
    using P = Pieces<kKind>;
    static_assert(kFusedRawBars % P::kRaw == 0 && kFusedRawBars % kConverterGroups == 0, "a barrier belongs to one place and one group");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const int bytes_a = p.box_rows * 128, stages = fused_stages(p.box_rows);
    const uint32_t smem_a = base, smem_b = base + stages * bytes_a, smem_c = base + kFusedStageBytes;
    const uint32_t bars = smem_c + kFusedRawBytes;
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (kFusedMostStages + s); };
    auto raw_full = [&](int s) { return bars + 8 * (2 * kFusedMostStages + s); };
    auto raw_empty = [&](int s) { return bars + 8 * (2 * kFusedMostStages + kFusedRawBars + s); };
    const uint32_t done = bars + 8 * (2 * kFusedMostStages + 2 * kFusedRawBars);
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up_word;
    volatile int *gave_up = &gave_up_word;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank(), ranks = cluster_ranks();
    const int64_t tile = blockIdx.x / ranks;
    const int64_t row0 = tile % p.row_tiles * kFusedRows;
    const int col0 = static_cast<int>(tile / p.row_tiles) * kFusedCols;
    const int all = (p.depth + kTileDepth - 1) / kTileDepth;
    const int first = static_cast<int>(static_cast<int64_t>(all) * rank / ranks);
    const int steps = static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / ranks) - first;   // at least one

    if (threadIdx.x == 0) {
        gave_up_word = 0;
        for (int s = 0; s < stages; ++s) {
            bar_init(full(s), 1 + kGroupWarps);
            bar_init(empty(s), 1);
        }
        for (int s = 0; s < kFusedRawBars; ++s) {
            bar_init(raw_full(s), 1);
            bar_init(raw_empty(s), kGroupWarps);
        }
        bar_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kConverterWarps + 1) tmem_alloc(smem_addr(&tmem_base), kFusedCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    next_may_start();   // not before: a block of the next launch must not take the tensor memory that this one is yet to allocate
    wait_for_previous();

    if (warp < kConverterWarps) {
        const int part = warp % kGroupWarps;
        int s = warp / kGroupWarps;
        uint32_t parity = 1;   // a stage that was never used counts as empty
        for (int k = s; k < steps; k += kConverterGroups) {
            uint4 codes[P::kCount];
            if constexpr (kVector) {
                const int b = k % kFusedRawBars;
                if (!bar_wait_warp(raw_full(b), k / kFusedRawBars & 1, gave_up)) break;
                read_codes<kKind>(smem_c + k % P::kRaw * P::kRawBytes, part, codes);
                __syncwarp();
                if (lane == 0) bar_arrive(raw_empty(b));
            } else {
                load_codes<kMode, kKind>(p, col0, first + k, part, codes);
            }
            if (!bar_wait_warp(empty(s), parity, gave_up)) break;
            store_codes<kKind, kHalf>(smem_b + s * kFusedBytesB, part, codes);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) bar_arrive(full(s));
            s += kConverterGroups;
            if (s >= stages) { s -= stages; parity ^= 1; }
        }
        if (warp < 4 && bar_wait_warp(done, 0, gave_up)) {
            tc_fence_after();
            const uint32_t part = base + (warp * 32 + lane) * (4 * kFusedPartPitch);
            if (row0 + warp * 32 < p.rows) {
#pragma unroll
                for (int c = 0; c < kFusedCols; c += 32) {
                    uint32_t acc[32];
                    tmem_ld32(tmem + (static_cast<uint32_t>(warp * 32) << 16) + c, acc);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(part + 4 * c + 16 * i), "r"(acc[4 * i]), "r"(acc[4 * i + 1]),
                                     "r"(acc[4 * i + 2]), "r"(acc[4 * i + 3]) : "memory");
                }
            }
            tc_fence_before();
        }
    } else if (warp == kConverterWarps) {
        bool ok = true;
        int k = 0, s = 0;
        uint32_t parity = 1;
        for (; k < steps; ++k) {
            ok = bar_wait_warp(empty(s), parity, gave_up);
            if (!ok) break;
            if (elect_one()) {
                bar_expect(full(s), bytes_a);   // rows behind the last token stay what they are: only their own sums see them
                tma_2d(smem_a + s * bytes_a, &map, (first + k) * kTileDepth, static_cast<int>(row0), full(s));
            }
            __syncwarp();
            if (++s == stages) { s = 0; parity ^= 1; }
        }
        // the last copies have landed before the block may end
        for (int i = 0; i < min(k, stages); ++i) {
            if (--s < 0) { s = stages - 1; parity ^= 1; }
            bar_drain(full(s), parity ^ 1);
        }
    } else if (warp == kConverterWarps + 2) {
        if constexpr (kVector) {
            constexpr int along = kKind == kInt4 ? kTileDepth / 2 : kTileDepth;   // bytes of 64 codes
            int k = 0;
            for (; k < steps; ++k) {
                const int b = k % kFusedRawBars, before = k - P::kRaw;
                if (before >= 0 && !bar_wait_warp(raw_empty(before % kFusedRawBars), before / kFusedRawBars & 1, gave_up)) break;
                if (elect_one()) {
                    const uint32_t to = smem_c + k % P::kRaw * P::kRawBytes;
                    bar_expect(raw_full(b), P::kRawBytes);
                    if (kMode == kForward) tma_2d(to, &code_map, (first + k) * along, col0, raw_full(b));
                    else tma_2d(to, &code_map, col0 / kTileDepth * along, (first + k) * kTileDepth, raw_full(b));
                }
                __syncwarp();
            }
            for (int i = max(0, k - P::kRaw); i < k; ++i) bar_drain(raw_full(i % kFusedRawBars), i / kFusedRawBars & 1);
        }
    } else {
        constexpr uint32_t kIdesc = (1u << 4) | (kHalf ? 0u : 1u << 7) | (kHalf ? 0u : 1u << 10) | (kMode != kForward ? 1u << 16 : 0u) |
                                    (static_cast<uint32_t>(kFusedCols >> 3) << 17) | (static_cast<uint32_t>(kFusedRows >> 4) << 24);
        constexpr uint32_t kStepB = kMode == kForward ? 32 : 2048;
        int k = 0, s = 0, last = 0;
        uint32_t parity = 0;
        for (; k < steps; ++k) {
            if (!bar_wait_warp(full(s), parity, gave_up)) break;
            tc_fence_after();
            if (elect_one()) {
                const uint32_t at = smem_a + s * bytes_a, bt = smem_b + s * kFusedBytesB;
#pragma unroll
                for (int i = 0; i < kTileDepth / 16; ++i)
                    mma_f16(tmem, smem_desc(at + i * 32, 16), smem_desc(bt + i * kStepB, 16), kIdesc, k > 0 || i > 0);
                mma_commit(k + 1 == steps ? done : empty(s));
            }
            __syncwarp();
            last = s;
            if (++s == stages) { s = 0; parity ^= 1; }
        }
        // the tensor cores have read their last stage before the block may end
        if (k == steps) bar_drain(done, 0);
        else if (k > 0) bar_drain(empty(last), s == 0 ? parity ^ 1 : parity);
    }
    __syncwarp();
    cluster_arrive_wait();   // all ranks' sums are in shared memory
    if (warp < kConverterWarps) {   // sixteen threads a row
        const int here = static_cast<int>(min(static_cast<int64_t>(kFusedRows), p.rows - row0));
        const int share = (here + static_cast<int>(ranks) - 1) / static_cast<int>(ranks);
        const int end = min(here, (static_cast<int>(rank) + 1) * share), c = (threadIdx.x & 15) * 4;
        const bool whole = !*gave_up;
        for (int r = static_cast<int>(rank) * share + (threadIdx.x >> 4); r - (lane >> 4) < end && whole; r += 2 * kConverterWarps) {
            float v[4] = {};
            if (r < end) {
                const uint32_t mine = base + r * (4 * kFusedPartPitch) + 4 * c;
                float part[kFusedMostRanks][4];
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
            }
            finish4<kMode, kHalf>(p, row0 + r, col0 + c, v, r < end);
        }
    }
    __syncwarp();
    cluster_arrive_wait();   // the others' sums stay until they have been read
    if (warp == kConverterWarps + 1) {
        tc_fence_after();
        tmem_free(tmem, kFusedCols);
    }
}

}  // namespace sq
