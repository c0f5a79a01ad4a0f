// Matrix products of the linear operators on the tensor cores (tcgen05): one operand is a 16-bit matrix that TMA
// brings into shared memory, the other one holds 8- or 4-bit codes that converter warps turn into 16-bit floats.
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
    int32_t vector;          // every row starts and ends on 16 bytes
    int32_t rows, cols;      // of the result
    int32_t depth;           // of the contraction
    int32_t row_tiles;
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

constexpr int kTileRows = 128;        // rows of a tile: the tensor memory's lanes
constexpr int kTileDepth = 64;        // of the contraction per stage: 128 bytes
constexpr int kConverterWarps = 8;
constexpr int kGemmThreads = 32 * (4 + kConverterWarps + 2);   // epilogue, converters, TMA, tensor cores

template <int kCols>
struct GemmShape {
    static constexpr int kBytesA = kTileRows * 128;
    static constexpr int kBytesB = kCols * 128;
    static constexpr int kStages = kCols == 256 ? 4 : kCols == 128 ? 6 : 8;
    static constexpr int kTmemCols = 2 * kCols;   // two accumulators: a tile's epilogue runs beside the next one's products
    static constexpr int kBars = 3 * kStages + 4;
    static constexpr int kSmem = 1024 + kStages * (kBytesA + kBytesB) + 8 * kBars + 16;
};

// One 16-byte piece of a coded row: 32 int4 codes or 16 8-bit codes.
template <int kKind>
struct Pieces {
    static constexpr int kPerRow = kKind == kInt4 ? 2 : 4;                        // pieces of a panel row (64 codes)
    static constexpr int kChunks = kKind == kInt4 ? 4 : 2;                        // 16-byte chunks of 16-bit floats a piece becomes
    static constexpr int kAhead = kKind == kInt4 ? 4 : 3;                         // stages whose codes a converter holds in registers
};

// Eight consecutive lanes take eight consecutive panel rows, so that their 16-byte stores, permuted by the row, cover
// all banks.
template <int kKind>
__device__ __forceinline__ void piece_place(int piece, int &row, int &sub)
{
    constexpr int rows = 32 / Pieces<kKind>::kPerRow;
    const int lane = piece & 31;
    row = (piece >> 5) * rows + lane % rows;
    sub = lane / rows;
}

// Where a converter thread reads: its pieces of a stage lie `rows` panel rows apart, which is as many rows of the
// operand (forward) or as many codes along a row (gradients).
template <int kMode, int kKind>
struct CodeCursor {
    static constexpr int kApart = 32 * kConverterWarps / Pieces<kKind>::kPerRow;   // panel rows between a thread's pieces
    const uint8_t *ptr;
    int row;   // of the operand
    int off;   // byte within the row

    __device__ __forceinline__ void start(const GemmArgs &p, int tid, int col0)
    {
        int r, sub;
        piece_place<kKind>(tid, r, sub);
        int first = sub * (kKind == kInt4 ? 32 : 16);
        if (kMode == kForward) {
            row = col0 + r;
        } else {
            row = r & 63;
            first += col0 + (r & ~63);
        }
        off = kKind == kInt4 ? first >> 1 : first;
        ptr = p.codes + static_cast<int64_t>(row) * p.code_pitch + off;
    }
    __device__ __forceinline__ void load(const GemmArgs &p, int i, uint4 &codes) const
    {
        const int r = kMode == kForward ? row + i * kApart : row;
        const int along = kMode == kForward ? 0 : i * (kKind == kInt4 ? kApart / 2 : kApart);
        codes = make_uint4(0, 0, 0, 0);
        if (r < p.code_rows && off + along < p.code_row_bytes) {
            const uint8_t *q = ptr + (kMode == kForward ? static_cast<int64_t>(i * kApart) * p.code_pitch : along);
            codes = p.vector ? ldg128(q) : load_bytes16(q, p.codes, p.codes + p.code_bytes);
        }
    }
    __device__ __forceinline__ void next(const GemmArgs &p)
    {
        if (kMode == kForward) {
            off += kKind == kInt4 ? kTileDepth / 2 : kTileDepth;
            ptr += kKind == kInt4 ? kTileDepth / 2 : kTileDepth;
        } else {
            row += kTileDepth;
            ptr += kTileDepth * p.code_pitch;
        }
    }
};

template <int kKind, bool kHalf>
__device__ __forceinline__ void store_piece(uint32_t panel, int piece, const uint4 &c)
{
    int row, sub;
    piece_place<kKind>(piece, row, sub);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    const uint32_t base = panel + row * 128;
#pragma unroll
    for (int j = 0; j < Pieces<kKind>::kChunks; ++j) {
        uint32_t o[4];
        if constexpr (kKind == kInt4) {
            int4_to_16<kHalf>(w[j], o);
        } else {
            int8_to_16<kHalf>(w[2 * j], o);
            int8_to_16<kHalf>(w[2 * j + 1], o + 2);
        }
        const uint32_t chunk = sub * Pieces<kKind>::kChunks + j;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(base + ((chunk ^ (row & 7)) << 4)), "r"(o[0]), "r"(o[1]),
                     "r"(o[2]), "r"(o[3]) : "memory");
    }
}

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
                const float4 s = __ldg(reinterpret_cast<const float4 *>(p.scales + col) + j);
                const float4 b = p.bias ? __ldg(reinterpret_cast<const float4 *>(p.bias + col) + j) : make_float4(0, 0, 0, 0);
                v[4 * j] = fmaf(v[4 * j], s.x, b.x);
                v[4 * j + 1] = fmaf(v[4 * j + 1], s.y, b.y);
                v[4 * j + 2] = fmaf(v[4 * j + 2], s.z, b.z);
                v[4 * j + 3] = fmaf(v[4 * j + 3], s.w, b.w);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int c = i < n ? col + i : col;
                v[i] = fmaf(v[i], __ldg(p.scales + c), p.bias ? __ldg(p.bias + c) : 0.0f);
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
                    const uint4 q = __ldg(reinterpret_cast<const uint4 *>(r) + j);
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
                    if (i < n) v[i] += to_float<kHalf>(__ldg(r + i));
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (8 * j < n) store8<kHalf>(out + 8 * j, v + 8 * j, n - 8 * j, p.out_vector);
}

// One persistent thread block a multiprocessor.  Roles: warps 0-3 epilogue (a warp reads the tensor memory's lanes of
// its own quarter), 4-11 converters, 12 copies the 16-bit operand by TMA, 13 issues the matrix instructions.  Stages of
// 64 of the contraction go round; "full" of a stage has two parts, the copy's and the converters'.
template <int kMode, int kKind, bool kHalf, int kCols>
__global__ void __launch_bounds__(kGemmThreads, 1) gemm_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ GemmArgs p)
{
    using S = GemmShape<kCols>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t smem_a = base, smem_b = base + S::kStages * S::kBytesA;
    const uint32_t bars = smem_b + S::kStages * S::kBytesB;
    auto full_a = [&](int s) { return bars + 8 * s; };
    auto full_b = [&](int s) { return bars + 8 * (S::kStages + s); };
    auto empty = [&](int s) { return bars + 8 * (2 * S::kStages + s); };
    auto acc_full = [&](int a) { return bars + 8 * (3 * S::kStages + a); };
    auto acc_empty = [&](int a) { return bars + 8 * (3 * S::kStages + 2 + a); };
    __shared__ uint32_t tmem_base;
    __shared__ int gave_up_word;
    volatile int *gave_up = &gave_up_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        gave_up_word = 0;
        for (int s = 0; s < S::kStages; ++s) {
            bar_init(full_a(s), 1);
            bar_init(full_b(s), kConverterWarps);
            bar_init(empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            bar_init(acc_full(a), 1);
            bar_init(acc_empty(a), 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 13) tmem_alloc(smem_addr(&tmem_base), S::kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    const int steps = (p.depth + kTileDepth - 1) / kTileDepth;

    if (warp < 4) {
        int n = 0;
        for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x, ++n) {
            const int a = n & 1;
            if (!bar_wait_warp(acc_full(a), (n >> 1) & 1, gave_up)) break;
            tc_fence_after();
            const int64_t row = (t % p.row_tiles) * kTileRows + warp * 32 + lane;
            const int col0 = static_cast<int>(t / p.row_tiles) * kCols;
            for (int c = 0; c < kCols; c += 32) {
                if (col0 + c >= p.cols) break;
                uint32_t acc[32];
                __syncwarp();
                tmem_ld32(tmem + (static_cast<uint32_t>(warp * 32) << 16) + a * kCols + c, acc);
                if (row < p.rows) finish32<kMode, kHalf>(p, row, col0 + c, acc);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(acc_empty(a));
        }
    } else if (warp < 4 + kConverterWarps) {
        constexpr int kThreads = 32 * kConverterWarps;
        constexpr int kPieces = kCols * Pieces<kKind>::kPerRow;           // of a stage
        constexpr int kMine = (kPieces + kThreads - 1) / kThreads;
        constexpr int kAhead = Pieces<kKind>::kAhead;
        const int tid = threadIdx.x - 128;
        uint4 codes[kAhead][kMine];
        CodeCursor<kMode, kKind> cursor;
        int64_t load_tile = blockIdx.x;
        int load_step = 0;
        auto load = [&](uint4 (&c)[kMine]) {
            if (load_tile >= p.tiles) return;
            if (load_step == 0) cursor.start(p, tid, static_cast<int>(load_tile / p.row_tiles) * kCols);
#pragma unroll
            for (int i = 0; i < kMine; ++i)
                if (kPieces % kThreads == 0 || tid < kPieces) cursor.load(p, i, c[i]);
            cursor.next(p);
            if (++load_step == steps) { load_step = 0; load_tile += gridDim.x; }
        };
#pragma unroll
        for (int d = 0; d < kAhead; ++d) load(codes[d]);
        const int64_t my_tiles = blockIdx.x < p.tiles ? (p.tiles - 1 - blockIdx.x) / gridDim.x + 1 : 0;
        const int64_t total = my_tiles * steps;
        bool ok = true;
        int s = 0;
        uint32_t parity = 1;   // a stage that was never used counts as empty
        for (int64_t it = 0; it < total && ok; it += kAhead) {
#pragma unroll
            for (int d = 0; d < kAhead; ++d) {
                if (it + d < total && ok) {
                    ok = bar_wait_warp(empty(s), parity, gave_up);
                    if (ok) {
#pragma unroll
                        for (int i = 0; i < kMine; ++i)
                            if (kPieces % kThreads == 0 || tid < kPieces)
                                store_piece<kKind, kHalf>(smem_b + s * S::kBytesB, tid + i * kThreads, codes[d][i]);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) bar_arrive(full_b(s));
                        load(codes[d]);
                        if (++s == S::kStages) { s = 0; parity ^= 1; }
                    }
                }
            }
        }
    } else if (warp == 4 + kConverterWarps) {
        if (lane == 0) {
            bool ok = true;
            int s = 0, issued = 0;
            uint32_t parity = 1;
            for (int64_t t = blockIdx.x; t < p.tiles && ok; t += gridDim.x) {
                const int row0 = static_cast<int>(t % p.row_tiles) * kTileRows;
                for (int k = 0; k < steps; ++k) {
                    ok = bar_wait(empty(s), parity, gave_up);
                    if (!ok) break;
                    bar_expect(full_a(s), S::kBytesA);
                    const uint32_t dst = smem_a + s * S::kBytesA;
                    tma_2d(dst, &map, k * kTileDepth, row0, full_a(s));
                    if (issued < S::kStages) ++issued;
                    if (++s == S::kStages) { s = 0; parity ^= 1; }
                }
            }
            // the last copies have landed before the block may end
            for (int i = 0; i < issued; ++i) {
                if (--s < 0) { s = S::kStages - 1; parity ^= 1; }
                bar_drain(full_a(s), parity ^ 1);
            }
        }
    } else if (lane == 0) {
        constexpr uint32_t kIdesc = (1u << 4) | (kHalf ? 0u : 1u << 7) | (kHalf ? 0u : 1u << 10) |
                                    (kMode != kForward ? 1u << 16 : 0u) |
                                    (static_cast<uint32_t>(kCols >> 3) << 17) | (static_cast<uint32_t>(kTileRows >> 4) << 24);
        constexpr uint32_t kStepA = 32, kStepB = kMode == kForward ? 32 : 2048;
        bool ok = true;
        int s = 0, n = 0;
        uint32_t parity = 0;
        int last_s = -1;
        for (int64_t t = blockIdx.x; t < p.tiles && ok; t += gridDim.x, ++n) {
            const int a = n & 1;
            ok = bar_wait(acc_empty(a), ((n >> 1) & 1) ^ 1, gave_up);
            if (!ok) break;
            tc_fence_after();
            for (int k = 0; k < steps; ++k) {
                ok = bar_wait(full_a(s), parity, gave_up) && bar_wait(full_b(s), parity, gave_up);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = smem_a + s * S::kBytesA, bt = smem_b + s * S::kBytesB;
#pragma unroll
                for (int i = 0; i < kTileDepth / 16; ++i)
                    mma_f16(tmem + a * kCols, smem_desc(at + i * kStepA, 16),
                            smem_desc(bt + i * kStepB, kMode == kForward ? 16 : 8192), kIdesc, k > 0 || i > 0);
                mma_commit(empty(s));
                last_s = s;
                if (++s == S::kStages) { s = 0; parity ^= 1; }
            }
            if (ok) mma_commit(acc_full(a));
        }
        // the tensor cores have read their last stage before the block may end: a stage's phase is complete when its
        // parity is the one this warp waited with
        if (last_s >= 0) bar_drain(empty(last_s), s == 0 ? parity ^ 1 : parity);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 13) {
        tc_fence_after();
        tmem_free(tmem, S::kTmemCols);
    }
}

}  // namespace sq
