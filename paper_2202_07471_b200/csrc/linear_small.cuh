// The forward product for few tokens, where reading the codes is all there is to do.
#pragma once

#include "linear_device.cuh"

namespace sq {

struct FewArgs {
    const uint16_t *x;
    int64_t x_stride;
    const uint8_t *codes;
    int64_t code_pitch, code_bytes;
    int32_t tokens, cin, cout;
    const float *scales, *bias;
    const uint16_t *residual;
    int64_t residual_stride;
    uint16_t *y;
    int64_t y_stride;
    int32_t act;
};

template <bool kHalf>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t a0, const uint32_t a1, const uint32_t a2, const uint32_t a3,
                                          const uint32_t b0, const uint32_t b1)
{
    if constexpr (kHalf)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Sixteen 16-bit values of a row from `first` on, zeros at and behind the row's end.  kAlign: bytes that rows start on (32, 16: and whole
// vectors of sixteen or eight) or 0.
template <int kAlign>
__device__ __forceinline__ void load_x16(const uint16_t *row, int first, int cin, uint4 (&v)[2])
{
    v[0] = v[1] = make_uint4(0, 0, 0, 0);
    if constexpr (kAlign == 32) {
        SQ_LINEAR_CHECK(first >= cin || (first + 16 <= cin && (reinterpret_cast<uintptr_t>(row + first) & 31) == 0), 1010);
        if (first < cin)
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(v[0].x), "=r"(v[0].y), "=r"(v[0].z), "=r"(v[0].w), "=r"(v[1].x), "=r"(v[1].y), "=r"(v[1].z), "=r"(v[1].w) : "l"(row + first));
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (kAlign == 16) {
                SQ_LINEAR_CHECK(first + 8 * h >= cin || (first + 8 * h + 8 <= cin && (reinterpret_cast<uintptr_t>(row + first) & 15) == 0), 1011);
                if (first + 8 * h < cin) v[h] = get(reinterpret_cast<const uint4 *>(row + first + 8 * h));
            } else {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = first + 8 * h + 2 * i;
                    w[i] = (k < cin ? static_cast<uint32_t>(get(row + k)) : 0u) | (k + 1 < cin ? static_cast<uint32_t>(get(row + k + 1)) << 16 : 0u);
                }
                v[h] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}

constexpr int kFewWarps = 8;       // share the contraction
constexpr int kFewRows = 16;       // output channels of a thread block
constexpr int kFewTokens = 8;      // of a tile

// Without a checkpoint (its 32 channels would be two thread blocks'): a thread block owns 16 channels, its warps take chunks of the
// contraction in turn and are summed at the end.  In a chunk (four lanes times 16 bytes of codes) lane (g, q) holds 16 bytes of the
// rows g and g + 8 and the same elements of the tokens g, g + 8, ..: the order of the contraction inside a matrix instruction is free as
// long as both operands agree, so nothing is shuffled.  A lane asks for the codes and the elements of x of its chunks at once, and
// nothing waits for another thread before the sum; every block reads all of x, mostly from its multiprocessor's L1.  A lane's elements
// of x are 32 or 64 neighbouring bytes: loads of 32 take whole sectors (loads of 16 use each sector twice: 8 tokens int4 4096 ->
// 11008 11.9 us, now 9.5).  Bound by the issue of instructions (about two a code) and the latency of a batch for one token, by the loads
// of x for many: int4 4096 -> 4096 1 / 8 / 16 / 32 tokens 4.8 / 5.0 / 6.2 / 10.1 us, 8192 -> 16384 one token 20.6 us (3.3 TB/s), codes
// from DRAM.  (128 channels a block, x through shared memory and the contraction shared by a cluster: 6.2 us for one token; 32 channels
// a block: 6.1, 8 tokens 6.6; sixteen tokens with one chunk in flight and three blocks a multiprocessor: 6.7.  mma.sync, since a step
// of 64 takes tcgen05 longer here.)
// kAlign: rows of x as load_x16 says; rows of codes start on 16 bytes unless it is 0.  kTiles: tiles of eight tokens of a thread block (y:
// the next tokens).
template <int kKind, bool kHalf, int kAlign, int kTiles>
__global__ void __launch_bounds__(32 * kFewWarps, kTiles == 1 ? 3 : 2) few_kernel(const __grid_constant__ FewArgs p)
{
    constexpr int kCodes = kKind == kInt4 ? 32 : 16;
    constexpr int kUnits = kCodes / 8;   // 16 bytes of x a lane, chunk and tile
    constexpr int kChunks = kTiles * kUnits <= 8 ? 2 : 1;   // in flight a warp
    constexpr int kSums = kTiles == 1 ? 2 : 1;              // a tile; two, so that matrix instructions do not wait for one another
    constexpr int kMine = kTiles <= 2 ? 1 : kTiles / 2;     // results a thread finishes
    __shared__ float part[kFewWarps][kTiles * kFewTokens][kFewRows];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int token0 = static_cast<int>(blockIdx.y) * (kTiles * kFewTokens), tokens = p.tokens - token0;   // from token0 on
    const uint16_t *const x_from = p.x + token0 * p.x_stride;
    const int row0 = static_cast<int>(blockIdx.x) * kFewRows;
    const int chunks = (p.cin + 4 * kCodes - 1) / (4 * kCodes);
    const int row_bytes = kKind == kInt4 ? (p.cin + 1) >> 1 : p.cin;
    // what the thread finishes: a channel of the tokens first, first + 16, ..
    const int first = threadIdx.x / kFewRows, row = row0 + static_cast<int>(threadIdx.x) % kFewRows;
    float scale = 0.0f, bias = 0.0f, res[kMine] = {};
    if (first < tokens && row < p.cout) {
        scale = get(p.scales + row);
        if (p.bias) bias = get(p.bias + row);
        if (p.residual)
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (first + 16 * j < tokens) res[j] = to_float<kHalf>(p.residual[(token0 + first + 16 * j) * p.residual_stride + row]);
    }
    float acc[kTiles][kSums][4] = {};
    [[maybe_unused]] const Int4To16<kHalf> int4;

    for (int c0 = warp; c0 < chunks; c0 += kFewWarps * kChunks) {
        uint4 codes[kChunks][2], x[kChunks][kUnits / 2][kTiles][2];
#pragma unroll
        for (int u = 0; u < kChunks; ++u) {
            const int piece = (c0 + u * kFewWarps) * 4 + q;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int at = row0 + g + 8 * r;
                codes[u][r] = make_uint4(0, 0, 0, 0);
                if (piece * 16 < row_bytes && at < p.cout) {
                    const uint8_t *from = p.codes + at * p.code_pitch + piece * 16;
                    SQ_LINEAR_CHECK(from >= p.codes && (kAlign ? from + 16 <= p.codes + p.code_bytes && (reinterpret_cast<uintptr_t>(from) & 15) == 0
                                                              : from < p.codes + p.code_bytes), 1012);
                    codes[u][r] = kAlign ? ldg128(from) : load_bytes16(from, p.codes, p.codes + p.code_bytes);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kChunks; ++u) {
            const int k = ((c0 + u * kFewWarps) * 4 + q) * kCodes;
#pragma unroll
            for (int i = 0; i < kUnits / 2; ++i)
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    const int row = g + 8 * t;
                    load_x16<kAlign>(x_from + row * p.x_stride, k + 16 * i, row < tokens ? p.cin : 0, x[u][i][t]);
                }
        }
#pragma unroll
        for (int u = 0; u < kChunks; ++u) {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                uint32_t a[2][4];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t w[4] = {codes[u][r].x, codes[u][r].y, codes[u][r].z, codes[u][r].w};
                    if constexpr (kKind == kInt4) {
                        int4(w[i], a[r]);
                    } else {
                        int8_to_16<kHalf>(w[2 * i], a[r]);
                        int8_to_16<kHalf>(w[2 * i + 1], a[r] + 2);
                    }
                }
#pragma unroll
                for (int t = 0; t < kTiles; ++t) mma_16816<kHalf>(acc[t][0], a[0][0], a[1][0], a[0][1], a[1][1], x[u][i / 2][t][i & 1].x, x[u][i / 2][t][i & 1].y);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) mma_16816<kHalf>(acc[t][kSums - 1], a[0][2], a[1][2], a[0][3], a[1][3], x[u][i / 2][t][i & 1].z, x[u][i / 2][t][i & 1].w);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            part[warp][8 * t + 2 * q + (i & 1)][g + 8 * (i >> 1)] = kSums == 1 ? acc[t][0][i] : acc[t][0][i] + acc[t][kSums - 1][i];
    __syncthreads();
    if (row >= p.cout) return;
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        const int token = first + 16 * j;
        if (token >= tokens) return;
        SQ_LINEAR_CHECK(token < kTiles * kFewTokens && token0 + token < p.tokens && row >= row0 && row < p.cout, 1013);
        float u = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) u += part[w][token][row - row0];
        p.y[(token0 + token) * p.y_stride + row] = to_16<kHalf>(act_value(fmaf(u, scale, bias), p.act) + res[j]);
    }
}

}  // namespace sq
