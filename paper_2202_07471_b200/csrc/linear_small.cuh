// The forward product for up to eight tokens, where reading the codes is all there is to do.
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

// Eight 16-bit values of a row from `first` on, zeros at and behind the row's end.
template <bool kVector>
__device__ __forceinline__ uint4 load_x8(const uint16_t *row, int first, int cin)
{
    if (first >= cin) return make_uint4(0, 0, 0, 0);
    if constexpr (kVector) {
        return get(reinterpret_cast<const uint4 *>(row + first));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = first + 2 * i;
            w[i] = (k < cin ? static_cast<uint32_t>(get(row + k)) : 0u) | (k + 1 < cin ? static_cast<uint32_t>(get(row + k + 1)) << 16 : 0u);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

constexpr int kFewWarps = 8;       // share the contraction
constexpr int kFewRows = 16;       // output channels of a thread block
constexpr int kFewTokens = 8;
constexpr int kFewChunks = 2;      // in flight a warp

// Without a checkpoint (its 32 channels would be two thread blocks'): a thread block owns 16 channels, its warps take chunks of the
// contraction in turn and are summed at the end.  In a chunk (four lanes times 16 bytes of codes) lane (g, q) holds 16 bytes of the
// rows g and g + 8 and the same elements of token g: the order of the contraction inside a matrix instruction is free as long as
// both operands agree, so nothing is shuffled.  A lane asks for the codes and the elements of x of two chunks at once, and
// nothing waits for another thread before the sum: for so few tokens x is small beside the codes although every block reads all
// of it.  Bound by the issue of instructions (about two a code) and the latency of a batch: one token int4 4096 -> 4096 4.3 us,
// 11008 -> 32768 51 us (3.5 TB/s); four chunks and two blocks a multiprocessor 4.35 and 64.  (128 channels a block, x through shared
// memory and the contraction shared by a cluster: 6.2 us.  mma.sync, since tcgen05 has no use for eight tokens: a step of 64
// takes longer there.)
// kVector: rows of codes and of x start on 16 bytes and are whole vectors.
template <int kKind, bool kHalf, bool kVector>
__global__ void __launch_bounds__(32 * kFewWarps, 3) few_kernel(const __grid_constant__ FewArgs p)
{
    constexpr int kCodes = kKind == kInt4 ? 32 : 16;
    constexpr int kUnits = kCodes / 8;   // 16 bytes of x a lane and chunk
    __shared__ float part[kFewWarps][kFewTokens][kFewRows];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int row0 = static_cast<int>(blockIdx.x) * kFewRows;
    const int chunks = (p.cin + 4 * kCodes - 1) / (4 * kCodes);
    const int row_bytes = kKind == kInt4 ? (p.cin + 1) >> 1 : p.cin;
    // the thread that finishes (token, row)
    const int token = threadIdx.x / kFewRows, row = row0 + static_cast<int>(threadIdx.x) % kFewRows;
    const bool mine = token < p.tokens && row < p.cout;
    float scale = 0.0f, bias = 0.0f, res = 0.0f;
    if (mine) {
        scale = get(p.scales + row);
        if (p.bias) bias = get(p.bias + row);
        if (p.residual) res = to_float<kHalf>(p.residual[token * p.residual_stride + row]);
    }
    float acc[2][4] = {};
    [[maybe_unused]] const Int4To16<kHalf> int4;

    for (int c0 = warp; c0 < chunks; c0 += kFewWarps * kFewChunks) {
        uint4 codes[kFewChunks][2], x[kFewChunks][kUnits];
#pragma unroll
        for (int u = 0; u < kFewChunks; ++u) {
            const int piece = (c0 + u * kFewWarps) * 4 + q;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int at = row0 + g + 8 * r;
                codes[u][r] = make_uint4(0, 0, 0, 0);
                if (piece * 16 < row_bytes && at < p.cout) {
                    const uint8_t *from = p.codes + at * p.code_pitch + piece * 16;
                    codes[u][r] = kVector ? ldg128(from) : load_bytes16(from, p.codes, p.codes + p.code_bytes);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kFewChunks; ++u) {
            const int k = ((c0 + u * kFewWarps) * 4 + q) * kCodes;
#pragma unroll
            for (int i = 0; i < kUnits; ++i)
                x[u][i] = g < p.tokens ? load_x8<kVector>(p.x + g * p.x_stride, k + 8 * i, p.cin) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < kFewChunks; ++u) {
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
                mma_16816<kHalf>(acc[0], a[0][0], a[1][0], a[0][1], a[1][1], x[u][i].x, x[u][i].y);
                mma_16816<kHalf>(acc[1], a[0][2], a[1][2], a[0][3], a[1][3], x[u][i].z, x[u][i].w);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[warp][2 * q + (i & 1)][g + 8 * (i >> 1)] = acc[0][i] + acc[1][i];
    __syncthreads();
    if (!mine) return;
    float u = 0.0f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) u += part[w][token][row - row0];
    p.y[token * p.y_stride + row] = to_16<kHalf>(act_value(fmaf(u, scale, bias), p.act) + res);
}

}  // namespace sq
