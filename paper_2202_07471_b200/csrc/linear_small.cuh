// The forward product for few tokens, where reading the codes is all there is to do: up to 32 tokens.
#pragma once

#include "linear_device.cuh"

namespace sq {

struct SmallArgs {
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
    uint8_t *z_codes, *z_exps;
    int64_t z_pitch, z_exps_pitch;
};

constexpr int kSmallRows = 32;      // output channels of a thread block: one checkpoint group
constexpr int kSmallWarps = 8;      // share the contraction

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
        return __ldg(reinterpret_cast<const uint4 *>(row + first));
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = first + 2 * i;
            w[i] = (k < cin ? static_cast<uint32_t>(__ldg(row + k)) : 0u) | (k + 1 < cin ? static_cast<uint32_t>(__ldg(row + k + 1)) << 16 : 0u);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// A thread block owns 32 channels; its warps take chunks of the contraction in turn (four lanes times 16 bytes of
// codes) and are summed at the end.  In a chunk lane (g, q) holds 16 bytes of rows g, g + 8, g + 16, g + 24 and the same
// elements of token g: the order of the contraction inside a matrix instruction is free as long as both operands
// agree, so nothing is shuffled.
// kVector: rows of codes and of x start on 16 bytes and are whole vectors.
template <int kKind, bool kHalf, int kTiles, bool kVector>
__global__ void __launch_bounds__(32 * kSmallWarps, 2) small_kernel(const __grid_constant__ SmallArgs p)
{
    constexpr int kCodes = kKind == kInt4 ? 32 : 16;      // codes of a lane's 16 bytes
    constexpr int kChunk = 4 * kCodes;
    constexpr int kAhead = kTiles == 1 ? 4 : 2;           // chunks in flight
    __shared__ float part[kSmallWarps][8 * kTiles][kSmallRows];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int row0 = blockIdx.x * kSmallRows;
    const int chunks = (p.cin + kChunk - 1) / kChunk;
    const int row_bytes = kKind == kInt4 ? (p.cin + 1) >> 1 : p.cin;
    float acc[2][kTiles][4] = {};

    for (int c0 = warp; c0 < chunks; c0 += kSmallWarps * kAhead) {
        uint4 codes[kAhead][4];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int off = ((c0 + u * kSmallWarps) * 4 + q) * 16;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = row0 + g + 8 * r;
                codes[u][r] = make_uint4(0, 0, 0, 0);
                if (off < row_bytes && row < p.cout) {
                    const uint8_t *at = p.codes + row * p.code_pitch + off;
                    codes[u][r] = kVector ? ldg128(at) : load_bytes16(at, p.codes, p.codes + p.code_bytes);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int k0 = ((c0 + u * kSmallWarps) * 4 + q) * kCodes;
            if (c0 + u * kSmallWarps >= chunks) break;
            uint32_t x[kTiles][kCodes / 2];
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
                const int token = 8 * n + g;
#pragma unroll
                for (int i = 0; i < kCodes / 8; ++i) {
                    const uint4 v = token < p.tokens ? load_x8<kVector>(p.x + token * p.x_stride, k0 + 8 * i, p.cin) : make_uint4(0, 0, 0, 0);
                    x[n][4 * i] = v.x; x[n][4 * i + 1] = v.y; x[n][4 * i + 2] = v.z; x[n][4 * i + 3] = v.w;
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t a[4][4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t w = j == 0 ? codes[u][r].x : j == 1 ? codes[u][r].y : j == 2 ? codes[u][r].z : codes[u][r].w;
                    if constexpr (kKind == kInt4) int4_to_16<kHalf>(w, a[r]);
                    else int8_to_16<kHalf>(w, a[r]);
                }
                constexpr int kSteps = kKind == kInt4 ? 2 : 1;   // matrix instructions of a word of codes
#pragma unroll
                for (int h = 0; h < kSteps; ++h)
#pragma unroll
                    for (int n = 0; n < kTiles; ++n) {
                        const uint32_t b0 = x[n][(j * kSteps + h) * 2], b1 = x[n][(j * kSteps + h) * 2 + 1];
                        mma_16816<kHalf>(acc[0][n], a[0][2 * h], a[1][2 * h], a[0][2 * h + 1], a[1][2 * h + 1], b0, b1);
                        mma_16816<kHalf>(acc[1][n], a[2][2 * h], a[3][2 * h], a[2][2 * h + 1], a[3][2 * h + 1], b0, b1);
                    }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][8 * n + 2 * q + (i & 1)][16 * b + g + 8 * (i >> 1)] = acc[b][n][i];
    __syncthreads();

    const int row = row0 + lane;
    const bool in = row < p.cout;
    for (int token = warp; token < p.tokens; token += kSmallWarps) {
        float u = 0.0f;
#pragma unroll
        for (int w = 0; w < kSmallWarps; ++w) u += part[w][token][lane];
        const float z = in ? fmaf(u, __ldg(p.scales + row), p.bias ? __ldg(p.bias + row) : 0.0f) : 0.0f;
        if (p.z_codes) {
            float a = fabsf(z);
#pragma unroll
            for (int s = 16; s; s >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, s));
            const uint32_t e = ckpt_exponent(a);
            p.z_codes[token * p.z_pitch + row] = static_cast<uint8_t>(ckpt_code(z, ckpt_inverse(e)));   // rows end on 32
            if (lane == 0) p.z_exps[token * p.z_exps_pitch + blockIdx.x] = static_cast<uint8_t>(e);
        }
        if (in) {
            float v = act_value(z, p.act);
            if (p.residual) v += to_float<kHalf>(p.residual[token * p.residual_stride + row]);
            p.y[token * p.y_stride + row] = to_16<kHalf>(v);
        }
    }
}

}  // namespace sq
