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

constexpr int kSmallWarps = 8;
constexpr int kSmallRows = 16 * kSmallWarps;   // output channels of a thread block
constexpr int kSmallChunks = 4;                // chunks of a block of the contraction; two blocks are in flight
constexpr int kSmallMostRanks = 8;             // thread blocks of a cluster, which share the contraction

template <int kKind, int kTiles>
struct SmallShape {
    static constexpr int kCodes = kKind == kInt4 ? 32 : 16;        // codes of a lane's 16 bytes
    static constexpr int kChunk = 4 * kCodes;                      // of four lanes
    static constexpr int kBlock = kSmallChunks * kChunk;           // elements of x a token and block
    static constexpr int kUnits = kBlock / 8;                      // the same in 16 bytes
    static constexpr int kPitch = 2 * kBlock + 64;                 // bytes of a token in shared memory: two tokens' halves of a load hit all banks
    static constexpr int kPartPitch = kSmallRows + 4;              // floats of a token's partial sums
    static constexpr int kTokens = 8 * kTiles;
    static constexpr int kSmem = 2 * kTokens * kPitch + 4 * kTokens * kPartPitch;
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

// A thread block owns 128 channels, a warp 16 of them; the ranks of a cluster share the contraction, so that everything a
// call reads is asked for at about once.  In a chunk, lane (g, q) holds 16 bytes of the rows g and g + 8 and the same elements
// of token g: the order of the contraction inside a matrix instruction is free as long as both operands agree, so nothing
// is shuffled.  x goes through shared memory, whose 16-byte units are kept in the order in which the four lanes of a
// token read them.  The ranks' sums are added in the order of the ranks.
// kVector: rows of codes and of x start on 16 bytes and are whole vectors.
template <int kKind, bool kHalf, int kTiles, bool kVector>
__global__ void __launch_bounds__(32 * kSmallWarps, 2) small_kernel(const __grid_constant__ SmallArgs p)
{
    using S = SmallShape<kKind, kTiles>;
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t xs = smem_addr(smem), part = xs + 2 * S::kTokens * S::kPitch;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const uint32_t rank = cluster_rank(), ranks = cluster_ranks();
    const int row0 = static_cast<int>(blockIdx.x / ranks) * kSmallRows;
    const int all = (p.cin + S::kBlock - 1) / S::kBlock;
    const int first = static_cast<int>(static_cast<int64_t>(all) * rank / ranks);
    const int blocks = static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / ranks) - first;
    const int row_bytes = kKind == kInt4 ? (p.cin + 1) >> 1 : p.cin;
    float acc[kTiles][4] = {};
    next_may_start();
    wait_for_previous();
    const int row = row0 + (warp & 3) * 32 + lane;   // that this thread finishes
    const bool in = row < p.cout;
    const float scale = in ? get(p.scales + row) : 0.0f, bias = in && p.bias ? get(p.bias + row) : 0.0f;

    auto load = [&](int b, uint4 (&c)[kSmallChunks][2]) {
        const int off0 = ((first + b) * kSmallChunks * 4 + q) * 16;
#pragma unroll
        for (int u = 0; u < kSmallChunks; ++u)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = row0 + 16 * warp + g + 8 * r, off = off0 + 64 * u;
                c[u][r] = make_uint4(0, 0, 0, 0);
                if (off < row_bytes && row < p.cout) {
                    const uint8_t *at = p.codes + row * p.code_pitch + off;
                    c[u][r] = kVector ? ldg128(at) : load_bytes16(at, p.codes, p.codes + p.code_bytes);
                }
            }
    };
    auto stage_x = [&](int b) {
        const uint32_t to = xs + (b & 1) * S::kTokens * S::kPitch;
        for (int i = threadIdx.x; i < p.tokens * S::kUnits; i += 32 * kSmallWarps) {
            const int token = i / S::kUnits, unit = i % S::kUnits;
            constexpr int kLane = S::kCodes / 8;   // units of a lane and chunk
            const int place = unit & ~(4 * kLane - 1) | unit % kLane * 4 | unit / kLane % 4;
            const uint32_t dst = to + token * S::kPitch + place * 16;
            const int k = (first + b) * S::kBlock + unit * 8;
            const uint16_t *row = p.x + token * p.x_stride;
            if constexpr (kVector) {
                const int bytes = k < p.cin ? 16 : 0;   // 0: zeros
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(bytes ? row + k : row), "r"(bytes) : "memory");
            } else {
                const uint4 w = load_x8<false>(row, k, p.cin);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto multiply = [&](int b, const uint4 (&c)[kSmallChunks][2]) {
        const uint32_t from = xs + (b & 1) * S::kTokens * S::kPitch + g * S::kPitch + q * 16;
#pragma unroll
        for (int u = 0; u < kSmallChunks; ++u)
#pragma unroll
            for (int i = 0; i < S::kCodes / 8; ++i) {
                uint32_t a[2][4];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t w[4] = {c[u][r].x, c[u][r].y, c[u][r].z, c[u][r].w};
                    if constexpr (kKind == kInt4) {
                        int4_to_16<kHalf>(w[i], a[r]);
                    } else {
                        int8_to_16<kHalf>(w[2 * i], a[r]);
                        int8_to_16<kHalf>(w[2 * i + 1], a[r] + 2);
                    }
                }
#pragma unroll
                for (int n = 0; n < kTiles; ++n) {
                    uint32_t x[4];
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                                 : "r"(from + 8 * n * S::kPitch + (u * (S::kChunk / 8) + 4 * i) * 16) : "memory");
                    mma_16816<kHalf>(acc[n], a[0][0], a[1][0], a[0][1], a[1][1], x[0], x[1]);
                    mma_16816<kHalf>(acc[n], a[0][2], a[1][2], a[0][3], a[1][3], x[2], x[3]);
                }
            }
    };

    uint4 codes[2][kSmallChunks][2];
#pragma unroll
    for (int d = 0; d < 2; ++d)
        if (d < blocks) {
            load(d, codes[d]);
            stage_x(d);
        } else {
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    for (int b0 = 0; b0 < blocks; b0 += 2) {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const int b = b0 + d;
            if (b >= blocks) break;
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncthreads();
            multiply(b, codes[d]);
            if (b + 2 < blocks) {
                __syncthreads();
                load(b + 2, codes[d]);
                stage_x(b + 2);
            } else {
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
        }
    }
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(part + 4 * ((8 * n + 2 * q + (i & 1)) * S::kPartPitch + 16 * warp + g + 8 * (i >> 1))), "f"(acc[n][i]) : "memory");
    cluster_arrive_wait();

    // a warp takes 32 channels, which share a checkpoint's exponent, of one of the rank's tokens
    for (int token = static_cast<int>(rank) + (warp >> 2) * static_cast<int>(ranks); token < p.tokens; token += 2 * static_cast<int>(ranks)) {
        if (row - lane >= p.cout) break;
        const uint32_t mine = part + 4 * (token * S::kPartPitch + (warp & 3) * 32 + lane);
        float v[kSmallMostRanks];
#pragma unroll
        for (uint32_t r = 0; r < kSmallMostRanks; ++r) {
            v[r] = 0.0f;
            if (r < ranks) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r]) : "r"(cluster_addr(mine, r)));
        }
        float res = 0.0f;
        if (p.residual && in) res = to_float<kHalf>(p.residual[token * p.residual_stride + row]);
        float u = 0.0f;
#pragma unroll
        for (int r = 0; r < kSmallMostRanks; ++r) u += v[r];
        const float z = fmaf(u, scale, bias);
        if (p.z_codes) {
            float a = fabsf(z);
#pragma unroll
            for (int s = 16; s; s >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, s));
            const uint32_t e = ckpt_exponent(a);
            p.z_codes[token * p.z_pitch + row] = static_cast<uint8_t>(ckpt_code(z, ckpt_inverse(e)));   // rows end on 32
            if (lane == 0) p.z_exps[token * p.z_exps_pitch + (row >> 5)] = static_cast<uint8_t>(e);
        }
        if (in) p.y[token * p.y_stride + row] = to_16<kHalf>(act_value(z, p.act) + res);
    }
    cluster_arrive_wait();   // the others' sums stay until they have been read
}

constexpr int kFewRows = 16;       // output channels of a thread block
constexpr int kFewTokens = 8;
constexpr int kFewChunks = 4;      // in flight a warp

// Up to eight tokens without a checkpoint: a thread block owns 16 channels, its warps take chunks of the contraction in
// turn and are summed at the end.  A lane asks for the codes and the elements of x of four chunks at once, and nothing
// waits for another thread before the sum: for so few tokens x is small beside the codes although every block reads all of it.
template <int kKind, bool kHalf, bool kVector>
__global__ void __launch_bounds__(32 * kSmallWarps, 2) few_kernel(const __grid_constant__ SmallArgs p)
{
    constexpr int kCodes = kKind == kInt4 ? 32 : 16;
    constexpr int kUnits = kCodes / 8;   // 16 bytes of x a lane and chunk
    __shared__ float part[kSmallWarps][kFewTokens][kFewRows];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int row0 = static_cast<int>(blockIdx.x) * kFewRows;
    const int chunks = (p.cin + 4 * kCodes - 1) / (4 * kCodes);
    const int row_bytes = kKind == kInt4 ? (p.cin + 1) >> 1 : p.cin;
    next_may_start();
    wait_for_previous();
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

    for (int c0 = warp; c0 < chunks; c0 += kSmallWarps * kFewChunks) {
        uint4 codes[kFewChunks][2], x[kFewChunks][kUnits];
#pragma unroll
        for (int u = 0; u < kFewChunks; ++u) {
            const int piece = (c0 + u * kSmallWarps) * 4 + q;
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
            const int k = ((c0 + u * kSmallWarps) * 4 + q) * kCodes;
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
                        int4_to_16<kHalf>(w[i], a[r]);
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
    for (int w = 0; w < kSmallWarps; ++w) u += part[w][token][row - row0];
    p.y[token * p.y_stride + row] = to_16<kHalf>(act_value(fmaf(u, scale, bias), p.act) + res);
}

}  // namespace sq
