// Row-wise kernels of the linear operators, bound by the bytes they move: 8-bit checkpoints, the gradient of the
// pre-activation with the sums over the tokens, and copies of rows that TMA cannot read.
#pragma once

#include <cooperative_groups.h>

#include "linear_device.cuh"

namespace sq {

constexpr int kRowThreads = 256;
constexpr int kRowPieces = 4;    // pieces of eight elements a thread: four loads in flight

// Eight 16-bit values of a row from `first` on, of which n are inside the row.
__device__ __forceinline__ uint4 load8(const uint16_t *at, int n, bool vector)
{
    if (vector && n >= 8) return get(reinterpret_cast<const uint4 *>(at));
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = (2 * i < n ? static_cast<uint32_t>(get(at + 2 * i)) : 0u) | (2 * i + 1 < n ? static_cast<uint32_t>(get(at + 2 * i + 1)) << 16 : 0u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void put8(uint16_t *at, const uint4 &v, int n, bool vector)
{
    if (vector && n >= 8) {
        *reinterpret_cast<uint4 *>(at) = v;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) at[i] = static_cast<uint16_t>(w[i >> 1] >> (16 * (i & 1)));
}
__device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// rows x pieces is below 2^31 in one launch.
struct RowArgs {
    const uint16_t *in;
    uint16_t *out;
    uint8_t *codes, *exps;
    int64_t in_stride, out_stride, code_pitch, exps_pitch;
    uint32_t rows, pieces;   // pieces of eight elements a row
    int32_t features, vector;
};

// Four lanes share a group of 32 features.
static __global__ void __launch_bounds__(kRowThreads) checkpoint_kernel(const RowArgs p)
{
    next_may_start();
    wait_for_previous();
    const uint32_t first = blockIdx.x * (kRowThreads * kRowPieces) + threadIdx.x, total = p.rows * p.pieces;
    uint4 v[kRowPieces];
    uint32_t row[kRowPieces];
    int col[kRowPieces];
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads;
        row[i] = at / p.pieces;
        col[i] = static_cast<int>(at - row[i] * p.pieces) * 8;
        v[i] = make_uint4(0, 0, 0, 0);
        if (at < total && col[i] < p.features) v[i] = load8(p.in + row[i] * p.in_stride + col[i], p.features - col[i], p.vector);
    }
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        float f[8], a = 0.0f;
        unpack8(v[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) a = max_nan(a, fabsf(f[j]));
        a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, 1));
        a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, 2));
        const uint32_t e = ckpt_exponent(a);
        const float inverse = ckpt_inverse(e);
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j >> 2] |= static_cast<uint32_t>(ckpt_code(f[j], inverse) & 255) << (8 * (j & 3));
        if (first + i * kRowThreads < total) {
            *reinterpret_cast<uint2 *>(p.codes + row[i] * p.code_pitch + col[i]) = make_uint2(w[0], w[1]);
            if ((threadIdx.x & 3) == 0) p.exps[row[i] * p.exps_pitch + (col[i] >> 5)] = static_cast<uint8_t>(e);
        }
    }
}

static __global__ void __launch_bounds__(kRowThreads) restore_kernel(const RowArgs p)
{
    next_may_start();
    wait_for_previous();
    const uint32_t first = blockIdx.x * (kRowThreads * kRowPieces) + threadIdx.x, total = p.rows * p.pieces;
    uint2 c[kRowPieces];
    uint32_t e[kRowPieces], row[kRowPieces];
    int col[kRowPieces];
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads;
        row[i] = at / p.pieces;
        col[i] = static_cast<int>(at - row[i] * p.pieces) * 8;
        c[i] = make_uint2(0, 0);
        e[i] = 0;
        if (at < total) {
            c[i] = get(reinterpret_cast<const uint2 *>(p.codes + row[i] * p.code_pitch + col[i]));
            e[i] = get(p.exps + row[i] * p.exps_pitch + (col[i] >> 5));
        }
    }
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        if (first + i * kRowThreads >= total || col[i] >= p.features) continue;
        uint32_t o[4];
        int8_to_16<false>(c[i].x, o);
        int8_to_16<false>(c[i].y, o + 2);
        const uint32_t scale = e[i] << 7 | e[i] << 23;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = mul2_bf16(o[j], scale);
        put8(p.out + row[i] * p.out_stride + col[i], make_uint4(o[0], o[1], o[2], o[3]), p.features - col[i], p.vector);
    }
}

// Codes to 16-bit floats, eight a thread and piece: rows of `code_pitch` bytes to rows that start on 16 bytes.
// vector: every row of codes starts on a piece's bytes.
template <int kKind, bool kHalf>
static __global__ void __launch_bounds__(kRowThreads) expand_kernel(const RowArgs p)
{
    constexpr int kBytes = kKind == kInt4 ? 4 : 8;   // of a piece
    next_may_start();
    wait_for_previous();
    const uint32_t first = blockIdx.x * (kRowThreads * kRowPieces) + threadIdx.x, total = p.rows * p.pieces;
    uint2 c[kRowPieces];
    uint32_t row[kRowPieces], piece[kRowPieces];
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads;
        row[i] = at / p.pieces;
        piece[i] = at - row[i] * p.pieces;
        c[i] = make_uint2(0, 0);
        if (at < total) {
            const uint8_t *q = p.codes + row[i] * p.code_pitch + piece[i] * kBytes;
            if (p.vector) {
                if (kKind == kInt4) c[i].x = get(reinterpret_cast<const uint32_t *>(q));
                else c[i] = get(reinterpret_cast<const uint2 *>(q));
            } else {
                const int left = static_cast<int>(p.code_pitch - piece[i] * kBytes);
                uint32_t w[2] = {0, 0};
#pragma unroll
                for (int b = 0; b < kBytes; ++b)
                    if (b < left) w[b >> 2] |= static_cast<uint32_t>(get(q + b)) << (8 * (b & 3));
                c[i] = make_uint2(w[0], w[1]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        if (first + i * kRowThreads >= total) continue;
        uint32_t o[4];
        if constexpr (kKind == kInt4) {
            int4_to_16<kHalf>(c[i].x, o);
        } else {
            int8_to_16<kHalf>(c[i].x, o);
            int8_to_16<kHalf>(c[i].y, o + 2);
        }
        *reinterpret_cast<uint4 *>(p.out + row[i] * p.out_stride + piece[i] * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// Rows that start anywhere to rows that start on 16 bytes, which TMA can read (the elements behind a row's end become 0).
static __global__ void __launch_bounds__(kRowThreads) align_kernel(const RowArgs p)
{
    next_may_start();
    wait_for_previous();
    const uint32_t first = blockIdx.x * (kRowThreads * kRowPieces) + threadIdx.x, total = p.rows * p.pieces;
    uint4 v[kRowPieces];
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads, row = at / p.pieces;
        const int col = static_cast<int>(at - row * p.pieces) * 8;
        if (at < total) v[i] = load8(p.in + row * p.in_stride + col, p.features - col, false);
    }
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads, row = at / p.pieces;
        if (at < total) *reinterpret_cast<uint4 *>(p.out + row * p.out_stride + (at - row * p.pieces) * 8) = v[i];
    }
}

struct SlopeArgs {
    const uint16_t *dy;
    int64_t dy_stride;
    int32_t dy_vector;
    const uint8_t *z_codes, *z_exps;   // null: no activation and no gradient of the scales
    int64_t z_pitch, z_exps_pitch;
    const float *scales, *bias;
    int64_t tokens;
    int32_t cout, act;
    uint16_t *dz, *dzs;                // null where not wanted
    int64_t pitch;                     // elements, a multiple of 8
    float *dbias, *dscales;            // null where not wanted
};

constexpr int kSlopeCols = 64;      // a thread block's columns: eight threads of eight, 32 rows at a time
constexpr int kSlopeCluster = 8;    // thread blocks that share the tokens of the same columns

// dz = dy * act'(zhat) in bf16, and times the scales; sums over the tokens of dz and of dz * (zhat - bias) / scale in
// fp32 from the unrounded products.  The thread blocks of a cluster each take a range of tokens; their sums meet
// through distributed shared memory in a fixed order, so that a call repeats to the bit.
static __global__ void __launch_bounds__(kRowThreads) slope_kernel(const __grid_constant__ SlopeArgs p)
{
    namespace cg = cooperative_groups;
    next_may_start();
    wait_for_previous();
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * kSlopeCols + tx * 8;
    const int n = p.cout - col;   // columns of this thread inside the row, possibly none
    __shared__ float part[kRowThreads / 32][2 * kSlopeCols];
    __shared__ float sums[2 * kSlopeCols];
    float scale[8], bias[8], db[8] = {}, ds[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        scale[i] = i < n ? get(p.scales + col + i) : 1.0f;
        bias[i] = i < n && p.bias ? get(p.bias + col + i) : 0.0f;
    }
    const int64_t share = ((p.tokens + ranks - 1) / ranks + 31) / 32 * 32;
    const int64_t end = min(p.tokens, (rank + 1) * share);
    if (n > 0)
#pragma unroll 2
        for (int64_t t = rank * share + ty; t < end; t += 32) {
            float dz[8];
            unpack8(load8(p.dy + t * p.dy_stride + col, n, p.dy_vector), dz);
            if (p.z_codes) {
                const uint2 c = get(reinterpret_cast<const uint2 *>(p.z_codes + t * p.z_pitch + col));
                const float zs = ckpt_scale(get(p.z_exps + t * p.z_exps_pitch + (col >> 5)));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = zs * static_cast<float>(static_cast<int8_t>((i < 4 ? c.x : c.y) >> (8 * (i & 3))));
                    if (i < n) {
                        dz[i] *= act_slope(z, p.act);
                        ds[i] = fmaf(dz[i], z - bias[i], ds[i]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) db[i] += dz[i];
            if (p.dz)
                *reinterpret_cast<uint4 *>(p.dz + t * p.pitch + col) = make_uint4(to_16x2<false>(dz[0], dz[1]), to_16x2<false>(dz[2], dz[3]),
                                                                                  to_16x2<false>(dz[4], dz[5]), to_16x2<false>(dz[6], dz[7]));
            if (p.dzs)
                *reinterpret_cast<uint4 *>(p.dzs + t * p.pitch + col) =
                    make_uint4(to_16x2<false>(dz[0] * scale[0], dz[1] * scale[1]), to_16x2<false>(dz[2] * scale[2], dz[3] * scale[3]),
                               to_16x2<false>(dz[4] * scale[4], dz[5] * scale[5]), to_16x2<false>(dz[6] * scale[6], dz[7] * scale[7]));
        }
    if (!p.dbias && !p.dscales) return;   // the same for all threads of the launch
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int s = 8; s <= 16; s <<= 1) {
            db[i] += __shfl_xor_sync(0xffffffffu, db[i], s);
            ds[i] += __shfl_xor_sync(0xffffffffu, ds[i], s);
        }
    if ((threadIdx.x & 31) < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            part[warp][tx * 8 + i] = db[i];
            part[warp][kSlopeCols + tx * 8 + i] = ds[i];
        }
    __syncthreads();
    if (threadIdx.x < 2 * kSlopeCols) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowThreads / 32; ++w) s += part[w][threadIdx.x];
        sums[threadIdx.x] = s;
    }
    cluster.sync();
    if (rank == 0 && threadIdx.x < 2 * kSlopeCols) {
        float s = 0.0f;
        for (int r = 0; r < ranks; ++r) s += cluster.map_shared_rank(sums, r)[threadIdx.x];
        const int c = blockIdx.x * kSlopeCols + (threadIdx.x & (kSlopeCols - 1));
        if (c < p.cout) {
            if (threadIdx.x < kSlopeCols) {
                if (p.dbias) p.dbias[c] = s;
            } else if (p.dscales) {
                p.dscales[c] = s / get(p.scales + c);
            }
        }
    }
    cluster.sync();   // the others' sums stay until rank 0 has read them
}

}  // namespace sq
