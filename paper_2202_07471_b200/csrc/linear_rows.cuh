// Row-wise kernels of the linear operators, bound by the bytes they move: 8-bit checkpoints, the gradient of the
// pre-activation with the sums over the tokens, and copies of rows that TMA cannot read.
#pragma once

#include "linear_device.cuh"

namespace sq {

constexpr int kRowThreads = 256;
constexpr int kRowPieces = 2;    // pieces of eight elements a thread (four and eight are no faster for large tensors and slower for small ones)

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
    uint32_t rows, pieces;   // pieces of eight elements (checkpoint_kernel: sixteen) a row
    uint32_t magic, shift;   // at / pieces = at * magic >> 32 >> shift for at < 2^31; magic 0: one piece a row
    int32_t features, vector;
};

__device__ __forceinline__ uint32_t row_of(const RowArgs &p, uint32_t at) { return p.magic ? __umulhi(at, p.magic) >> p.shift : at; }

// Pieces of sixteen elements; two lanes share a group of 32 features.
static __global__ void __launch_bounds__(kRowThreads) checkpoint_kernel(const RowArgs p)
{
    const uint32_t first = blockIdx.x * (kRowThreads * kRowPieces) + threadIdx.x, total = p.rows * p.pieces;
    uint4 v[kRowPieces][2];
    uint32_t row[kRowPieces];
    int col[kRowPieces];
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads;
        row[i] = row_of(p, at);
        col[i] = static_cast<int>(at - row[i] * p.pieces) * 16;
        const int n = at < total ? p.features - col[i] : 0;
        const uint16_t *from = p.in + row[i] * p.in_stride + col[i];
#pragma unroll
        for (int h = 0; h < 2; ++h) v[i][h] = n > 8 * h ? load8(from + 8 * h, n - 8 * h, p.vector) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        float f[2][8], a = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unpack8(v[i][h], f[h]);
#pragma unroll
            for (int j = 0; j < 8; ++j) a = max_nan(a, fabsf(f[h][j]));
        }
        a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, 1));
        const uint32_t e = ckpt_exponent(a);
        const float inverse = ckpt_inverse(e);
        const uint4 w = make_uint4(ckpt_codes(f[0], inverse), ckpt_codes(f[0] + 4, inverse), ckpt_codes(f[1], inverse), ckpt_codes(f[1] + 4, inverse));
        if (first + i * kRowThreads < total) {
            SQ_LINEAR_CHECK(row[i] < p.rows && col[i] >= 0 && col[i] + 16 <= p.code_pitch && (col[i] >> 5) < p.exps_pitch, 1050);
            *reinterpret_cast<uint4 *>(p.codes + row[i] * p.code_pitch + col[i]) = w;
            if ((threadIdx.x & 1) == 0) p.exps[row[i] * p.exps_pitch + (col[i] >> 5)] = static_cast<uint8_t>(e);
        }
    }
}

static __global__ void __launch_bounds__(kRowThreads) restore_kernel(const RowArgs p)
{
    const uint32_t first = blockIdx.x * (kRowThreads * kRowPieces) + threadIdx.x, total = p.rows * p.pieces;
    uint2 c[kRowPieces];
    uint32_t e[kRowPieces], row[kRowPieces];
    int col[kRowPieces];
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads;
        row[i] = row_of(p, at);
        col[i] = static_cast<int>(at - row[i] * p.pieces) * 8;
        c[i] = make_uint2(0, 0);
        e[i] = 0;
        if (at < total) {
            SQ_LINEAR_CHECK(row[i] < p.rows && col[i] >= 0 && col[i] + 8 <= p.code_pitch && (col[i] >> 5) < p.exps_pitch, 1051);
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
    [[maybe_unused]] const Int4To16<kHalf> int4;
    const uint32_t first = blockIdx.x * (kRowThreads * kRowPieces) + threadIdx.x, total = p.rows * p.pieces;
    uint2 c[kRowPieces];
    uint32_t row[kRowPieces], piece[kRowPieces];
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads;
        row[i] = row_of(p, at);
        piece[i] = at - row[i] * p.pieces;
        c[i] = make_uint2(0, 0);
        if (at < total) {
            const uint8_t *q = p.codes + row[i] * p.code_pitch + piece[i] * kBytes;
            SQ_LINEAR_CHECK(row[i] < p.rows && piece[i] < p.pieces && piece[i] * 8 + 8 <= p.out_stride, 1052);
            SQ_LINEAR_CHECK(p.vector ? piece[i] * kBytes + kBytes <= p.code_pitch : piece[i] * kBytes < p.code_pitch, 1053);
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
            int4(c[i].x, o);
        } else {
            int8_to_16<kHalf>(c[i].x, o);
            int8_to_16<kHalf>(c[i].y, o + 2);
        }
        *reinterpret_cast<uint4 *>(p.out + row[i] * p.out_stride + piece[i] * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// Rows of bytes that start anywhere to rows that start on 16 bytes, which TMA can read (what lies behind a row's last byte is not used).
struct CopyJob {
    const uint8_t *in, *end;   // end: of what may be read
    uint8_t *out;
    int64_t in_pitch, out_pitch;
    uint32_t rows, pieces;     // of 16 bytes a row
    uint32_t magic, shift;     // as in RowArgs
};

// Two jobs in one launch: the first `blocks` thread blocks take the first.
static __global__ void __launch_bounds__(kRowThreads) copy_kernel(const __grid_constant__ CopyJob a, const __grid_constant__ CopyJob b, uint32_t blocks)
{
    const bool second = blockIdx.x >= blocks;
    const CopyJob &p = second ? b : a;
    const uint32_t first = (blockIdx.x - (second ? blocks : 0)) * (kRowThreads * kRowPieces) + threadIdx.x, total = p.rows * p.pieces;
#pragma unroll
    for (int i = 0; i < kRowPieces; ++i) {
        const uint32_t at = first + i * kRowThreads, row = p.magic ? __umulhi(at, p.magic) >> p.shift : at, piece = at - row * p.pieces;
        SQ_LINEAR_CHECK(at >= total || (row < p.rows && piece < p.pieces && piece * 16 + 16 <= p.out_pitch), 1054);
        if (at < total)
            *reinterpret_cast<uint4 *>(p.out + row * p.out_pitch + piece * 16) = load_bytes16(p.in + row * p.in_pitch + piece * 16, p.in, p.end);
    }
}

struct SlopeArgs {
    const uint16_t *dy;
    int64_t dy_stride;
    const uint8_t *z_codes, *z_exps;   // null: no activation and no gradient of the scales
    int64_t z_pitch, z_exps_pitch;
    const float *scales, *bias;
    int64_t tokens;
    int32_t cout, act;
    uint16_t *dz, *dzs;                // null where not wanted
    int64_t pitch;                     // elements, a multiple of 8
    float *dbias, *dscales;            // null where not wanted
    int64_t share;                     // tokens of a thread block
    float *partial;                    // [shares][2][cout] sums of the shares; null: there is one
    int32_t shares;
};

constexpr int kSlopeCols = 64;      // a thread block's columns: sixteen threads of four, 16 rows at a time
constexpr int kSlopeRows = kRowThreads / 16;
constexpr int kSlopeBatch = 4;      // rows a thread has in flight
constexpr int kSlopeBlocks = 592;   // wanted of a launch: four a multiprocessor of a B200
constexpr int kSlopeLeast = 64;     // tokens of a share
// A group's exponent leaves its values 255 codes: for the exponents of groups whose largest value is between 2^-2 and 2^6 a block makes
// tables of gelu' or silu' first (8 KB), if its share is long enough to pay for 2048 of them; they hold what act_slopes gives.
// 4096 x 4096, sums only, gelu 30 -> 18.5 us, silu 26 -> 18.9; 16384 x 11008 290 -> 161 (42 instructions an element without, which bound it).  With every other
// group off the tables 31.4 and 309: warps take both ways.
constexpr uint32_t kSlopeTables = 8, kSlopeFirst = 119;
constexpr int kSlopeTableLeast = 128;   // tokens of a share

template <int kValue>
struct Count {
    static constexpr int value = kValue;
};

// Four 16-bit values of a row, of which n are inside the row.
__device__ __forceinline__ uint2 load4(const uint16_t *at, int n, bool vector)
{
    if (vector && n >= 4) return get(reinterpret_cast<const uint2 *>(at));
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = (2 * i < n ? static_cast<uint32_t>(get(at + 2 * i)) : 0u) | (2 * i + 1 < n ? static_cast<uint32_t>(get(at + 2 * i + 1)) << 16 : 0u);
    return make_uint2(w[0], w[1]);
}

// dz = dy * act'(zhat) in bf16, and times the scales; sums over the tokens of dz and of dz * (zhat - bias) / scale in
// fp32 from the unrounded products.  bf16, since dz and dz * s are the tensor cores' operands: half a step of each term, which makes the gradients' distance
// from their formulas 0.0024 of their norm instead of the 0.0017 that the rounding of the result alone leaves.  Thread blocks share the tokens; the sums of their shares go through global memory and are
// added in their order by sums_kernel, so that a call repeats to the bit.  What the kernel needs is loads in flight: four columns a
// thread keep sums and factors in few registers.  (Eight columns a thread and shares joined by clusters of eight, which allow 264
// blocks at once, took 34 to 50 us for 4096 x 4096.)
// kAct: kActNone and so on, or kNoZ where zhat is not needed.  kVector: whole vectors of four, rows of dy start on 8 bytes.
constexpr int kNoZ = -1;
template <int kAct, bool kVector>
__global__ void __launch_bounds__(kRowThreads, 4) slope_kernel(const __grid_constant__ SlopeArgs p)
{
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * kSlopeCols + tx * 4;
    const int n = kVector ? (col < p.cout ? 4 : 0) : p.cout - col;   // columns of this thread inside the row, possibly none
    __shared__ float part[kRowThreads / 32][2 * kSlopeCols];
    constexpr bool kTable = kAct == kActGelu || kAct == kActSilu;
    __shared__ float table[kTable ? kSlopeTables : 1][256];
    [[maybe_unused]] uint32_t tables = 0;
    if constexpr (kTable)
        if (p.share >= kSlopeTableLeast) {
            tables = kSlopeTables;
            for (uint32_t i = 2 * threadIdx.x; i < kSlopeTables * 256; i += 2 * kRowThreads) {
                const float unit = ckpt_scale(kSlopeFirst + (i >> 8));
                const float z[2] = {unit * static_cast<float>(static_cast<int8_t>(i)), unit * static_cast<float>(static_cast<int8_t>(i + 1))};
                float slope[2];
                act_slopes<kAct>(z, slope);
                *reinterpret_cast<float2 *>(&table[i >> 8][i & 255]) = make_float2(slope[0], slope[1]);
            }
            __syncthreads();
        }
    float scale[4], bias[4], db[4] = {}, ds[4] = {};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        scale[i] = i < n && p.dzs ? get(p.scales + col + i) : 1.0f;
        bias[i] = i < n && p.bias ? get(p.bias + col + i) : 0.0f;
    }
    const int64_t end = min(p.tokens, (blockIdx.y + 1) * p.share);
    if (n > 0) {
        int64_t t0 = blockIdx.y * p.share + ty;
        const uint16_t *dy_at = p.dy + t0 * p.dy_stride + col;
        const uint8_t *zc_at = p.z_codes + t0 * p.z_pitch + col, *ze_at = p.z_exps + t0 * p.z_exps_pitch + (col >> 5);
        const int64_t out0 = t0 * p.pitch + col;
        uint16_t *dz_at = p.dz + out0, *dzs_at = p.dzs + out0;
        // whole batches without a look at the end, then what is left row by row
        auto rows = [&](auto count) {
            constexpr int kCount = decltype(count)::value;
            uint2 dy[kCount];
            [[maybe_unused]] uint32_t zc[kCount], ze[kCount];
#pragma unroll
            for (int b = 0; b < kCount; ++b) {
                SQ_LINEAR_CHECK(t0 + b * kSlopeRows < p.tokens && dy_at == p.dy + (t0 + b * kSlopeRows) * p.dy_stride + col && col + (kVector ? 4 : 1) <= p.cout, 1055);
                if constexpr (kVector) dy[b] = get(reinterpret_cast<const uint2 *>(dy_at));
                else dy[b] = load4(dy_at, n, false);
                dy_at += kSlopeRows * p.dy_stride;
                if constexpr (kAct != kNoZ) {
                    SQ_LINEAR_CHECK(col + 4 <= p.z_pitch && zc_at == p.z_codes + (t0 + b * kSlopeRows) * p.z_pitch + col &&
                                    ze_at == p.z_exps + (t0 + b * kSlopeRows) * p.z_exps_pitch + (col >> 5), 1056);
                    zc[b] = get(reinterpret_cast<const uint32_t *>(zc_at));
                    ze[b] = get(ze_at);
                    zc_at += kSlopeRows * p.z_pitch;
                    ze_at += kSlopeRows * p.z_exps_pitch;
                }
            }
#pragma unroll
            for (int b = 0; b < kCount; ++b) {
                float dz[4] = {__uint_as_float(dy[b].x << 16), __uint_as_float(dy[b].x & 0xffff0000u), __uint_as_float(dy[b].y << 16),
                               __uint_as_float(dy[b].y & 0xffff0000u)};
                if constexpr (kAct != kNoZ) {
                    const float zs = ckpt_scale(ze[b]);
                    float z[4], slope[4];
                    const bool known = kTable && ze[b] - kSlopeFirst < tables;
                    if (!known || p.dscales)
#pragma unroll
                        for (int i = 0; i < 4; ++i) z[i] = zs * static_cast<float>(static_cast<int8_t>(zc[b] >> (8 * i)));
                    if (known) {
                        const float *at = table[kTable ? ze[b] - kSlopeFirst : 0];
#pragma unroll
                        for (int i = 0; i < 4; ++i) slope[i] = at[zc[b] >> (8 * i) & 255];
                    } else {
                        act_slopes<kAct>(z, slope);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (kVector || i < n) dz[i] *= slope[i];   // behind the row's end an exponent may stand for NaN
                    if (p.dscales)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (kVector || i < n) ds[i] = fmaf(dz[i], z[i] - bias[i], ds[i]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) db[i] += dz[i];
                SQ_LINEAR_CHECK(col + 4 <= p.pitch && dz_at == p.dz + (t0 + b * kSlopeRows) * p.pitch + col && dzs_at == p.dzs + (t0 + b * kSlopeRows) * p.pitch + col, 1057);
                if (p.dz) *reinterpret_cast<uint2 *>(dz_at) = make_uint2(to_16x2<false>(dz[0], dz[1]), to_16x2<false>(dz[2], dz[3]));
                if (p.dzs)
                    *reinterpret_cast<uint2 *>(dzs_at) = make_uint2(to_16x2<false>(dz[0] * scale[0], dz[1] * scale[1]),
                                                                    to_16x2<false>(dz[2] * scale[2], dz[3] * scale[3]));
                dz_at += kSlopeRows * p.pitch;
                dzs_at += kSlopeRows * p.pitch;
            }
        };
        for (; t0 + (kSlopeBatch - 1) * kSlopeRows < end; t0 += kSlopeBatch * kSlopeRows) rows(Count<kSlopeBatch>{});
        for (; t0 < end; t0 += kSlopeRows) rows(Count<1>{});
    }
    if (!p.dbias && !p.dscales) return;   // the same for all threads of the launch
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        db[i] += __shfl_xor_sync(0xffffffffu, db[i], 16);
        ds[i] += __shfl_xor_sync(0xffffffffu, ds[i], 16);
    }
    if ((threadIdx.x & 31) < 16)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            part[warp][tx * 4 + i] = db[i];
            part[warp][kSlopeCols + tx * 4 + i] = ds[i];
        }
    __syncthreads();
    const int which = threadIdx.x / kSlopeCols, c = blockIdx.x * kSlopeCols + static_cast<int>(threadIdx.x) % kSlopeCols;
    if (which < 2 && c < p.cout) {
        SQ_LINEAR_CHECK(!p.partial || blockIdx.y < static_cast<unsigned>(p.shares), 1058);
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kRowThreads / 32; ++w) s += part[w][threadIdx.x];
        if (p.partial) p.partial[(static_cast<int64_t>(blockIdx.y) * 2 + which) * p.cout + c] = s;
        else if (which == 0 && p.dbias) p.dbias[c] = s;
        else if (which == 1 && p.dscales) p.dscales[c] = s / get(p.scales + c);
    }
}

static __global__ void __launch_bounds__(kRowThreads) sums_kernel(const __grid_constant__ SlopeArgs p)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x;
    if (i >= 2 * static_cast<int64_t>(p.cout)) return;
    const bool scales = i >= p.cout;
    const int64_t c = scales ? i - p.cout : i;
    if (scales ? !p.dscales : !p.dbias) return;
    float s = 0.0f;
#pragma unroll 8
    for (int r = 0; r < p.shares; ++r) s += get(p.partial + static_cast<int64_t>(r) * 2 * p.cout + i);
    if (scales) p.dscales[c] = s / get(p.scales + c);
    else p.dbias[c] = s;
}

}  // namespace sq
