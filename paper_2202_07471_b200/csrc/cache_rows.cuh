// Keys and values into the cache and back.
#pragma once

#include <type_traits>

#include "cache_device.cuh"

namespace sq {

struct MoveArgs {
    uint8_t *cache;
    CacheRows r;
    uint16_t *k, *v;               // read: written
    int64_t k_stride, k_head, v_stride, v_head;   // elements from row to row and from head to head
    int32_t vector;                // all rows of k and v start on 16 bytes
    int32_t blocks;                // of heads, kMoveHeads each
};

constexpr int kMoveThreads = 256;
constexpr int kMoveLoads = 4;      // 16-byte pieces of k or v that a lane has in flight
// Heads of a row that a warp takes: a lane has 8 channels of a head's key or value at a time.
template <int D>
constexpr int kMoveHeads = kMoveLoads * 128 / D;

// Lane's i-th piece: (head of the block, key or value, word).
template <int D>
struct Piece {
    int head, word;
    bool value;
    __device__ __forceinline__ explicit Piece(int i)
    {
        const int at = i * 32 + (threadIdx.x & 31);
        word = at % (D / 8);
        value = at / (D / 8) % 2;
        head = at / (D / 4);
    }
};

// Where a row is in the cache: its granules (of head 0) and its place in one, or null.
struct Place {
    uint8_t *granule;
    int t;
};
template <int D>
__device__ __forceinline__ Place place_of(const MoveArgs &p, int64_t row, int &b, int64_t &position)
{
    b = sequence_of(p.r, row);
    position = -1;
    if (b < 0) return {nullptr, 0};
    const int64_t last = p.r.starts ? row_start(p.r, b + 1) : row + 1;
    position = length_of(p.r, b) - (last - row);
    if (position < 0) return {nullptr, 0};
    const int column = static_cast<int>(position) / p.r.page_size, in = static_cast<int>(position) - column * p.r.page_size;
    const int64_t page = page_of(p.r, b, column);
    if (page < 0) return {nullptr, 0};
    const int granules = p.r.page_size / kGranule;
    return {p.cache + (page * p.r.kv_heads * granules + in / kGranule) * CacheFormat<D>::kBytes, in % kGranule};
}

// A warp quantizes kMoveHeads heads of a row: the loads of keys and values, which no position is needed for, are in flight while it looks up where
// the row belongs.  Four lanes hold the channels that share a scale.  x / s is rounded from a product with the reciprocal that is corrected by its remainder
// (an fma yields it exactly), so that a quotient of exactly one half, the only one that matters, is one.
template <int D, bool kHalf>
__global__ void __launch_bounds__(kMoveThreads)
cache_write_kernel(const __grid_constant__ MoveArgs p)
{
    using F = CacheFormat<D>;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kMoveThreads / 32) + (threadIdx.x >> 5);
    const int64_t row = unit / p.blocks;
    const int head0 = static_cast<int>(unit % p.blocks) * kMoveHeads<D>;
    if (row >= p.r.rows) return;
    uint4 x[kMoveLoads];
    const auto load = [&](auto on_vectors) {
#pragma unroll
        for (int i = 0; i < kMoveLoads; ++i) {
            const Piece<D> at(i);
            const int head = head0 + at.head;
            x[i] = make_uint4(0, 0, 0, 0);
            if (head < p.r.kv_heads)
                x[i] = load8(at.value ? p.v + row * p.v_stride + head * p.v_head + 8 * at.word : p.k + row * p.k_stride + head * p.k_head + 8 * at.word,
                             decltype(on_vectors)::value);
        }
    };
    if (p.vector) load(std::true_type{});
    else load(std::false_type{});
    int b;
    int64_t position;
    const Place to = place_of<D>(p, row, b, position);
    if (!to.granule) return;
    const int64_t head_bytes = static_cast<int64_t>(p.r.page_size / kGranule) * F::kBytes;
#pragma unroll
    for (int i = 0; i < kMoveLoads; ++i) {
        const Piece<D> at(i);
        const int head = head0 + at.head;
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        float f[8], top = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f[e] = to_float<kHalf>(static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1))));
            top = max_nan(top, fabsf(f[e]));
        }
        top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // to four significant bits, ties to even; whether a quotient is a tie shows in fp32
        const uint32_t bits = __float_as_uint(__fdiv_rn(top, 7.0f));
        float scale = __uint_as_float((bits + 0x7ffffu + (bits >> 20 & 1)) & ~0xfffffu);
        uint32_t word = 0;
        if (top < kScaleLeast) {
            scale = 0.0f;
        } else if (!(top < kScaleMost)) {
            scale = __uint_as_float(0x7f800000u);
        } else {
            const float inverse = __frcp_rn(scale);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = __fmul_rn(f[e], inverse);
                const float quotient = fmaf(fmaf(-q, scale, f[e]), inverse, q);
                word |= (__float_as_uint(__fadd_rn(quotient, 12582912.0f)) & 15u) << (4 * (e >> 1) + 16 * (e & 1));   // 1.5 * 2^23: rounded to an integer, ties to even
            }
        }
        if (head < p.r.kv_heads) {
            uint8_t *granule = to.granule + head * head_bytes;
            SQ_LINEAR_CHECK(granule >= p.cache && granule + F::kBytes <= p.cache + p.r.page_count * p.r.kv_heads * head_bytes, 2000);
            *reinterpret_cast<uint32_t *>(granule + (at.value ? F::value_word(to.t, at.word) : F::key_word(to.t, at.word))) = word;
            if (at.word % 4 == 0)
                *reinterpret_cast<uint16_t *>(granule + (at.value ? F::value_scale(to.t, at.word / 4) : F::key_scale(to.t, at.word / 4))) =
                    static_cast<uint16_t>(__float_as_uint(scale) >> 16);
        }
    }
}

// Zeros for rows that are in a sequence but before its first position, or in a page that is not there; rows in no sequence stay as they are.
template <int D, bool kHalf>
__global__ void __launch_bounds__(kMoveThreads)
cache_read_kernel(const __grid_constant__ MoveArgs p)
{
    using F = CacheFormat<D>;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kMoveThreads / 32) + (threadIdx.x >> 5);
    const int64_t row = unit / p.blocks;
    const int head0 = static_cast<int>(unit % p.blocks) * kMoveHeads<D>;
    if (row >= p.r.rows) return;
    int b;
    int64_t position;
    const Place from = place_of<D>(p, row, b, position);
    if (b < 0) return;
    const int64_t head_bytes = static_cast<int64_t>(p.r.page_size / kGranule) * F::kBytes;
    uint32_t word[kMoveLoads], scale[kMoveLoads];
#pragma unroll
    for (int i = 0; i < kMoveLoads; ++i) {
        const Piece<D> at(i);
        const int head = head0 + at.head;
        word[i] = scale[i] = 0;
        if (from.granule && head < p.r.kv_heads) {
            const uint8_t *granule = from.granule + head * head_bytes;
            SQ_LINEAR_CHECK(granule >= p.cache && granule + F::kBytes <= p.cache + p.r.page_count * p.r.kv_heads * head_bytes, 2001);
            word[i] = *reinterpret_cast<const uint32_t *>(granule + (at.value ? F::value_word(from.t, at.word) : F::key_word(from.t, at.word)));
            scale[i] = *reinterpret_cast<const uint16_t *>(granule + (at.value ? F::value_scale(from.t, at.word / 4) : F::key_scale(from.t, at.word / 4)));
        }
    }
    const CodePairs<kHalf> pairs;
#pragma unroll
    for (int i = 0; i < kMoveLoads; ++i) {
        const Piece<D> at(i);
        const int head = head0 + at.head;
        if (head >= p.r.kv_heads) continue;
        const uint32_t s = scale_twice<kHalf>(scale[i], false);
        uint32_t out[4];
        pairs(word[i], pairs.scales(s), out);
        uint16_t *to = at.value ? p.v + row * p.v_stride + head * p.v_head + 8 * at.word : p.k + row * p.k_stride + head * p.k_head + 8 * at.word;
        if (p.vector) {
            *reinterpret_cast<uint4 *>(to) = make_uint4(out[0], out[1], out[2], out[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) to[e] = static_cast<uint16_t>(out[e / 2] >> (16 * (e & 1)));
        }
    }
}

}  // namespace sq
