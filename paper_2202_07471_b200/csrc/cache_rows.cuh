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
    __device__ __forceinline__ explicit Piece(unsigned i)
    {
        const unsigned at = i * 32 + (threadIdx.x & 31);
        word = static_cast<int>(at % (D / 8));
        value = at / (D / 8) % 2;
        head = static_cast<int>(at / (D / 4));
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

// The larger of two magnitudes in each half, NaN if either is one.
template <bool kHalf>
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b)
{
    uint32_t r;
    if constexpr (kHalf) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The scale of a group whose largest magnitude is `top` (at most 11 significant bits): top / 7, correctly rounded by the remainder of a product with the
// reciprocal (an fma yields it exactly; to 24 bits, so that a tie between two scales shows), then to four significant bits, ties to even.
__device__ __forceinline__ float group_scale(float top)
{
    if (top < kScaleLeast) return 0.0f;
    if (!(top < kScaleMost)) return __uint_as_float(0x7f800000u);
    const float q = __fmul_rn(top, 1.0f / 7.0f);
    const uint32_t bits = __float_as_uint(fmaf(fmaf(-q, 7.0f, top), 1.0f / 7.0f, q));
    return __uint_as_float((bits + 0x7ffffu + (bits >> 20 & 1)) & ~0xfffffu);
}
// Codes of 8 values, two values an instruction.  x / s comes from a product with the reciprocal that is corrected by its remainder: whatever the reciprocal's last bits, a
// quotient of k + 1/2, the only one that matters, comes out as such.  Adding 1.5 * 2^23 and taking it off rounds to an integer, ties to even; the integers, as digits of 16, make the
// halves of a word, with 8 added to each (0x8888) so that none is negative, which the last step takes off.
template <bool kHalf>
__device__ __forceinline__ uint32_t group_codes(const uint32_t (&w)[4], float scale)
{
    if (!(scale > 0.0f && scale < __uint_as_float(0x7f800000u))) return 0;
    float inverse;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(scale));
    const Two by(inverse, inverse), minus(-scale, -scale), up(12582912.0f, 12582912.0f), down(-12582912.0f, -12582912.0f), digit(16.0f, 16.0f);
    Two sum(0.0f, 0.0f);
#pragma unroll
    for (int p = 3; p >= 0; --p) {
        const Two x(to_float<kHalf>(static_cast<uint16_t>(w[p])), to_float<kHalf>(static_cast<uint16_t>(w[p] >> 16)));
        const Two q = mul(x, by);
        const Two rounded = add(add(fma(fma(q, minus, x), by, q), up), down);
        sum = p == 3 ? rounded : fma(sum, digit, rounded);
    }
    float low, high;
    add(sum, Two(8388608.0f + 34952.0f, 8388608.0f + 34952.0f)).get(low, high);   // 2^23 and 0x8888: the low 16 bits
    return __byte_perm(__float_as_uint(low), __float_as_uint(high), 0x5410) ^ 0x88888888u;
}

// A warp quantizes kMoveHeads heads of a row: the loads of keys and values, which no position is needed for, are in flight while it looks up where
// the row belongs.  Four lanes hold the channels that share a scale.  Instructions bound it next to the bytes: 29,656 rows of 8 heads of 128
// channels took 68 us with 31 instructions a value (83 % of the issue slots), and take 57 with two values an instruction, magnitudes compared in 16 bits and rows and heads
// that need no division; the bytes alone are 21 us.
template <int D, bool kHalf>
__global__ void __launch_bounds__(kMoveThreads)
cache_write_kernel(const __grid_constant__ MoveArgs p)
{
    using F = CacheFormat<D>;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kMoveThreads / 32) + (threadIdx.x >> 5);
    const int head0 = static_cast<int>(blockIdx.y) * kMoveHeads<D>;
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
        uint32_t both = larger2<kHalf>(larger2<kHalf>(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), larger2<kHalf>(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
        both = larger2<kHalf>(both, __shfl_xor_sync(0xffffffffu, both, 1));
        both = larger2<kHalf>(both, __shfl_xor_sync(0xffffffffu, both, 2));
        const float scale = group_scale(max_nan(to_float<kHalf>(static_cast<uint16_t>(both)), to_float<kHalf>(static_cast<uint16_t>(both >> 16))));
        const uint32_t word = group_codes<kHalf>(w, scale);
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

// As many lanes as in the write, a word of codes and 16 bytes of results each: 53,488 rows of 8 heads of 128 channels 59 us, 4.7 TB/s of what has to be
// moved; 64 in fp16, whose values are rounded once at every magnitude (59 with the scale rounded first; 63 with a vote on which of the two a warp's scales want).
// Zeros for rows that are in a sequence but before its first position, or in a page that is not there; rows in no sequence stay as they are.
template <int D, bool kHalf>
__global__ void __launch_bounds__(kMoveThreads)
cache_read_kernel(const __grid_constant__ MoveArgs p)
{
    using F = CacheFormat<D>;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kMoveThreads / 32) + (threadIdx.x >> 5);
    const int head0 = static_cast<int>(blockIdx.y) * kMoveHeads<D>;
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
        uint32_t out[4];
        pairs.rounded_once(word[i], scale[i], out);
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
