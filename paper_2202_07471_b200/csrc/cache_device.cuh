// A key/value cache held in 4 bits: its format, and what the kernels that write, read and attend to it share.
//
// The cache is made of granules: 16 positions of one page and one kv head, 18 * d bytes (d channels: 64, 128 or 256).  32 neighbouring channels of a
// position's key or value share a scale s, the largest magnitude over 7 rounded to four significant bits (ties to even); the code of x is rint(x / s), which is
// never outside -7..7 since s is at most 1/17 too small (7.44 steps at 8.5 rounded down to 8).  A value, code * s, has three bits times four and is exact in bf16, so that
// everything that reads the cache sees the same numbers.
//   0       codes of the keys    [slab][position][word % 4][word / 4]      a word: 8 codes of neighbouring channels, 32 bits; a slab: 128 channels (64)
//   8 d     codes of the values  [slab][position / 2][word % 8][position % 2][word / 8]
//   16 d    scales of the keys   [position][group], bf16
//   17 d    scales of the values [slab][position / 2][group % 2][group / 2][position % 2], bf16
// The orders are those in which the lanes of a warp hold the operands of a matrix instruction: a lane reads 16 bytes at a time, neighbouring lanes
// neighbouring ones.  Code e of a word is in bits 4 * (e / 2) + 16 * (e % 2), so that one shift and one mask yield a pair of neighbours in the halves of a register.
#pragma once

#include "linear_device.cuh"

namespace sq {

constexpr int kGranule = 16;            // positions
constexpr int kGroup = 32;              // channels that share a scale
constexpr float kScaleLeast = 7.888609052210118e-31f;   // 2^-100: smaller groups are zeros
constexpr float kScaleMost = 1.329227995784916e36f;     // 2^120: from here on, and for infinities and NaN, the group's values are NaN

template <int D>
struct CacheFormat {
    static_assert(D == 64 || D == 128 || D == 256, "head dimensions");
    static constexpr int kBytes = 18 * D;
    static constexpr int kSlabs = D > 128 ? D / 128 : 1, kSlab = D / kSlabs;
    static constexpr int kWords = kSlab / 8, kGroups = kSlab / kGroup;    // of a position and slab
    static constexpr int kKeyScales = 16 * D, kValues = 8 * D, kValueScales = 17 * D;
    // bytes from the granule's start; word, group: over all slabs
    __host__ __device__ static constexpr int key_word(int t, int word)
    {
        return 4 * (word / kWords * 16 * kWords + t * kWords + word % 4 * (kWords / 4) + word % kWords / 4);
    }
    __host__ __device__ static constexpr int value_word(int t, int word)
    {
        return kValues + 4 * (word / kWords * 16 * kWords + (t >> 1) * 2 * kWords + word % 8 * (kWords / 4) + (t & 1) * (kWords / 8) + word % kWords / 8);
    }
    __host__ __device__ static constexpr int key_scale(int t, int group) { return kKeyScales + 2 * (t * (D / kGroup) + group); }
    __host__ __device__ static constexpr int value_scale(int t, int group)
    {
        return kValueScales + 2 * (group / kGroups * 16 * kGroups + (t >> 1) * 2 * kGroups + group % 2 * kGroups + group % kGroups / 2 * 2 + (t & 1));
    }
};

// Where rows of keys, values or queries belong: rows starts[b] .. starts[b + 1] are the last positions of sequence b, of lens[b] in all.  Nothing that the
// arrays hold leads outside the tensors: lengths are cut to what the page table's rows cover, rows to those there are, and pages outside the cache count as not there.
struct CacheRows {
    const int32_t *lens, *pages, *starts;   // starts: null: row b is the last position of sequence b
    int64_t pages_stride;
    int32_t batch, width, page_size, kv_heads;
    int64_t page_count, rows;
};
__device__ __forceinline__ int64_t row_start(const CacheRows &r, int64_t b)
{
    if (!r.starts) return b;
    return max(static_cast<int64_t>(0), min(r.rows, static_cast<int64_t>(r.starts[b])));
}
__device__ __forceinline__ int length_of(const CacheRows &r, int64_t b)
{
    const int64_t most = min(static_cast<int64_t>(r.width) * r.page_size, static_cast<int64_t>(1) << 30);
    return static_cast<int>(max(static_cast<int64_t>(0), min(most, static_cast<int64_t>(r.lens[b]))));
}
// The page, or -1.
__device__ __forceinline__ int64_t page_of(const CacheRows &r, int64_t b, int column)
{
    const int32_t p = r.pages[b * r.pages_stride + column];
    return p >= 0 && p < r.page_count ? p : -1;
}
// The sequence that a row belongs to, or -1; the same row in all lanes of a warp.  Each round of loads leaves a 32nd of the sequences.
__device__ __forceinline__ int sequence_of(const CacheRows &r, int64_t row)
{
    if (!r.starts) return row < r.batch ? static_cast<int>(row) : -1;
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = r.batch;   // starts[lo] <= row < starts[hi], if it is in any
    while (hi - lo > 1) {
        const int stride = (hi - lo + 31) / 32, at = lo + (lane + 1) * stride;
        const unsigned below = __ballot_sync(0xffffffffu, at < hi && row_start(r, at) <= row);
        const int n = __popc(below);
        const int next = lo + n * stride;
        hi = min(hi, next + stride);
        lo = next;
    }
    return row >= row_start(r, lo) && row < row_start(r, lo + 1) ? lo : -1;
}

// ---------------------------------------------------------------- codes to floats

// The halves of a register, both or one of them twice.
__device__ __forceinline__ uint32_t half_twice(uint32_t two, bool high)
{
    uint32_t r;
    if (high) asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tmov.b32 %0, {h, h};\n\t}" : "=r"(r) : "r"(two));
    else asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tmov.b32 %0, {l, l};\n\t}" : "=r"(r) : "r"(two));
    return r;
}

// What the conversion of a word wants of its scales (both halves in the values' type).
template <bool kHalf>
struct PairScales {
    uint32_t scale, other, eight;   // s; bf16: -136 s, 8 s
};

// A word's (or two half words') codes, pair p of them in bits 4 p of both halves, times the pair's scales.  The integer pipe, which shifts and masks, has half the
// rate of the one that multiplies, and is what the conversion is bound by: so pairs are taken out where they lie, with one shift a word.
//   bf16  pairs 0 and 2 (after the shift): the bits of code + 8 become the low mantissa bits of 128, and one multiply-add by s takes 136 s off, exactly (five bits
//         times four).  Pairs 1 and 3 lie in bits 4 to 7, the upper three of the mantissa and the lowest of the exponent: with all other bits zero that is a number
//         near the smallest there is, 16 (code + 8) 2^-133, which a multiply-add makes code / 8, and a product with 8 s the value.
//   fp16  the mantissa holds bits 4 to 7 too: 1024 + 8 + code, and 1024 + 16 (code + 8) = 1152 + 16 code; taking 1032 off, and 1152 (over 16), leaves the code.  No
//         offset times a scale here, for which large scales leave no room.
template <bool kHalf>
struct CodePairs {
    uint32_t mask, flip, mask_high, flip_high;
    __device__ __forceinline__ CodePairs()
    {
        // from registers that the compiler cannot see through, see Int4To16
        asm volatile("mov.b32 %0, 0x000f000f;" : "=r"(mask));
        asm volatile("mov.b32 %0, %1;" : "=r"(flip) : "n"(kHalf ? 0x64086408u : 0x43084308u));
        asm volatile("mov.b32 %0, 0x00f000f0;" : "=r"(mask_high));
        asm volatile("mov.b32 %0, %1;" : "=r"(flip_high) : "n"(kHalf ? 0x64806480u : 0x00800080u));
    }
    static __device__ __forceinline__ PairScales<kHalf> scales(uint32_t s)
    {
        PairScales<kHalf> r;
        r.scale = s;
        if constexpr (kHalf) {
            r.other = r.eight = 0;   // not used
        } else {
            r.other = mul2_bf16(s, 0xc308c308u);   // -136
            r.eight = mul2_bf16(s, 0x41004100u);   // 8
        }
        return r;
    }
    // The halves of pair p as described, before arithmetic; upper: w >> 8.
    __device__ __forceinline__ uint32_t bits(uint32_t w, uint32_t upper, int p) const
    {
        const uint32_t from = p < 2 ? w : upper;
        uint32_t u;
        if (p & 1) asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(u) : "r"(from), "r"(mask_high), "r"(flip_high));   // (from & mask) ^ flip
        else asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(u) : "r"(from), "r"(mask), "r"(flip));
        return u;
    }
    __device__ __forceinline__ void operator()(uint32_t w, const PairScales<kHalf> &s, uint32_t (&out)[4]) const
    {
        const uint32_t upper = w >> 8;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            uint32_t u = bits(w, upper, p);
            if constexpr (kHalf) {
                u = p & 1 ? fma2<true>(u, 0x2c002c00u, 0xd480d480u) : fma2<true>(u, 0x3c003c00u, 0xe408e408u);   // u / 16 - 72, u - 1032
                asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(out[p]) : "r"(u), "r"(s.scale));
            } else if (p & 1) {
                out[p] = mul2_bf16(fma2<false>(u, 0x7e807e80u, 0xbf80bf80u), s.eight);   // u 2^126 - 1
            } else {
                out[p] = fma2<false>(u, s.scale, s.other);
            }
        }
    }
    // A word's values, rounded to nearest once whatever the scale is.  In fp16 a scale below 2^-21 loses bits and one from 2^16 on is infinite, though its products with
    // codes may be numbers; so the codes are taken 2^-12 (2) times as large, exactly, and the scale 2^12 (1/2) times, where it is a number of four bits: below 2^-33
    // it is not, but then all values are rounded to 0, and from 2^17 on any number makes infinities of codes other than 0.  The operator above takes the scale as fp16 holds it.
    __device__ __forceinline__ void rounded_once(uint32_t w, uint32_t scale, uint32_t (&out)[4]) const
    {
        if constexpr (kHalf) {
            const float s = __uint_as_float(scale << 16);
            const bool small = s < 0.00390625f;
            const float moved = small ? s * 4096.0f : s * 0.5f, held = s < __uint_as_float(0x7f800000u) ? fminf(moved, 65504.0f) : s;
            const uint32_t k = to_16x2<true>(held, held), upper = w >> 8;
            const uint32_t even = small ? 0x0c000c00u : 0x40004000u, even_less = small ? 0xb408b408u : 0xe808e808u;   // 2^-12 and 2, -1032 times that
            const uint32_t odd = small ? 0x01000100u : 0x30003000u, odd_less = small ? 0xa480a480u : 0xd880d880u;     // a sixteenth of that, -72 times it
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t u = bits(w, upper, p), code = p & 1 ? fma2<true>(u, odd, odd_less) : fma2<true>(u, even, even_less);
                asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(out[p]) : "r"(code), "r"(k));
            }
        } else {
            (*this)(w, scales(half_twice(scale, false)), out);
        }
    }
};
// The same scale in both halves; `two` holds two bf16 scales, `high` says which.
template <bool kHalf>
__device__ __forceinline__ uint32_t scale_twice(uint32_t two, bool high)
{
    if constexpr (kHalf) {
        const float s = __uint_as_float(high ? two & 0xffff0000u : two << 16);
        return to_16x2<true>(s, s);
    } else {
        return half_twice(two, high);
    }
}
// Two bf16 scales in the values' type.
template <bool kHalf>
__device__ __forceinline__ uint32_t scale_pair(uint32_t two)
{
    if constexpr (kHalf) return to_16x2<true>(__uint_as_float(two << 16), __uint_as_float(two & 0xffff0000u));
    else return two;
}

// ---------------------------------------------------------------- copies, arithmetic

// A contiguous copy into shared memory; 16-byte addresses and sizes.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ Two add(Two a, Two b)
{
    Two r(0ull);
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// 8 values of 16 bits from any 2-byte address.
__device__ __forceinline__ uint4 load8(const uint16_t *p, bool vector)
{
    if (vector) return *reinterpret_cast<const uint4 *>(p);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = get(p + 2 * i) | static_cast<uint32_t>(get(p + 2 * i + 1)) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace sq
