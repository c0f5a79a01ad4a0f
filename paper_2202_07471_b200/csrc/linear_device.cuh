// Device helpers of the linear operators: codes to 16-bit floats, the 8-bit checkpoint format, activations,
// mbarriers, TMA and tcgen05 wrappers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace sq {

enum { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };
enum CodeKind { kInt4 = 0, kInt8 = 1 };

// Set by a kernel of this file's users that gave up a bounded wait (read and cleared by squant_device_status()).
static __device__ int g_linear_status = 0;

// ---------------------------------------------------------------- checked build
// Built with -DSQUANT_DEBUG_BOUNDS the kernels check the indices that they form into shared memory, tensor memory and the tensors; a failed check is
// counted and its site recorded (read and cleared by squant_debug_violations()).  The regular build compiles the checks away.
static __device__ unsigned g_linear_violations = 0;
static __device__ int g_linear_site = 0;
#ifdef SQUANT_DEBUG_BOUNDS
static __device__ __noinline__ void linear_debug_fail(int site)
{
    atomicAdd(&g_linear_violations, 1u);
    atomicCAS(&g_linear_site, 0, site);
}
#define SQ_LINEAR_CHECK(cond, site) do { if (!(cond)) linear_debug_fail(site); } while (0)
#else
#define SQ_LINEAR_CHECK(cond, site) do {} while (0)
#endif

// ---------------------------------------------------------------- 8-bit checkpoints
//
// 32 consecutive features of a row share a power of two: with a = max|v|, E = max(1, exponent field of a - 6) and
// q = clamp(rint(v * 2^(127 - E)), -127, 127); the value is q * 2^(E - 127).  E = 255 marks a group with an infinity
// or a NaN: its values are NaN.  A power of two costs up to one bit against a scale of absmax / 127, and makes every
// value exact in bfloat16 (seven significant bits), so that the tensor cores read what was stored.
__device__ __forceinline__ uint32_t ckpt_exponent(float absmax)   // absmax: NaN if any value is
{
    const uint32_t field = __float_as_uint(absmax) >> 23;
    return field >= 255u ? 255u : field < 7u ? 1u : field - 6u;
}
__device__ __forceinline__ float ckpt_inverse(uint32_t e)   // 2^(127 - E); 0 for a group that is not finite
{
    return e == 255u ? 0.0f : __uint_as_float((254u - e) << 23);
}
// Codes of four values, the first in the low byte.  The product with a power of two is exact unless it is far below one half;
// adding 1.5 * 2^23 rounds it to an integer, ties to even, whose low byte is the code.  In a group that is not finite the codes are 0.
__device__ __forceinline__ uint32_t ckpt_codes(const float *v, float inverse)
{
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(__fadd_rn(fminf(fmaxf(__fmul_rn(v[i], inverse), -127.0f), 127.0f), 12582912.0f));
    const uint32_t w = __byte_perm(__byte_perm(u[0], u[1], 0x0040), __byte_perm(u[2], u[3], 0x0040), 0x5410);
    return inverse == 0.0f ? 0u : w;
}
__device__ __forceinline__ float ckpt_scale(uint32_t e) { return __uint_as_float(e << 23); }   // 255: inf, 0 * inf = NaN
// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// ---------------------------------------------------------------- activations (fp32)

// Two fp32 operations in one instruction.
struct Two {
    uint64_t v;
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit Two(uint64_t u) : v(u) {}
    __device__ __forceinline__ void get(float &a, float &b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ Two fma(Two a, Two b, Two c)
{
    Two r(0ull);
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Two mul(Two a, Two b)
{
    Two r(0ull);
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

// P(N(0, 1) < z) of two values and e = exp(-z^2 / 2).  With a = |z| the upper tail is e times a polynomial in u = 1 / (1 + 0.3 a)
// without a constant term, since exp(a^2 / 2) P falls like 1 / a.  The coefficients are a weighted least-squares fit of
// erfcx(a / sqrt 2) / 2 over [0, 14], at most 1.7e-7 of the value off with these coefficients; beyond, the value is no normal fp32 number.
// The tail is off by that and by what the rounding of -z^2 / 2 and expf's argument makes of e, which grows with it: 9e-7 of itself up to |z| = 4, 2e-6
// up to 6, 8e-6 up to 13, and expf's own last places; 1 + erf(z / sqrt 2) would keep no digit of it there.  gelu and its slope share e.  Two values at a
// time take 23 instructions, erfcf() and expf() of both about 180.
__device__ __forceinline__ void normal_below(float z0, float z1, float &p0, float &p1, float &e0, float &e1)
{
    float x0, x1, d0, d1, h0, h1;
    const Two z(z0, z1), half(-0.5f, -0.5f);
    mul(mul(z, half), z).get(x0, x1);
    e0 = __expf(x0);
    e1 = __expf(x1);
    fma(Two(fabsf(z0), fabsf(z1)), Two(0.3f, 0.3f), Two(1.0f, 1.0f)).get(d0, d1);
    const Two u(__fdividef(1.0f, d0), __fdividef(1.0f, d1));
    Two q(0.03567597f, 0.03567597f);
    q = fma(q, u, Two(-0.15720823f, -0.15720823f));
    q = fma(q, u, Two(0.20636259f, 0.20636259f));
    q = fma(q, u, Two(-0.05369217f, -0.05369217f));
    q = fma(q, u, Two(0.1285662f, 0.1285662f));
    q = fma(q, u, Two(0.0999121f, 0.0999121f));
    q = fma(q, u, Two(0.12075418f, 0.12075418f));
    q = fma(q, u, Two(0.11962928f, 0.11962928f));
    mul(mul(q, u), Two(e0, e1)).get(h0, h1);
    p0 = z0 < 0.0f ? h0 : 1.0f - h0;
    p1 = z1 < 0.0f ? h1 : 1.0f - h1;
}
// 0 from z = -87.3 on, where 1 + exp(-z) is more than the division takes and the value less than 1.2e-38.
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

// act(v) of all values: one branch for all.
template <int kCount>
__device__ __forceinline__ void act_values(float (&v)[kCount], int act)
{
    if (act == kActRelu) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];   // keeps a NaN
    } else if (act == kActGelu) {
#pragma unroll
        for (int i = 0; i < kCount; i += 2) {
            float p0, p1, e0, e1;
            normal_below(v[i], v[i + 1], p0, p1, e0, e1);
            v[i] *= p0;
            v[i + 1] *= p1;
        }
    } else if (act == kActSilu) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) v[i] *= sigmoid(v[i]);
    }
}
__device__ __forceinline__ float act_value(float z, int act)
{
    float v[2] = {z, z};
    act_values(v, act);
    return v[0];
}
// act'(z)
template <int kAct, int kCount>
__device__ __forceinline__ void act_slopes(const float (&z)[kCount], float (&slope)[kCount])
{
#pragma unroll
    for (int i = 0; i < kCount; i += 2) {
        if constexpr (kAct == kActGelu) {
            float p0, p1, e0, e1;
            normal_below(z[i], z[i + 1], p0, p1, e0, e1);
            slope[i] = fmaf(z[i] * 0.39894228040143268f, e0, p0);
            slope[i + 1] = fmaf(z[i + 1] * 0.39894228040143268f, e1, p1);
        } else {
#pragma unroll
            for (int j = i; j < i + 2; ++j) {
                const float p = kAct == kActSilu ? sigmoid(z[j]) : 0.0f;
                slope[j] = kAct == kActSilu ? p * fmaf(z[j], 1.0f - p, 1.0f) : kAct == kActRelu ? (z[j] > 0.0f ? 1.0f : 0.0f) : 1.0f;
            }
        }
    }
}

// ---------------------------------------------------------------- 16-bit types

template <bool kHalf>
__device__ __forceinline__ float to_float(uint16_t v)
{
    if constexpr (kHalf) return __half2float(__ushort_as_half(v));
    else return __uint_as_float(static_cast<uint32_t>(v) << 16);
}
template <bool kHalf>
__device__ __forceinline__ uint16_t to_16(float v)
{
    if constexpr (kHalf) return __half_as_ushort(__float2half_rn(v));
    else return __bfloat16_as_ushort(__float2bfloat16_rn(v));
}
template <bool kHalf>
__device__ __forceinline__ uint32_t to_16x2(float lo, float hi)
{
    if constexpr (kHalf) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
}

template <bool kHalf>
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    if constexpr (kHalf) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    else asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t sub2_bf16(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t mul2_bf16(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Eight int4 codes (low nibble first) to four pairs of 16-bit floats, exactly.  A code's nibble n, its sign bit
// flipped, becomes the low mantissa bits of 128 (bf16) or 1024 (fp16), which gives 128 + n + 8; the odd codes' nibbles
// sit three bits further up (the word shifted by one), which gives 128 + 8 (n + 8).  One fused multiply-add on the
// pair takes the offsets off and divides the odd code by 8: three instructions a pair and one shift a word.  The constants come from
// registers that the compiler cannot see through: known ones it writes into the instructions, which hold one each, and
// takes five instructions a pair.
template <bool kHalf>
struct Int4To16 {
    uint32_t mask, flip, factor, offset;
    __device__ __forceinline__ Int4To16()
    {
        asm volatile("mov.b32 %0, 0x0078000f;" : "=r"(mask));
        asm volatile("mov.b32 %0, %1;" : "=r"(flip) : "n"(kHalf ? 0x64406408u : 0x43404308u));
        asm volatile("mov.b32 %0, %1;" : "=r"(factor) : "n"(kHalf ? 0x30003c00u : 0x3e003f80u));   // (1, 1/8), low half first
        asm volatile("mov.b32 %0, %1;" : "=r"(offset) : "n"(kHalf ? 0xd840e408u : 0xc1c0c308u));   // fp16 (-1032, -136), bf16 (-136, -24)
    }
    __device__ __forceinline__ void operator()(uint32_t w, uint32_t out[4]) const
    {
        const uint32_t s = w >> 1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t v = __byte_perm(w, s, 0x0400u | (0x0101u * j));   // byte 0: w's byte j, byte 2: s's byte j
            uint32_t u;
            asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(u) : "r"(v), "r"(mask), "r"(flip));   // (v & mask) ^ flip
            out[j] = fma2<kHalf>(u, factor, offset);
        }
    }
};

// Four int8 codes to two pairs of 16-bit floats, exactly.  bf16 has seven mantissa bits: the low seven bits L of a
// byte give 128 + L, its sign bit S gives 128 + 128 S as exponent bit; the difference is L - 128 S.
template <bool kHalf>
__device__ __forceinline__ void int8_to_16(uint32_t w, uint32_t out[2])
{
    if constexpr (kHalf) {
        const uint32_t u = w ^ 0x80808080u;                              // 1024 + (code + 128)
        out[0] = fma2<true>(__byte_perm(u, 0x64u, 0x4140), 0x3c003c00u, 0xe480e480u);
        out[1] = fma2<true>(__byte_perm(u, 0x64u, 0x4342), 0x3c003c00u, 0xe480e480u);
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t h = __byte_perm(w, 0x43u, j ? 0x4342 : 0x4140);
            out[j] = sub2_bf16(h & 0xff7fff7fu, h & 0xff80ff80u);
        }
    }
}

// ---------------------------------------------------------------- loads

// Not read-only (.nc): the residual may be the output.
template <typename T>
__device__ __forceinline__ T get(const T *p) { return *p; }

__device__ __forceinline__ uint4 ldg128(const void *p)
{
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// 16 bytes from any address: five aligned words, shifted.  Words that are not wholly inside [lo, hi) are put
// together from the bytes that are; other bytes read as zero.
static __device__ __noinline__ uint4 load_bytes16(const uint8_t *p, const uint8_t *lo, const uint8_t *hi)
{
    const uint8_t *a = reinterpret_cast<const uint8_t *>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t{3});
    const unsigned sh = static_cast<unsigned>(reinterpret_cast<uintptr_t>(p) & 3) * 8;
    uint32_t w[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const uint8_t *q = a + 4 * i;
        if (q >= lo && q + 4 <= hi) {
            SQ_LINEAR_CHECK((reinterpret_cast<uintptr_t>(q) & 3) == 0, 1000);
            w[i] = get(reinterpret_cast<const uint32_t *>(q));
        } else {
            uint32_t v = 0;
            for (int b = 0; b < 4; ++b)
                if (q + b >= lo && q + b < hi) v |= static_cast<uint32_t>(get(q + b)) << (8 * b);
            w[i] = v;
        }
    }
    return make_uint4(__funnelshift_r(w[0], w[1], sh), __funnelshift_r(w[1], w[2], sh), __funnelshift_r(w[2], w[3], sh),
                      __funnelshift_r(w[3], w[4], sh));
}

// ---------------------------------------------------------------- mbarriers, TMA, tcgen05

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// End of the block's dynamic shared memory, which starts at `from`.
__device__ __forceinline__ uint32_t smem_end(const void *from)
{
    uint32_t bytes;
    asm("mov.u32 %0, %%dynamic_smem_size;" : "=r"(bytes));
    return smem_addr(from) + bytes;
}

// True for one lane of a converged warp, always the same one.  The compiler knows that there is one: under a comparison
// of the lane's number instead, copies and matrix instructions, whose operands are uniform registers, cost several times the issue time.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Tries of a wait.  The hardware parks a try for 4 us before it fails (4,096 tries: 16.5 ms), so that a wait gives up after a second.  The longest
// one that goes well is for a tile's sums, at most kLongestSum terms of a contraction: below a millisecond.
constexpr int kWaitLimit = 1 << 18;
#ifdef SQUANT_DEBUG_BOUNDS
static __device__ int g_wait_limit = kWaitLimit;   // tests of the checked build shorten it
__device__ __forceinline__ int wait_limit() { return *const_cast<volatile int *>(&g_wait_limit); }
#else
__device__ __forceinline__ int wait_limit() { return kWaitLimit; }
#endif

// False when the wait ran out or another thread of the block gave up (*gave_up is shared by the block).
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *gave_up, int limit = wait_limit())
{
    for (int i = 0; i < limit; ++i) {
        if (bar_try(bar, parity)) return true;
        if (*gave_up) return false;
    }
    *gave_up = 1;
    atomicExch(&g_linear_status, 1);
    return false;
}
// The same for a whole warp, which goes on or gives up together.
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, volatile int *gave_up)
{
    return __all_sync(0xffffffffu, bar_wait(bar, parity, gave_up));
}
// A wait on its own, at a barrier that nobody arrives at.
static __global__ void wait_kernel(int limit)
{
    __shared__ uint64_t bar;
    __shared__ int gave_up;
    if (threadIdx.x == 0) {
        gave_up = 0;
        bar_init(smem_addr(&bar), 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) bar_wait(smem_addr(&bar), 0, &gave_up, limit);
}
// The wait for one's own copies after the block has given up: bounded (16 ms), without a look at the flag.
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity)
{
    for (int i = 0; i < (1 << 12); ++i)
        if (bar_try(bar, parity)) return;
}

__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_ranks()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive_wait()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle.  A panel has rows of 64 16-bit elements (128 bytes), its eight
// 16-byte pieces permuted by the row's low three bits; eight rows are 1024 bytes.
//   contraction along the rows' 64 elements ("K-major"): 1024 bytes between groups of eight rows; the next 16 elements
//   of the contraction are 32 bytes on
//   contraction over the rows ("MN-major"): the panel's 64 elements are 64 columns of the tile, `panel` bytes to the
//   next 64; 1024 bytes between groups of eight rows, 16 of which a matrix instruction takes: the next start 2048 on
// The low word holds the address and the leading distance in 16 bytes (so 16 bytes further is one more); the high word is the
// same for all: 1024 bytes between groups, version 1, swizzle mode 2.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t leading) { return ((addr & 0x3ffffu) >> 4) | ((leading >> 4) << 16); }

__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

__device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns));
}
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// a, b: low words of the operands' descriptors
__device__ __forceinline__ void mma_f16(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)), "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

}  // namespace sq
