// Host side of the key/value cache's operators: validation, choice of kernels, launches (C ABI of include/squant.h).
#include "squant.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <random>

#include "cache_device.cuh"
#include "cache_prompt.cuh"
#include "cache_rows.cuh"
#include "cache_step.cuh"
#include "squant_host.h"

namespace {

constexpr int kMaxDevices = 64;
constexpr int kB200Sms = 148;
constexpr int64_t kMaxRows = 1ll << 30;
constexpr int64_t kMaxStride = 1ll << 36;

#define SQ_CUDA(call)                                                      \
    do {                                                                   \
        cudaError_t e__ = (call);                                          \
        if (e__ != cudaSuccess) return sq_host::cuda_failed(e__, #call);   \
    } while (0)

inline bool misaligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }
inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
// Rows and heads that start on 16 bytes.
inline bool on_vectors(const void *p, int64_t stride, int64_t head) { return !misaligned(p, 16) && stride % 8 == 0 && head % 8 == 0; }

template <typename Args>
int launch(void (*kernel)(Args), dim3 grid, int threads, int smem, cudaStream_t stream, const Args &args)
{
    kernel<<<grid, threads, smem, stream>>>(args);
    SQ_CUDA(cudaGetLastError());
    sq_host::count_launch();
    return SQUANT_OK;
}
// The same for kernels that take more shared memory than is had for nothing; `ready` is the kernel's own.
template <typename Args>
int launch_large(void (*kernel)(Args), std::atomic<bool> (&ready)[kMaxDevices], int64_t grid, int threads, int smem, cudaStream_t stream, const Args &args)
{
    int device;
    SQ_CUDA(cudaGetDevice(&device));
    if (device >= kMaxDevices || !ready[device].load(std::memory_order_relaxed)) {
        SQ_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (device < kMaxDevices) ready[device].store(true, std::memory_order_relaxed);
    }
    return launch(kernel, dim3(static_cast<unsigned>(grid)), threads, smem, stream, args);
}

int check(const squant_cache_rows &r, uint32_t dtype)
{
    if (r.head_dim != 64 && r.head_dim != 128 && r.head_dim != 256) return SQUANT_ERR_SHAPE;
    if (r.page_size < sq::kGranule || r.page_size % sq::kGranule || r.page_size > (1 << 24) || r.kv_heads < 1 || r.kv_heads > (1 << 16)) return SQUANT_ERR_SHAPE;
    if (r.page_count < 0 || r.page_count > (1ll << 31) || r.batch < 0 || r.batch > kMaxRows || r.width < 0 || r.rows < 0 || r.rows > kMaxRows) return SQUANT_ERR_SHAPE;
    // granules are counted in 32 bits: 2 TB of them (a page's are fewer than 2^37, all of them may be more than 64 bits hold)
    if (r.page_count > ((1ll << 31) - 1) / (static_cast<int64_t>(r.kv_heads) * (r.page_size / sq::kGranule))) return SQUANT_ERR_SHAPE;
    if (r.batch > 1 && (r.pages_stride < r.width || r.pages_stride > kMaxStride)) return SQUANT_ERR_SHAPE;
    if (!r.starts && r.rows != r.batch) return SQUANT_ERR_SHAPE;
    if (dtype > SQUANT_FP16) return SQUANT_ERR_MODE;
    if (r.batch > 0 && r.rows > 0) {
        if (!r.lens || (r.width > 0 && !r.pages) || (r.page_count > 0 && !r.data)) return SQUANT_ERR_NULL;
        if (misaligned(r.data, 16) || misaligned(r.lens, 4) || misaligned(r.pages, 4) || misaligned(r.starts, 4)) return SQUANT_ERR_ALIGN;
    }
    return SQUANT_OK;
}
bool nothing(const squant_cache_rows &r) { return r.batch == 0 || r.rows == 0; }

// Rows `stride` elements apart of `heads` heads `head` elements apart; one that is written may not lie in another.
bool bad_strides(int64_t stride, int64_t head, int64_t heads, int64_t rows, int64_t dim, bool written)
{
    if (stride < 0 || head < 0 || stride > kMaxStride || head > kMaxStride) return true;
    if (!written) return false;
    if (heads > 1 && rows > 1) return !(head >= dim && stride >= (heads - 1) * head + dim) && !(stride >= dim && head >= dim && rows - 1 <= (head - dim) / stride);   // no product of rows: it may overflow
    return (heads > 1 && head < dim) || (rows > 1 && stride < dim);
}

sq::CacheRows rows_of(const squant_cache_rows &r)
{
    sq::CacheRows c{};
    c.lens = r.lens;
    c.pages = r.pages;
    c.starts = r.starts;
    c.pages_stride = r.pages_stride;
    c.batch = r.batch;
    c.width = r.width;
    c.page_size = r.page_size;
    c.kv_heads = r.kv_heads;
    c.page_count = r.page_count;
    c.rows = r.rows;
    return c;
}

// ---- write and read

int check(const squant_cache_move_args *args, bool write)
{
    if (!args) return SQUANT_ERR_NULL;
    const squant_cache_move_args &a = *args;
    if (int rc = check(a.rows, a.dtype)) return rc;
    const squant_cache_rows &r = a.rows;
    if (bad_strides(a.k_stride, a.k_head_stride, r.kv_heads, r.rows, r.head_dim, !write) ||
        bad_strides(a.v_stride, a.v_head_stride, r.kv_heads, r.rows, r.head_dim, !write)) return SQUANT_ERR_SHAPE;
    if (nothing(r)) return SQUANT_OK;
    if (!a.k || !a.v) return SQUANT_ERR_NULL;
    if (misaligned(a.k, 2) || misaligned(a.v, 2)) return SQUANT_ERR_ALIGN;
    return SQUANT_OK;
}

template <int D>
int move(const squant_cache_move_args &a, bool write, cudaStream_t stream)
{
    sq::MoveArgs m{};
    m.cache = static_cast<uint8_t *>(a.rows.data);
    m.r = rows_of(a.rows);
    m.k = static_cast<uint16_t *>(a.k);
    m.v = static_cast<uint16_t *>(a.v);
    m.k_stride = a.k_stride;
    m.k_head = a.k_head_stride;
    m.v_stride = a.v_stride;
    m.v_head = a.v_head_stride;
    m.vector = on_vectors(a.k, a.k_stride, a.k_head_stride) && on_vectors(a.v, a.v_stride, a.v_head_stride);
    const bool half = a.dtype == SQUANT_FP16;
    const auto kernel = write ? (half ? sq::cache_write_kernel<D, true> : sq::cache_write_kernel<D, false>)
                              : (half ? sq::cache_read_kernel<D, true> : sq::cache_read_kernel<D, false>);
    const dim3 grid(static_cast<unsigned>((a.rows.rows + sq::kMoveThreads / 32 - 1) / (sq::kMoveThreads / 32)),
                    static_cast<unsigned>((a.rows.kv_heads + sq::kMoveHeads<D> - 1) / sq::kMoveHeads<D>));   // at most 32,768 high
    return launch(kernel, grid, sq::kMoveThreads, 0, stream, m);
}

int move(const squant_cache_move_args *args, bool write, void *cuda_stream)
{
    if (int rc = check(args, write)) return rc;
    const squant_cache_rows &r = args->rows;
    if (nothing(r) || (write && (r.width == 0 || r.page_count == 0))) return SQUANT_OK;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return r.head_dim == 64 ? move<64>(*args, write, stream) : r.head_dim == 128 ? move<128>(*args, write, stream) : move<256>(*args, write, stream);
}

// ---- attention

// For exponents of 2.
float scale_log2(const squant_cache_attention_args &a) { return static_cast<float>(static_cast<double>(a.scale) * 1.4426950408889634); }

int check(const squant_cache_attention_args *args)
{
    if (!args) return SQUANT_ERR_NULL;
    const squant_cache_attention_args &a = *args;
    if (int rc = check(a.rows, a.dtype)) return rc;
    const squant_cache_rows &r = a.rows;
    if (a.group < 1 || a.group > (1 << 16) || a.most < 0) return SQUANT_ERR_SHAPE;
    const int64_t heads = static_cast<int64_t>(r.kv_heads) * a.group;
    if (heads > (1 << 20) || r.rows * a.group >= (1ll << 31)) return SQUANT_ERR_SHAPE;
    // units of a tile are counted in 32 bits, with the group's share in them
    if (std::min<int64_t>(static_cast<int64_t>(r.width) * r.page_size, 1ll << 30) * a.group >= (1ll << 37)) return SQUANT_ERR_SHAPE;
    if (bad_strides(a.q_stride, a.q_head_stride, heads, r.rows, r.head_dim, false) ||
        bad_strides(a.out_stride, a.out_head_stride, heads, r.rows, r.head_dim, true)) return SQUANT_ERR_SHAPE;
    if (!std::isfinite(scale_log2(a))) return SQUANT_ERR_MODE;
    if (nothing(r)) return SQUANT_OK;
    if (!a.q || !a.out) return SQUANT_ERR_NULL;
    if (misaligned(a.q, 2) || misaligned(a.out, 2) || misaligned(a.lse, 4)) return SQUANT_ERR_ALIGN;
    return SQUANT_OK;
}

// Rows of a sequence, at most, as far as the host knows.
int64_t most_rows(const squant_cache_attention_args &a)
{
    if (!a.rows.starts) return 1;
    return a.most > 0 ? std::min<int64_t>(a.most, a.rows.rows) : a.rows.rows;
}
// cache_step_kernel reads the cache once for each of its tiles, cache_prompt_kernel once for 256 rows but at the cost of 128: the line is drawn at as many rows times heads (16
// sequences of 3,000 to 8,000 positions, 8 kv heads; us of step and prompt: 64 channels 97 and 112 for 64 rows, 112 and 109 for 80; 128 channels 131 and 136 for 40, 152 and 136
// for 48; 256 channels 255 and 288 for 48, 308 and 277 for 56.  Sequences of 200 to 900: 30 and 34, 31 and 37; 35 and 42, 40 and 49; 69 and 66, 91 and 75).
// Tiles of 16 rows pay where two of 8 take more than one and a half times as long, which with 128 channels they do not: 16 rows' sums
// and a unit's scores do not fit in 128 registers (32 rows in tiles of 8 and of 16: 64 channels 77 and 60, 128 channels 120 and 120, 256 channels 238 and 175).
constexpr int most_step_rows(int dim) { return dim == 64 ? 64 : dim == 128 ? 40 : 48; }
static_assert(std::max({most_step_rows(64), most_step_rows(128), most_step_rows(256)}) <= sq::kWholeRows, "as exact in either kernel");
constexpr int step_tiles(int dim) { return dim == 128 ? 1 : 2; }   // of 8 rows, beyond 8

int plan(const squant_cache_attention_args &a)
{
    if (nothing(a.rows)) return 0;
    const int64_t rows = most_rows(a) * a.group;
    if (rows > most_step_rows(a.rows.head_dim)) return SQUANT_CACHE_PROMPT;
    return rows <= 8 || step_tiles(a.rows.head_dim) == 1 ? SQUANT_CACHE_STEP : SQUANT_CACHE_STEP_16;
}

// Thread blocks and the workspace's parts.
struct StepPlan {
    int64_t blocks = 0, tickets = 0, bytes = 0;
};
template <int D, int kTiles>
StepPlan step_plan(const squant_cache_attention_args &a)
{
    using S = sq::StepShape<D, kTiles>;
    const squant_cache_rows &r = a.rows;
    // units, at most: no more blocks than one a unit and warp of a block
    const int64_t tiles = (r.rows * a.group + static_cast<int64_t>(std::min<int64_t>(r.batch, r.rows)) * (S::kRows - 1)) / S::kRows;
    const int64_t positions = std::min<int64_t>(static_cast<int64_t>(r.width) * r.page_size, 1ll << 30);
    const double units = static_cast<double>(tiles) * r.kv_heads * std::max<int64_t>(1, (positions + S::kPositions - 1) / S::kPositions);
    StepPlan s;
    s.blocks = static_cast<int64_t>(std::min<double>(kB200Sms * S::kBlocks, std::ceil(units / sq::kStepWarps)));
    s.tickets = up(8 * s.blocks, 128);
    s.bytes = s.tickets + s.blocks * S::kParts * S::kPart * 4;
    return s;
}
template <int D>
StepPlan prompt_plan(const squant_cache_attention_args &a)
{
    using S = sq::PromptShape<D>;
    const squant_cache_rows &r = a.rows;
    const int64_t tiles = (r.rows * a.group + static_cast<int64_t>(std::min<int64_t>(r.batch, r.rows)) * (S::kRows - 1)) / S::kRows;
    const int64_t positions = std::min<int64_t>(static_cast<int64_t>(r.width) * r.page_size, 1ll << 30);
    const double units = static_cast<double>(tiles) * r.kv_heads * (positions / S::kRows + 2);
    StepPlan s;
    s.blocks = static_cast<int64_t>(std::min<double>(kB200Sms, units));
    s.tickets = up(8 * s.blocks, 128);
    s.bytes = s.tickets + 2 * s.blocks * S::kPart * 4;
    return s;
}
template <int D>
int64_t attention_bytes(const squant_cache_attention_args &a)
{
    switch (plan(a)) {
        case SQUANT_CACHE_STEP: return step_plan<D, 1>(a).bytes;
        case SQUANT_CACHE_STEP_16: return step_plan<D, step_tiles(D)>(a).bytes;
        case SQUANT_CACHE_PROMPT: return prompt_plan<D>(a).bytes;
        default: return 0;
    }
}
int64_t attention_bytes(const squant_cache_attention_args &a)
{
    return a.rows.head_dim == 64 ? attention_bytes<64>(a) : a.rows.head_dim == 128 ? attention_bytes<128>(a) : attention_bytes<256>(a);
}

// A number that no other call of any process has put into this call's workspace, 48 bits and not 0.
unsigned long long nonce()
{
    static std::atomic<unsigned long long> next{[] {
        std::random_device device;
        return static_cast<unsigned long long>(device()) << 32 | device();
    }()};
    const unsigned long long n = next.fetch_add(1, std::memory_order_relaxed) & ((1ull << 48) - 1);
    return n ? n : nonce();
}

sq::AttendArgs attend_args(const squant_cache_attention_args &a, const StepPlan &s)
{
    sq::AttendArgs p{};
    p.cache = static_cast<const uint8_t *>(a.rows.data);
    p.r = rows_of(a.rows);
    p.q = static_cast<const uint16_t *>(a.q);
    p.q_stride = a.q_stride;
    p.q_head = a.q_head_stride;
    p.out = static_cast<uint16_t *>(a.out);
    p.out_stride = a.out_stride;
    p.out_head = a.out_head_stride;
    p.lse = a.lse;
    p.group = a.group;
    p.q_vector = on_vectors(a.q, a.q_stride, a.q_head_stride);
    p.out_vector = on_vectors(a.out, a.out_stride, a.out_head_stride);
    p.scale_log2 = scale_log2(a);
    p.tickets = static_cast<unsigned long long *>(a.workspace);
    p.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(a.workspace) + s.tickets);
    p.nonce = nonce();
    return p;
}
template <int D, bool kHalf, int kTiles>
int step(const squant_cache_attention_args &a, cudaStream_t stream)
{
    const StepPlan s = step_plan<D, kTiles>(a);
    static std::atomic<bool> ready[kMaxDevices];
    return launch_large(sq::cache_step_kernel<D, kHalf, kTiles>, ready, s.blocks, sq::kStepThreads, sq::StepShape<D, kTiles>::kSmem, stream, attend_args(a, s));
}
template <int D, bool kHalf>
int prompt(const squant_cache_attention_args &a, cudaStream_t stream)
{
    const StepPlan s = prompt_plan<D>(a);
    static std::atomic<bool> ready[kMaxDevices];
    return launch_large(sq::cache_prompt_kernel<D, kHalf>, ready, s.blocks, sq::PromptShape<D>::kThreads, sq::PromptShape<D>::kSmem, stream, attend_args(a, s));
}
template <int D>
int attention(const squant_cache_attention_args &a, cudaStream_t stream)
{
    const bool half = a.dtype == SQUANT_FP16;
    switch (plan(a)) {
        case SQUANT_CACHE_STEP: return half ? step<D, true, 1>(a, stream) : step<D, false, 1>(a, stream);
        case SQUANT_CACHE_STEP_16: return half ? step<D, true, step_tiles(D)>(a, stream) : step<D, false, step_tiles(D)>(a, stream);
        default: return half ? prompt<D, true>(a, stream) : prompt<D, false>(a, stream);
    }
}

}  // namespace

namespace sq_host {

cudaError_t take_cache_status(int *status)
{
    cudaError_t e = cudaMemcpyFromSymbol(status, sq::g_linear_status, sizeof(int));
    const int zero = 0;
    if (e == cudaSuccess && *status) e = cudaMemcpyToSymbol(sq::g_linear_status, &zero, sizeof(int));
    return e;
}

cudaError_t take_cache_violations(unsigned *count, int *site)
{
    cudaError_t e = cudaMemcpyFromSymbol(count, sq::g_linear_violations, sizeof(unsigned));
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(site, sq::g_linear_site, sizeof(int));
    const unsigned zero = 0;
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(sq::g_linear_violations, &zero, sizeof(zero));
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(sq::g_linear_site, &zero, sizeof(zero));
    return e;
}

cudaError_t set_cache_wait_limit(int tries)
{
#ifdef SQUANT_DEBUG_BOUNDS
    return cudaMemcpyToSymbol(sq::g_wait_limit, &tries, sizeof(int));
#else
    return tries >= 0 ? cudaSuccess : cudaErrorInvalidValue;
#endif
}

}  // namespace sq_host

extern "C" {

int squant_cache_write(const squant_cache_move_args *args, void *cuda_stream) { return move(args, true, cuda_stream); }
int squant_cache_read(const squant_cache_move_args *args, void *cuda_stream) { return move(args, false, cuda_stream); }

int64_t squant_cache_attention_workspace(const squant_cache_attention_args *args)
{
    if (int rc = check(args)) return rc;
    return attention_bytes(*args);
}

int squant_cache_attention_plan(const squant_cache_attention_args *args)
{
    if (int rc = check(args)) return rc;
    return plan(*args);
}

int squant_cache_attention(const squant_cache_attention_args *args, void *cuda_stream)
{
    if (int rc = check(args)) return rc;
    const squant_cache_attention_args &a = *args;
    const int64_t need = attention_bytes(a);
    if (need == 0) return SQUANT_OK;
    if (!a.workspace || misaligned(a.workspace, 16) || a.workspace_bytes < need) return SQUANT_ERR_WORKSPACE;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return a.rows.head_dim == 64 ? attention<64>(a, stream) : a.rows.head_dim == 128 ? attention<128>(a, stream) : attention<256>(a, stream);
}

}  // extern "C"
