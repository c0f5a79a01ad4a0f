// Host side of the linear operators: validation, choice of kernels, launches (C ABI of include/squant.h).
#include "squant.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>

#include "linear_dense.cuh"
#include "linear_device.cuh"
#include "linear_gemm.cuh"
#include "linear_rows.cuh"
#include "linear_small.cuh"
#include "squant_host.h"

namespace {

constexpr int kMaxDevices = 64;
constexpr int kB200Sms = 148;   // for squant_linear_plan
constexpr int64_t kMaxRows = 1ll << 30;
// Up to as many tokens fused_kernel turns the codes into floats on the way to the tensor cores; beyond, they are expanded once (4096 -> 4096 int4, fused and
// expanded: 256 tokens 16.9 and 21.3 us, 384 tokens 33 and 21.5).  For narrow results the line would lie higher, since dense_kernel gives a tile's whole
// contraction to one pair of thread blocks (300 tokens 11008 -> 64 int4 14 and 31 us, 4096 -> 1024 int8 14.5 and 18.4).
constexpr int kExpandBeyond = 256;
// few_kernel is faster up to eight tokens.  Its rows of x and codes start on 16 bytes; others it reads in small pieces, which beyond this many codes costs more
// than to copy them for fused_kernel.  Fewer than 4096 channels count as that: the GPU is not full.
constexpr int64_t kFewOddCodes = 1ll << 23;
// Beyond eight tokens, it reads all of x once for 16 channels, and from 33 tokens on the codes for 32 tokens anew, so that its time grows with tokens
// times codes while fused_kernel starts at 6 to 10 us: the lines are drawn at this many codes times tiles of eight tokens, a contraction of less than 2048
// counted as that (a block's warps do not all have work) and fewer than 4096 channels, all blocks of tokens together, as that.
constexpr int64_t kFewWork = 3ll << 25, kFewWorkBeyond32 = 1ll << 26;

// Contractions that fused_kernel's thread blocks and few_kernel's warps can share so that no sum has more than kLongestSum terms.
constexpr int64_t kLongestFused = sq::kLongestSum * std::min(sq::kFusedMostRanks, sq::kFewWarps);

#define SQ_CUDA(call)                                                      \
    do {                                                                   \
        cudaError_t e__ = (call);                                          \
        if (e__ != cudaSuccess) return sq_host::cuda_failed(e__, #call);   \
    } while (0)

inline bool misaligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }
inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
// Rows that start on 16 bytes (one row: only its own start counts).
inline bool rows_on_vectors(const void *p, int64_t stride, int64_t rows) { return !misaligned(p, 16) && (rows <= 1 || stride % 8 == 0); }

int device_sms(int &device, int &sms)
{
    SQ_CUDA(cudaGetDevice(&device));
    SQ_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    return SQUANT_OK;
}

// Clusters of `cluster` thread blocks.  Not with programmatic stream serialization: with it (every kernel letting the next one start
// at once and waiting for the one before) a call was 0.2 to 1 us a launch shorter, but some hundred backward calls in a row without a
// synchronization stopped for good.
template <typename... Params, typename... Args>
int launch(void (*kernel)(Params...), dim3 grid, dim3 cluster, int threads, int smem, cudaStream_t stream, const Args &...args)
{
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {cluster.x, cluster.y, 1};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SQ_CUDA(cudaLaunchKernelEx(&cfg, kernel, args...));
    sq_host::count_launch();
    return SQUANT_OK;
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encoder(EncodeTiled &fn)
{
    static std::atomic<void *> cached{nullptr};
    void *p = cached.load(std::memory_order_acquire);
    if (!p) {
        cudaDriverEntryPointQueryResult found;
        SQ_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found));
        if (found != cudaDriverEntryPointSuccess || !p) return sq_host::cuda_failed(cudaErrorNotSupported, "cuTensorMapEncodeTiled");
        cached.store(p, std::memory_order_release);
    }
    fn = reinterpret_cast<EncodeTiled>(p);
    return SQUANT_OK;
}

// A two-dimensional map.  The driver's function wants a current context, which a thread has once the runtime has set it up there: in a
// thread that has done nothing on the GPU yet, the current device is set and the call made again.
int encode(CUtensorMap &map, CUtensorMapDataType type, const void *p, const cuuint64_t (&dims)[2], const cuuint64_t (&strides)[1],
           const cuuint32_t (&box)[2], const cuuint32_t (&step)[2], CUtensorMapSwizzle swizzle, CUtensorMapL2promotion promotion)
{
    EncodeTiled fn;
    if (int rc = encoder(fn)) return rc;
    for (int attempt = 0;; ++attempt) {
        const CUresult r = fn(&map, type, 2, const_cast<void *>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, promotion,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (r == CUDA_SUCCESS) return SQUANT_OK;
        if (r != CUDA_ERROR_INVALID_CONTEXT || attempt) return sq_host::cuda_failed(cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
        int device;
        SQ_CUDA(cudaGetDevice(&device));
        SQ_CUDA(cudaSetDevice(device));
    }
}

// A 16-bit matrix [rows][cols] whose boxes are 64 elements wide and `box_rows` high; elements outside read as zero.
int matrix_map(CUtensorMap &map, const void *p, int64_t rows, int64_t cols, int64_t stride, bool half, int box_rows)
{
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(2 * (rows <= 1 ? up(cols, 8) : stride))};
    const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)}, step[2] = {1, 1};
    return encode(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, p, dims, strides, box, step,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

// Codes as bytes [rows][pitch].
int code_matrix_map(CUtensorMap &map, const void *p, int64_t rows, int64_t pitch, int box_bytes, int box_rows)
{
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(pitch), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(pitch)};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_bytes), static_cast<cuuint32_t>(box_rows)}, step[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, p, dims, strides, box, step, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B);
}

// As many thread blocks share a tile's contraction as there are multiprocessors (each holds two blocks) and stages for, and as its length asks for.
// x: [rows][depth] 16-bit.
template <int kMode, int kKind, bool kHalf>
int fused(const void *x, int64_t x_stride, sq::GemmArgs a, int device, int sms, cudaStream_t stream)
{
    auto kernel = sq::fused_kernel<kMode, kKind, kHalf>;
    static std::atomic<bool> ready[kMaxDevices];
    if (device >= kMaxDevices || !ready[device].load(std::memory_order_relaxed)) {
        SQ_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sq::kFusedSmem));
        if (device < kMaxDevices) ready[device].store(true, std::memory_order_relaxed);
    }
    a.box_rows = static_cast<int32_t>(std::min<int64_t>(sq::kFusedTokens, up(a.rows, 16)));
    CUtensorMap map, code_map;
    if (int rc = matrix_map(map, x, a.rows, a.depth, x_stride, kHalf, a.box_rows)) return rc;
    const int bytes = kKind == sq::kInt4 ? 32 : 64;   // of 64 codes
    if (int rc = kMode == sq::kForward ? code_matrix_map(code_map, a.codes, a.code_rows, a.code_pitch, bytes, sq::kFusedCols)
                                       : code_matrix_map(code_map, a.codes, a.code_rows, a.code_pitch, 2 * bytes, sq::kTileDepth)) return rc;
    a.row_tiles = (a.rows + sq::kFusedTokens - 1) / sq::kFusedTokens;
    a.tiles = static_cast<int64_t>(a.row_tiles) * ((static_cast<int64_t>(a.cols) + sq::kFusedCols - 1) / sq::kFusedCols);
    const int64_t steps = (static_cast<int64_t>(a.depth) + sq::kTileDepth - 1) / sq::kTileDepth;
    const int64_t needed = (a.depth + sq::kLongestSum - 1) / sq::kLongestSum;   // at most kFusedMostRanks: kLongestFused
    const unsigned ranks = static_cast<unsigned>(std::max(needed, std::min({static_cast<int64_t>(sq::kFusedMostRanks), 2 * sms / a.tiles, steps / 2})));
    return launch(kernel, dim3(static_cast<unsigned>(a.tiles * ranks)), dim3(ranks), sq::kFusedThreads, sq::kFusedSmem, stream, map, code_map, a);
}

template <int kMode, bool kHalf, int kCols>
int launch_dense(const CUtensorMap &map_a, const CUtensorMap &map_b, sq::GemmArgs a, int device, int sms, cudaStream_t stream)
{
    auto kernel = sq::dense_kernel<kMode, kHalf, kCols>;
    constexpr int smem = sq::DenseShape<kCols>::kSmem;
    static std::atomic<bool> ready[kMaxDevices];
    if (device >= kMaxDevices || !ready[device].load(std::memory_order_relaxed)) {
        SQ_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (device < kMaxDevices) ready[device].store(true, std::memory_order_relaxed);
    }
    a.row_tiles = (a.rows + sq::kPairRows - 1) / sq::kPairRows;
    a.tiles = static_cast<int64_t>(a.row_tiles) * ((static_cast<int64_t>(a.cols) + kCols - 1) / kCols);
    return launch(kernel, dim3(2 * static_cast<unsigned>(std::min<int64_t>(a.tiles, sms / 2))), dim3(2), sq::kDenseThreads, smem, stream, map_a, map_b, a);
}

// Bytes of the sums that the parts of a long contraction hand on.
int64_t sums_bytes(int64_t rows, int64_t cols, int64_t depth) { return depth > sq::kLongestSum ? rows * up(cols, 32) * 4 : 0; }

// Tiles of 256 or 128 columns, whichever is done in fewer waves; a wave of narrow tiles takes about 0.6 of one of wide tiles.
bool wide_tiles(int64_t rows, int64_t cols, int64_t sms)
{
    const int64_t row_tiles = (rows + sq::kPairRows - 1) / sq::kPairRows, pairs = sms / 2;
    const int64_t wide = (row_tiles * ((cols + 255) / 256) + pairs - 1) / pairs, narrow = (row_tiles * ((cols + 127) / 128) + pairs - 1) / pairs;
    return 10 * wide <= 6 * narrow;
}

// The product of two 16-bit matrices: `a` as gemm's 16-bit operand, `b` [cols][depth] (forward) or [depth][cols].
// sums: sums_bytes() of workspace.
template <int kMode, bool kHalf>
int dense(const void *a, int64_t a_stride, const void *b, int64_t b_stride, sq::GemmArgs g, void *sums, int device, int sms, cudaStream_t stream)
{
    const bool use_wide = wide_tiles(g.rows, g.cols, sms);
    CUtensorMap map_a, map_b;
    if (int rc = kMode == sq::kWeightGrad ? matrix_map(map_a, a, g.depth, g.rows, a_stride, kHalf, sq::kTileDepth)
                                          : matrix_map(map_a, a, g.rows, g.depth, a_stride, kHalf, 128)) return rc;
    if (int rc = kMode == sq::kForward ? matrix_map(map_b, b, g.cols, g.depth, b_stride, kHalf, use_wide ? 128 : 64)
                                       : matrix_map(map_b, b, g.depth, g.cols, b_stride, kHalf, sq::kTileDepth)) return rc;
    const int64_t steps = (static_cast<int64_t>(g.depth) + sq::kTileDepth - 1) / sq::kTileDepth;
    const int64_t parts = (g.depth + sq::kLongestSum - 1) / sq::kLongestSum;
    if (parts > 1) g.sums = static_cast<float *>(sums);
    g.sums_pitch = up(g.cols, 32);
    for (int64_t part = 0; part < parts; ++part) {
        g.first_step = static_cast<int32_t>(steps * part / parts);
        g.steps = static_cast<int32_t>(steps * (part + 1) / parts) - g.first_step;
        g.sums_in = part > 0;
        g.sums_out = part + 1 < parts;
        if (int rc = use_wide ? launch_dense<kMode, kHalf, 256>(map_a, map_b, g, device, sms, stream)
                              : launch_dense<kMode, kHalf, 128>(map_a, map_b, g, device, sms, stream)) return rc;
    }
    return SQUANT_OK;
}

enum class RowKernel { kCheckpoint, kRestore, kExpandInt4Bf16, kExpandInt4Fp16, kExpandInt8Bf16, kExpandInt8Fp16 };

// With 2^(L-1) < by <= 2^L and magic = floor(2^(31+L) / by) + 1, at * magic / 2^(31+L) exceeds at / by by less than at / 2^(31+L) < 1 / by.
void division(uint32_t by, uint32_t &magic, uint32_t &shift)
{
    uint32_t bits = 0;
    while ((1ull << bits) < by) ++bits;
    magic = bits ? static_cast<uint32_t>((1ull << (31 + bits)) / by + 1) : 0;
    shift = bits ? bits - 1 : 0;
}

// Rows of `bytes` bytes to rows that start on 16 bytes.
struct Copy {
    const void *in = nullptr;   // null: nothing to copy
    int64_t rows = 0, bytes = 0, pitch = 0;
    void *out = nullptr;
    int64_t out_pitch() const { return up(bytes, 16); }
    int64_t out_bytes() const { return in ? rows * out_pitch() : 0; }
};

// Both in one launch where they are not very large, else in ranges of rows.
int launch_copies(const Copy &a, const Copy &b, cudaStream_t stream)
{
    const auto job = [](const Copy &c, int64_t row, int64_t rows) {
        sq::CopyJob j{};
        if (!c.in || rows <= 0) return j;
        j.in = static_cast<const uint8_t *>(c.in) + row * c.pitch;
        j.end = static_cast<const uint8_t *>(c.in) + (c.rows - 1) * c.pitch + c.bytes;
        j.out = static_cast<uint8_t *>(c.out) + row * c.out_pitch();
        j.in_pitch = c.pitch;
        j.out_pitch = c.out_pitch();
        j.rows = static_cast<uint32_t>(rows);
        j.pieces = static_cast<uint32_t>(c.out_pitch() / 16);
        division(j.pieces, j.magic, j.shift);
        return j;
    };
    const auto blocks = [](const sq::CopyJob &j) {
        return static_cast<uint32_t>((static_cast<int64_t>(j.rows) * j.pieces + sq::kRowThreads * sq::kRowPieces - 1) / (sq::kRowThreads * sq::kRowPieces));
    };
    const int64_t limit = (1ll << 31) - 4096;
    const auto pieces = [](const Copy &c) { return c.in ? c.rows * (c.out_pitch() / 16) : 0; };
    if (pieces(a) <= limit && pieces(b) <= limit) {
        const sq::CopyJob ja = job(a, 0, a.rows), jb = job(b, 0, b.rows);
        const uint32_t ba = blocks(ja), bb = blocks(jb);
        return ba + bb ? launch(sq::copy_kernel, dim3(ba + bb), dim3(1), sq::kRowThreads, 0, stream, ja, jb, ba) : SQUANT_OK;
    }
    for (const Copy *c : {&a, &b}) {
        if (!c->in) continue;
        const int64_t most = std::max<int64_t>(1, limit / (c->out_pitch() / 16));
        for (int64_t r = 0; r < c->rows; r += most) {
            const sq::CopyJob j = job(*c, r, std::min(most, c->rows - r));
            if (int rc = launch(sq::copy_kernel, dim3(blocks(j)), dim3(1), sq::kRowThreads, 0, stream, j, sq::CopyJob{}, blocks(j))) return rc;
        }
    }
    return SQUANT_OK;
}

// Launches over ranges of rows, so that indices within a launch fit 32 bits.
int launch_rows(RowKernel which, sq::RowArgs a, int64_t rows, cudaStream_t stream)
{
    const int64_t most = std::max<int64_t>(1, ((1ll << 31) - 4096) / a.pieces);
    division(a.pieces, a.magic, a.shift);
    for (int64_t r = 0; r < rows; r += most) {
        sq::RowArgs b = a;
        b.rows = static_cast<uint32_t>(std::min(most, rows - r));
        if (b.in) b.in += r * a.in_stride;
        if (b.out) b.out += r * a.out_stride;
        if (b.codes) b.codes += r * a.code_pitch;
        if (b.exps) b.exps += r * a.exps_pitch;
        const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(b.rows) * b.pieces + sq::kRowThreads * sq::kRowPieces - 1) / (sq::kRowThreads * sq::kRowPieces));
        void (*kernel)(sq::RowArgs) = nullptr;
        switch (which) {
            case RowKernel::kCheckpoint: kernel = sq::checkpoint_kernel; break;
            case RowKernel::kRestore: kernel = sq::restore_kernel; break;
            case RowKernel::kExpandInt4Bf16: kernel = sq::expand_kernel<sq::kInt4, false>; break;
            case RowKernel::kExpandInt4Fp16: kernel = sq::expand_kernel<sq::kInt4, true>; break;
            case RowKernel::kExpandInt8Bf16: kernel = sq::expand_kernel<sq::kInt8, false>; break;
            case RowKernel::kExpandInt8Fp16: kernel = sq::expand_kernel<sq::kInt8, true>; break;
        }
        if (int rc = launch(kernel, dim3(grid), dim3(1), sq::kRowThreads, 0, stream, b)) return rc;
    }
    return SQUANT_OK;
}

int restore(const squant_checkpoint_data &from, int64_t rows, int32_t features, void *out, int64_t stride, cudaStream_t stream)
{
    sq::RowArgs r{};
    r.out = static_cast<uint16_t *>(out);
    r.out_stride = stride;
    r.codes = reinterpret_cast<uint8_t *>(from.codes);
    r.exps = from.exps;
    r.code_pitch = up(features, 32);
    r.exps_pitch = r.code_pitch / 32;
    r.pieces = static_cast<uint32_t>(r.code_pitch / 8);
    r.features = features;
    r.vector = rows_on_vectors(out, stride, rows);
    return launch_rows(RowKernel::kRestore, r, rows, stream);
}

// Codes [cout][cin] to 16-bit floats [cout][cin rounded up to 8].
int expand(const int8_t *codes, int64_t cout, int32_t cin, bool packed, bool half, void *out, cudaStream_t stream)
{
    sq::RowArgs r{};
    r.codes = reinterpret_cast<uint8_t *>(const_cast<int8_t *>(codes));
    r.code_pitch = packed ? (static_cast<int64_t>(cin) + 1) / 2 : cin;
    r.out = static_cast<uint16_t *>(out);
    r.out_stride = up(cin, 8);
    r.pieces = static_cast<uint32_t>(r.out_stride / 8);
    r.features = cin;
    const int64_t piece = packed ? 4 : 8;
    r.vector = !misaligned(codes, piece) && r.code_pitch % piece == 0;
    return launch_rows(packed ? (half ? RowKernel::kExpandInt4Fp16 : RowKernel::kExpandInt4Bf16)
                              : (half ? RowKernel::kExpandInt8Fp16 : RowKernel::kExpandInt8Bf16), r, cout, stream);
}

bool good_dims(int64_t tokens, int64_t cin, int64_t cout)
{
    return tokens >= 0 && tokens <= kMaxRows && cin >= 1 && cin <= kMaxRows && cout >= 1 && cout <= kMaxRows && cin * cout <= (1ll << 40);
}
bool good_stride(int64_t stride, int64_t cols, int64_t rows) { return rows <= 1 || (stride >= cols && stride <= (1ll << 36)); }
bool bad_checkpoint(const squant_checkpoint_data &c) { return misaligned(c.codes, 16) || misaligned(c.exps, 16); }

// ---- forward

// Bytes of a row of codes, and whether every row starts on 16 bytes.
int64_t code_pitch(int32_t cin, uint32_t flags) { return flags & SQUANT_FLAG_PACK_INT4 ? (static_cast<int64_t>(cin) + 1) / 2 : cin; }
bool codes_on_vectors(const int8_t *codes, int64_t pitch) { return !misaligned(codes, 16) && pitch % 16 == 0; }

// Bytes that rows of x start on for few_kernel (0: any, or rows of codes that start off 16), and the calls it takes.
int few_align(const squant_linear_args &a)
{
    if (!codes_on_vectors(a.codes, code_pitch(a.cin, a.flags)) || !rows_on_vectors(a.x, a.x_stride, a.tokens) || a.cin % 8) return 0;
    return a.cin % 16 || misaligned(a.x, 32) || (a.tokens > 1 && a.x_stride % 16) ? 16 : 32;
}
// Thread blocks that share the tokens: four tiles each.
int64_t few_blocks(int64_t tokens) { return (tokens + 4 * sq::kFewTokens - 1) / (4 * sq::kFewTokens); }
bool few(const squant_linear_args &a)
{
    if (a.z.codes || a.tokens > kExpandBeyond || a.cin > kLongestFused) return false;
    if (a.tokens <= sq::kFewTokens) return few_align(a) || a.cin * std::max<int64_t>(a.cout, 4096) <= kFewOddCodes;
    const int64_t blocks = few_blocks(a.tokens), tiles = a.tokens > 2 * sq::kFewTokens ? 4 : 2;
    const int64_t codes = std::max<int64_t>(a.cin, 2048) * std::max<int64_t>(a.cout * blocks, 4096);
    return codes * tiles <= (blocks > 1 ? kFewWorkBeyond32 : kFewWork) && few_align(a) == 32;
}

// Parts of the workspace: copies of x and of the codes with rows that TMA can read, or the codes as 16-bit floats and the sums of a long contraction.
struct ForwardPlan {
    bool dense = false;
    Copy x, codes;
    int64_t wide_bytes = 0;   // the codes as 16-bit floats
    int64_t bytes = 0;
};

ForwardPlan forward_plan(const squant_linear_args &a)
{
    ForwardPlan p;
    p.dense = a.tokens > kExpandBeyond || a.cin > kLongestFused;
    if (few(a)) return p;
    uint8_t *at = static_cast<uint8_t *>(a.workspace);
    if (!rows_on_vectors(a.x, a.x_stride, a.tokens)) p.x = {a.x, a.tokens, 2 * static_cast<int64_t>(a.cin), 2 * (a.tokens > 1 ? a.x_stride : a.cin), at};
    const int64_t pitch = code_pitch(a.cin, a.flags);
    if (!p.dense && !codes_on_vectors(a.codes, pitch)) p.codes = {a.codes, a.cout, pitch, pitch, at ? at + p.x.out_bytes() : nullptr};
    p.wide_bytes = p.dense ? a.cout * up(a.cin, 8) * 2 : 0;
    p.bytes = p.x.out_bytes() + p.codes.out_bytes() + p.wide_bytes + (p.dense ? sums_bytes(a.tokens, a.cout, a.cin) : 0);
    return p;
}

int check(const squant_linear_args *args)
{
    if (!args) return SQUANT_ERR_NULL;
    const squant_linear_args &a = *args;
    if (!good_dims(a.tokens, a.cin, a.cout)) return SQUANT_ERR_SHAPE;
    if (!good_stride(a.x_stride, a.cin, a.tokens) || !good_stride(a.y_stride, a.cout, a.tokens) ||
        (a.residual && !good_stride(a.residual_stride, a.cout, a.tokens))) return SQUANT_ERR_SHAPE;
    if (a.dtype > SQUANT_FP16 || a.act > SQUANT_ACT_SILU || (a.flags & ~SQUANT_FLAG_PACK_INT4)) return SQUANT_ERR_MODE;
    if (!a.codes || !a.scales) return SQUANT_ERR_NULL;
    if (a.tokens > 0 && (!a.x || !a.y)) return SQUANT_ERR_NULL;
    if (a.z.codes && !a.z.exps) return SQUANT_ERR_NULL;
    if (misaligned(a.x, 2) || misaligned(a.y, 2) || misaligned(a.residual, 2) || misaligned(a.scales, 4) || misaligned(a.bias, 4) ||
        (a.z.codes && bad_checkpoint(a.z))) return SQUANT_ERR_ALIGN;
    return SQUANT_OK;
}

template <int kKind, bool kHalf>
int forward(const squant_linear_args &a, cudaStream_t stream)
{
    const int64_t pitch = code_pitch(a.cin, a.flags);
    const int64_t z_pitch = up(a.cout, 32);
    if (few(a)) {
        sq::FewArgs s{};
        s.x = static_cast<const uint16_t *>(a.x);
        s.x_stride = a.x_stride;
        s.codes = reinterpret_cast<const uint8_t *>(a.codes);
        s.code_pitch = pitch;
        s.code_bytes = pitch * a.cout;
        s.tokens = static_cast<int32_t>(a.tokens);
        s.cin = a.cin;
        s.cout = a.cout;
        s.scales = a.scales;
        s.bias = a.bias;
        s.residual = static_cast<const uint16_t *>(a.residual);
        s.residual_stride = a.residual_stride;
        s.y = static_cast<uint16_t *>(a.y);
        s.y_stride = a.y_stride;
        s.act = static_cast<int32_t>(a.act);
        const int align = few_align(a);
        const auto kernel = a.tokens > 2 * sq::kFewTokens ? sq::few_kernel<kKind, kHalf, 32, 4>
                            : a.tokens > sq::kFewTokens   ? sq::few_kernel<kKind, kHalf, 32, 2>
                            : align == 32                 ? sq::few_kernel<kKind, kHalf, 32, 1>
                            : align == 16                 ? sq::few_kernel<kKind, kHalf, 16, 1>
                                                          : sq::few_kernel<kKind, kHalf, 0, 1>;
        const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(a.cout) + sq::kFewRows - 1) / sq::kFewRows);
        return launch(kernel, dim3(grid, static_cast<unsigned>(few_blocks(a.tokens))), dim3(1), 32 * sq::kFewWarps, 0, stream, s);
    }
    int device, sms;
    if (int rc = device_sms(device, sms)) return rc;
    const ForwardPlan plan = forward_plan(a);
    if (int rc = launch_copies(plan.x, plan.codes, stream)) return rc;
    const void *x = plan.x.in ? plan.x.out : a.x;
    const int64_t x_stride = plan.x.in ? plan.x.out_pitch() / 2 : a.x_stride;
    sq::GemmArgs g{};
    g.rows = static_cast<int32_t>(a.tokens);
    g.cols = a.cout;
    g.depth = a.cin;
    g.out = static_cast<uint16_t *>(a.y);
    g.out_stride = a.y_stride;
    g.out_vector = rows_on_vectors(a.y, a.y_stride, a.tokens);
    g.scales = a.scales;
    g.bias = a.bias;
    g.param_vector = !misaligned(a.scales, 16) && !misaligned(a.bias, 16);
    g.residual = static_cast<const uint16_t *>(a.residual);
    g.residual_stride = a.residual_stride;
    g.residual_vector = rows_on_vectors(a.residual, a.residual_stride, a.tokens);
    g.act = static_cast<int32_t>(a.act);
    g.z_codes = reinterpret_cast<uint8_t *>(a.z.codes);
    g.z_exps = a.z.exps;
    g.z_pitch = z_pitch;
    g.z_exps_pitch = z_pitch / 32;
    if (plan.dense) {
        uint8_t *b = static_cast<uint8_t *>(a.workspace) + plan.x.out_bytes();
        if (int rc = expand(a.codes, a.cout, a.cin, kKind == sq::kInt4, kHalf, b, stream)) return rc;
        return dense<sq::kForward, kHalf>(x, x_stride, b, up(a.cin, 8), g, b + plan.wide_bytes, device, sms, stream);
    }
    g.codes = static_cast<const uint8_t *>(plan.codes.in ? plan.codes.out : a.codes);
    g.code_pitch = plan.codes.in ? plan.codes.out_pitch() : pitch;
    g.code_rows = a.cout;
    return fused<sq::kForward, kKind, kHalf>(x, x_stride, g, device, sms, stream);
}

// ---- backward

// What the gradients need of dy * act'(zhat): parts of the workspace, each [tokens][pitch] bf16.
struct SlopePlan {
    bool dzs = false, dz = false, any = false, dense = false;
    int64_t pitch = 0, slope_bytes = 0;
    int64_t share = 0, shares = 1;   // tokens of a thread block of slope_kernel
    int64_t partial_bytes = 0;       // behind dzs and dz: sums of the shares
    Copy codes;               // a copy of the codes with rows that TMA can read
    int64_t wide_bytes = 0;   // behind them: that copy or the codes as 16-bit floats, then the input as 16-bit floats
    int64_t bytes = 0;        // behind these the sums of a long contraction, of dx and then of dweight
};

SlopePlan slope_plan(const squant_linear_grad_args &a)
{
    SlopePlan s;
    s.pitch = up(a.cout, 8);
    s.dzs = a.dx && a.tokens > 0;
    s.dz = a.dweight && a.tokens > 0 && (a.act != SQUANT_ACT_NONE || !rows_on_vectors(a.dy, a.dy_stride, a.tokens));
    s.any = s.dzs || s.dz || a.dbias || a.dscales;
    const int64_t columns = (static_cast<int64_t>(a.cout) + sq::kSlopeCols - 1) / sq::kSlopeCols;
    s.shares = std::max<int64_t>(1, std::min(sq::kSlopeBlocks / columns, (a.tokens + sq::kSlopeLeast - 1) / sq::kSlopeLeast));
    s.share = std::max<int64_t>(1, (a.tokens + s.shares - 1) / s.shares);
    if (s.shares > 1 && (a.dbias || a.dscales)) s.partial_bytes = up(s.shares * 2 * a.cout * 4, 16);
    s.slope_bytes = (s.dzs + s.dz) * a.tokens * s.pitch * 2 + s.partial_bytes;
    s.dense = s.dzs && (a.tokens > kExpandBeyond || a.cout > kLongestFused);
    const int64_t row = up(a.cin, 8) * 2;
    const int64_t pitch = code_pitch(a.cin, a.flags);
    if (s.dzs && !s.dense && !codes_on_vectors(a.codes, pitch))
        s.codes = {a.codes, a.cout, pitch, pitch, a.workspace ? static_cast<uint8_t *>(a.workspace) + s.slope_bytes : nullptr};
    s.wide_bytes = std::max({s.dense ? a.cout * row : 0, s.codes.out_bytes(), a.dweight ? a.tokens * row : 0});
    s.bytes = s.slope_bytes + s.wide_bytes + std::max(s.dense ? sums_bytes(a.tokens, a.cin, a.cout) : 0, a.dweight ? sums_bytes(a.cout, a.cin, a.tokens) : 0);
    return s;
}

int check(const squant_linear_grad_args *args)
{
    if (!args) return SQUANT_ERR_NULL;
    const squant_linear_grad_args &a = *args;
    if (!good_dims(a.tokens, a.cin, a.cout)) return SQUANT_ERR_SHAPE;
    if (!good_stride(a.dy_stride, a.cout, a.tokens) || (a.dx && !good_stride(a.dx_stride, a.cin, a.tokens)) ||
        (a.dweight && !good_stride(a.dweight_stride, a.cin, a.cout))) return SQUANT_ERR_SHAPE;
    if (a.act > SQUANT_ACT_SILU || (a.flags & ~SQUANT_FLAG_PACK_INT4)) return SQUANT_ERR_MODE;
    if (a.dx && (!a.codes || !a.scales)) return SQUANT_ERR_NULL;
    if (a.dscales && !a.scales) return SQUANT_ERR_NULL;
    if (a.tokens > 0) {
        if (!a.dy) return SQUANT_ERR_NULL;
        if ((a.act != SQUANT_ACT_NONE || a.dscales) && (!a.z.codes || !a.z.exps)) return SQUANT_ERR_NULL;
        if (a.dweight && (!a.x.codes || !a.x.exps)) return SQUANT_ERR_NULL;
    }
    if (misaligned(a.dy, 2) || misaligned(a.dx, 2) || misaligned(a.dweight, 2) || misaligned(a.scales, 4) || misaligned(a.bias, 4) ||
        misaligned(a.dbias, 4) || misaligned(a.dscales, 4) || bad_checkpoint(a.z) || bad_checkpoint(a.x)) return SQUANT_ERR_ALIGN;
    return SQUANT_OK;
}

int slope(const squant_linear_grad_args &a, const SlopePlan &plan, uint16_t *dzs, uint16_t *dz, float *partial, cudaStream_t stream)
{
    sq::SlopeArgs s{};
    s.dy = static_cast<const uint16_t *>(a.dy);
    s.dy_stride = a.dy_stride;
    const bool need_z = a.act != SQUANT_ACT_NONE || a.dscales;
    s.z_codes = need_z ? reinterpret_cast<const uint8_t *>(a.z.codes) : nullptr;
    s.z_exps = need_z ? a.z.exps : nullptr;
    s.z_pitch = up(a.cout, 32);
    s.z_exps_pitch = s.z_pitch / 32;
    s.scales = a.scales;
    s.bias = a.bias;
    s.tokens = a.tokens;
    s.cout = a.cout;
    s.act = static_cast<int32_t>(a.act);
    s.dz = dz;
    s.dzs = dzs;
    s.pitch = plan.pitch;
    s.dbias = a.dbias;
    s.dscales = a.dscales;
    s.share = plan.share;
    s.shares = static_cast<int32_t>(plan.shares);
    s.partial = plan.partial_bytes ? partial : nullptr;
    const unsigned columns = static_cast<unsigned>((static_cast<int64_t>(a.cout) + sq::kSlopeCols - 1) / sq::kSlopeCols);
    const bool vector = a.cout % 4 == 0 && !misaligned(a.dy, 8) && (a.tokens <= 1 || a.dy_stride % 4 == 0);
    void (*kernel)(sq::SlopeArgs) = nullptr;
    if (!need_z) kernel = vector ? sq::slope_kernel<sq::kNoZ, true> : sq::slope_kernel<sq::kNoZ, false>;
    else if (a.act == SQUANT_ACT_NONE) kernel = vector ? sq::slope_kernel<sq::kActNone, true> : sq::slope_kernel<sq::kActNone, false>;
    else if (a.act == SQUANT_ACT_RELU) kernel = vector ? sq::slope_kernel<sq::kActRelu, true> : sq::slope_kernel<sq::kActRelu, false>;
    else if (a.act == SQUANT_ACT_GELU) kernel = vector ? sq::slope_kernel<sq::kActGelu, true> : sq::slope_kernel<sq::kActGelu, false>;
    else kernel = vector ? sq::slope_kernel<sq::kActSilu, true> : sq::slope_kernel<sq::kActSilu, false>;
    if (int rc = launch(kernel, dim3(columns, static_cast<unsigned>(plan.shares)), dim3(1), sq::kRowThreads, 0, stream, s)) return rc;
    if (!s.partial) return SQUANT_OK;
    const unsigned grid = static_cast<unsigned>((2 * static_cast<int64_t>(a.cout) + sq::kRowThreads - 1) / sq::kRowThreads);
    return launch(sq::sums_kernel, dim3(grid), dim3(1), sq::kRowThreads, 0, stream, s);
}

}  // namespace

namespace sq_host {

cudaError_t take_linear_status(int *status)
{
    cudaError_t e = cudaMemcpyFromSymbol(status, sq::g_linear_status, sizeof(int));
    const int zero = 0;
    if (e == cudaSuccess && *status) e = cudaMemcpyToSymbol(sq::g_linear_status, &zero, sizeof(int));
    return e;
}

cudaError_t take_linear_violations(unsigned *count, int *site)
{
    cudaError_t e = cudaMemcpyFromSymbol(count, sq::g_linear_violations, sizeof(unsigned));
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(site, sq::g_linear_site, sizeof(int));
    const unsigned zero = 0;
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(sq::g_linear_violations, &zero, sizeof(zero));
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(sq::g_linear_site, &zero, sizeof(zero));
    return e;
}

}  // namespace sq_host

extern "C" {

int squant_checkpoint(const void *x, int64_t rows, int32_t features, int64_t stride, const squant_checkpoint_data *to, void *cuda_stream)
{
    if (!to) return SQUANT_ERR_NULL;
    if (!good_dims(rows, features, 1) || !good_stride(stride, features, rows)) return SQUANT_ERR_SHAPE;
    if (rows == 0) return SQUANT_OK;
    if (!x || !to->codes || !to->exps) return SQUANT_ERR_NULL;
    if (misaligned(x, 2) || bad_checkpoint(*to)) return SQUANT_ERR_ALIGN;
    sq::RowArgs r{};
    r.in = static_cast<const uint16_t *>(x);
    r.in_stride = stride;
    r.codes = reinterpret_cast<uint8_t *>(to->codes);
    r.exps = to->exps;
    r.code_pitch = up(features, 32);
    r.exps_pitch = r.code_pitch / 32;
    r.pieces = static_cast<uint32_t>(r.code_pitch / 16);
    r.features = features;
    r.vector = rows_on_vectors(x, stride, rows);
    return launch_rows(RowKernel::kCheckpoint, r, rows, static_cast<cudaStream_t>(cuda_stream));
}

int squant_checkpoint_restore(const squant_checkpoint_data *from, int64_t rows, int32_t features, void *out, int64_t stride,
                              void *cuda_stream)
{
    if (!from) return SQUANT_ERR_NULL;
    if (!good_dims(rows, features, 1) || !good_stride(stride, features, rows)) return SQUANT_ERR_SHAPE;
    if (rows == 0) return SQUANT_OK;
    if (!out || !from->codes || !from->exps) return SQUANT_ERR_NULL;
    if (misaligned(out, 2) || bad_checkpoint(*from)) return SQUANT_ERR_ALIGN;
    return restore(*from, rows, features, out, stride, static_cast<cudaStream_t>(cuda_stream));
}

int squant_debug_linear_wait_expires(int32_t max_tries, void *cuda_stream)
{
    if (max_tries < 1 || max_tries > 4096) return SQUANT_ERR_SHAPE;
    return launch(sq::wait_kernel, dim3(1), dim3(1), 32, 0, static_cast<cudaStream_t>(cuda_stream), max_tries);
}

int squant_debug_linear_wait_limit(int32_t tries)
{
    if (tries < -1 || tries > sq::kWaitLimit) return SQUANT_ERR_SHAPE;
#ifdef SQUANT_DEBUG_BOUNDS
    const int limit = tries < 0 ? sq::kWaitLimit : tries;
    SQ_CUDA(cudaDeviceSynchronize());
    SQ_CUDA(cudaMemcpyToSymbol(sq::g_wait_limit, &limit, sizeof(int)));
    return 1;   // this library was built with the checks
#else
    return SQUANT_OK;
#endif
}

int64_t squant_linear_workspace(const squant_linear_args *args)
{
    if (int rc = check(args)) return rc;
    return forward_plan(*args).bytes;
}

int squant_linear_plan(const squant_linear_args *args)
{
    if (int rc = check(args)) return rc;
    const squant_linear_args &a = *args;
    if (a.tokens == 0) return 0;
    if (few(a)) return SQUANT_LINEAR_FEW;
    if (!forward_plan(a).dense) return SQUANT_LINEAR_FUSED;
    return wide_tiles(a.tokens, a.cout, kB200Sms) ? SQUANT_LINEAR_DENSE_WIDE : SQUANT_LINEAR_DENSE;
}

int squant_linear(const squant_linear_args *args, void *cuda_stream)
{
    if (int rc = check(args)) return rc;
    const squant_linear_args &a = *args;
    if (a.tokens == 0) return SQUANT_OK;
    const int64_t need = forward_plan(a).bytes;
    if (need && (!a.workspace || misaligned(a.workspace, 16) || a.workspace_bytes < need)) return SQUANT_ERR_WORKSPACE;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool half = a.dtype == SQUANT_FP16;
    if (a.flags & SQUANT_FLAG_PACK_INT4) return half ? forward<sq::kInt4, true>(a, stream) : forward<sq::kInt4, false>(a, stream);
    return half ? forward<sq::kInt8, true>(a, stream) : forward<sq::kInt8, false>(a, stream);
}

int64_t squant_linear_backward_workspace(const squant_linear_grad_args *args)
{
    if (int rc = check(args)) return rc;
    return slope_plan(*args).bytes;
}

int squant_linear_backward(const squant_linear_grad_args *args, void *cuda_stream)
{
    if (int rc = check(args)) return rc;
    const squant_linear_grad_args &a = *args;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const SlopePlan plan = slope_plan(a);
    if (plan.bytes && (!a.workspace || misaligned(a.workspace, 16) || a.workspace_bytes < plan.bytes)) return SQUANT_ERR_WORKSPACE;
    int device, sms;
    if (int rc = device_sms(device, sms)) return rc;
    uint16_t *dzs = plan.dzs ? static_cast<uint16_t *>(a.workspace) : nullptr;
    uint16_t *dz = plan.dz ? static_cast<uint16_t *>(a.workspace) + (plan.dzs ? a.tokens * plan.pitch : 0) : nullptr;
    float *partial = reinterpret_cast<float *>(static_cast<uint8_t *>(a.workspace) + plan.slope_bytes - plan.partial_bytes);
    if (plan.any)
        if (int rc = slope(a, plan, dzs, dz, partial, stream)) return rc;
    uint8_t *wide = static_cast<uint8_t *>(a.workspace) + plan.slope_bytes, *sums = wide + plan.wide_bytes;
    if (plan.dzs) {
        const bool packed = a.flags & SQUANT_FLAG_PACK_INT4;
        sq::GemmArgs g{};
        g.rows = static_cast<int32_t>(a.tokens);
        g.cols = a.cin;
        g.depth = a.cout;
        g.out = static_cast<uint16_t *>(a.dx);
        g.out_stride = a.dx_stride;
        g.out_vector = rows_on_vectors(a.dx, a.dx_stride, a.tokens);
        if (plan.dense) {
            if (int rc = expand(a.codes, a.cout, a.cin, packed, false, wide, stream)) return rc;
            if (int rc = dense<sq::kInputGrad, false>(dzs, plan.pitch, wide, up(a.cin, 8), g, sums, device, sms, stream)) return rc;
        } else {
            if (int rc = launch_copies(plan.codes, Copy{}, stream)) return rc;
            g.codes = static_cast<const uint8_t *>(plan.codes.in ? plan.codes.out : a.codes);
            g.code_pitch = plan.codes.in ? plan.codes.out_pitch() : code_pitch(a.cin, a.flags);
            g.code_rows = a.cout;
            if (int rc = packed ? fused<sq::kInputGrad, sq::kInt4, false>(dzs, plan.pitch, g, device, sms, stream)
                                : fused<sq::kInputGrad, sq::kInt8, false>(dzs, plan.pitch, g, device, sms, stream)) return rc;
        }
    }
    if (a.dweight) {
        if (a.tokens == 0) {
            SQ_CUDA(cudaMemset2DAsync(a.dweight, 2 * (a.cout == 1 ? a.cin : a.dweight_stride), 0, 2 * static_cast<size_t>(a.cin), a.cout, stream));
            return SQUANT_OK;
        }
        if (int rc = restore(a.x, a.tokens, a.cin, wide, up(a.cin, 8), stream)) return rc;
        sq::GemmArgs g{};
        g.rows = a.cout;
        g.cols = a.cin;
        g.depth = static_cast<int32_t>(a.tokens);
        g.out = static_cast<uint16_t *>(a.dweight);
        g.out_stride = a.dweight_stride;
        g.out_vector = rows_on_vectors(a.dweight, a.dweight_stride, a.cout);
        if (int rc = dense<sq::kWeightGrad, false>(dz ? dz : a.dy, dz ? plan.pitch : a.dy_stride, wide, up(a.cin, 8), g, sums, device, sms, stream)) return rc;
    }
    return SQUANT_OK;
}

}  // extern "C"
