// Quantisation to e4m3 with a scale for each block of 128: rows of activations (blocks of 1 x 128 along the features of a worker's block) and weights
// (blocks of 128 x 128).  Every value is read once, held in registers while the block's largest magnitude is found, and written once.
#include <algorithm>
#include <cstring>

#include "common.h"
#include "eight_bit.h"

namespace distdl {

constexpr int kQuantThreads = 256;
constexpr int kMaxRowWorkers = 8;
constexpr int kMaxGridWorkers = 16;

struct QuantRowsParams {
    const void *x[kMaxRowWorkers];
    uint8_t *q[kMaxRowWorkers];
    float *s[kMaxRowWorkers];
    int64_t nb;
    int32_t bf, blocks;                    // features and blocks of a worker's row
};

// What bounds it: HBM, read once and written once.  B200: 8192 x 8192 bf16 36.5 us (5.6 TB/s), 4096 x 8192 fp32 28.5 (5.9); rows of 1001, which take
// 2-byte loads and byte stores whose number is what counts, 32.8 us for 8192 x 4004 (3.0 TB/s); 256 x 8192, in a graph, 2.4 us with x in L2, 3.5 from HBM.
// A thread block takes kSpan blocks side by side of rows r0, r0 + 1, ...: half a warp a block and row, kDepth rows of each in flight.  The scales of a block
// lie row by row, so those of the thread block's rows fill whole lines in L2 before they leave.
constexpr int kSpan = 4;
constexpr int kRowsAtOnce = kQuantThreads / kBlockLanes / kSpan;
constexpr int kDepth = 4;

template <typename T, int VW>
__global__ void __launch_bounds__(kQuantThreads)
quantize_rows_kernel(const __grid_constant__ QuantRowsParams P) {
    stream_enter();
    const int lane = threadIdx.x % kBlockLanes, unit = threadIdx.x / kBlockLanes;
    const int block = blockIdx.y * kSpan + unit % kSpan, worker = blockIdx.z;
    const int64_t row0 = (int64_t)blockIdx.x * (kRowsAtOnce * kDepth) + unit / kSpan;
    const int at = block * kScaleBlock + lane * VW;
    Eight<T> x[kDepth];
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
        const int64_t row = row0 + d * kRowsAtOnce;
        x[d].template load<VW>(reinterpret_cast<const T *>(P.x[worker]) + row * P.bf + at, row < P.nb ? P.bf - at : 0);
    }
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
        const int64_t row = row0 + d * kRowsAtOnce;
        float v[8];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = x[d].get(i);
            top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
        }
        const BlockScale s = block_scale(block_max(top));
        if (row >= P.nb || block >= P.blocks) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], s.inverse);
        store_e4m3<VW>(v, P.q[worker] + row * P.bf + at, P.bf - at);
        if (lane == 0) P.s[worker][block * P.nb + row] = s.scale;
    }
}

struct QuantWeightsParams {
    const void *w[kMaxGridWorkers];
    uint8_t *q[kMaxGridWorkers];
    float *s[kMaxGridWorkers];
    int32_t rows, cols;                    // of a worker's block
};

// What bounds it: HBM.  B200, 8192 x 8192 on 4 x 4 workers: fp32 52.2 us (6.4 TB/s), bf16 33.8 (6.0); 2048 x 1001 on the same grid 35.5 (4.6). A thread
// block holds a block of 128 x 128, so that its largest value is known without a second read: a warp reads its rows in pieces of 32 VW values, 64 values a
// thread.
template <typename T, int VW>
__global__ void __launch_bounds__(kQuantThreads)
quantize_weights_kernel(const __grid_constant__ QuantWeightsParams P) {
    stream_enter();
    __shared__ uint32_t tops[kQuantThreads / 32];
    constexpr int kRuns = 4 / VW;                              // a lane's runs of VW values in a row
    constexpr int kRows = kScaleBlock / (kQuantThreads / 32);  // rows of a warp
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int row0 = blockIdx.y * kScaleBlock + warp * kRows, col0 = blockIdx.x * kScaleBlock + lane * VW;
    const T *w = reinterpret_cast<const T *>(P.w[blockIdx.z]);
    constexpr int kWords = VW * (int)sizeof(T) / 4 > 0 ? VW * (int)sizeof(T) / 4 : 1;
    uint32_t raw[kRows][kRuns][kWords];
    uint32_t top = 0;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int u = 0; u < kRuns; ++u)
            ld_bytes<VW * (int)sizeof(T)>(w + (int64_t)(row0 + r) * P.cols + col0 + u * 32 * VW, raw[r][u], row0 + r < P.rows && col0 + u * 32 * VW < P.cols);
    const auto value = [&](int r, int u, int i) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(raw[r][u][i]);
        else return __uint_as_float(i & 1 ? raw[r][u][i >> 1] & 0xffff0000u : raw[r][u][i >> 1] << 16);
    };
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int u = 0; u < kRuns; ++u)
#pragma unroll
            for (int i = 0; i < VW; ++i) top = max(top, __float_as_uint(value(r, u, i)) & 0x7fffffffu);
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) tops[warp] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQuantThreads / 32; ++i) top = max(top, tops[i]);
    const BlockScale s = block_scale(top);
    if (threadIdx.x == 0) P.s[blockIdx.z][(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s.scale;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int u = 0; u < kRuns; ++u)
            if (row0 + r < P.rows && col0 + u * 32 * VW < P.cols) {
                float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < VW; ++i) v[i] = __fmul_rn(value(r, u, i), s.inverse);
                const uint32_t bytes = pack_e4m3(v[0], v[1], v[2], v[3]);
                st_bytes<VW>(P.q[blockIdx.z] + (int64_t)(row0 + r) * P.cols + col0 + u * 32 * VW, &bytes);
            }
}

static distdl_status_t quantize_rows_impl(int64_t nb, int64_t nf, int32_t pf, const void *const *x, distdl_dtype_t t, void *const *q, void *const *s,
                                          void *stream) {
    const char *what = "quantize_rows";
    clear_error();
    if (nb < 0 || nf < 1 || pf < 1) return fail(DISTDL_ERR_INVALID_ARG, "%s: non-positive size", what);
    if (t != DISTDL_F32 && t != DISTDL_BF16) return fail(DISTDL_ERR_INVALID_ARG, "%s: inputs are F32 or BF16", what);
    if (pf > kMaxRowWorkers) return fail(DISTDL_ERR_UNSUPPORTED, "%s: more than %d workers", what, kMaxRowWorkers);
    if (nf % pf) return fail(DISTDL_ERR_SHAPE, "%s: features not divisible by the workers", what);
    const int64_t bf = nf / pf, blocks = scale_blocks(bf), tiles = (nb + kRowsAtOnce * kDepth - 1) / (kRowsAtOnce * kDepth);
    if (bf > 1 << 24 || tiles > INT32_MAX) return fail(DISTDL_ERR_UNSUPPORTED, "%s: more than 2^24 features a worker or 2^31 tiles of 16 rows", what);
    if (nb == 0) return DISTDL_OK;
    distdl_status_t st;
    if ((st = check_blocks(what, "x", x, pf)) || (st = check_blocks(what, "q", q, pf)) || (st = check_blocks(what, "s", s, pf))) return st;
    QuantRowsParams P;
    memset(&P, 0, sizeof(P));
    for (int j = 0; j < pf; ++j) {
        P.x[j] = x[j];
        P.q[j] = (uint8_t *)q[j];
        P.s[j] = (float *)s[j];
    }
    P.nb = nb;
    P.bf = (int32_t)bf;
    P.blocks = (int32_t)blocks;
    int device;
    if ((st = current_device(what, x[0], &device))) return st;
    const dim3 grid((unsigned)tiles, (unsigned)((blocks + kSpan - 1) / kSpan), (unsigned)pf);
    const auto launch = [&](auto kernel) { launch_in_stream(kernel, grid, dim3(kQuantThreads), 0, (cudaStream_t)stream, P); };
    // the widest runs that the rows' length allows, 16 bytes at most (see element_of)
    if (t == DISTDL_BF16) {
        if (bf % 8 == 0) launch(quantize_rows_kernel<bf16, 8>);
        else if (bf % 2 == 0) launch(quantize_rows_kernel<bf16, 2>);
        else launch(quantize_rows_kernel<bf16, 1>);
    } else {
        if (bf % 4 == 0) launch(quantize_rows_kernel<float, 4>);
        else if (bf % 2 == 0) launch(quantize_rows_kernel<float, 2>);
        else launch(quantize_rows_kernel<float, 1>);
    }
    DISTDL_CUDA_CHECK(cudaGetLastError());
    return DISTDL_OK;
}

static distdl_status_t quantize_weights_impl(int64_t nfi, int64_t nfo, int32_t pfo, int32_t pfi, const void *const *w, distdl_dtype_t t, void *const *q,
                                             void *const *s, void *stream) {
    const char *what = "quantize_weights";
    clear_error();
    if (nfi < 1 || nfo < 1 || pfo < 1 || pfi < 1) return fail(DISTDL_ERR_INVALID_ARG, "%s: non-positive size", what);
    if (t != DISTDL_F32 && t != DISTDL_BF16) return fail(DISTDL_ERR_INVALID_ARG, "%s: weights are F32 or BF16", what);
    if (pfo > 8 || pfi > 8 || pfo * pfi > kMaxGridWorkers)
        return fail(DISTDL_ERR_UNSUPPORTED, "%s: worker grid larger than 8 per side or %d workers", what, kMaxGridWorkers);
    if (nfi % pfi || nfo % pfo) return fail(DISTDL_ERR_SHAPE, "%s: features not divisible by the worker grid", what);
    const int64_t rows = nfo / pfo, cols = nfi / pfi;
    if (rows > 1 << 22 || cols > 1 << 22) return fail(DISTDL_ERR_UNSUPPORTED, "%s: more than 2^22 rows or columns a worker", what);
    const int n = pfo * pfi;
    distdl_status_t st;
    if ((st = check_blocks(what, "w", w, n)) || (st = check_blocks(what, "q", q, n)) || (st = check_blocks(what, "s", s, n))) return st;
    QuantWeightsParams P;
    memset(&P, 0, sizeof(P));
    for (int i = 0; i < n; ++i) {
        P.w[i] = w[i];
        P.q[i] = (uint8_t *)q[i];
        P.s[i] = (float *)s[i];
    }
    P.rows = (int32_t)rows;
    P.cols = (int32_t)cols;
    int device;
    if ((st = current_device(what, w[0], &device))) return st;
    const dim3 grid((unsigned)scale_blocks(cols), (unsigned)scale_blocks(rows), (unsigned)n);
    const auto launch = [&](auto kernel) { launch_in_stream(kernel, grid, dim3(kQuantThreads), 0, (cudaStream_t)stream, P); };
    if (t == DISTDL_BF16) {
        if (cols % 4 == 0) launch(quantize_weights_kernel<bf16, 4>);
        else if (cols % 2 == 0) launch(quantize_weights_kernel<bf16, 2>);
        else launch(quantize_weights_kernel<bf16, 1>);
    } else {
        if (cols % 4 == 0) launch(quantize_weights_kernel<float, 4>);
        else if (cols % 2 == 0) launch(quantize_weights_kernel<float, 2>);
        else launch(quantize_weights_kernel<float, 1>);
    }
    DISTDL_CUDA_CHECK(cudaGetLastError());
    return DISTDL_OK;
}

}  // namespace distdl

extern "C" distdl_status_t distdl_quantize_rows(int64_t nb, int64_t nf, int32_t pf, const void *const *x, distdl_dtype_t t, void *const *q,
                                                void *const *s, void *stream) {
    return distdl::quantize_rows_impl(nb, nf, pf, x, t, q, s, stream);
}

extern "C" distdl_status_t distdl_quantize_weights(int64_t nfi, int64_t nfo, int32_t pfo, int32_t pfi, const void *const *w, distdl_dtype_t t,
                                                   void *const *q, void *const *s, void *stream) {
    return distdl::quantize_weights_impl(nfi, nfo, pfo, pfi, w, t, q, s, stream);
}
