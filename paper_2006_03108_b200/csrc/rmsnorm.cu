// Root-mean-square norm over features split over workers, with the residual's addition, 16 / 32-bit and 8-bit outputs, and its adjoint.
//
// The paper's algorithm would be: every worker sums the squares of its features, R over the workers, B of the mean back, a product on every worker.
// All workers' blocks lie in one memory, so a group of threads walks a sample's blocks through the list of workers and the sum stays on the chip.
//
// A sample's features are cut into chunks of eight values, sixteen chunks to a block of 128 (the blocks of a worker's last features are padded), so that
// half a warp holds a block whatever the sizes and finds its scale by itself.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "common.h"
#include "eight_bit.h"

namespace distdl {

constexpr int kNormMaxWorkers = 8;
constexpr int kNormMaxThreads = 1024;

struct NormParams {
    const void *x[kNormMaxWorkers], *res[kNormMaxWorkers];
    const float *gamma[kNormMaxWorkers];
    void *h[kNormMaxWorkers], *y[kNormMaxWorkers];
    uint8_t *q[kNormMaxWorkers];
    float *qs[kNormMaxWorkers];
    float *rstd;
    int64_t nb;
    int32_t bf, nf;
    int32_t worker_chunks, chunks;         // chunks of a worker's padded row, of a sample
    int32_t group;                         // threads on a sample: 16, or a multiple of 32
    float eps;
    bool add, sum, out, eight;             // there is a residual, h, y, q
};

// Where a chunk lies: its worker, its first element there, and what the worker's row has from there on.
struct ChunkAt {
    int worker, at, left;
    template <int VW, typename P>
    static __device__ __forceinline__ ChunkAt of(const P &p, int chunk) {
        ChunkAt c;
        c.worker = chunk / p.worker_chunks;
        const int in = chunk - c.worker * p.worker_chunks;
        c.at = in / kBlockLanes * kScaleBlock + in % kBlockLanes * VW;
        c.left = chunk < p.chunks ? p.bf - c.at : 0;
        if (chunk >= p.chunks) c.worker = 0;
        return c;
    }
};

// Sum over the threads of a sample's group; every one gets it.  Groups of more than a warp are the whole block.
__device__ __forceinline__ float group_sum(float v, int group, float *shared) {
    for (int d = min(group, 32) / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (group > 32) {
        const int warps = group / 32;
        if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = v;
        __syncthreads();
        v = (int)threadIdx.x % 32 < warps ? shared[threadIdx.x % 32] : 0.f;
        for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    }
    return v;
}

// Eight products of a lane with gamma, whose rows are read again for every sample and so stay in L1.
template <int VW>
__device__ __forceinline__ void load_gamma(const float *g, int left, float *v) {
#pragma unroll
    for (int r = 0; r < 8 / VW; ++r) {
        const bool there = r * kBlockLanes * VW < left;
        const float *p = g + r * kBlockLanes * VW;
        if constexpr (VW >= 4) {
#pragma unroll
            for (int i = 0; i < VW; i += 4) {
                const float4 f = there ? __ldg(reinterpret_cast<const float4 *>(p + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
                v[r * VW + i] = f.x, v[r * VW + i + 1] = f.y, v[r * VW + i + 2] = f.z, v[r * VW + i + 3] = f.w;
            }
        } else if constexpr (VW == 2) {
            const float2 f = there ? __ldg(reinterpret_cast<const float2 *>(p)) : make_float2(0.f, 0.f);
            v[2 * r] = f.x, v[2 * r + 1] = f.y;
        } else {
            v[r] = there ? __ldg(p) : 0.f;
        }
    }
}

template <typename T, int VW>
__device__ __forceinline__ Eight<T> norm_input(const NormParams &P, int64_t row, const ChunkAt &c) {
    Eight<T> x;
    x.template load<VW>(reinterpret_cast<const T *>(P.x[c.worker]) + row * P.bf + c.at, c.left);
    return x;
}
template <typename T, int VW>
__device__ __forceinline__ Eight<T> norm_residual(const NormParams &P, int64_t row, const ChunkAt &c) {
    Eight<T> x;
    x.template load<VW>(reinterpret_cast<const T *>(P.res[c.worker]) + row * P.bf + c.at, c.left);
    return x;
}
template <typename T>
__device__ __forceinline__ void norm_add(Eight<T> &x, const Eight<T> &res) {
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = __fadd_rn(x.get(i), res.get(i));
    x.set(s);
}
// The outputs of a chunk: all lanes of its block are here.
template <typename T, int VW>
__device__ __forceinline__ void norm_write(const NormParams &P, int64_t row, const ChunkAt &c, const Eight<T> &h, float rstd) {
    float y[8];
    load_gamma<VW>(P.gamma[c.worker] + c.at, c.left, y);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __fmul_rn(__fmul_rn(h.get(i), rstd), y[i]);
    const int64_t at = row * P.bf + c.at;
    if (P.out) {
        Eight<T> o;
        o.set(y);
        o.template store<VW>(reinterpret_cast<T *>(P.y[c.worker]) + at, c.left);
    }
    if (P.eight) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
        const BlockScale s = block_scale(block_max(top));
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __fmul_rn(y[i], s.inverse);
        store_e4m3<VW>(y, P.q[c.worker] + at, c.left);
        if (threadIdx.x % kBlockLanes == 0 && c.left > 0) P.qs[c.worker][c.at / kScaleBlock * P.nb + row] = s.scale;
    }
}

// V: chunks of a thread, which stay in registers between the two passes over the sample; 0: any number, read again.
//
// What bounds it: HBM for many samples -- every input is read once and every output written once -- and the latency of one pass for few.  B200, bf16 with
// residual, h, y, q: 8192 x 8192 on four workers 107 us (5.7 TB/s, 0.87 of the copy rate), 8192 x 4096 53 (5.7), 32768 x 512 29 (5.2), 4000 x 2 x 1415
// 39 (2.6; an access of 2 bytes for every value, and their number is what counts); fp32 8192 x 8192 207 (5.5); one sample of 8192 with h, q in a graph 3.3 us.
// Four chunks in bfloat16 spill 48 bytes of a thread's 64 registers.
template <typename T, int VW, int V>
__global__ void __launch_bounds__(kNormMaxThreads)
rmsnorm_kernel(const __grid_constant__ NormParams P) {
    stream_enter();
    __shared__ float shared[32];
    const int t = threadIdx.x % P.group;
    const int64_t first = (int64_t)blockIdx.x * (blockDim.x / P.group) + threadIdx.x / P.group;
    const bool there = first < P.nb;                   // groups past the last sample read and write nothing
    const int64_t row = there ? first : P.nb - 1;
    float squares = 0.f;
    if constexpr (V > 0) {
        ChunkAt c[V];
        Eight<T> h[V], res[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            c[v] = ChunkAt::of<VW>(P, t + v * P.group);
            if (!there) c[v].left = 0;
            h[v] = norm_input<T, VW>(P, row, c[v]);
        }
        if (P.add) {
#pragma unroll
            for (int v = 0; v < V; ++v) res[v] = norm_residual<T, VW>(P, row, c[v]);
#pragma unroll
            for (int v = 0; v < V; ++v) norm_add(h[v], res[v]);
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) squares = fmaf(h[v].get(i), h[v].get(i), squares);
        const float rstd = 1.f / sqrtf(group_sum(squares, P.group, shared) / (float)P.nf + P.eps);
        if (there && t == 0 && P.rstd) P.rstd[row] = rstd;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (P.sum) h[v].template store<VW>(reinterpret_cast<T *>(P.h[c[v].worker]) + row * P.bf + c[v].at, c[v].left);
            norm_write<T, VW>(P, row, c[v], h[v], rstd);
        }
    } else {
        // one sample a block: whole blocks of 128 walk together
        const auto input = [&](const ChunkAt &c) {
            Eight<T> h = norm_input<T, VW>(P, row, c);
            if (P.add) norm_add(h, norm_residual<T, VW>(P, row, c));
            return h;
        };
        for (int k = t; k < P.chunks; k += P.group) {
            const Eight<T> h = input(ChunkAt::of<VW>(P, k));
#pragma unroll
            for (int i = 0; i < 8; ++i) squares = fmaf(h.get(i), h.get(i), squares);
        }
        const float rstd = 1.f / sqrtf(group_sum(squares, P.group, shared) / (float)P.nf + P.eps);
        if (t == 0 && P.rstd) P.rstd[row] = rstd;
        for (int k = t; k - t < P.chunks; k += P.group) {
            const ChunkAt c = ChunkAt::of<VW>(P, k);
            const Eight<T> h = input(c);
            if (P.sum) h.template store<VW>(reinterpret_cast<T *>(P.h[c.worker]) + row * P.bf + c.at, c.left);
            norm_write<T, VW>(P, row, c, h, rstd);
        }
    }
}

// ------------------------------------------------------------------------------------------
// Adjoint
// ------------------------------------------------------------------------------------------
struct NormAdjParams {
    const void *dy[kNormMaxWorkers], *dres[kNormMaxWorkers], *h[kNormMaxWorkers];
    const float *gamma[kNormMaxWorkers];
    void *dh[kNormMaxWorkers];
    float *dgamma[kNormMaxWorkers];
    const float *rstd;
    float *partial;                        // [thread blocks][chunks * 8]: sums over a thread block's samples, in the chunks' order
    float *dots;                           // [nb]: sum over the features of gamma dy h, where a kernel of its own takes it
    int64_t nb;
    int32_t bf, nf;
    int32_t worker_chunks, chunks;
    int32_t group;
    int32_t rows;                          // thread blocks over the samples
    bool add, params;
};

template <typename T, typename TG>
__device__ __forceinline__ float norm_dot(const float *g, const Eight<TG> &dy, const Eight<T> &h) {
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) dot = fmaf(g[i] * dy.get(i), h.get(i), dot);
    return dot;
}

// Many features: the sums over a sample's features, a thread block a sample.
template <typename T, typename TG, int VW>
__global__ void __launch_bounds__(kNormMaxThreads)
rmsnorm_dots_kernel(const __grid_constant__ NormAdjParams P) {
    stream_enter();
    __shared__ float shared[32];
    const int64_t row = blockIdx.x;
    float dot = 0.f;
    for (int k = threadIdx.x; k < P.chunks; k += blockDim.x) {
        const ChunkAt c = ChunkAt::of<VW>(P, k);
        Eight<TG> dy;
        Eight<T> h;
        dy.template load<VW>(reinterpret_cast<const TG *>(P.dy[c.worker]) + row * P.bf + c.at, c.left);
        h.template load<VW>(reinterpret_cast<const T *>(P.h[c.worker]) + row * P.bf + c.at, c.left);
        float gamma[8];
        load_gamma<VW>(P.gamma[c.worker] + c.at, c.left, gamma);
        dot += norm_dot(gamma, dy, h);
    }
    dot = group_sum(dot, (int)blockDim.x, shared);
    if (threadIdx.x == 0) P.dots[row] = dot;
}

// Threads of a multiprocessor by a thread's chunks: what their registers allow, and the most of a thread block
constexpr int adj_resident(bool all_bf16, int v) { return v > 1 ? 512 : all_bf16 ? 768 : 640; }

// Persistent: a thread keeps its V chunks of the features for all samples of its group (P.rows * groups apart) and sums dgamma in registers; the groups of
// a block add up through shared memory, the blocks through `partial` and a second kernel, each in a fixed order. GIVEN: the sample's sums are there already
// and blockIdx.y is a piece of the features (more than some 8192 features in 32 bits, 16384 in 16: no thread block holds a sample and its sums of dgamma;
// dy and h are read twice then).
//
// What bounds it: HBM, with one sample in work and the next on its way in every thread block; a thread block a sample and multiprocessor in flight reached
// half of it. B200, with dres, the fold of dgamma included: 8192 x 8192 bf16 92 us (5.8 TB/s, 0.9 of the copy rate), 8192 x 4096 48 (5.6), 4096 x 4096 fp32
// 46 (5.9), 1021 x 5000 fp32 in rows of 1250 (8-byte loads) 18.5 (4.4), 1000 x 32768 bf16 74 (3.5; 5.3 with what is read twice). Two chunks without look-ahead,
// beyond 5120 features with a 32-bit type, lose nothing by it: 8192 x 8192 bf16 with fp32 gradients 158 (5.9), fp32 171 (6.3); 4096 x 5120 with one chunk
// 51 (5.7).  Four in bfloat16, beyond 8192 features, do, and spill 116 to 280 bytes a thread: 4096 x 12288 119 (3.4), 4096 x 16384 135 (4.0).
template <typename T, typename TG, int VW, int V, bool GIVEN>
__global__ void __launch_bounds__(adj_resident(sizeof(T) + sizeof(TG) <= 4, V), 1)
rmsnorm_adj_kernel(const __grid_constant__ NormAdjParams P) {
    stream_enter();
    __shared__ float shared[2][32];
    __shared__ float sums[GIVEN ? 1 : 32 * V * 8];
    const int t = threadIdx.x % P.group, g = threadIdx.x / P.group, groups = blockDim.x / P.group;
    const int chunk0 = t + blockIdx.y * P.group * V;
    ChunkAt c[V];
    constexpr bool kHold = V == 1;         // gamma in registers; else it comes from L1 for every sample
    float gamma[kHold ? V : 1][8], dgamma[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = ChunkAt::of<VW>(P, chunk0 + v * P.group);
        if (kHold) load_gamma<VW>(P.gamma[c[v].worker] + c[v].at, c[v].left, gamma[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dgamma[v][i] = 0.f;
    }
    const int64_t step = (int64_t)P.rows * groups;
    int turn = 0;
    struct Sample {
        Eight<TG> dy[V], dres[V];
        Eight<T> h[V];
        float rstd, dot;
    };
    const auto load = [&](Sample &s, int64_t row) {
        const bool there = row < P.nb;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int left = there ? c[v].left : 0;
            const int64_t at = row * P.bf + c[v].at;
            s.dy[v].template load<VW>(reinterpret_cast<const TG *>(P.dy[c[v].worker]) + at, left);
            s.h[v].template load<VW>(reinterpret_cast<const T *>(P.h[c[v].worker]) + at, left);
            s.dres[v].template load<VW>(reinterpret_cast<const TG *>(P.dres[c[v].worker]) + at, P.add ? left : 0);
        }
        s.rstd = there ? P.rstd[row] : 0.f;
        if constexpr (GIVEN) s.dot = there ? P.dots[row] : 0.f;
    };
    // the next sample is on its way while this one is worked on, where there are registers for it
    constexpr bool kAhead = V == 1 || (sizeof(T) + sizeof(TG) <= 4 && V == 2);
    Sample s, next;
    if (kAhead) load(next, (int64_t)blockIdx.x * groups + g);
    for (int64_t first = (int64_t)blockIdx.x * groups; first < P.nb; first += step, turn ^= 1) {
        const int64_t row = first + g;
        const bool there = row < P.nb;
        if (kAhead) {
            s = next;
            load(next, row + step);
        } else {
            load(s, row);
        }
        const auto &dy = s.dy, &dres = s.dres;
        const auto &h = s.h;
        const float rstd = s.rstd;
        float dot = 0.f;
        if constexpr (GIVEN) {
            dot = s.dot;
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!kHold) load_gamma<VW>(P.gamma[c[v].worker] + c[v].at, c[v].left, gamma[0]);
                dot += norm_dot(gamma[kHold ? v : 0], dy[v], h[v]);
            }
            dot = group_sum(dot, P.group, shared[turn]);
        }
        // hhat * mean(gamma dy hhat) * rstd as a product with hhat: h times the square of rstd would be the same, but a root above 2^64 has no square in fp32,
        // and a sample of zeros would be 0 * infinity
        const float back = rstd * (dot * rstd / (float)P.nf);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float o[8];
            if (!kHold) load_gamma<VW>(P.gamma[c[v].worker] + c[v].at, c[v].left, gamma[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = dy[v].get(i), x = h[v].get(i);
                const float hat = x * rstd;
                o[i] = fmaf(rstd, gamma[kHold ? v : 0][i] * d, dres[v].get(i)) - hat * back;
                dgamma[v][i] = fmaf(d, hat, dgamma[v][i]);
            }
            Eight<TG> e;
            e.set(o);
            e.template store<VW>(reinterpret_cast<TG *>(P.dh[c[v].worker]) + row * P.bf + c[v].at, there ? c[v].left : 0);
        }
    }
    if (!P.params) return;
    if constexpr (!GIVEN) {
        if (groups > 1) {                                          // groups of 16 or 32 threads: one after the other
            for (int k = 0; k < groups; ++k) {
                __syncthreads();
                if (g == k) {
#pragma unroll
                    for (int v = 0; v < V; ++v)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float *s = &sums[(t + v * P.group) * 8 + i];
                            *s = k ? *s + dgamma[v][i] : dgamma[v][i];
                        }
                }
            }
            if (g != groups - 1) return;                           // the last group's threads hold the sums' last terms
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) dgamma[v][i] = sums[(t + v * P.group) * 8 + i];
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int chunk = chunk0 + v * P.group;
        if (chunk < P.chunks) {
            float4 *o = reinterpret_cast<float4 *>(P.partial + ((int64_t)blockIdx.x * P.chunks + chunk) * 8);
            o[0] = make_float4(dgamma[v][0], dgamma[v][1], dgamma[v][2], dgamma[v][3]);
            o[1] = make_float4(dgamma[v][4], dgamma[v][5], dgamma[v][6], dgamma[v][7]);
        }
    }
}

// dgamma: the thread blocks' sums, 32 slices of them by a warp each, the slices in order.
constexpr int kFoldColumns = 32, kFoldSlices = 32;
template <int VW>
__global__ void __launch_bounds__(kFoldColumns * kFoldSlices)
rmsnorm_fold_kernel(const __grid_constant__ NormAdjParams P) {
    stream_enter();
    __shared__ float part[kFoldSlices][kFoldColumns];
    const int column = blockIdx.x * kFoldColumns + threadIdx.x % kFoldColumns, slice = threadIdx.x / kFoldColumns, columns = P.chunks * 8;
    const int per = (P.rows + kFoldSlices - 1) / kFoldSlices, r0 = slice * per, r1 = min(P.rows, r0 + per);
    float s = 0.f;
    for (int r = r0; r < r1; r += 8) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = r + i < r1 ? P.partial[(int64_t)(r + i) * columns + column] : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[i];
    }
    part[slice][threadIdx.x % kFoldColumns] = s;
    __syncthreads();
    if (slice) return;
    for (int k = 1; k < kFoldSlices; ++k) s += part[k][threadIdx.x];
    const int chunk = column / 8, worker = chunk / P.worker_chunks, in = chunk - worker * P.worker_chunks;
    const int at = in / kBlockLanes * kScaleBlock + element_of<VW>(in % kBlockLanes, column % 8);
    if (at < P.bf) P.dgamma[worker][at] = s;
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------
struct NormShape {
    int64_t bf, chunks;
    int32_t worker_chunks;
};
static distdl_status_t norm_shape(const char *what, int64_t nb, int64_t nf, int32_t pf, NormShape *s) {
    if (nb < 0 || nf < 1 || pf < 1) return fail(DISTDL_ERR_INVALID_ARG, "%s: non-positive size", what);
    if (pf > kNormMaxWorkers) return fail(DISTDL_ERR_UNSUPPORTED, "%s: more than %d workers", what, kNormMaxWorkers);
    if (nf % pf) return fail(DISTDL_ERR_SHAPE, "%s: features not divisible by the workers", what);
    if (nf > 1 << 20 || nb > INT32_MAX) return fail(DISTDL_ERR_UNSUPPORTED, "%s: more than 2^20 features or 2^31 samples", what);
    s->bf = nf / pf;
    s->worker_chunks = (int32_t)scale_blocks(s->bf) * kBlockLanes;
    s->chunks = (int64_t)s->worker_chunks * pf;
    return DISTDL_OK;
}
static bool float_type(distdl_dtype_t t) { return t == DISTDL_F32 || t == DISTDL_BF16; }
static int run_width(int64_t bf, bool all_bf16) {
    for (int w = all_bf16 ? 8 : 4; w > 1; w /= 2)
        if (bf % w == 0) return w;
    return 1;
}
// Threads for n chunks at a time: groups of 16 or 32 share a block of 128 threads, larger ones are whole warps and a block.
static int group_of(int64_t n, int most) { return n <= kBlockLanes ? kBlockLanes : (int)std::min<int64_t>((n + 31) / 32 * 32, most); }
static int block_of(int group) { return group > 32 ? group : 128; }

template <typename T, int VW>
static void norm_launch(NormParams &P, cudaStream_t stream, int sms) {
    // chunks of a thread: four of 16 bytes (two of 32, or of narrower pieces) where the samples fill the device, else as few as a block of 1024 threads allows
    constexpr int kMost = sizeof(T) == 2 && VW == 8 ? 4 : 2;
    int v = P.nb >= 2 * sms ? kMost : 1;
    while (v < kMost && P.chunks > (int64_t)v * kNormMaxThreads) v *= 2;
    P.group = group_of((P.chunks + v - 1) / v, kNormMaxThreads);
    const bool again = P.chunks > (int64_t)v * P.group;
    const int threads = block_of(P.group), per = threads / P.group;
    const dim3 grid((unsigned)((P.nb + per - 1) / per));
    const auto launch = [&](auto kernel) { launch_in_stream(kernel, grid, dim3((unsigned)threads), 0, stream, P); };
    if (again) launch(rmsnorm_kernel<T, VW, 0>);
    else if (v == 1) launch(rmsnorm_kernel<T, VW, 1>);
    else if (v == 2) launch(rmsnorm_kernel<T, VW, 2>);
    else if constexpr (kMost == 4) launch(rmsnorm_kernel<T, VW, 4>);
}

static distdl_status_t rmsnorm_fwd_impl(int64_t nb, int64_t nf, int32_t pf, const void *const *x, const void *const *residual, const void *const *gamma,
                                        const double *eps, distdl_dtype_t t, void *const *h, void *const *y, void *const *q, void *const *qs, void *rstd,
                                        void *stream) {
    const char *what = "rmsnorm_fwd";
    clear_error();
    NormShape s;
    distdl_status_t st;
    if ((st = norm_shape(what, nb, nf, pf, &s))) return st;
    if (!float_type(t)) return fail(DISTDL_ERR_INVALID_ARG, "%s: values are F32 or BF16", what);
    // below 2^-120 the squares of what weighs against eps are subnormal in fp32, and their sum is no longer good to its roundings
    if (!eps || !(*eps >= 0x1p-120) || !std::isfinite((float)*eps)) return fail(DISTDL_ERR_INVALID_ARG, "%s: eps must be a number from 2^-120 on", what);
    if (!h && !y && !q && !rstd) return fail(DISTDL_ERR_INVALID_ARG, "%s: no output", what);
    if (!q != !qs) return fail(DISTDL_ERR_INVALID_ARG, "%s: q and qs come together", what);
    if (nb == 0) return DISTDL_OK;
    if ((st = check_blocks(what, "x", x, pf)) || (st = check_blocks(what, "gamma", gamma, pf))) return st;
    if (residual && (st = check_blocks(what, "residual", residual, pf))) return st;
    if (h && (st = check_blocks(what, "h", h, pf))) return st;
    if (y && (st = check_blocks(what, "y", y, pf))) return st;
    if (q && ((st = check_blocks(what, "q", q, pf)) || (st = check_blocks(what, "qs", qs, pf)))) return st;
    if (rstd && !aligned16(rstd)) return fail(DISTDL_ERR_ALIGNMENT, "%s: rstd not 16-byte aligned", what);
    NormParams P;
    memset(&P, 0, sizeof(P));
    for (int j = 0; j < pf; ++j) {
        P.x[j] = x[j];
        P.gamma[j] = (const float *)gamma[j];
        if (residual) P.res[j] = residual[j];
        if (h) P.h[j] = h[j];
        if (y) P.y[j] = y[j];
        if (q) P.q[j] = (uint8_t *)q[j], P.qs[j] = (float *)qs[j];
    }
    P.rstd = (float *)rstd;
    P.nb = nb;
    P.bf = (int32_t)s.bf;
    P.nf = (int32_t)nf;
    P.worker_chunks = s.worker_chunks;
    P.chunks = (int32_t)s.chunks;
    P.eps = (float)*eps;
    P.add = residual != nullptr;
    P.sum = h != nullptr;
    P.out = y != nullptr;
    P.eight = q != nullptr;
    int device, sms;
    if ((st = current_device(what, x[0], &device)) || (st = multiprocessors(device, &sms))) return st;
    const int vw = run_width(s.bf, t == DISTDL_BF16);
    const cudaStream_t in = (cudaStream_t)stream;
    if (t == DISTDL_BF16 && vw == 8) norm_launch<bf16, 8>(P, in, sms);
    else if (t == DISTDL_BF16) vw == 4 ? norm_launch<bf16, 4>(P, in, sms) : vw == 2 ? norm_launch<bf16, 2>(P, in, sms) : norm_launch<bf16, 1>(P, in, sms);
    else vw == 4 ? norm_launch<float, 4>(P, in, sms) : vw == 2 ? norm_launch<float, 2>(P, in, sms) : norm_launch<float, 1>(P, in, sms);
    DISTDL_CUDA_CHECK(cudaGetLastError());
    return DISTDL_OK;
}

// Chunks a thread keeps in the adjoint, and whether a sample's features fit one thread block (else a kernel of its own takes the sums over them).
struct AdjShape {
    int v, group, threads;
    bool given;
    int32_t rows;                          // thread blocks over the samples
    int pieces;                            // of the features
};
static AdjShape adj_shape(int64_t nb, int64_t chunks, bool all_bf16, int sms) {
    AdjShape a;
    // one chunk where a multiprocessor has two thread blocks of them (16 bits) or holds a sample and the next one (32 bits)
    a.v = chunks <= (all_bf16 ? 384 : 640) ? 1 : all_bf16 && chunks > 2 * adj_resident(true, 2) ? 4 : 2;
    a.group = group_of((chunks + a.v - 1) / a.v, adj_resident(all_bf16, a.v));
    a.given = chunks > (int64_t)a.v * a.group;
    if (a.given) a.group = 256;
    a.threads = block_of(a.group);
    a.pieces = a.given ? (int)((chunks + (int64_t)a.v * a.group - 1) / ((int64_t)a.v * a.group)) : 1;
    const int64_t resident = (int64_t)sms * (adj_resident(all_bf16, a.v) / a.threads), groups = a.threads / a.group;
    a.rows = (int32_t)std::max<int64_t>(1, std::min<int64_t>((nb + groups - 1) / groups, resident / a.pieces));
    return a;
}
static int64_t adj_workspace(const AdjShape &a, int64_t nb, int64_t chunks) { return (int64_t)a.rows * chunks * 8 * 4 + (a.given ? (nb + 3) / 4 * 16 : 0); }

template <typename T, typename TG, int VW>
static void adj_launch(NormAdjParams &P, const AdjShape &a, cudaStream_t stream) {
    constexpr int kMost = sizeof(T) == 2 && sizeof(TG) == 2 ? 4 : 2;
    const dim3 grid((unsigned)a.rows, (unsigned)a.pieces), block((unsigned)a.threads);
    if (a.given) {
        launch_in_stream(rmsnorm_dots_kernel<T, TG, VW>, dim3((unsigned)P.nb), dim3(512), 0, stream, P);
        launch_in_stream(rmsnorm_adj_kernel<T, TG, VW, kMost, true>, grid, block, 0, stream, P);
    } else if (a.v == 1) {
        launch_in_stream(rmsnorm_adj_kernel<T, TG, VW, 1, false>, grid, block, 0, stream, P);
    } else if (a.v == 2) {
        launch_in_stream(rmsnorm_adj_kernel<T, TG, VW, 2, false>, grid, block, 0, stream, P);
    } else {
        launch_in_stream(rmsnorm_adj_kernel<T, TG, VW, kMost, false>, grid, block, 0, stream, P);
    }
    if (P.params) launch_in_stream(rmsnorm_fold_kernel<VW>, dim3((unsigned)(P.chunks * 8 / kFoldColumns)), dim3(kFoldColumns * kFoldSlices), 0, stream, P);
}
template <typename T, typename TG>
static void adj_launch_width(NormAdjParams &P, const AdjShape &a, int vw, cudaStream_t stream) {
    if constexpr (sizeof(T) == 2 && sizeof(TG) == 2)
        if (vw == 8) return adj_launch<T, TG, 8>(P, a, stream);
    if (vw == 4) adj_launch<T, TG, 4>(P, a, stream);
    else if (vw == 2) adj_launch<T, TG, 2>(P, a, stream);
    else adj_launch<T, TG, 1>(P, a, stream);
}

static distdl_status_t rmsnorm_adj_impl(int64_t nb, int64_t nf, int32_t pf, const void *const *dy, const void *const *dres, const void *const *h,
                                        const void *const *gamma, const void *rstd, distdl_dtype_t t, distdl_dtype_t tg, void *const *dh,
                                        void *const *dgamma, void *workspace, int64_t workspace_bytes, void *stream) {
    const char *what = "rmsnorm_adj";
    clear_error();
    NormShape s;
    distdl_status_t st;
    if ((st = norm_shape(what, nb, nf, pf, &s))) return st;
    if (!float_type(t) || !float_type(tg)) return fail(DISTDL_ERR_INVALID_ARG, "%s: values are F32 or BF16", what);
    if (dgamma && (st = check_blocks(what, "dgamma", dgamma, pf))) return st;
    int device, sms;
    NormAdjParams P;
    memset(&P, 0, sizeof(P));
    if (nb == 0) {                          // a sum over no samples
        if (!dgamma) return DISTDL_OK;
        if ((st = current_device(what, dgamma[0], &device))) return st;
        for (int j = 0; j < pf; ++j) DISTDL_CUDA_CHECK(cudaMemsetAsync(dgamma[j], 0, (size_t)s.bf * 4, (cudaStream_t)stream));
        return DISTDL_OK;
    }
    if ((st = check_blocks(what, "dy", dy, pf)) || (st = check_blocks(what, "h", h, pf)) || (st = check_blocks(what, "gamma", gamma, pf)) ||
        (st = check_blocks(what, "dh", dh, pf)))
        return st;
    if (dres && (st = check_blocks(what, "dres", dres, pf))) return st;
    if (!rstd || !workspace) return fail(DISTDL_ERR_INVALID_ARG, "%s: rstd or workspace is NULL", what);
    if (!aligned16(rstd) || !aligned16(workspace)) return fail(DISTDL_ERR_ALIGNMENT, "%s: rstd or workspace not 16-byte aligned", what);
    if ((st = current_device(what, dy[0], &device)) || (st = multiprocessors(device, &sms))) return st;
    const bool all_bf16 = t == DISTDL_BF16 && tg == DISTDL_BF16;
    const AdjShape a = adj_shape(nb, s.chunks, all_bf16, sms);
    const int64_t need = adj_workspace(a, nb, s.chunks);
    if (workspace_bytes < need)
        return fail(DISTDL_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld are needed", what, (long long)workspace_bytes, (long long)need);
    for (int j = 0; j < pf; ++j) {
        P.dy[j] = dy[j];
        P.dres[j] = dres ? dres[j] : nullptr;
        P.h[j] = h[j];
        P.gamma[j] = (const float *)gamma[j];
        P.dh[j] = dh[j];
        if (dgamma) P.dgamma[j] = (float *)dgamma[j];
    }
    P.rstd = (const float *)rstd;
    P.partial = (float *)workspace;
    P.dots = (float *)workspace + (int64_t)a.rows * s.chunks * 8;
    P.nb = nb;
    P.bf = (int32_t)s.bf;
    P.nf = (int32_t)nf;
    P.worker_chunks = s.worker_chunks;
    P.chunks = (int32_t)s.chunks;
    P.group = a.group;
    P.rows = a.rows;
    P.add = dres != nullptr;
    P.params = dgamma != nullptr;
    const int vw = run_width(s.bf, all_bf16);
    const cudaStream_t in = (cudaStream_t)stream;
    if (t == DISTDL_BF16) tg == DISTDL_BF16 ? adj_launch_width<bf16, bf16>(P, a, vw, in) : adj_launch_width<bf16, float>(P, a, vw, in);
    else tg == DISTDL_BF16 ? adj_launch_width<float, bf16>(P, a, vw, in) : adj_launch_width<float, float>(P, a, vw, in);
    DISTDL_CUDA_CHECK(cudaGetLastError());
    return DISTDL_OK;
}

}  // namespace distdl

extern "C" distdl_status_t distdl_rmsnorm_fwd(int64_t nb, int64_t nf, int32_t pf, const void *const *x, const void *const *residual,
                                              const void *const *gamma, const double *eps, distdl_dtype_t t, void *const *h, void *const *y, void *const *q,
                                              void *const *qs, void *rstd, void *stream) {
    return distdl::rmsnorm_fwd_impl(nb, nf, pf, x, residual, gamma, eps, t, h, y, q, qs, rstd, stream);
}

extern "C" distdl_status_t distdl_rmsnorm_adj_workspace(int64_t nb, int64_t nf, int32_t pf, int64_t *bytes) {
    using namespace distdl;
    clear_error();
    NormShape s;
    const distdl_status_t st = norm_shape("rmsnorm_adj_workspace", nb, nf, pf, &s);
    if (st) return st;
    if (!bytes) return fail(DISTDL_ERR_INVALID_ARG, "rmsnorm_adj_workspace: NULL argument");
    int device = 0, sms = 0;
    DISTDL_CUDA_CHECK(cudaGetDevice(&device));
    if (device < 0 || device >= kMaxDevicesPerProcess) return fail(DISTDL_ERR_UNSUPPORTED, "rmsnorm_adj_workspace: device index %d", device);
    if (const distdl_status_t found = multiprocessors(device, &sms)) return found;
    // enough for either type of the values
    const auto bytes_for = [&](bool all_bf16) { return adj_workspace(adj_shape(nb, s.chunks, all_bf16, sms), nb, s.chunks); };
    *bytes = std::max<int64_t>(16, std::max(bytes_for(true), bytes_for(false)));
    return DISTDL_OK;
}

extern "C" distdl_status_t distdl_rmsnorm_adj(int64_t nb, int64_t nf, int32_t pf, const void *const *dy, const void *const *dres, const void *const *h,
                                              const void *const *gamma, const void *rstd, distdl_dtype_t t, distdl_dtype_t tg, void *const *dh,
                                              void *const *dgamma, void *workspace, int64_t workspace_bytes, void *stream) {
    return distdl::rmsnorm_adj_impl(nb, nf, pf, dy, dres, h, gamma, rstd, t, tg, dh, dgamma, workspace, workspace_bytes, stream);
}
