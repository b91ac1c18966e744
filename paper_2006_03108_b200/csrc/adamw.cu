// AdamW over lists of tensors: decoupled weight decay, states in fp32 or in 8 bits with a scale for each block of 128, optional bfloat16 copies of
// the weights.  One launch takes up to kTensorsAtOnce tensors of any sizes.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "common.h"
#include "eight_bit.h"

namespace distdl {

constexpr int kAdamThreads = 256;
// Blocks of 128 of a thread block's tile.  fp32 states: one for each half warp, and more thread blocks to hide the loads; 8-bit states: two, since what a
// thread does before its first element counts there (67 M weights, B200: 294 us against 300; 200 against 240).
__host__ __device__ constexpr int tile_blocks(bool eight) { return eight ? 32 : 16; }
// Tensors of a launch.  Its parameters hold them all, 21 KB; lists of up to 24 go with 1.7, which saves 0.65 us of a call's 4.6.
constexpr int kTensorsAtOnce = 320, kFewTensors = 24;

struct AdamTensor {
    float *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    uint16_t *copy;
    int64_t n;
};
struct AdamCommon {
    int32_t count, first_tensor;                         // tensors of this launch; number of its first one in the call
    float beta1, one_beta1, beta2, one_beta2, eps, decay;
    float log_beta1, log_beta2;
    float lr_decay, grad_scale;
    float rate, root;                                    // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    uint32_t seed, step;
    const float *live;                                   // {lr, t, gradient scale} on the device, or null: what stands above
};
template <int N>
struct AdamParams : AdamCommon {
    AdamTensor tensor[N];
    uint32_t first_tile[N + 1];                          // of each tensor, and behind the last
};
static_assert(sizeof(AdamParams<kTensorsAtOnce>) < 32700, "kernel parameters");

// 32 well mixed bits of 32: multiplications by odd constants and shifted copies.
__host__ __device__ __forceinline__ uint32_t mixed(uint32_t x) {
    x ^= x >> 16;
    x *= 0xB504F333u;
    x ^= x >> 15;
    x *= 0x93CD3A2Du;
    return x ^ (x >> 16);
}

// The larger one, or NaN.
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float reciprocal(float v) {      // of a normal number, to 2^-23
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
// Root to 2^-23 or so, subnormal numbers included.
__device__ __forceinline__ float root(float v) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

struct AdamStep {
    float rate, root, decay, grad_scale;                 // decay: lr times the decay
    uint32_t key;
};

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 pair_at(const float *v) { return make_float2(v[0], v[1]); }
__device__ __forceinline__ void pair_to(float *v, float2 w) { v[0] = w.x, v[1] = w.y; }

// Two elements at a time: what bounds steps with 8-bit states is the number of instructions, and these do two elements' products or sums each.
template <bool EIGHT>
__device__ __forceinline__ void adam_pair(const AdamCommon &P, const AdamStep &s, float *p, const float *g, float *m, float *v) {
    const float2 w = pair_at(p), h = __fmul2_rn(pair_at(g), both(s.grad_scale));
    const float2 a = __ffma2_rn(both(P.beta1), pair_at(m), __fmul2_rn(both(P.one_beta1), h));
    const float2 b = __ffma2_rn(both(P.beta2), pair_at(v), __fmul2_rn(__fmul2_rn(both(P.one_beta2), h), h));
    const float2 r = make_float2(root(b.x), root(b.y));
    const float2 below = __ffma2_rn(r, both(s.root), both(P.eps));
    const float2 step = __fmul2_rn(__fmul2_rn(both(s.rate), a), make_float2(reciprocal(below.x), reciprocal(below.y)));
    pair_to(p, __ffma2_rn(__ffma2_rn(both(s.decay), w, step), both(-1.f), w));          // the weight is rounded once
    pair_to(m, a);
    pair_to(v, EIGHT ? r : b);
}

// What bounds it: HBM with fp32 states (67 M weights in 16 tensors, bf16 copies: 295 us, 6.8 TB/s; 150 tensors of 5 to 1,000,003 elements, 17 M in all,
// without: 73 us, 6.6 TB/s), HBM and the issue of instructions about equally with 8-bit ones (200 us, 6.1 TB/s; at 110 instructions an element it was 262
// us, now there are 76; 24 to 36 bytes of a thread are spilled for five blocks a multiprocessor).  Tensors are found by a binary search over their first
// tiles in the launch's parameters, so that one launch takes 320 of any sizes.  Whole blocks by 16-byte accesses (the tensors' addresses are on 16-byte
// boundaries), half a warp a block.  The last elements of a tensor go one by one.
template <typename TG, bool EIGHT, int N>
__global__ void __launch_bounds__(kAdamThreads, EIGHT ? 5 : 1)
adamw_kernel(const __grid_constant__ AdamParams<N> P) {
    stream_enter();
    int lo = 0, hi = P.count;                                                     // the tensor of this tile
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (P.first_tile[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const AdamTensor &T = P.tensor[lo];
    const int64_t tile0 = (int64_t)(blockIdx.x - P.first_tile[lo]) * (tile_blocks(EIGHT) * kScaleBlock);
    const int lane = threadIdx.x % kBlockLanes;
    AdamStep s = {P.rate, P.root, P.lr_decay, P.grad_scale, 0u};
    uint32_t step = P.step;
    if (P.live) {
        const float lr = P.live[0], t = P.live[1];
        s.rate = lr / -expm1f(t * P.log_beta1);
        s.root = rsqrtf(-expm1f(t * P.log_beta2));
        s.decay = lr * P.decay;
        s.grad_scale = P.live[2];
        step = (uint32_t)t;
    }
    if (EIGHT) s.key = mixed(P.seed + step * 0x9E3779B9u) + (uint32_t)(P.first_tensor + lo) * 0xA54FF53Bu;
    for (int b = threadIdx.x / kBlockLanes; b < tile_blocks(EIGHT); b += kAdamThreads / kBlockLanes) {
        const int64_t block0 = tile0 + (int64_t)b * kScaleBlock;
        const int64_t warp0 = tile0 + (int64_t)(b & ~1) * kScaleBlock;            // both blocks of a warp walk together
        if (warp0 >= T.n) break;
        constexpr int VW = 4;
        const int64_t at = block0 + lane * VW;
        const int64_t left64 = T.n - at;
        const bool whole = block0 + kScaleBlock <= T.n;
        const int left = whole ? 1024 : (int)max((int64_t)-1024, left64);
        float p[8], g[8], m[8], v[8];
        Eight<float> raw;
        Eight<TG> rawg;
        const auto element = [&](int i) { return i / VW * (kBlockLanes * VW) + i % VW; };       // from `at`
        if (whole) {
            raw.template load<VW>(T.p + at, left);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = raw.get(i);
            rawg.template load<VW>(reinterpret_cast<const TG *>(T.g) + at, left);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = rawg.get(i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool there = element(i) < left;
                p[i] = there ? T.p[at + element(i)] : 0.f;
                g[i] = 0.f;
                if (there) {
                    if constexpr (sizeof(TG) == 4) g[i] = reinterpret_cast<const float *>(T.g)[at + element(i)];
                    else g[i] = __uint_as_float((uint32_t) reinterpret_cast<const uint16_t *>(T.g)[at + element(i)] << 16);
                }
            }
        }
        if constexpr (!EIGHT) {
            float *tm = reinterpret_cast<float *>(T.m), *tv = reinterpret_cast<float *>(T.v);
            if (whole) {
                raw.template load<VW>(tm + at, left);
#pragma unroll
                for (int i = 0; i < 8; ++i) m[i] = raw.get(i);
                raw.template load<VW>(tv + at, left);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = raw.get(i);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    m[i] = element(i) < left ? tm[at + element(i)] : 0.f;
                    v[i] = element(i) < left ? tv[at + element(i)] : 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 8; i += 2) adam_pair<false>(P, s, p + i, g + i, m + i, v + i);
            if (whole) {
                raw.set(m);
                raw.template store<VW>(tm + at, left);
                raw.set(v);
                raw.template store<VW>(tv + at, left);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (element(i) < left) tm[at + element(i)] = m[i], tv[at + element(i)] = v[i];
            }
        } else {
            uint8_t *tm = reinterpret_cast<uint8_t *>(T.m), *tv = reinterpret_cast<uint8_t *>(T.v);
            uint32_t cm[2] = {0u, 0u}, cv[2] = {0u, 0u};                          // four codes a word
            if (whole) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    ld_bytes<4>(tm + at + r * kBlockLanes * VW, &cm[r]);
                    ld_bytes<4>(tv + at + r * kBlockLanes * VW, &cv[r]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (element(i) < left) {
                        cm[i / 4] |= (uint32_t)tm[at + element(i)] << (i % 4 * 8);
                        cv[i / 4] |= (uint32_t)tv[at + element(i)] << (i % 4 * 8);
                    }
            }
            const int64_t block = block0 / kScaleBlock;
            const bool any = block0 < T.n;
            const float sm = any ? T.ms[block] : 0.f, sv = any ? T.vs[block] : 0.f;
            unpack_e4m3(cm[0], m);
            unpack_e4m3(cm[1], m + 4);
            unpack_e4m3(cv[0], v);
            unpack_e4m3(cv[1], v + 4);
            float topm = 0.f, topv = 0.f;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                pair_to(m + i, __fmul2_rn(pair_at(m + i), both(sm)));
                const float2 r = __fmul2_rn(pair_at(v + i), both(sv));
                pair_to(v + i, __fmul2_rn(r, r));
                adam_pair<true>(P, s, p + i, g + i, m + i, v + i);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!whole && element(i) >= left) m[i] = v[i] = 0.f;
                topm = max_or_nan(topm, fabsf(m[i]));
                topv = max_or_nan(topv, v[i]);
            }
            const BlockScale nm = block_scale(block_max(__float_as_uint(topm) & 0x7fffffffu)), nv = block_scale(block_max(__float_as_uint(topv) & 0x7fffffffu));
            if (lane == 0 && any) T.ms[block] = nm.scale, T.vs[block] = nv.scale;
            // a block of 128 elements lies in one piece of 2^32
            const uint32_t x = (uint32_t)at * 0x9E3779B9u + (uint32_t)((uint64_t)at >> 32) * 0xA54FF53Bu + s.key;
            // A magnitude a up to 448 is rounded up or down to an e4m3 value by 16 random bits: floor(a / width + u) widths, width = distance of the e4m3
            // values at a, u = random / 2^16.  Times 2^-120, a's bits from 20 on are its code -- exponents are 120 apart, and where e4m3 numbers have one
            // width, fp32 numbers have too -- and the 20 bits below are the rest, so u is added to them as bits 4 to 19 and what carries carries as it
            // should. What is no number gives any code (its block's scale is none either).
            uint32_t c[8], d[8];                                                  // codes in the highest bytes
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float2 am = __fmul2_rn(__fmul2_rn(pair_at(m + i), both(nm.inverse)), both(0x1p-120f));
                const float2 av = __fmul2_rn(__fmul2_rn(pair_at(v + i), both(nv.inverse)), both(0x1p-120f));
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t bits = mixed(x + (uint32_t)element(i + k) * 0x9E3779B9u);
                    const uint32_t y = __float_as_uint(k ? am.y : am.x) + ((bits & 0xffffu) << 4);          // the sign stays where it is
                    uint32_t z = __float_as_uint(k ? av.y : av.x) + (bits >> 16 << 4);
                    if (v[i + k] > 0.f) z = max(z, 1u << 20);
                    c[i + k] = y << 4 | (__float_as_uint(m[i + k]) & 0x80000000u);
                    d[i + k] = z << 4;
                }
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const auto four = [r](const uint32_t *w) {
                    return __byte_perm(__byte_perm(w[4 * r], w[4 * r + 1], 0x0073), __byte_perm(w[4 * r + 2], w[4 * r + 3], 0x0073), 0x5410);
                };
                cm[r] = four(c);
                cv[r] = four(d) & 0x7f7f7f7fu;
            }
            if (whole) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    st_bytes<4>(tm + at + r * kBlockLanes * VW, &cm[r]);
                    st_bytes<4>(tv + at + r * kBlockLanes * VW, &cv[r]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (element(i) < left) {
                        tm[at + element(i)] = (uint8_t)(cm[i / 4] >> (i % 4 * 8));
                        tv[at + element(i)] = (uint8_t)(cv[i / 4] >> (i % 4 * 8));
                    }
            }
        }
        if (whole) {
            raw.set(p);
            raw.template store<VW>(T.p + at, left);
            if (T.copy) {
                Eight<bf16> c;
                c.set(p);
                c.template store<VW>(reinterpret_cast<bf16 *>(T.copy) + at, left);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (element(i) < left) {
                    T.p[at + element(i)] = p[i];
                    if (T.copy) T.copy[at + element(i)] = (uint16_t)pack_bf16(p[i], 0.f);
                }
        }
    }
}

static bool rate_like(double v) { return std::isfinite(v) && v >= 0; }

static distdl_status_t adamw_impl(int32_t count, const int64_t *elems, void *const *p, const void *const *g, distdl_dtype_t tg, void *const *m,
                                  void *const *v, void *const *ms, void *const *vs, distdl_dtype_t state, void *const *copies, const double *hyper,
                                  int64_t step, int64_t seed, const void *live, void *stream) {
    const char *what = "adamw_step";
    clear_error();
    if (count < 0 || !hyper || (count > 0 && !elems)) return fail(DISTDL_ERR_INVALID_ARG, "%s: NULL argument or negative count", what);
    if (count > DISTDL_MAX_TENSORS) return fail(DISTDL_ERR_UNSUPPORTED, "%s: more than %d tensors", what, DISTDL_MAX_TENSORS);
    if (tg != DISTDL_F32 && tg != DISTDL_BF16) return fail(DISTDL_ERR_INVALID_ARG, "%s: gradients are F32 or BF16", what);
    if (state != DISTDL_F32 && state != DISTDL_E4M3) return fail(DISTDL_ERR_INVALID_ARG, "%s: states are F32 or E4M3", what);
    const double lr = hyper[0], beta1 = hyper[1], beta2 = hyper[2], eps = hyper[3], decay = hyper[4], scale = hyper[5];
    if (!rate_like(lr) || !rate_like(decay) || !std::isfinite(scale)) return fail(DISTDL_ERR_INVALID_ARG, "%s: learning rate, decay or gradient scale", what);
    if (!(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1)) return fail(DISTDL_ERR_INVALID_ARG, "%s: betas lie in [0, 1)", what);
    if (!std::isfinite((float)eps) || !(eps >= 0x1p-120)) return fail(DISTDL_ERR_INVALID_ARG, "%s: eps must be a number from 2^-120 on", what);
    if (step < 1 && !live) return fail(DISTDL_ERR_INVALID_ARG, "%s: steps are counted from 1", what);
    const bool eight = state == DISTDL_E4M3;
    if (count > 0 && (!p || !g || !m || !v || (eight && (!ms || !vs)))) return fail(DISTDL_ERR_INVALID_ARG, "%s: NULL argument", what);
    const void *some = nullptr;
    for (int i = 0; i < count; ++i) {
        if (elems[i] < 0) return fail(DISTDL_ERR_INVALID_ARG, "%s: tensor %d has %lld elements", what, i, (long long)elems[i]);
        if (elems[i] > (int64_t)1 << 40) return fail(DISTDL_ERR_UNSUPPORTED, "%s: tensor %d has more than 2^40 elements", what, i);
        if (elems[i] == 0) continue;
        const void *const need[6] = {p[i], g[i], m[i], v[i], eight ? ms[i] : p[i], eight ? vs[i] : p[i]};
        for (const void *a : need) {
            if (!a) return fail(DISTDL_ERR_INVALID_ARG, "%s: a buffer of tensor %d is NULL", what, i);
            if (!aligned16(a)) return fail(DISTDL_ERR_ALIGNMENT, "%s: a buffer of tensor %d is not 16-byte aligned", what, i);
        }
        if (copies && copies[i] && !aligned16(copies[i])) return fail(DISTDL_ERR_ALIGNMENT, "%s: copies[%d] not 16-byte aligned", what, i);
        some = p[i];
    }
    if (live && !aligned16(live)) return fail(DISTDL_ERR_ALIGNMENT, "%s: live not 16-byte aligned", what);
    if (!some) return DISTDL_OK;
    int device;
    if (const distdl_status_t st = current_device(what, some, &device)) return st;

    AdamParams<kTensorsAtOnce> P;
    P.beta1 = (float)beta1;
    P.one_beta1 = (float)(1 - beta1);
    P.beta2 = (float)beta2;
    P.one_beta2 = (float)(1 - beta2);
    P.log_beta1 = (float)std::log(beta1);                        // beta = 0: minus infinity, and 1 - beta^t = 1
    P.log_beta2 = (float)std::log(beta2);
    P.eps = (float)eps;
    P.decay = (float)decay;
    P.lr_decay = (float)(lr * decay);
    P.grad_scale = (float)scale;
    P.rate = live ? 0.f : (float)(lr / (1 - std::pow(beta1, (double)step)));
    P.root = live ? 0.f : (float)(1 / std::sqrt(1 - std::pow(beta2, (double)step)));
    P.seed = (uint32_t)((uint64_t)seed ^ ((uint64_t)seed >> 32));
    P.step = (uint32_t)step;
    P.live = (const float *)live;
    const auto launch_of = [&](const auto &params, auto few, uint32_t tiles) {
        constexpr int N = decltype(few)::value;
        const auto with = [&](auto kernel) { launch_in_stream(kernel, dim3(tiles), dim3(kAdamThreads), 0, (cudaStream_t)stream, params); };
        if (tg == DISTDL_F32) eight ? with(adamw_kernel<float, true, N>) : with(adamw_kernel<float, false, N>);
        else eight ? with(adamw_kernel<bf16, true, N>) : with(adamw_kernel<bf16, false, N>);
    };
    const auto launch = [&](uint32_t tiles) {
        if (P.count > kFewTensors) return launch_of(P, std::integral_constant<int, kTensorsAtOnce>(), tiles);
        AdamParams<kFewTensors> few;
        static_cast<AdamCommon &>(few) = P;
        std::copy(P.tensor, P.tensor + P.count, few.tensor);
        std::copy(P.first_tile, P.first_tile + P.count + 1, few.first_tile);
        launch_of(few, std::integral_constant<int, kFewTensors>(), tiles);
    };
    P.count = 0;
    P.first_tensor = 0;
    P.first_tile[0] = 0;
    for (int i = 0; i < count; ++i) {
        const int64_t tile = tile_blocks(eight) * kScaleBlock, tiles = (elems[i] + tile - 1) / tile;
        if (P.count == kTensorsAtOnce || (P.count > 0 && P.first_tile[P.count] + tiles > INT32_MAX)) {
            if (P.first_tile[P.count]) launch(P.first_tile[P.count]);
            P.first_tensor = i;
            P.count = 0;
        }
        AdamTensor &T = P.tensor[P.count];
        T.p = (float *)p[i];
        T.g = g[i];
        T.m = m[i];
        T.v = v[i];
        T.ms = eight ? (float *)ms[i] : nullptr;
        T.vs = eight ? (float *)vs[i] : nullptr;
        T.copy = copies ? (uint16_t *)copies[i] : nullptr;
        T.n = elems[i];
        P.first_tile[P.count + 1] = P.first_tile[P.count] + (uint32_t)tiles;
        ++P.count;
    }
    if (P.first_tile[P.count]) launch(P.first_tile[P.count]);
    DISTDL_CUDA_CHECK(cudaGetLastError());
    return DISTDL_OK;
}

}  // namespace distdl

extern "C" distdl_status_t distdl_adamw_step(int32_t count, const int64_t *elems, void *const *p, const void *const *g, distdl_dtype_t tg, void *const *m,
                                             void *const *v, void *const *ms, void *const *vs, distdl_dtype_t state, void *const *copies,
                                             const double *hyper, int64_t step, int64_t seed, const void *live, void *stream) {
    return distdl::adamw_impl(count, elems, p, g, tg, m, v, ms, vs, state, copies, hyper, step, seed, live, stream);
}
