// Values in 8 bits with a scale for each block of 128, and the way a block's values lie in registers: shared by the quantisation, the norm and the
// optimiser.  Half a warp holds a block, eight values a lane.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.h"

namespace distdl {

constexpr int kScaleBlock = 128;                 // values under one scale
constexpr int kBlockLanes = 16;                  // lanes that hold a block, eight values each

inline int64_t scale_blocks(int64_t n) { return (n + kScaleBlock - 1) / kScaleBlock; }

// Host: a list of n blocks, none missing, on 16-byte boundaries.
inline distdl_status_t check_blocks(const char *what, const char *name, const void *const *p, int n) {
    if (!p) return fail(DISTDL_ERR_INVALID_ARG, "%s: %s is NULL", what, name);
    for (int i = 0; i < n; ++i) {
        if (!p[i]) return fail(DISTDL_ERR_INVALID_ARG, "%s: %s[%d] is NULL", what, name, i);
        if (!aligned16(p[i])) return fail(DISTDL_ERR_ALIGNMENT, "%s: %s[%d] not 16-byte aligned", what, name, i);
    }
    return DISTDL_OK;
}

// Host: the current device, which the call runs on, and that a buffer of the call is memory it can reach.  A launch on another device's memory would be
// a fault on the GPU.
inline distdl_status_t current_device(const char *what, const void *buffer, int *device) {
    DISTDL_CUDA_CHECK(cudaGetDevice(device));
    if (*device < 0 || *device >= kMaxDevicesPerProcess)
        return fail(DISTDL_ERR_UNSUPPORTED, "%s: device index %d: at most %d devices per process", what, *device, kMaxDevicesPerProcess);
    cudaPointerAttributes a;
    DISTDL_CUDA_CHECK(cudaPointerGetAttributes(&a, buffer));
    if (a.type == cudaMemoryTypeUnregistered) return fail(DISTDL_ERR_INVALID_ARG, "%s: a buffer is no device memory", what);
    if (a.type == cudaMemoryTypeDevice && a.device != *device)
        return fail(DISTDL_ERR_INVALID_ARG, "%s: a buffer is on device %d, the current one is %d", what, a.device, *device);
    return DISTDL_OK;
}

// Multiprocessors of a device (looked up once).
inline distdl_status_t multiprocessors(int device, int *sms) {
    static int known[kMaxDevicesPerProcess] = {0};
    std::lock_guard<std::mutex> lock(setup_mutex());
    if (!known[device]) DISTDL_CUDA_CHECK(cudaDeviceGetAttribute(&known[device], cudaDevAttrMultiProcessorCount, device));
    *sms = known[device];
    return DISTDL_OK;
}

#ifdef __CUDACC__
struct bf16 {
    uint16_t bits;
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {      // nearest even
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {     // nearest even, at most 448; a lowest
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | (uint32_t)hi << 16;
}

__device__ __forceinline__ void unpack_e4m3(uint32_t codes, float *v) {      // exact
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(codes >> (16 * i))));
        asm("{\n.reg .b16 lo, hi;\nmov.b32 {lo, hi}, %2;\ncvt.f32.f16 %0, lo;\ncvt.f32.f16 %1, hi;\n}" : "=f"(v[2 * i]), "=f"(v[2 * i + 1]) : "r"(h));
    }
}

// Accesses of B bytes to global memory.  Loads are coherent (a buffer may be worked on in place).  Wide ones pass L1 by, since every byte is read once; rows
// that are no whole number of wide ones are read in pieces that share sectors of 32 bytes, which L1 keeps for the next piece.
// What is not there is 0, by a predicate on the load itself: a branch around narrow ones would wait for each.
template <int B>
__device__ __forceinline__ void ld_bytes(const void *p, uint32_t *v, bool there = true) {
    const uint32_t t = there;
    if constexpr (B == 16)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %5, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\nmov.b32 %2, 0;\nmov.b32 %3, 0;\n@p ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n}"
                     : "=&r"(v[0]), "=&r"(v[1]), "=&r"(v[2]), "=&r"(v[3]) : "l"(p), "r"(t) : "memory");
    else if constexpr (B == 8)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %3, 0;\nmov.b32 %0, 0;\nmov.b32 %1, 0;\n@p ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];\n}"
                     : "=&r"(v[0]), "=&r"(v[1]) : "l"(p), "r"(t) : "memory");
    else if constexpr (B == 4)
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\nmov.b32 %0, 0;\n@p ld.global.u32 %0, [%1];\n}" : "=&r"(v[0]) : "l"(p), "r"(t) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %2, 0;\nmov.b32 %0, 0;\n@p ld.global.u16 %0, [%1];\n}" : "=&r"(v[0]) : "l"(p), "r"(t) : "memory");
}
template <int B>
__device__ __forceinline__ void st_bytes(void *p, const uint32_t *v) {
    if constexpr (B == 16) *reinterpret_cast<uint4 *>(p) = make_uint4(v[0], v[1], v[2], v[3]);
    else if constexpr (B == 8) *reinterpret_cast<uint2 *>(p) = make_uint2(v[0], v[1]);
    else if constexpr (B == 4) *reinterpret_cast<uint32_t *>(p) = v[0];
    else if constexpr (B == 2) *reinterpret_cast<uint16_t *>(p) = (uint16_t)v[0];
    else *reinterpret_cast<uint8_t *>(p) = (uint8_t)v[0];
}

// A lane's eight values of a block, as they lie in memory (bfloat16: two to a word).  Value i of lane l is element element_of<VW>(l, i) of the block: runs
// of VW elements, the runs of the sixteen lanes side by side, so that an access of the lanes is one piece of memory whatever VW is.  VW divides the
// rows' length and is at most 16 bytes of the widest type at hand.
template <int VW>
__host__ __device__ __forceinline__ constexpr int element_of(int lane, int i) { return i / VW * (kBlockLanes * VW) + lane * VW + i % VW; }

template <typename T>
struct Eight {
    static constexpr bool kHalf = sizeof(T) == 2;
    uint32_t w[kHalf ? 4 : 8];
    __device__ __forceinline__ float get(int i) const {
        if constexpr (!kHalf) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
    }
    __device__ __forceinline__ void set(const float *v) {         // each rounded once to the type
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if constexpr (!kHalf) w[i] = __float_as_uint(v[i]);
            else if (i & 1) w[i >> 1] = pack_bf16(v[i - 1], v[i]);
    }
    // p: the block's first element of this lane; left: elements of the row from there on (none: 0 or less).  What is not there is 0.
    template <int VW>
    __device__ __forceinline__ void load(const T *p, int left) {
        if constexpr (VW == 1 && kHalf) {
            uint32_t v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) ld_bytes<2>(p + r * kBlockLanes, v + r, r * kBlockLanes < left);
#pragma unroll
            for (int r = 0; r < 4; ++r) w[r] = v[2 * r] | v[2 * r + 1] << 16;
        } else {
            constexpr int words = VW * (int)sizeof(T) / 4;
#pragma unroll
            for (int r = 0; r < 8 / VW; ++r) ld_bytes<VW * (int)sizeof(T)>(p + r * kBlockLanes * VW, w + r * words, r * kBlockLanes * VW < left);
        }
    }
    template <int VW>
    __device__ __forceinline__ void store(T *p, int left) const {
#pragma unroll
        for (int r = 0; r < 8 / VW; ++r)
            if (r * kBlockLanes * VW < left) {
                if constexpr (VW == 1 && kHalf) {
                    const uint32_t v = r & 1 ? w[r >> 1] >> 16 : w[r >> 1];
                    st_bytes<2>(p + r * kBlockLanes, &v);
                } else {
                    constexpr int words = VW * (int)sizeof(T) / 4 > 0 ? VW * (int)sizeof(T) / 4 : 1;
                    st_bytes<VW * (int)sizeof(T)>(p + r * kBlockLanes * VW, w + r * words);
                }
            }
    }
};

// Largest magnitude of a block from the bit patterns of its values without sign: their order as integers is that of the numbers, infinity above them,
// NaN above infinity -- so that neither is lost, as a maximum of numbers would lose a NaN.  The sixteen lanes of a block get it.
__device__ __forceinline__ uint32_t block_max(uint32_t bits) {
#pragma unroll
    for (int d = kBlockLanes / 2; d; d >>= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, d));
    return bits;
}
struct BlockScale {
    float scale, inverse;
};
__device__ __forceinline__ BlockScale block_scale(uint32_t max_bits) {
    const float a = __uint_as_float(max(max_bits, 0x0d800000u));          // 2^-100
    return {__fdiv_rn(a, 448.f), __fdiv_rn(448.f, a)};
}
// Eight scaled values of a lane to a row of bytes.
template <int VW>
__device__ __forceinline__ void store_e4m3(const float *v, uint8_t *p, int left) {
    const uint32_t w[2] = {pack_e4m3(v[0], v[1], v[2], v[3]), pack_e4m3(v[4], v[5], v[6], v[7])};
#pragma unroll
    for (int r = 0; r < 8 / VW; ++r)
        if (r * kBlockLanes * VW < left) {
            if constexpr (VW >= 4) st_bytes<VW>(p + r * kBlockLanes * VW, w + r * VW / 4);
            else {
                const uint32_t part = w[r * VW / 4] >> (r * VW % 4 * 8);
                st_bytes<VW>(p + r * kBlockLanes * VW, &part);
            }
        }
}
#endif

}  // namespace distdl
