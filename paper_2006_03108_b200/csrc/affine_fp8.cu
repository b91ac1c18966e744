// Distributed affine layer on a Pfo x Pfi worker grid with activations and weights in 8 bits (e4m3 values with a scale for each 1 x 128 of a sample and
// each 128 x 128 of a weight block): forward  y_i = R_j (x_j W_ij^T) (+ b_i)  and adjoint  dx_j = R_i (dy_i W_ij).
//
// B and R are as in the bfloat16 layer (affine.cu): blocks of x are read through L2, and R goes on in the accumulator in worker order.  The scales change
// every 128 of the contraction, on both sides, so a product of 128 is all that the tensor cores may add up by themselves: it is finished in tensor memory,
// and the epilogue warps add it, times its two scales, to sums in their registers, while the next 128 are multiplied into the other half of tensor memory.
// The sums are fp32 throughout, in the order of the k-blocks.
//
// The forward pass takes the weights as the K-major operand, the adjoint takes the same bytes as the MN-major one; a scale block is 128 x 128, so both
// read the same scales.  Every wait is bounded, as in affine.cu.
#include <cuda.h>

#include <algorithm>
#include <cstring>

#include "common.h"
#include "distdl_selftest.h"
#include "eight_bit.h"
#include "tcgen05.h"
#include "tma.h"

namespace distdl {

constexpr int kF8K = 128;                                   // of the contraction at a time: one scale, one 128-byte swizzle row
constexpr int kF8Rows = 128;                                // rows of a thread block's tile
constexpr int kF8MaxWorkers = 16;

__device__ int g_fp8_status = 0;                            // 0 or DISTDL_ERR_TIMEOUT
int fp8_take_status() {
    int st = 0;
    if (cudaMemcpyFromSymbol(&st, g_fp8_status, sizeof(int)) != cudaSuccess) return -1;
    if (st) {
        const int zero = 0;
        cudaMemcpyToSymbol(g_fp8_status, &zero, sizeof(int));
    }
    return st;
}

struct AffineF8Params {
    CUtensorMap a_map[8];                                   // activation blocks (x_j forward, dy_i adjoint)
    CUtensorMap w_map[kF8MaxWorkers];                       // weight blocks, worker order i * pfi + j
    const float *as[8];                                     // scales of the activations [k-blocks][nb]
    const float *ws[kF8MaxWorkers];                         // scales of the weights
    void *out[8];
    const float *bias[8];
    int32_t nb, pfi;
    int32_t blk_out, blk_red;                               // columns of an output block, contraction inside one worker
    int32_t nred;                                           // workers summed over
    int32_t kpw;                                            // k-blocks of a worker
    int32_t ws_k, ws_n;                                     // steps in the weights' scales: to the next k-block, the next 128 columns
    int32_t nout, tiles, splits;                            // output blocks; tiles and splits of the contraction (pairs)
    int32_t adjoint, out_bf16;
    int32_t out_wide, out_lines;                            // every output block begins on a 32-byte boundary; and is rows of whole 128 bytes of fp32
};

__device__ __forceinline__ bool f8_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag) {
    return bounded_wait(bar, parity, abort_flag, &g_fp8_status, kWaitLimitCycles);
}
// kind::f8f6f4, K = 32: both operands e4m3 (formats 0), D = fp32
__device__ __forceinline__ void umma_f8(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_f8_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// Instruction descriptor: D = fp32 [4,6) = 1, A = B = e4m3 [7,10) = [10,13) = 0, A major bit 15, B major bit 16 (1 = MN-major), N >> 3 in [17,23),
// M >> 4 in [24,29).
__host__ __device__ constexpr uint32_t f8_instr(int m, int n, int a_mn, int b_mn) {
    return (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// Arrival at a barrier of another block of the cluster.  What it releases is tensor memory (the fence before it sees to that), so it takes no fence at the
// cluster's scope: that one, once a k-block for each warp, was the largest stall of the kernel.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar_cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster_addr) : "memory");
}
// 64 columns of tensor memory, and the wait for them.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, uint32_t *v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,"
        "%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
        "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31]),
          "=r"(v[32]), "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]), "=r"(v[37]), "=r"(v[38]), "=r"(v[39]),
          "=r"(v[40]), "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]), "=r"(v[46]), "=r"(v[47]),
          "=r"(v[48]), "=r"(v[49]), "=r"(v[50]), "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]), "=r"(v[55]),
          "=r"(v[56]), "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]), "=r"(v[61]), "=r"(v[62]), "=r"(v[63])
        : "r"(taddr) : "memory");
}
// 4 bytes, or four zeros, to shared memory, and an arrival at a barrier once this thread's copies so far are there.
__device__ __forceinline__ void copy_float_async(uint32_t dst, const float *src, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4u : 0u) : "memory");
}
__device__ __forceinline__ void arrive_after_copies(uint32_t bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// ------------------------------------------------------------------------------------------
// Batches over 128: a pair of blocks owns a 256 x TN tile (cta_group::2, 128 rows and half of the weights' columns each); a cluster of S pairs shares the
// k-blocks of a tile, in S runs one after the other, and adds up the S sums through distributed shared memory in that order.
//
// What bounds it.  The tensor cores take 600 clocks for a k-block of a 256 x 256 tile, and 32 KB for it come into each SM.  Large products run at what
// power and L2 allow: 2048 x 8192 x 8192 in 127 to 132 us from machine to machine (2080 to 2160 TFLOP/s; 1.07 GB from L2, 8.1 to 8.5 TB/s) in a burst,
// 4096 x 8192 x 8192 in 235 to 245 us, 274 us (2010 TFLOP/s at 1.48 GHz and 1 kW) when it goes on for seconds -- the same loop with all k-blocks added
// up in tensor memory, without scales, takes 218 and 250.  Small ones are bound by what surrounds the k-blocks, some 5 to 8 us: 256 x 8192 x 8192 26 us
// (adjoint 25), 777 x 3120 x 1312 14.6 us.  256 columns in runs spill 36 bytes a thread.  On the way (2048 x 8192 x 8192, us): an arrival at the other
// block with release at the cluster's scope, a fence for every warp and k-block, 336; without 192; scalar sums instead of pairs put together by moves
// 167; pairs that go on from tile to tile 152; one barrier for a product and its stage instead of two 143; eight summing warps with 64-column loads
// instead of sixteen with 32-column ones 135; a second thread that issues products 127. Halves of tiles for the last turn cost the other turns more than
// they gained (133).
// ------------------------------------------------------------------------------------------
constexpr int kF8Tail = 1024 + 512;                         // alignment, barriers
constexpr int kF8ScaleSlots = 8;                            // k-blocks whose scales are on their way or waited for
constexpr int kF8ScaleSlot = kF8Rows + 8;                   // floats: the rows' scales, the two column halves' weight scales
template <int TN>
struct F8Cfg {
    static constexpr int kSumWarps = 8;                     // 32 rows and half of the columns each
    static constexpr int kCols = TN / 2;
    static constexpr int kBuffers = 512 / TN;               // products in tensor memory
    static constexpr int kThreads = 128 + 32 * kSumWarps;   // warp 0: TMA, 1: MMA and tensor memory, 2: scales, 3: MMA, 4..: sums
    static constexpr int kABytes = kF8Rows * kF8K;          // 16 KB
    static constexpr int kBBytes = TN / 2 * kF8K;
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = 196608 / kStageBytes;    // 6 or 8
    static constexpr int kPitch = TN + 4;                   // floats of a row of sums in shared memory; spreads rows over the banks
    static constexpr int kScaleBytes = kF8ScaleSlots * kF8ScaleSlot * 4;
    static constexpr int kSmemBytes = kStages * kStageBytes + kScaleBytes + kF8Tail;
    static_assert(kF8Rows * kPitch * 4 <= kStages * kStageBytes, "the sums take the ring's place");
    static_assert(TN % kScaleBlock == 0, "");
    static_assert(tensor_blocks_fit(kSmemBytes, 512), "affine_fp8_pair_kernel");
    static constexpr int kBars = 2 * kStages + kBuffers + 2 * kF8ScaleSlots;
    static_assert(kBars * 8 + 8 <= 512, "barriers");
    // a stage's next product waits for the sums to have taken its last one: its barrier is never two turns ahead of them
    static_assert(kStages >= kBuffers, "as many stages as products");
};

// Tiles in groups of eight rows of tiles, column by column inside a group, so that what runs at a time shares its rows and columns in L2.
constexpr int kF8GroupRows = 8;
struct F8Tile {
    int m0, n0, oblk;                                       // first row of the tile, first column inside the output block
    template <int TN>
    static __device__ __forceinline__ F8Tile of(const AffineF8Params &P, int tile) {
        const int row_tiles = (P.nb + 2 * kF8Rows - 1) / (2 * kF8Rows), per_block = (P.blk_out + TN - 1) / TN, columns = P.nout * per_block;
        const int group = tile / (kF8GroupRows * columns), first = group * kF8GroupRows, rows = min(kF8GroupRows, row_tiles - first);
        const int in = tile - first * columns, column = in / rows;
        F8Tile t;
        t.m0 = (first + in - column * rows) * 2 * kF8Rows;
        t.oblk = column / per_block;
        t.n0 = (column - t.oblk * per_block) * TN;
        return t;
    }
};

// 4 values of a row.
__device__ __forceinline__ void f8_store4(const AffineF8Params &P, int oblk, int64_t at, float4 v) {
    if (P.out_bf16) *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(P.out[oblk]) + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    else *reinterpret_cast<float4 *>(reinterpret_cast<float *>(P.out[oblk]) + at) = v;
}
// 16 values of a row: two 16-byte stores, or one of 32 bytes where the buffer allows it.
__device__ __forceinline__ void f8_store(const AffineF8Params &P, int oblk, int64_t at, const float *v) {
    if (P.out_bf16) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        uint16_t *p = reinterpret_cast<uint16_t *>(P.out[oblk]) + at;
        if (P.out_wide) {
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                         ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
        } else {
            st_bytes<16>(p, w);
            st_bytes<16>(p + 8, w + 4);
        }
    } else {
        float *p = reinterpret_cast<float *>(P.out[oblk]) + at;
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            if (P.out_wide) {
                asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                             ::"l"(p + i), "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]), "f"(v[i + 3]), "f"(v[i + 4]), "f"(v[i + 5]), "f"(v[i + 6]), "f"(v[i + 7]) : "memory");
            } else {
                *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                *reinterpret_cast<float4 *>(p + i + 4) = make_float4(v[i + 4], v[i + 5], v[i + 6], v[i + 7]);
            }
        }
    }
}

// 32 fp32 values of each lane's row, rows row0 + lane, columns from column on: four lanes exchange quarters, so that a store writes 128 bytes of each of
// eight rows; 32 bytes of each of 32 rows keep L2 busy with four times the requests.  Where a row of the output is whole lines, and fp32 (B200, us):
// 1024 x 512 x 16384 30.4 without, 25.6 so, 4096 x 1024 x 1024 12.5 and 11.4, 2048 x 8192 x 8192 137.5 and 134.7; rows that are no whole lines, and bfloat16
// ones with half the bytes, lose by the exchange what they gain (777 x 3120 x 1312 14.2 and 14.4; in bfloat16 1321 x 2496 x 4704 26.6 and 27.3).
__device__ __forceinline__ void f8_store_rows(const AffineF8Params &P, int oblk, int row0, int column, uint32_t *w) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 1; d < 4; d *= 2) {
        const bool odd = lane & d;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u & d) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t &lo = w[8 * u + i], &hi = w[8 * (u + d) + i];
                const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? lo : hi, d);
                lo = odd ? got : lo;
                hi = odd ? hi : got;
            }
        }
    }
    column += (lane & 3) * 8;
    if (column >= P.blk_out) return;                        // whole groups of 16: blocks are multiples of that
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int row = row0 + (lane & ~3) + k;
        if (row >= P.nb) break;
        uint8_t *p = reinterpret_cast<uint8_t *>(P.out[oblk]) + ((int64_t)row * P.blk_out + column) * 4;
        const uint32_t *v = w + 8 * k;
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    }
}

// SPLIT: a cluster of S pairs takes one tile.  Otherwise a pair goes from tile to tile, and copies and products of the next one begin while the
// sums of the last one are written.
template <int TN, bool SPLIT>
__global__ void __launch_bounds__(F8Cfg<TN>::kThreads, 1)
affine_fp8_pair_kernel(const __grid_constant__ AffineF8Params P) {
    stream_enter();
    using C = F8Cfg<TN>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;           // the swizzle is a function of address bits [7,10)
    uint8_t *aligned = smem_raw + (base - raw);
    const float *scales = reinterpret_cast<const float *>(aligned + C::kStages * C::kStageBytes);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + C::kStages * C::kStageBytes + C::kScaleBytes);
    const uint32_t bar_full = smem_u32(bars);
    const uint32_t bar_done = bar_full + 8 * C::kStages;    // a stage's product of 128 is in tensor memory, and the stage is empty
    const uint32_t bar_free = bar_done + 8 * C::kStages;    // a part of tensor memory has been read
    const uint32_t bar_scale = bar_free + 8 * C::kBuffers;               // a k-block's scales are in shared memory
    const uint32_t bar_scale_free = bar_scale + 8 * kF8ScaleSlots;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + C::kBars);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t crank = cluster_ctarank(), prank = crank & 1, leader = crank & ~1u;
    const int splits = SPLIT ? P.splits : 1, split = SPLIT ? (int)crank / 2 : 0;
    const int first_tile = (int)blockIdx.x / (2 * splits), tile_step = (int)gridDim.x / (2 * splits);
    const int all = P.nred * P.kpw;
    const int kb0 = (int)((int64_t)all * split / splits), kb1 = (int)((int64_t)all * (split + 1) / splits);

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_done + 8 * s, 1);
        }
        for (int b = 0; b < C::kBuffers; ++b) mbar_init(bar_free + 8 * b, 2 * C::kSumWarps);     // the summing warps of both blocks
        for (int s = 0; s < kF8ScaleSlots; ++s) {
            mbar_init(bar_scale + 8 * s, 32);               // the lanes that copy
            mbar_init(bar_scale_free + 8 * s, C::kSumWarps); // the summing warps
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    cluster_sync_all();
    tcgen05_fence_after();
    const uint32_t tmem = *tmem_slot;

    // 256 columns: a summing thread holds 128 sums.  The launch gives all of the 384 threads 168 registers; the first four warps hand 128 of theirs over to
    // the eight that sum (40 + 2 * 232 = 3 * 168).
    if (warp < 4) {
        if constexpr (TN == 256) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 0) {
            if (lane == 0) {
                uint32_t s = 0, phase = 0;
                bool ok = true;
                for (int tile = first_tile; ok && tile < P.tiles; tile += tile_step) {
                    const F8Tile t = F8Tile::of<TN>(P, tile);
                    int r = kb0 / P.kpw, kin = kb0 - r * P.kpw;
                    const int row = t.m0 + (int)prank * kF8Rows, column = t.n0 + (int)prank * (TN / 2);
                    for (int kb = kb0; kb < kb1; ++kb) {
                        ok = f8_wait(bar_done + 8 * s, phase ^ 1, abort_flag);
                        if (!ok) break;
                        const uint32_t full = bar_full + 8 * s, full_leader = map_to_cta(full, leader), sa = base + s * C::kStageBytes;
                        const CUtensorMap *wmap = &P.w_map[P.adjoint ? r * P.pfi + t.oblk : t.oblk * P.pfi + r];
                        if (prank == 0) mbar_expect_tx(full, 2 * C::kStageBytes);
                        tma_load_2d_pair(sa, &P.a_map[r], kin * kF8K, row, full_leader);                                  // box {128 k, 128 rows}
                        if (!P.adjoint) tma_load_2d_pair(sa + C::kABytes, wmap, kin * kF8K, column, full_leader);         // box {128 k, TN / 2 rows}
                        else tma_load_2d_pair(sa + C::kABytes, wmap, column, kin * kF8K, full_leader);                    // box {TN / 2 columns, 128 k}
                        if (++kin == P.kpw) {
                            kin = 0;
                            ++r;
                        }
                        if (++s == C::kStages) {
                            s = 0;
                            phase ^= 1;
                        }
                    }
                }
                if (*abort_flag) {
                    // give copies that are still in flight time to land before the block retires
                    const uint64_t t0 = global_timer();
                    while (global_timer() - t0 < 1000000ull) {}
                }
            }
        } else if (warp & 1) {
            // Two warps issue products, every other one each: they are independent of one another, and a thread alone takes 750 clocks for the two waits,
            // the four instructions and the commit of one, where the tensor cores take 300 to 600.
            if (lane == 0 && prank == 0) {
                const uint32_t idesc = f8_instr(2 * kF8Rows, TN, 0, P.adjoint);
                // K-major: 8-row groups 1024 bytes apart, a K step of 32 values is 32 bytes.  MN-major: rows of TN / 2 columns (128-byte swizzle, or 64-byte
                // where that is 64), 8-k groups 8 rows apart, a K step of 32 rows.
                constexpr uint32_t row = TN / 2;
                const uint64_t a0 = smem_desc(base, 16, 1024);
                uint64_t b0 = smem_desc(base + C::kABytes, P.adjoint ? C::kBBytes : 16, P.adjoint ? 8 * row : 1024);
                if (TN == 128 && P.adjoint) b0 = (b0 & ~((uint64_t)7 << 61)) | (uint64_t)4 << 61;
                const uint64_t bstep = P.adjoint ? 32 * row >> 4 : 32 >> 4;
                const uint16_t mask = (uint16_t)(3u << leader);
                static_assert(C::kStages % 2 == 0 && C::kBuffers % 2 == 0, "each of the two warps has stages and buffers of its own");
                const uint32_t total = first_tile < P.tiles ? (uint32_t)((P.tiles - first_tile + tile_step - 1) / tile_step * (kb1 - kb0)) : 0u;
                uint32_t s = (uint32_t)warp >> 1, phase = 0, buf = s, bphase = 1;
                for (uint32_t it = s; it < total; it += 2) {
                    if (!f8_wait(bar_free + 8 * buf, bphase, abort_flag) || !f8_wait(bar_full + 8 * s, phase, abort_flag)) break;
                    tcgen05_fence_after();
                    const uint64_t off = (uint64_t)(s * (C::kStageBytes >> 4)), a = a0 + off, b = b0 + off;
                    const uint32_t d = tmem + buf * TN;
                    umma_f8_pair(d, a, b, idesc, 0u);
                    umma_f8_pair(d, a + 2, b + bstep, idesc, 1u);
                    umma_f8_pair(d, a + 4, b + 2 * bstep, idesc, 1u);
                    umma_f8_pair(d, a + 6, b + 3 * bstep, idesc, 1u);
                    tcgen05_commit_mask(bar_done + 8 * s, mask);
                    if ((s += 2) >= C::kStages) {
                        s -= C::kStages;
                        phase ^= 1;
                    }
                    if ((buf += 2) >= C::kBuffers) {
                        buf -= C::kBuffers;
                        bphase ^= 1;
                    }
                }
            }
        } else if (warp == 2) {
            // scales: four rows a lane, and a weight block's by each of the first lanes, up to eight k-blocks ahead of the sums
            uint32_t s = 0, phase = 0;
            bool ok = true;
            for (int tile = first_tile; ok && tile < P.tiles; tile += tile_step) {
                const F8Tile t = F8Tile::of<TN>(P, tile);
                int r = kb0 / P.kpw, kin = kb0 - r * P.kpw;
                const int row0 = t.m0 + (int)prank * kF8Rows + lane, col = t.n0 + lane * kScaleBlock;
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = __all_sync(0xffffffffu, f8_wait(bar_scale_free + 8 * s, phase ^ 1, abort_flag));
                    if (!ok) break;
                    const uint32_t slot = smem_u32(scales) + s * (kF8ScaleSlot * 4);
                    const float *a = P.as[r] + (int64_t)kin * P.nb;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int row = row0 + 32 * i;
                        copy_float_async(slot + 4 * (lane + 32 * i), a + min(row, P.nb - 1), row < P.nb);
                    }
                    if (lane < TN / kScaleBlock) {
                        const float *w = P.ws[P.adjoint ? r * P.pfi + t.oblk : t.oblk * P.pfi + r] + (int64_t)kin * P.ws_k;
                        copy_float_async(slot + 4 * (kF8Rows + lane), w + (col < P.blk_out ? (int64_t)(col / kScaleBlock) * P.ws_n : 0), col < P.blk_out);
                    }
                    arrive_after_copies(bar_scale + 8 * s);
                    if (++kin == P.kpw) {
                        kin = 0;
                        ++r;
                    }
                    if (++s == kF8ScaleSlots) {
                        s = 0;
                        phase ^= 1;
                    }
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
        __syncwarp();
        tcgen05_fence_before();
        cluster_sync_all();
        if (SPLIT) cluster_sync_all();
        if (warp == 1) {
            tcgen05_fence_after();
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
        }
    } else {
        if constexpr (TN == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        const int quarter = warp & 3, col = ((warp - 4) >> 2) * C::kCols;   // tensor-memory lanes [32 q, 32 q + 32), columns from col
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)col;
        const uint32_t free_leader = map_to_cta(bar_free, leader);
        const float *my_scale = scales + quarter * 32 + lane, *w_scale = scales + kF8Rows + col / kScaleBlock;
        uint32_t s = 0, phase = 0, it = 0, slot = 0, sphase = 0;
        float scale = 0.f;
        // the scale of the next k-block
        const auto next_scale = [&]() {
            if (!__all_sync(0xffffffffu, f8_wait(bar_scale + 8 * slot, sphase, abort_flag))) return false;
            scale = my_scale[slot * kF8ScaleSlot] * w_scale[slot * kF8ScaleSlot];
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_scale_free + 8 * slot);
            if (++slot == kF8ScaleSlots) {
                slot = 0;
                sphase ^= 1;
            }
            return true;
        };
        bool ok = true;
        for (int tile = first_tile; ok && tile < P.tiles; tile += tile_step) {
            float2 acc[C::kCols / 2];
#pragma unroll
            for (int i = 0; i < C::kCols / 2; ++i) acc[i] = make_float2(0.f, 0.f);
            for (int kb = kb0; kb < kb1; ++kb, ++it) {
                const uint32_t buf = it % C::kBuffers;
                if (!(ok = next_scale())) break;
                ok = __all_sync(0xffffffffu, f8_wait(bar_done + 8 * s, phase, abort_flag));
                if (!ok) break;
                tcgen05_fence_after();
                const float now = scale;
#pragma unroll
                for (int c = 0; c < C::kCols; c += 64) {
                    uint32_t v[64];
                    tmem_ld64(taddr + buf * TN + c, v);
                    if (c + 64 == C::kCols) {                               // this part of tensor memory may be written again
                        tcgen05_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(free_leader + 8 * buf);
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i)                            // two sums at an instruction
                        acc[c / 2 + i] = __ffma2_rn(make_float2(now, now), make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), acc[c / 2 + i]);
                }
                if (++s == C::kStages) {
                    s = 0;
                    phase ^= 1;
                }
            }
            if (!ok) break;
            const F8Tile t = F8Tile::of<TN>(P, tile);
            const int m0 = t.m0 + (int)prank * kF8Rows;
            const float *bias = P.bias[t.oblk];
            if constexpr (!SPLIT) {
                const int row = m0 + quarter * 32 + lane;
                if (P.out_lines) {
#pragma unroll
                    for (int c = 0; c < C::kCols; c += 32) {
                        const int column = t.n0 + col + c;
                        uint32_t w[32];
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            const float4 b = bias && column < P.blk_out ? __ldg(reinterpret_cast<const float4 *>(bias + column + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
                            const float2 lo = acc[(c + i) / 2], hi = acc[(c + i) / 2 + 1];
                            w[i] = __float_as_uint(lo.x + b.x), w[i + 1] = __float_as_uint(lo.y + b.y);
                            w[i + 2] = __float_as_uint(hi.x + b.z), w[i + 3] = __float_as_uint(hi.y + b.w);
                        }
                        f8_store_rows(P, t.oblk, m0 + quarter * 32, column, w);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < C::kCols; c += 16) {
                        const int column = t.n0 + col + c;
                        if (column >= P.blk_out) continue;                      // whole groups of 16: blocks are multiples of that
                        float o[16];
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float4 b = bias ? __ldg(reinterpret_cast<const float4 *>(bias + column + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
                            const float2 lo = acc[(c + i) / 2], hi = acc[(c + i) / 2 + 1];
                            o[i] = lo.x + b.x, o[i + 1] = lo.y + b.y, o[i + 2] = hi.x + b.z, o[i + 3] = hi.y + b.w;
                        }
                        if (row < P.nb) f8_store(P, t.oblk, (int64_t)row * P.blk_out + column, o);
                    }
                }
            } else {
                // every product has been taken, so the ring is free: the sums as [row][column]
                float *o = reinterpret_cast<float *>(aligned) + (quarter * 32 + lane) * C::kPitch + col;
#pragma unroll
                for (int i = 0; i < C::kCols / 2; i += 2) *reinterpret_cast<float4 *>(o + 2 * i) = make_float4(acc[i].x, acc[i].y, acc[i + 1].x, acc[i + 1].y);
                tcgen05_fence_before();
                cluster_sync_all();                                         // every block's sums are in place
                const int r0 = kF8Rows * split / splits, r1 = kF8Rows * (split + 1) / splits;
#pragma unroll
                for (int u = 0; u < TN / 128; ++u) {
                    const int c = 128 * u + 4 * lane, column = t.n0 + c;
                    if (column >= P.blk_out || *abort_flag) continue;
                    const float4 b = bias ? __ldg(reinterpret_cast<const float4 *>(bias + column)) : make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int rl = r0 + warp - 4; rl < r1; rl += 4 * C::kSumWarps) {
                        float4 v[4];                                        // four rows in flight: a block has 32 of them at least
                        const auto at_row = [&](int i) { return base + (uint32_t)(((rl + i * C::kSumWarps) * C::kPitch + c) * 4); };
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = ld_cluster_f4(map_to_cta(at_row(i), prank));
                        for (int q = 1; q < splits; ++q) {
                            float4 w[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) w[i] = ld_cluster_f4(map_to_cta(at_row(i), (uint32_t)(2 * q) + prank));
#pragma unroll
                            for (int i = 0; i < 4; ++i) v[i].x += w[i].x, v[i].y += w[i].y, v[i].z += w[i].z, v[i].w += w[i].w;
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int row = m0 + rl + i * C::kSumWarps;
                            if (row >= P.nb) continue;
                            v[i].x += b.x, v[i].y += b.y, v[i].z += b.z, v[i].w += b.w;
                            const int64_t at = (int64_t)row * P.blk_out + column;
                            f8_store4(P, t.oblk, at, v[i]);
                        }
                    }
                }
            }
        }
        // A cluster whose waits ran out still meets at its barriers: once more here, and before the sums are read (SPLIT, above).
        if (SPLIT && !ok) cluster_sync_all();
        tcgen05_fence_before();
        cluster_sync_all();                                                 // nobody retires while a peer uses its memory or its barriers
    }
}

// ------------------------------------------------------------------------------------------
// Few samples (a batch of at most 128): the weights are the M operand, 128 output features a block, the batch takes N = 16, 32, 64 or 128 columns.  A
// cluster of S blocks shares the k-blocks of the features in S runs and adds up the S sums through distributed shared memory in that order.  What bounds it
// is the stream of the weights: two blocks an SM (one from N = 64 on, whose sums need the registers of two) keep it going, and its first copies leave
// before anything else is set up.  8192 x 8192 weights (B200, cold, in a graph): one sample 16.0 us (adjoint 15.5) -- of which the weights take 10.4 at the copy
// rate, from 0.7 us after the start on -- 32 samples 17.2, 64 19.9, 128 22.7.
// ------------------------------------------------------------------------------------------
constexpr int kF8WBytes = 128 * kF8K;
constexpr int kF8FewMaxStages = 12;
constexpr int kF8FewMaxSmem = 220 * 1024;                   // one block an SM; half of it: two

struct AffineF8FewParams {
    AffineF8Params p;
    int32_t split, stages;
};
template <int N>
struct F8FewCfg {
    static constexpr int kParts = N >= 64 ? 2 : 1;          // summing warps: four for each part of the columns
    static constexpr int kCols = N / kParts;
    static constexpr int kThreads = 128 + 128 * kParts;     // warp 0: TMA, 1: MMA and tensor memory, 3: MMA, 4..: sums
    static constexpr int kBlocksPerSm = N >= 64 ? 1 : 2;
    static constexpr int kStageBytes = kF8WBytes + N * kF8K;
    static constexpr int kBuffers = N >= 128 ? 2 : 4;       // products in tensor memory
    static constexpr int kTmemCols = kBuffers * N;
    static constexpr int kScaleBytes = 4 * kParts * 2 * kCols * 4;          // two sets of a k-block's scales for each summing warp
    static constexpr int kTail = kF8Tail + kScaleBytes;
    static constexpr int kMinStages = (512 * N + kStageBytes - 1) / kStageBytes;      // the sums take the ring's place
    static constexpr int stages(int budget) { return (budget - kTail) / kStageBytes < kF8FewMaxStages ? (budget - kTail) / kStageBytes : kF8FewMaxStages; }
    static constexpr int smem(int budget) { return stages(budget) * kStageBytes + kTail; }
    static_assert((2 * kF8FewMaxStages + kBuffers) * 8 + 8 <= 512, "barriers");
    static_assert((kF8FewMaxSmem / kBlocksPerSm - kTail) / kStageBytes >= kMinStages, "room for the sums");
    // a stage's next product waits for the sums to have taken its last one: its barrier is never two turns ahead of them
    static_assert((kF8FewMaxSmem / kBlocksPerSm - kTail) / kStageBytes >= kBuffers, "as many stages as products");
};
template <int N>
constexpr bool few_blocks_fit() {
    using C = F8FewCfg<N>;
    return tensor_blocks_fit(C::smem(kF8FewMaxSmem), C::kTmemCols) && tensor_blocks_fit(C::smem(kF8FewMaxSmem / C::kBlocksPerSm), C::kTmemCols);
}
static_assert(few_blocks_fit<16>() && few_blocks_fit<32>() && few_blocks_fit<64>() && few_blocks_fit<128>(), "tensor_blocks_fit: affine_fp8_few_kernel");
template <int C>
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t *v) {
    if constexpr (C == 16) tmem_ld16(taddr, v);
    else if constexpr (C == 32) tmem_ld32(taddr, v);
    else tmem_ld64(taddr, v);
}

template <int N>
__global__ void __launch_bounds__(F8FewCfg<N>::kThreads, F8FewCfg<N>::kBlocksPerSm)
affine_fp8_few_kernel(const __grid_constant__ AffineF8FewParams Q) {
    stream_enter();
    using C = F8FewCfg<N>;
    const AffineF8Params &P = Q.p;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t *aligned = smem_raw + (base - raw);
    float *scales = reinterpret_cast<float *>(aligned + Q.stages * C::kStageBytes);
    uint64_t *bars = reinterpret_cast<uint64_t *>(aligned + Q.stages * C::kStageBytes + C::kScaleBytes);
    const uint32_t bar_full = smem_u32(bars);
    const uint32_t bar_done = bar_full + 8 * kF8FewMaxStages;       // a stage's product is in tensor memory, and the stage is empty
    const uint32_t bar_free = bar_done + 8 * kF8FewMaxStages;       // a part of tensor memory has been read
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + 2 * kF8FewMaxStages + C::kBuffers);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank();
    const int tile = (int)blockIdx.x / Q.split;
    const int tiles_per_block = (P.blk_out + 127) / 128;
    const int oblk = tile / tiles_per_block;
    const int n0 = (tile - oblk * tiles_per_block) * 128;   // first output feature inside the block
    const int all = P.nred * P.kpw;
    const int kb0 = (int)((int64_t)all * rank / Q.split), kb1 = (int)((int64_t)all * (rank + 1) / Q.split);
    const int stages = Q.stages;

    // one k-block's copies
    const auto copy = [&](int kb, uint32_t s) {
        const int r = kb / P.kpw, k = (kb - r * P.kpw) * kF8K;
        const uint32_t full = bar_full + 8 * s, sa = base + s * C::kStageBytes;
        const CUtensorMap *wmap = &P.w_map[P.adjoint ? r * P.pfi + oblk : oblk * P.pfi + r];
        mbar_expect_tx(full, C::kStageBytes);
        if (!P.adjoint) tma_load_2d(sa, wmap, k, n0, full);                                // K-major: box {128 k, 128 features}
        else tma_load_2d(sa, wmap, n0, k, full);                                           // MN-major: box {128 features, 128 k}
        tma_load_2d(sa + kF8WBytes, &P.a_map[r], k, 0, full);                              // box {128 k, N rows}
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_done + 8 * s, 1);
        }
        for (int b = 0; b < C::kBuffers; ++b) mbar_init(bar_free + 8 * b, 4 * C::kParts);
        *abort_flag = 0;
        fence_barrier_init();
        for (int kb = kb0; kb < min(kb1, kb0 + stages); ++kb) copy(kb, (uint32_t)(kb - kb0));
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"((uint32_t)C::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t s = 0, phase = 0;
            for (int kb = kb0 + stages; kb < kb1; ++kb) {
                if (!f8_wait(bar_done + 8 * s, phase, abort_flag)) break;
                copy(kb, s);
                if (++s == (uint32_t)stages) {
                    s = 0;
                    phase ^= 1;
                }
            }
            if (*abort_flag) {
                const uint64_t t0 = global_timer();
                while (global_timer() - t0 < 1000000ull) {}
            }
        }
        __syncwarp();
    } else if (warp < 4 && (warp & 1)) {
        // two warps issue products, every other one each (see the pair kernel)
        if (lane == 0) {
            const uint32_t idesc = f8_instr(128, N, P.adjoint, 0);
            const uint64_t a0 = smem_desc(base, P.adjoint ? kF8WBytes : 16, 1024);
            const uint64_t astep = P.adjoint ? 32 * 128 >> 4 : 32 >> 4;
            const uint64_t b0 = smem_desc(base + kF8WBytes, 16, 1024);
            uint32_t s = (uint32_t)warp >> 1, phase = 0, buf = s, bphase = 1;
            if (s >= (uint32_t)stages) s -= stages, phase ^= 1;
            for (int kb = kb0 + (warp >> 1); kb < kb1; kb += 2) {
                if (!f8_wait(bar_free + 8 * buf, bphase, abort_flag) || !f8_wait(bar_full + 8 * s, phase, abort_flag)) break;
                tcgen05_fence_after();
                const uint64_t off = (uint64_t)(s * (C::kStageBytes >> 4)), a = a0 + off, b = b0 + off;
                const uint32_t d = tmem + buf * N;
                umma_f8(d, a, b, idesc, 0u);
                umma_f8(d, a + astep, b + 2, idesc, 1u);
                umma_f8(d, a + 2 * astep, b + 4, idesc, 1u);
                umma_f8(d, a + 3 * astep, b + 6, idesc, 1u);
                tcgen05_commit(bar_done + 8 * s);
                s += 2;
                while (s >= (uint32_t)stages) s -= stages, phase ^= 1;
                if ((buf += 2) >= C::kBuffers) {
                    buf -= C::kBuffers;
                    bphase ^= 1;
                }
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        // A lane is a feature; the samples' scales, times the weights' one, go through shared memory of the warp's own, two sets in turn.
        const int quarter = warp & 3, col0 = ((warp - 4) >> 2) * C::kCols;
        constexpr int kPer = (C::kCols + 31) / 32, kAhead = 4;
        float *mine = scales + (warp - 4) * 2 * C::kCols;
        int r = kb0 / P.kpw, kin = kb0 - r * P.kpw;
        // the next k-block's scales, those of columns `lane`, `lane` + 32, ..., and the weights' one: multiplied when they are used, not waited for here
        const auto fetch = [&](float *s, float &w) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) s[i] = 0.f;
            if (r >= P.nred) return;
            w = __ldg(P.ws[P.adjoint ? r * P.pfi + oblk : oblk * P.pfi + r] + (int64_t)kin * P.ws_k + (int64_t)(n0 / kScaleBlock) * P.ws_n);
            const float *a = P.as[r] + (int64_t)kin * P.nb;
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (col0 + lane + 32 * i < P.nb) s[i] = __ldg(a + col0 + lane + 32 * i);
            if (++kin == P.kpw) {
                kin = 0;
                ++r;
            }
        };
        float next[kAhead][kPer], wnext[kAhead] = {};
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(next[i], wnext[i]);
        float2 acc[C::kCols / 2];
#pragma unroll
        for (int i = 0; i < C::kCols / 2; ++i) acc[i] = make_float2(0.f, 0.f);
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)col0;
        uint32_t s = 0, phase = 0, buf = 0;
        bool ok = true;
        for (int kb = kb0; ok && kb < kb1; kb += kAhead) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (kb + u >= kb1) break;
                float *set = mine + (u & 1) * C::kCols;
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (C::kCols % 32 == 0 || lane + 32 * i < C::kCols) set[lane + 32 * i] = next[u][i] * wnext[u];
                fetch(next[u], wnext[u]);
                __syncwarp();
                ok = __all_sync(0xffffffffu, f8_wait(bar_done + 8 * s, phase, abort_flag));
                if (!ok) break;
                tcgen05_fence_after();
                uint32_t v[C::kCols];
                tmem_ld<C::kCols>(taddr + buf * N, v);
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar_free + 8 * buf);
#pragma unroll
                for (int i = 0; i < C::kCols; i += 4) {
                    const float4 f = *reinterpret_cast<const float4 *>(set + i);
                    float2 &lo = acc[i / 2], &hi = acc[i / 2 + 1];
                    lo = __ffma2_rn(make_float2(f.x, f.y), make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), lo);
                    hi = __ffma2_rn(make_float2(f.z, f.w), make_float2(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), hi);
                }
                if (++s == (uint32_t)stages) {
                    s = 0;
                    phase ^= 1;
                }
                if (++buf == C::kBuffers) buf = 0;
            }
        }
        // every product has been taken, so the ring is free: the sums as [sample][feature]
        if (ok) {
            float *part = reinterpret_cast<float *>(aligned) + col0 * 128 + quarter * 32 + lane;
#pragma unroll
            for (int i = 0; i < C::kCols / 2; ++i) {
                part[(2 * i) * 128] = acc[i].x;
                part[(2 * i + 1) * 128] = acc[i].y;
            }
        }
    }
    tcgen05_fence_before();
    cluster_sync_all();                                     // every block's sums are in place
    if (!*abort_flag) {
        const int rows = (P.nb + Q.split - 1) / Q.split, row0 = rank * rows, row1 = min(P.nb, row0 + rows);
        const int f = 4 * lane;
        if (n0 + f < P.blk_out) {
            const float4 bias = P.bias[oblk] ? __ldg(reinterpret_cast<const float4 *>(P.bias[oblk] + n0 + f)) : make_float4(0.f, 0.f, 0.f, 0.f);
            for (int row = row0 + warp; row < row1; row += C::kThreads / 32) {
                const uint32_t addr = base + (uint32_t)((row * 128 + f) * 4);
                float4 o = ld_cluster_f4(map_to_cta(addr, 0));
                for (int q = 1; q < Q.split; ++q) {
                    const float4 v = ld_cluster_f4(map_to_cta(addr, (uint32_t)q));
                    o.x += v.x, o.y += v.y, o.z += v.z, o.w += v.w;
                }
                o.x += bias.x, o.y += bias.y, o.z += bias.z, o.w += bias.w;
                const int64_t at = (int64_t)row * P.blk_out + n0 + f;
                f8_store4(P, oblk, at, o);
            }
        }
    }
    cluster_sync_all();                                     // nobody retires while a peer reads its shared memory
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::kTmemCols) : "memory");
    }
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------
// Row-major matrix of bytes [rows, cols]; box = {box_cols (inner, 128 or 64), box_rows}, swizzled by its inner extent.
static bool make_map_u8(CUtensorMap *m, const void *ptr, int64_t rows, int64_t cols, int box_cols, int box_rows) {
    EncodeTiledFn fn = tensor_map_encoder();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)cols};
    const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              box_cols == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles of 256 or 128 columns, the contraction in one, two or four runs: the one with the least time by its clusters' turns.  Measured (B200, us): the
// first tile without its k-blocks, each further one (a pair goes on while sums are written), a k-block.  The narrow tile reads a half more through L2 for
// the same work, but fills SMs that wide ones leave idle; so do runs, which cost a meeting of their blocks (256 x 8192 x 8192: 256 columns in 1, 2, 4 runs
// 33.6, 24.9, 52.4; 128 columns 25.4, 33.8, 63.3.  2048 x 8192 x 8192: 127, 180, 295; 151, 256, 425.  200 x 8192 x 1024: 31.4, 21.5, 16.4; 24.4, 16.0,
// 12.6).
struct F8Shape {
    void (*kernel)(AffineF8Params);
    int tn, splits, threads, smem;
    double first, next, kblock;
};
constexpr int kF8Shapes = 6;
static const F8Shape kF8Shape[kF8Shapes] = {
    {affine_fp8_pair_kernel<256, false>, 256, 1, F8Cfg<256>::kThreads, F8Cfg<256>::kSmemBytes, 6.2, 1.8, 0.44},
    {affine_fp8_pair_kernel<256, true>, 256, 2, F8Cfg<256>::kThreads, F8Cfg<256>::kSmemBytes, 8.3, 0.0, 0.48},
    {affine_fp8_pair_kernel<256, true>, 256, 4, F8Cfg<256>::kThreads, F8Cfg<256>::kSmemBytes, 10.1, 0.0, 0.48},
    {affine_fp8_pair_kernel<128, false>, 128, 1, F8Cfg<128>::kThreads, F8Cfg<128>::kSmemBytes, 5.1, 1.2, 0.31},
    {affine_fp8_pair_kernel<128, true>, 128, 2, F8Cfg<128>::kThreads, F8Cfg<128>::kSmemBytes, 6.5, 0.0, 0.32},
    {affine_fp8_pair_kernel<128, true>, 128, 4, F8Cfg<128>::kThreads, F8Cfg<128>::kSmemBytes, 7.8, 0.0, 0.32},
};

// The shape for a layer of `all` k-blocks and nout output blocks of blk_out columns, its tiles and how many of its clusters run at a time; clusters: of each
// shape.
struct F8Choice {
    const F8Shape *shape;
    int64_t tiles, at_once;
};
static F8Choice f8_choose(int64_t nb, int nout, int64_t blk_out, int64_t all, const int *clusters) {
    const int64_t row_tiles = (nb + 2 * kF8Rows - 1) / (2 * kF8Rows);
    F8Choice c = {};
    double best = 0;
    for (int i = 0; i < kF8Shapes; ++i) {
        const F8Shape &s = kF8Shape[i];
        if ((s.splits > 1 && all < 4 * s.splits) || clusters[i] < 1) continue;
        const int64_t tiles = row_tiles * nout * ((blk_out + s.tn - 1) / s.tn), turns = (tiles + clusters[i] - 1) / clusters[i];
        const double again = s.splits > 1 ? s.first : s.next;
        const double us = s.first + (double)turns * (double)((all + s.splits - 1) / s.splits) * s.kblock + (double)(turns - 1) * again;
        if (!c.shape || us < best) {
            best = us;
            c = {&s, tiles, clusters[i]};
        }
    }
    return c;
}

// One-time set-up of a device: kernel attributes, and how many clusters of each shape run at a time.
static distdl_status_t f8_setup(int device, int sms, const int **clusters) {
    static bool configured_on[kMaxDevicesPerProcess] = {false};
    static int clusters_on[kMaxDevicesPerProcess][kF8Shapes];
    std::lock_guard<std::mutex> setup_lock(setup_mutex());
    if (!configured_on[device]) {
        for (int i = 0; i < kF8Shapes; ++i) {
            const F8Shape &s = kF8Shape[i];
            DISTDL_CUDA_CHECK(cudaFuncSetAttribute(s.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, s.smem));
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(2 * s.splits * sms));
            cfg.blockDim = dim3((unsigned)s.threads);
            cfg.dynamicSmemBytes = (size_t)s.smem;
            cudaLaunchAttribute attr = {};
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = 2u * s.splits;
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            DISTDL_CUDA_CHECK(cudaOccupancyMaxActiveClusters(&clusters_on[device][i], s.kernel, &cfg));
        }
        for (const auto kernel : {affine_fp8_few_kernel<16>, affine_fp8_few_kernel<32>, affine_fp8_few_kernel<64>, affine_fp8_few_kernel<128>})
            DISTDL_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kF8FewMaxSmem));
        configured_on[device] = true;
    }
    *clusters = clusters_on[device];
    return DISTDL_OK;
}

template <int N>
static void launch_few(const AffineF8Params &P, int64_t tiles, int sms, cudaStream_t stream) {
    // blocks of a tile: doubled while the device holds them all at a time and every block keeps four k-blocks
    using C = F8FewCfg<N>;
    AffineF8FewParams Q;
    Q.p = P;
    Q.split = 1;
    const int64_t all = (int64_t)P.nred * P.kpw;
    while (Q.split < 8 && tiles * Q.split * 2 <= C::kBlocksPerSm * sms && all >= 4 * 2 * Q.split) Q.split *= 2;
    const int budget = C::kBlocksPerSm == 1 || tiles * Q.split <= sms ? kF8FewMaxSmem : kF8FewMaxSmem / 2;
    Q.stages = C::stages(budget);
    const int smem = C::smem(budget);
    launch_clusters_in_stream(affine_fp8_few_kernel<N>, (unsigned)Q.split, dim3((unsigned)(tiles * Q.split)), dim3(C::kThreads), (size_t)smem, stream, Q);
}

static distdl_status_t affine_fp8_impl(int64_t nb, int64_t nfi, int64_t nfo, int32_t pfo, int32_t pfi, const void *const *act, const void *const *act_scales,
                                       const void *const *w, const void *const *ws, const void *const *bias, distdl_dtype_t t, void *const *out, void *stream,
                                       bool adjoint, const char *what) {
    clear_error();
    if (nb < 1 || nfi < 1 || nfo < 1 || pfo < 1 || pfi < 1) return fail(DISTDL_ERR_INVALID_ARG, "%s: non-positive size", what);
    if (t != DISTDL_F32 && t != DISTDL_BF16) return fail(DISTDL_ERR_INVALID_ARG, "%s: results are F32 or BF16", what);
    if (nfi % pfi || nfo % pfo) return fail(DISTDL_ERR_SHAPE, "%s: features not divisible by the worker grid", what);
    const int64_t bfi = nfi / pfi, bfo = nfo / pfo;
    if (bfi % 16 || bfo % 16)
        return fail(DISTDL_ERR_UNSUPPORTED, "%s: per-worker feature blocks must be multiples of 16 (rows of whole 16-byte units)", what);
    if (pfo > 8 || pfi > 8 || pfo * pfi > kF8MaxWorkers)
        return fail(DISTDL_ERR_UNSUPPORTED, "%s: worker grid larger than 8 per side or %d workers", what, kF8MaxWorkers);
    if (nb > (1 << 20) || bfi > (1 << 22) || bfo > (1 << 22)) return fail(DISTDL_ERR_UNSUPPORTED, "%s: more than 2^20 samples or 2^22 features a worker", what);
    const int nact = adjoint ? pfo : pfi, nout = adjoint ? pfi : pfo, grid = pfo * pfi;
    distdl_status_t st;
    if ((st = check_blocks(what, adjoint ? "dy" : "x", act, nact)) || (st = check_blocks(what, adjoint ? "dys" : "xs", act_scales, nact)) ||
        (st = check_blocks(what, "w", w, grid)) || (st = check_blocks(what, "ws", ws, grid)) || (st = check_blocks(what, adjoint ? "dx" : "y", out, nout)))
        return st;
    for (int i = 0; bias && i < nout; ++i)
        if (bias[i] && !aligned16(bias[i])) return fail(DISTDL_ERR_ALIGNMENT, "%s: bias[%d] not 16-byte aligned", what, i);
    int device, sms;
    if ((st = current_device(what, act[0], &device)) || (st = multiprocessors(device, &sms))) return st;
    if (!tensor_map_encoder()) return fail(DISTDL_ERR_CUDA, "%s: cuTensorMapEncodeTiled is not available", what);

    AffineF8Params P;
    memset(&P, 0, sizeof(P));
    P.nb = (int32_t)nb;
    P.pfi = pfi;
    P.blk_out = (int32_t)(adjoint ? bfi : bfo);
    P.blk_red = (int32_t)(adjoint ? bfo : bfi);
    P.nred = nact;
    P.kpw = (int32_t)scale_blocks(P.blk_red);
    const int32_t scale_cols = (int32_t)scale_blocks(bfi);
    P.ws_k = adjoint ? scale_cols : 1;
    P.ws_n = adjoint ? 1 : scale_cols;
    P.adjoint = adjoint ? 1 : 0;
    P.out_bf16 = t == DISTDL_BF16;
    P.nout = nout;
    P.out_wide = 1;
    P.out_lines = t == DISTDL_F32 && P.blk_out % 32 == 0;
    for (int i = 0; i < nact; ++i) P.as[i] = (const float *)act_scales[i];
    for (int i = 0; i < grid; ++i) P.ws[i] = (const float *)ws[i];
    for (int i = 0; i < nout; ++i) {
        P.out[i] = out[i];
        if (reinterpret_cast<uintptr_t>(out[i]) & 31u) P.out_wide = P.out_lines = 0;
        P.bias[i] = bias ? (const float *)bias[i] : nullptr;
    }

    const int *clusters;
    if ((st = f8_setup(device, sms, &clusters))) return st;
    const bool few = nb <= kF8Rows;
    const int n = nb <= 16 ? 16 : nb <= 32 ? 32 : nb <= 64 ? 64 : 128;
    F8Choice choice = {};
    if (!few) {
        choice = f8_choose(nb, nout, P.blk_out, (int64_t)P.nred * P.kpw, clusters);
        if (!choice.shape) return fail(DISTDL_ERR_CUDA, "%s: no cluster of two blocks fits the device", what);
    }
    const F8Shape *const shape = choice.shape;
    for (int i = 0; i < nact; ++i)
        if (!make_map_u8(&P.a_map[i], act[i], nb, P.blk_red, kF8K, few ? n : kF8Rows))
            return fail(DISTDL_ERR_CUDA, "%s: tensor map of activation block %d failed", what, i);
    for (int i = 0; i < grid; ++i) {
        // weights: the columns of a tile that a block stages, by 128 of the contraction
        const int columns = few ? 128 : shape->tn / 2;
        const bool ok = adjoint ? make_map_u8(&P.w_map[i], w[i], bfo, bfi, columns, kF8K) : make_map_u8(&P.w_map[i], w[i], bfo, bfi, kF8K, columns);
        if (!ok) return fail(DISTDL_ERR_CUDA, "%s: tensor map of weight block %d failed", what, i);
    }
    const cudaStream_t in = (cudaStream_t)stream;
    if (few) {
        const int64_t tiles = nout * scale_blocks(P.blk_out);
        if (n == 16) launch_few<16>(P, tiles, sms, in);
        else if (n == 32) launch_few<32>(P, tiles, sms, in);
        else if (n == 64) launch_few<64>(P, tiles, sms, in);
        else launch_few<128>(P, tiles, sms, in);
    } else {
        if (choice.tiles * 2 * shape->splits > INT32_MAX / 2) return fail(DISTDL_ERR_UNSUPPORTED, "%s: too many tiles", what);
        P.tiles = (int32_t)choice.tiles;
        P.splits = shape->splits;
        const unsigned count = (unsigned)(shape->splits > 1 ? choice.tiles : std::min(choice.tiles, choice.at_once));
        const unsigned blocks = 2u * shape->splits;            // of a cluster
        launch_clusters_in_stream(shape->kernel, blocks, dim3(blocks * count), dim3((unsigned)shape->threads), (size_t)shape->smem, in, P);
    }
    DISTDL_CUDA_CHECK(cudaGetLastError());
    return DISTDL_OK;
}

}  // namespace distdl

extern "C" distdl_status_t distdl_affine_fp8_fwd(int64_t nb, int64_t nfi, int64_t nfo, int32_t pfo, int32_t pfi, const void *const *x,
                                                 const void *const *xs, const void *const *w, const void *const *ws, const void *const *bias,
                                                 distdl_dtype_t t, void *const *y, void *stream) {
    return distdl::affine_fp8_impl(nb, nfi, nfo, pfo, pfi, x, xs, w, ws, bias, t, y, stream, false, "affine_fp8_fwd");
}

extern "C" distdl_status_t distdl_affine_fp8_adj(int64_t nb, int64_t nfi, int64_t nfo, int32_t pfo, int32_t pfi, const void *const *dy,
                                                 const void *const *dys, const void *const *w, const void *const *ws, distdl_dtype_t t, void *const *dx,
                                                 void *stream) {
    return distdl::affine_fp8_impl(nb, nfi, nfo, pfo, pfi, dy, dys, w, ws, nullptr, t, dx, stream, true, "affine_fp8_adj");
}

extern "C" distdl_status_t distdl_selftest_affine_fp8_shape(int64_t nb, int64_t nfi, int64_t nfo, int32_t pfo, int32_t pfi, int32_t adjoint,
                                                            const int32_t *clusters, int32_t *columns, int32_t *runs, int64_t *tiles, int64_t *at_once) {
    using namespace distdl;
    const char *what = "selftest_affine_fp8_shape";
    clear_error();
    if (!columns || !runs || !tiles || !at_once) return fail(DISTDL_ERR_INVALID_ARG, "%s: NULL argument", what);
    if (nb <= kF8Rows || nfi < 1 || nfo < 1 || pfo < 1 || pfi < 1 || nfi % pfi || nfo % pfo) return fail(DISTDL_ERR_INVALID_ARG, "%s: sizes", what);
    if (!clusters) {
        int device, sms;
        const int *found;
        DISTDL_CUDA_CHECK(cudaGetDevice(&device));
        if (device < 0 || device >= kMaxDevicesPerProcess) return fail(DISTDL_ERR_UNSUPPORTED, "%s: device index %d", what, device);
        if (const distdl_status_t st = multiprocessors(device, &sms)) return st;
        if (const distdl_status_t st = f8_setup(device, sms, &found)) return st;
        clusters = found;
    }
    const int64_t bfi = nfi / pfi, bfo = nfo / pfo;
    const F8Choice c = f8_choose(nb, adjoint ? pfi : pfo, adjoint ? bfi : bfo, adjoint ? pfo * scale_blocks(bfo) : pfi * scale_blocks(bfi), clusters);
    if (!c.shape) return fail(DISTDL_ERR_CUDA, "%s: no cluster of two blocks fits the device", what);
    *columns = c.shape->tn;
    *runs = c.shape->splits;
    *tiles = c.tiles;
    *at_once = c.at_once;
    return DISTDL_OK;
}
