// fp4_tile.cuh -- what the tcgen05 kernels of the 4-bit floating-point operators
// share: single-CTA and CTA-pair forms of loads and commits, the epilogue's way
// to memory, tensor maps.
#pragma once

#include "fp4.cuh"
#include "internal.h"
#include "mbarrier.cuh"
#include "tcgen05.cuh"

namespace mnmt {

constexpr int F4_BM = 128;  // rows of a tile per CTA
constexpr int F4_BLK = 2048;  // a warp's staging block: 32 rows of 64 bytes

// An epilogue warp has read an accumulator (tcgen05.wait::ld): the leader's MMAs
// may overwrite it.  Relaxed: nothing in memory is handed over, and a release
// would wait for the warp's own stores of the tile before (16384 x 8192 x 2048: 142 us).
template <int CG>
__device__ __forceinline__ void f4_release(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(CG == 1 ? bar : t2_mapa(bar, 0)) : "memory");
}

// One lane of a converged warp.  The producer and MMA warps of a fast kernel run
// their loops with all lanes and issue from this one by predicate (on): operands
// that every lane computes alike stay in uniform registers, where a branch on the
// lane costs a move per operand and instruction.
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t on;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(on));
    return on;
}
template <int CG>
__device__ __forceinline__ void f4_load_on(uint32_t on, uint32_t dst, const CUtensorMap *tm, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(bar), "r"(on)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t"
            "@q cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}" ::"r"(
                dst),
            "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(bar), "r"(on)
            : "memory");
}
__device__ __forceinline__ void expect_tx_on(uint32_t on, uint32_t bar, uint32_t bytes) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
                 "r"(bytes), "r"(on)
                 : "memory");
}
template <int CG>
__device__ __forceinline__ void f4_commit_on(uint32_t on, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
            "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
            "r"(on)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t"
            "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(bar),
            "h"((uint16_t)3), "r"(on)
            : "memory");
}

template <int CG>
__device__ __forceinline__ void f4_load(uint32_t dst, const CUtensorMap *tm, int x, int y, uint32_t bar) {
    if constexpr (CG == 1) tma_load_2d(dst, tm, x, y, bar);
    else t2_load(dst, tm, x, y, bar);
}
template <int CG>
__device__ __forceinline__ void f4_commit(uint32_t bar) {
    if constexpr (CG == 1) mma_commit(bar);
    else t2_commit(bar);
}

struct F4Out {
    void *y;
    long ldy;
    int type;   // MNMT_F32 / BF16 / F16
    int vec;    // 16-byte stores are aligned
    int relu;
    float alpha;
    const float *bias;
};

// 32 outputs of a row, rounded, into staging blocks (row = lane): one of 32
// 16-bit outputs, or half h of 32 fp32 ones
__device__ __forceinline__ void f4_stage16(uint8_t *blk, const float (&v)[32], int type) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int c = 0; c < 4; c++) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float lo = v[8 * c + 2 * i], hi = v[8 * c + 2 * i + 1];
            if (type == MNMT_BF16) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __half2 h = __floats2half2_rn(lo, hi);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
        *reinterpret_cast<uint4 *>(blk + lane * 64 + t2_chunk<64>(lane, c)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <int H>
__device__ __forceinline__ void f4_stage32(uint8_t *blk, const float (&v)[32]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int c = 0; c < 4; c++)
        *reinterpret_cast<float4 *>(blk + lane * 64 + t2_chunk<64>(lane, c)) =
            make_float4(v[16 * H + 4 * c], v[16 * H + 4 * c + 1], v[16 * H + 4 * c + 2], v[16 * H + 4 * c + 3]);
}

// 32 columns of a warp's 32 rows (a row per lane) from column col on: through the
// staging block (32 x 16-bit or 16 x fp32 columns) so that the stores write whole
// 64-byte runs, eight rows at a time.
__device__ __forceinline__ void f4_store_block(const F4Out &o, uint8_t *blk, const float (&v)[32], int row0, int col, int M, int N) {
    const int lane = threadIdx.x & 31, rl = lane >> 2, c = lane & 3;
    const bool f32 = o.type == MNMT_F32, whole = o.vec && row0 + 32 <= M && col + 32 <= N;
    const int es = f32 ? 4 : 2, per = 16 / es;
    const long step = 8 * o.ldy * es;  // bytes between the rows that a lane stores
    uint8_t *dst = static_cast<uint8_t *>(o.y) + ((row0 + rl) * o.ldy + col) * es + 16 * c;
    const uint8_t *src = blk + rl * 64 + t2_chunk<64>(rl, c);  // rows 8 apart have the same swizzle
#pragma unroll
    for (int h = 0; h < 2; h++) {
        if (h == 1 && !f32) break;
        __syncwarp();  // the block has been read
        if (!f32) f4_stage16(blk, v, o.type);
        else if (h == 0) f4_stage32<0>(blk, v);
        else f4_stage32<1>(blk, v);
        __syncwarp();
        if (whole) {
#pragma unroll
            for (int i = 0; i < 4; i++) *reinterpret_cast<uint4 *>(dst + i * step + 64 * h) = *reinterpret_cast<const uint4 *>(src + 512 * i);
        } else {
            const int n = N - col - 16 * h - per * c;
            for (int i = 0; i < 4; i++) {
                if (row0 + rl + 8 * i >= M || n <= 0) continue;
                const uint4 w = *reinterpret_cast<const uint4 *>(src + 512 * i);
                uint8_t *d = dst + i * step + 64 * h;
                if (o.vec && n >= per) {
                    *reinterpret_cast<uint4 *>(d) = w;
                    continue;
                }
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
                if (f32) {
#pragma unroll
                    for (int k = 0; k < 4; k++)
                        if (k < n) reinterpret_cast<uint32_t *>(d)[k] = u[k];
                } else {
#pragma unroll
                    for (int k = 0; k < 8; k++)
                        if (k < n) reinterpret_cast<uint16_t *>(d)[k] = (uint16_t)(u[k >> 1] >> (16 * (k & 1)));
                }
            }
        }
    }
}

// two-dimensional tensor map: w x h elements, rows `stride` bytes apart, boxes of bw x bh
inline bool encode(CUtensorMap *tm, CUtensorMapDataType type, const void *p, cuuint64_t w, cuuint64_t h, cuuint64_t stride, cuuint32_t bw, cuuint32_t bh,
            CUtensorMapSwizzle sw) {
    cuuint64_t dims[2] = {w, h}, strides[1] = {stride};
    cuuint32_t box[2] = {bw, bh}, estr[2] = {1, 1};
    return tma_encoder()(tm, type, 2, const_cast<void *>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// whether every 16-byte store of the epilogue is aligned
inline bool out_vec(const void *y, long ldy, int type) {
    return (reinterpret_cast<uintptr_t>(y) & 15) == 0 && ldy * (type == MNMT_F32 ? 4 : 2) % 16 == 0;
}

// cluster and launch attributes of a tile kernel (programmatic launch outside stream captures, as launch_pdl)
inline cudaLaunchConfig_t f4_config(int cg, int units, int threads, size_t smem, cudaStream_t st, cudaLaunchAttribute (&attr)[2]) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(cg * units));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    int n = 0;
    if (cg == 2) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = 2;
        attr[n].val.clusterDim.y = 1;
        attr[n++].val.clusterDim.z = 1;
    }
    cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &cs) != cudaSuccess) cs = cudaStreamCaptureStatusNone;
    if (cs != cudaStreamCaptureStatusActive) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cfg;
}

}  // namespace mnmt
