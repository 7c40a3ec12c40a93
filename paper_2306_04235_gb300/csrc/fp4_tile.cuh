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
constexpr int F4_EPI_WARPS = 8;
constexpr int F4_THREADS = 64 + F4_EPI_WARPS * 32;  // producer warp, MMA warp, epilogue warps
constexpr int F4_BLK = 2048;  // a staging block: 32 rows of 64 bytes

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

__device__ __forceinline__ void f4_epi_sync() { asm volatile("bar.sync 1, %0;" ::"n"(F4_EPI_WARPS * 32) : "memory"); }

struct F4Out {
    void *y;
    long ldy;
    int type;   // MNMT_F32 / BF16 / F16
    int tma;    // tmY describes y
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

// a staged block to y where no tensor map describes it: coalesced single elements
__device__ __forceinline__ void f4_store_plain(const F4Out &o, const uint8_t *blk, int row0, int col0, int M, int N) {
    const int lane = threadIdx.x & 31;
    if (o.type == MNMT_F32) {
        const int c = lane & 15;
        for (int r = lane >> 4; r < 32; r += 2)
            if (row0 + r < M && col0 + c < N)
                static_cast<float *>(o.y)[(row0 + r) * o.ldy + col0 + c] =
                    *reinterpret_cast<const float *>(blk + r * 64 + t2_chunk<64>(r, c >> 2) + 4 * (c & 3));
    } else {
        for (int r = 0; r < 32; r++)
            if (row0 + r < M && col0 + lane < N)
                static_cast<uint16_t *>(o.y)[(row0 + r) * o.ldy + col0 + lane] =
                    *reinterpret_cast<const uint16_t *>(blk + r * 64 + t2_chunk<64>(r, lane >> 3) + 2 * (lane & 7));
    }
}

// 32 columns of a warp's 32 rows (a row per lane) from column col on: one block
// of 16-bit outputs or two of fp32, staged in the two blocks at stg by turns
__device__ __forceinline__ void f4_store_block(const F4Out &o, const CUtensorMap *tmY, uint8_t *stg, uint32_t &blocks, const float (&v)[32], int row0,
                                               int col, int M, int N) {
    const int lane = threadIdx.x & 31;
    const bool f32 = o.type == MNMT_F32;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        if (h == 1 && !f32) break;
        uint8_t *blk = stg + (blocks & 1) * F4_BLK;
        if (o.tma) {
            if (lane == 0) t2_store_wait_read<1>();  // the store before the last has read this block
            __syncwarp();
        }
        if (!f32) f4_stage16(blk, v, o.type);
        else if (h == 0) f4_stage32<0>(blk, v);
        else f4_stage32<1>(blk, v);
        if (o.tma) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (col + 16 * h < N) t2_store(tmY, col + 16 * h, row0, s_addr(blk));
                t2_store_commit();
            }
        } else {
            __syncwarp();
            f4_store_plain(o, blk, row0, col + 16 * h, M, N);
            __syncwarp();
        }
        blocks++;
    }
}

// two-dimensional tensor map: w x h elements, rows `stride` bytes apart, boxes of bw x bh
inline bool encode(CUtensorMap *tm, CUtensorMapDataType type, const void *p, cuuint64_t w, cuuint64_t h, cuuint64_t stride, cuuint32_t bw, cuuint32_t bh,
            CUtensorMapSwizzle sw, bool load) {
    cuuint64_t dims[2] = {w, h}, strides[1] = {stride};
    cuuint32_t box[2] = {bw, bh}, estr[2] = {1, 1};
    return tma_encoder()(tm, type, 2, const_cast<void *>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
                         load ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// the map of an output matrix in the epilogue's boxes; o.tma: whether there is one
inline void encode_out(CUtensorMap *tm, F4Out &o, int M, int N) {
    const int es = o.type == MNMT_F32 ? 4 : 2;
    const CUtensorMapDataType t = o.type == MNMT_F32    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                  : o.type == MNMT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    o.tma = (reinterpret_cast<uintptr_t>(o.y) & 15) == 0 && o.ldy * es % 16 == 0 && o.ldy * es < ((long)1 << 40) &&
            encode(tm, t, o.y, N, M, (cuuint64_t)o.ldy * es, 64 / es, 32, CU_TENSOR_MAP_SWIZZLE_64B, false);
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
