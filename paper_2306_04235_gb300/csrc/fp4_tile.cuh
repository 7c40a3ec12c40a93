// fp4_tile.cuh -- what the tcgen05 kernels of the 4-bit floating-point operators
// share: single-CTA and CTA-pair forms of loads and commits, the epilogue's way
// to memory, tensor maps.
#pragma once

#include <type_traits>

#include "fp4.cuh"
#include "mbarrier.cuh"
#include "row_pass.cuh"
#include "tcgen05.cuh"
#include "train.h"

namespace mnmt {

constexpr int F4_BM = 128;  // rows of a tile per CTA

// mbar_wait.  Most waits end within the first tries, each of which suspends the
// thread for a while; reading the device clock before them costs each its latency.
// (A function that calls none: with mbar_wait called here 8192^3 took 177 us, 160 so.)
static __device__ __noinline__ bool f4_wait_slow(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < 8; i++)
        if (mbar_try(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    while (!mbar_try(bar, parity))
        if (global_ns() - t0 > MNMT_WAIT_NS) return false;
    return true;
}
__device__ __forceinline__ bool f4_wait(uint32_t bar, uint32_t parity) { return mbar_test(bar, parity) || f4_wait_slow(bar, parity); }

// An epilogue warp has read an accumulator (tcgen05.wait::ld): the leader's MMAs
// may overwrite it.  Relaxed: nothing in memory is handed over, and a release
// would wait for the warp's own stores of the tile before (16384 x 8192 x 2048: 142 us, 109 so).
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
    int al;     // every row starts on 32 bytes (2), 16 bytes (1), less (0)
    int tma;    // stores by TMA
    int relu;
    float alpha;
    const float *bias;
};

// The tiles of a unit (CTA or pair), every units-th one, without divisions after
// the first: the dimension of fewer tiles runs fastest, so that the larger operand
// is read by units that run at the same time.
struct F4Walk {
    int fast, slow, f, end, df, ds;
    bool m_fast;
    __device__ __forceinline__ F4Walk(int mt, int nt, int unit, int units) {
        m_fast = mt <= nt;
        f = m_fast ? mt : nt, end = m_fast ? nt : mt;
        fast = unit % f, slow = unit / f;
        df = units % f, ds = units / f;
    }
    __device__ __forceinline__ bool more() const { return slow < end; }
    __device__ __forceinline__ int m() const { return m_fast ? fast : slow; }
    __device__ __forceinline__ int n() const { return m_fast ? slow : fast; }
    __device__ __forceinline__ void next() {
        fast += df, slow += ds;
        if (fast >= f) fast -= f, slow++;
    }
};

// two fp32 at a time: sums and products, each rounded (the pair instructions of this part)
__device__ __forceinline__ unsigned long long f4_two(float lo, float hi) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void f4_untwo(unsigned long long v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ unsigned long long f4_add2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long f4_mul2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// outputs c .. c + 1 of a row as a word of type's 16 bits
__device__ __forceinline__ uint32_t f4_pair(float lo, float hi, int type) {
    if (type == MNMT_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// `rows` rows of n bytes from a block as f4_store_block leaves it.  Out of line where
// the kernel's loops need no registers across the call (single CTAs: 512 x 32001 x 512
// 21.5 us, inline 24.8; gradients: 64 x 32000 x 511 84.6, 94.7), inline on pairs (16384 x
// 8190 x 2048 122 us, out of line 157).
__device__ __forceinline__ void f4_block_out(uint8_t *dst, long ld, uint32_t bits, const uint8_t *blk, bool f32, int n, int rows) {
    const int lane = threadIdx.x & 31, rb = f32 ? 128 : 64;
    auto store = [&](auto unit) {
        using T = decltype(unit);
        const int lanes = rb / (int)sizeof(T), at = lane % lanes * (int)sizeof(T);
        if (at >= n) return;
#pragma unroll 8
        for (int r = lane / lanes; r < rows; r += 32 / lanes)
            *reinterpret_cast<T *>(dst + r * ld + at) =
                *reinterpret_cast<const T *>(blk + r * rb + (f32 ? t2_chunk<128>(r, at >> 4) : t2_chunk<64>(r, at >> 4)) + (at & 15));
    };
    if (bits % 8 == 0) store(uint2{});
    else if (bits % 4 == 0) store(uint32_t{});
    else store(uint16_t{});
}
static __device__ __noinline__ void f4_block_out_call(uint8_t *dst, long ld, uint32_t bits, const uint8_t *blk, bool f32, int n, int rows) {
    f4_block_out(dst, ld, bits, blk, f32, n, rows);
}

// 32 columns of a warp's 32 rows (a row per lane) from column col on, from
// registers: a lane stores its row in whole 32-byte sectors (o.al, all columns in the matrix).
__device__ __forceinline__ void f4_store_rows(const F4Out &o, const float (&v)[32], int row0, int col, int M) {
    const int lane = threadIdx.x & 31;
    const bool f32 = o.type == MNMT_F32;
    if (row0 + lane >= M) return;
    uint8_t *dst = static_cast<uint8_t *>(o.y) + ((row0 + lane) * o.ldy + col) * (f32 ? 4 : 2);
    if (f32) {
        uint32_t w[32];
#pragma unroll
        for (int i = 0; i < 32; i++) w[i] = __float_as_uint(v[i]);
        if (o.al == 2) {
#pragma unroll
            for (int i = 0; i < 4; i++) st32(dst + 32 * i, w + 8 * i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) reinterpret_cast<uint4 *>(dst)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
    } else {
        uint32_t w[16];
        if (o.type == MNMT_BF16) {
#pragma unroll
            for (int i = 0; i < 16; i++) w[i] = f4_pair(v[2 * i], v[2 * i + 1], MNMT_BF16);
        } else {
#pragma unroll
            for (int i = 0; i < 16; i++) w[i] = f4_pair(v[2 * i], v[2 * i + 1], MNMT_F16);
        }
        if (o.al == 2) {
            st32(dst, w);
            st32(dst + 32, w + 8);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) reinterpret_cast<uint4 *>(dst)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
    }
}

// The same of any alignment and cut off at the matrix's edge, turned in shared memory
// first (blk: BLK bytes, 32 rows of 16-bit outputs or more), so that lanes next to
// each other store what is next to each other in a row, 8, 4 or 2 bytes each as the
// rows are aligned (4052 x 25146 x 115 to fp32 110 us; in pieces of 32 bytes of a
// row 232).
template <int BLK, bool INLINE>
__device__ __forceinline__ void f4_store_block(const F4Out &o, uint8_t *blk, const float (&v)[32], int row0, int col, int M, int N) {
    const int lane = threadIdx.x & 31;
    const bool f32 = o.type == MNMT_F32;
    const int es = f32 ? 4 : 2, rb = 32 * es, pass = BLK / rb < 32 ? BLK / rb : 32;  // bytes of a row; rows at a time
    const int n = (N - col < 32 ? N - col : 32) * es;                               // bytes to store of each
    uint8_t *dst = static_cast<uint8_t *>(o.y) + (row0 * o.ldy + col) * es;
    const long ld = o.ldy * es;
    const uint32_t bits = (uint32_t)reinterpret_cast<uintptr_t>(o.y) | (uint32_t)ld | (uint32_t)n;
    for (int r0 = 0; r0 < 32; r0 += pass) {
        __syncwarp();  // the block has been read
        if (lane >= r0 && lane < r0 + pass) {
            if (f32) {
#pragma unroll
                for (int c = 0; c < 8; c++)
                    *reinterpret_cast<uint4 *>(blk + (lane - r0) * 128 + t2_chunk<128>(lane - r0, c)) =
                        make_uint4(__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]), __float_as_uint(v[4 * c + 2]), __float_as_uint(v[4 * c + 3]));
            } else {
#pragma unroll
                for (int c = 0; c < 4; c++)
                    *reinterpret_cast<uint4 *>(blk + (lane - r0) * 64 + t2_chunk<64>(lane - r0, c)) =
                        make_uint4(f4_pair(v[8 * c], v[8 * c + 1], o.type), f4_pair(v[8 * c + 2], v[8 * c + 3], o.type),
                                   f4_pair(v[8 * c + 4], v[8 * c + 5], o.type), f4_pair(v[8 * c + 6], v[8 * c + 7], o.type));
            }
        }
        __syncwarp();
        if constexpr (INLINE) f4_block_out(dst + r0 * ld, ld, bits, blk, f32, n, min(pass, M - row0 - r0));
        else f4_block_out_call(dst + r0 * ld, ld, bits, blk, f32, n, min(pass, M - row0 - r0));
    }
}

// The same by TMA (o.tma): blocks of 32 rows x 64 bytes (fp32 with RB = 128: 128) of
// tensor map tm, staged in BLOCKS blocks at stg by turns; `sent` counts them.
template <int RB, int BLOCKS>
__device__ __forceinline__ void f4_send_block(const F4Out &o, const CUtensorMap *tm, uint8_t *stg, uint32_t &sent, const float (&v)[32], int row0, int col,
                                              int N) {
    const int lane = threadIdx.x & 31;
    auto send = [&](auto first) {
        constexpr int C0 = decltype(first)::value;
        uint8_t *blk = stg + (sent++ & (BLOCKS - 1)) * (32 * RB);
        if (lane == 0) t2_store_wait_read<BLOCKS - 1>();  // the block's earlier store has read it
        __syncwarp();
        if (o.type == MNMT_F32) {
#pragma unroll
            for (int c = 0; c < RB / 16; c++)
                *reinterpret_cast<uint4 *>(blk + lane * RB + t2_chunk<RB>(lane, c)) =
                    make_uint4(__float_as_uint(v[C0 + 4 * c]), __float_as_uint(v[C0 + 4 * c + 1]), __float_as_uint(v[C0 + 4 * c + 2]),
                               __float_as_uint(v[C0 + 4 * c + 3]));
        } else {
#pragma unroll
            for (int c = 0; c < 4; c++)
                *reinterpret_cast<uint4 *>(blk + lane * 64 + t2_chunk<64>(lane, c)) =
                    make_uint4(f4_pair(v[8 * c], v[8 * c + 1], o.type), f4_pair(v[8 * c + 2], v[8 * c + 3], o.type),
                               f4_pair(v[8 * c + 4], v[8 * c + 5], o.type), f4_pair(v[8 * c + 6], v[8 * c + 7], o.type));
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            if (col + C0 < N) t2_store(tm, col + C0, row0, s_addr(blk));
            t2_store_commit();
        }
    };
    send(std::integral_constant<int, 0>{});
    if constexpr (RB == 64)
        if (o.type == MNMT_F32) send(std::integral_constant<int, 16>{});
}

// two-dimensional tensor map: w x h elements, rows `stride` bytes apart, boxes of bw x bh
inline bool encode(CUtensorMap *tm, CUtensorMapDataType type, const void *p, cuuint64_t w, cuuint64_t h, cuuint64_t stride, cuuint32_t bw, cuuint32_t bh,
            CUtensorMapSwizzle sw) {
    cuuint64_t dims[2] = {w, h}, strides[1] = {stride};
    cuuint32_t box[2] = {bw, bh}, estr[2] = {1, 1};
    return tma_encoder()(tm, type, 2, const_cast<void *>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, sw,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether rows of cols elements can be stored by TMA: it stores 16 bytes at a time, so
// a row that ends within 16 bytes would take what lies beside it along.
inline bool tma_output(const F4Out &o, int cols) { return o.al && (long)cols * (o.type == MNMT_F32 ? 4 : 2) % 16 == 0; }

// the map for f4_send_block<RB, ...>
template <int RB>
bool encode_out(CUtensorMap *tm, const F4Out &o, int rows, int cols) {
    const bool f32 = o.type == MNMT_F32, wide = f32 && RB == 128;
    const int es = f32 ? 4 : 2;
    return encode(tm, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, o.y, cols, rows, (cuuint64_t)o.ldy * es,
                  (wide ? 128 : 64) / es, 32, wide ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

inline int out_alignment(const void *y, long ldy, int type) {
    return type == MNMT_F32 ? row_alignment(static_cast<const float *>(y), ldy) : row_alignment(static_cast<const uint16_t *>(y), ldy);
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
