// seq_tile.cuh -- tiles of 128 rows of one head, as the tcgen05 kernels of
// attention over sequences move and multiply them.
//
// A tile in shared memory: DH / 64 boxes of 128 rows x 64 elements (128 bytes),
// 128-byte swizzle, as TMA leaves them (heads of fewer than 64 or 128 elements are
// filled up with zeros).  Read with K-major rows it is an operand whose sum runs
// over the head's elements; read MN-major, one whose sum runs over the rows.
#pragma once

#include "fp4_tile.cuh"
#include "seq_attn.cuh"

namespace mnmt {

constexpr int SQ_ROWS = 128;  // rows of a tile
template <int DH, int ROWS = SQ_ROWS>
__host__ __device__ constexpr int sq_bytes() { return DH / 64 * ROWS * 128; }

// dimensions {element, head, row}: the coordinates of a box may start at a negative row or end past the last (zeros)
inline bool sq_map(CUtensorMap *tm, const HeadRows &x, int rows, int heads, int dh, int box_rows) {
    cuuint64_t dims[3] = {(cuuint64_t)dh, (cuuint64_t)heads, (cuuint64_t)rows}, strides[2] = {(cuuint64_t)x.hd * 2, (cuuint64_t)x.ld * 2};
    cuuint32_t box[3] = {64, 1, (cuuint32_t)box_rows}, estr[3] = {1, 1, 1};
    return tma_encoder()(tm, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, x.p, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// the tile from row on of a head (one thread): completes on bar, which expects sq_bytes<DH>()
template <int DH, int ROWS = SQ_ROWS>
__device__ __forceinline__ void sq_load(uint32_t dst, const CUtensorMap *tm, int head, int row, uint32_t bar) {
    mbar_expect_tx(bar, sq_bytes<DH, ROWS>());
#pragma unroll
    for (int b = 0; b < DH / 64; b++)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst + b * ROWS * 128),
            "l"(reinterpret_cast<uint64_t>(tm)), "r"(64 * b), "r"(head), "r"(row), "r"(bar)
            : "memory");
}

// Descriptor of a tile and what step k of 16 reduction indices adds to it: K-major (the sum
// runs over the head's elements) and MN-major (over the tile's rows)
__device__ __forceinline__ uint64_t sq_k(uint32_t tile) { return sw128_desc(tile); }
template <int ROWS = SQ_ROWS>
__host__ __device__ constexpr uint64_t sq_k_step(int k) { return (uint64_t)(((k >> 2) * (ROWS * 128) + (k & 3) * 32) >> 4); }
template <int ROWS = SQ_ROWS>
__device__ __forceinline__ uint64_t sq_mn(uint32_t tile) {
    return (uint64_t)((tile >> 4) & 0x3FFFu) | ((uint64_t)((ROWS * 128) >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__host__ __device__ constexpr uint64_t sq_mn_step(int k) { return (uint64_t)(k * 2048 >> 4); }
// kind::f16, D fp32 of 128 x n; bf: bf16 operands; b_mn: B is MN-major
__host__ __device__ constexpr uint32_t sq_idesc(int n, bool bf, bool b_mn) {
    return (1u << 4) | ((bf ? 1u : 0u) << 7) | ((bf ? 1u : 0u) << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// MMAs and commits of a converged warp, by one lane (on; see elect_one): issued under a branch on
// the lane they took 100 to 130 cycles each, and set the pace of every kernel here.
__device__ __forceinline__ void sq_mma(uint32_t on, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)
        : "memory");
}
// A from tensor memory: lane = row, a column holds two elements
__device__ __forceinline__ void sq_mma_ta(uint32_t on, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15]));  // nothing in memory: loads of what comes next may go before it
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]));
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <bool BF>
__device__ __forceinline__ uint32_t sq_pack(float lo, float hi) {
    uint32_t r;
    if constexpr (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ unsigned long long sq_fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// the 32 lanes' bits of columns lo .. hi - 1 of a block of 32
__device__ __forceinline__ uint32_t sq_bits(int lo, int hi) {
    const uint32_t up = hi >= 32 ? 0xFFFFFFFFu : hi <= 0 ? 0u : (1u << hi) - 1u;
    return lo >= 32 ? 0u : lo <= 0 ? up : up & ~((1u << lo) - 1u);
}

// A column range of a row stored from fp32: COLS elements from element c0 on, those below dh, in 16-byte pieces
template <bool BF, int COLS>
__device__ __forceinline__ void sq_store(void *row, int c0, int dh, const float (&v)[COLS]) {
#pragma unroll
    for (int c = 0; c < COLS; c += 8)
        if (c0 + c < dh)
            *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(row) + c0 + c) =
                make_uint4(sq_pack<BF>(v[c], v[c + 1]), sq_pack<BF>(v[c + 2], v[c + 3]), sq_pack<BF>(v[c + 4], v[c + 5]), sq_pack<BF>(v[c + 6], v[c + 7]));
}

// COLS elements (16-bit, packed two to a word) of a warp's 32 rows, a row per lane, stored through
// `stage` (32 rows of 2 COLS bytes of the warp's own, 16-byte pieces at piece ^ row) so that
// lanes next to each other store what is next to each other (a row's pieces from its own lane:
// an instruction to 32 rows, and twice the time of the rest of a short sequence's epilogue).
// live: the rows to store; n: elements of a row, a multiple of 8.
template <int COLS>
__device__ __forceinline__ void sq_store_rows(uint8_t *stage, const uint32_t (&w)[COLS / 2], uint16_t *row0, long ld, uint32_t live, int n) {
    constexpr int P = COLS / 8;  // pieces of a row
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int c = 0; c < P; c++)
        *reinterpret_cast<uint4 *>(stage + lane * (16 * P) + 16 * ((c & ~7) | ((c ^ lane) & (P < 8 ? P - 1 : 7)))) =
            make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < P; i++) {
        const int r = i * (32 / P) + lane / P, c = lane % P;
        if (((live >> r) & 1u) && 8 * c < n)
            *reinterpret_cast<uint4 *>(row0 + r * ld + 8 * c) =
                *reinterpret_cast<const uint4 *>(stage + r * (16 * P) + 16 * ((c & ~7) | ((c ^ r) & (P < 8 ? P - 1 : 7))));
    }
    __syncwarp();
}

// all threads of the cluster, whole warps
__device__ __forceinline__ void sq_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 sq_remote(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}

__device__ __forceinline__ float2 sq_remote2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
    return v;
}

// launch_pdl in clusters of `ctas`
template <typename... KArgs, typename... Args>
cudaError_t sq_launch(void (*kernel)(KArgs...), unsigned grid, int ctas, int threads, size_t smem, cudaStream_t st, Args &&...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (ctas > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)ctas;
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
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Args &&>(args)...);
}

// what was written to or read from shared memory comes before copies into it by TMA (all threads, before a barrier)
__device__ __forceinline__ void sq_before_copies() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// mbar_try of a whole warp: the vote on its own predicate, so that all lanes have the same answer
__device__ __forceinline__ bool sq_try_all(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "vote.sync.all.pred p, p, 0xFFFFFFFF;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Waits of a kernel's roles: a wait that gives up sets `failed` in shared memory and the
// status, and every role leaves its loop at its next wait.  What comes behind a warp's wait takes
// whole warps (tcgen05.ld and st, votes), so its lanes give up as one, by votes: looking
// for themselves, one might see the phase end that another had just given up.
static __device__ __noinline__ bool sq_wait_warp(volatile int *failed, int *status, uint32_t bar, uint32_t parity) {
    unsigned long long t0 = 0;
    for (int i = 0;; i++) {
        if (sq_try_all(bar, parity)) return true;
        if (i < 8) continue;
        if (i == 8) t0 = global_ns();
        if (__any_sync(0xFFFFFFFFu, *failed || global_ns() - t0 > MNMT_WAIT_NS)) break;
    }
    if ((threadIdx.x & 31) == 0) {
        *failed = 1;
        set_status(status, MNMT_ETIMEOUT);
    }
    return false;
}
static __device__ __noinline__ bool sq_wait_one(volatile int *failed, int *status, uint32_t bar, uint32_t parity) {
    for (int i = 0; i < 8; i++)
        if (mbar_try(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    while (!mbar_try(bar, parity))
        if (*failed || global_ns() - t0 > MNMT_WAIT_NS) {
            *failed = 1;
            set_status(status, MNMT_ETIMEOUT);
            return false;
        }
    return true;
}
struct SqWaits {
    volatile int *failed;
    int *status;
    // A whole warp: alike in all lanes.  The first look may suspend the warp for a while: one that
    // never does sent most waits into the call (3 x 2500..4095 rows of 16 heads of 128, gradients: 400 us, 366 so).
    __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) const {
        return sq_try_all(bar, parity) || sq_wait_warp(failed, status, bar, parity);
    }
    // one lane
    __device__ __forceinline__ bool one(uint32_t bar, uint32_t parity) const {
        return mbar_test(bar, parity) || sq_wait_one(failed, status, bar, parity);
    }
    // whether a role has given up: alike in all lanes of a warp
    __device__ __forceinline__ bool given_up() const { return __any_sync(0xFFFFFFFFu, *failed); }
};

}  // namespace mnmt
