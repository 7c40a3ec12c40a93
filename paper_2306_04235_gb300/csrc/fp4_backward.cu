// fp4_backward.cu -- gradients of the linear on microscaled 4-bit floating-point
// operands (include/mnmt.h, mnmt_fp4_linear_backward).
//
//   gX[m][k] = in_x alpha_w sum_n G[m][n] W[n][k]
//   gW[n][k] = in_w alpha_x sum_m G[m][n] X[m][k],   gb[n] = sum_m G[m][n]
// The output gradients stay bf16, so both products run on tcgen05 kind::f16: a
// code times its block scale (a power of two, or an E4M3 number) has at most six
// significant bits and is exact in bf16, products are exact in fp32.
//
// fp4_backward_prepare, one pass over the operands (memory): W and X decoded to
// bf16 in their stored order, column sums of G over 256 rows at a time, and a
// copy of G where TMA cannot read it (rows not 16-byte aligned).
// fp4_backward_gemm, both products in one persistent launch (tensor cores): the
// reduction index is the row of a stored operand, so the MMAs read W, X and (for
// gW) G "MN-major" from tiles as they lie in memory: no transposed copies.  The
// epilogue warps sum the bias gradient while the first tile is multiplied,
// gather the straight-through masks of a tile before its sums are ready, and
// store through shared memory by TMA.
#include <type_traits>

#include "fp4.cuh"
#include "fp4_tile.cuh"
#include "internal.h"

namespace mnmt {
namespace {

constexpr int GB_ROWS = 256;  // rows of G per partial column sum

struct PrepArgs {
    Fp4Args w, x;
    const __nv_bfloat16 *g;
    long ldg;
    __nv_bfloat16 *w16, *x16, *g16;  // each may be null
    float *part;                     // [ceil(M / 256)][N], may be null
    int M, N, K, pk, pn;
    int bw, bx;                      // blocks of W, of X; the rest take G
};

// rows of a packed matrix as bf16 (without the tensor scale); a thread takes 32 elements of a row
template <bool NV>
MNMT_DEV void decode_rows(const Fp4Args &q, __nv_bfloat16 *out, int ld, long first, long step) {
    const int groups = fp4_div_up(q.cols, 32), tiles_k = fp4_tiles_k(q.cols, NV);
    const long total = (long)q.rows * groups;
    for (long i = first; i < total; i += step) {
        const int row = (int)(i / groups), c = (int)(i - (long)row * groups) * 32;
        const uint4 codes = *reinterpret_cast<const uint4 *>(q.codes + (size_t)row * fp4_pitch(q.cols) + (c >> 1));
        const uint32_t cw[4] = {codes.x, codes.y, codes.z, codes.w};
        float S[2];
        const uint8_t *sp = q.scales + fp4_scale_at(row, c / fp4_block(NV), tiles_k);
        S[0] = fp4_scale_of<NV>(sp[0], 1.0f).S;
        S[1] = NV ? fp4_scale_of<NV>(sp[1], 1.0f).S : S[0];
        __nv_bfloat16 *o = out + (size_t)row * ld + c;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            uint32_t w[4];
#pragma unroll
            for (int b = 0; b < 4; b++) {
                const float2 f = fp4_float2((cw[j] >> (8 * b)) & 0xFFu);
                const __nv_bfloat162 h = __floats2bfloat162_rn(__fmul_rn(f.x, S[j >> 1]), __fmul_rn(f.y, S[j >> 1]));
                w[b] = *reinterpret_cast<const uint32_t *>(&h);
            }
            if (c + 8 * j < ld) *reinterpret_cast<uint4 *>(o + 8 * j) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

template <bool NV>
__global__ void __launch_bounds__(256) fp4_backward_prepare(PrepArgs a) {
    pdl_grid_wait();
    if ((int)blockIdx.x < a.bw) {
        decode_rows<NV>(a.w, a.w16, a.pk, (long)blockIdx.x * 256 + threadIdx.x, (long)a.bw * 256);
        return;
    }
    if ((int)blockIdx.x < a.bw + a.bx) {
        decode_rows<NV>(a.x, a.x16, a.pk, (long)(blockIdx.x - a.bw) * 256 + threadIdx.x, (long)a.bx * 256);
        return;
    }
    // 256 rows x 256 columns of G per block and step: a thread takes eight columns of every eighth row
    __shared__ float red[8][257];
    const int strips = fp4_div_up(a.N, 256), chunks = fp4_div_up(a.M, GB_ROWS);
    const bool vec = (reinterpret_cast<uintptr_t>(a.g) & 15) == 0 && a.ldg % 8 == 0;
    const int cg = (threadIdx.x & 31) * 8, rr = threadIdx.x >> 5;
    for (long i = (int)blockIdx.x - a.bw - a.bx; i < (long)strips * chunks; i += (int)gridDim.x - a.bw - a.bx) {
        const int chunk = (int)(i / strips), c = (int)(i - (long)chunk * strips) * 256 + cg;
        float s[8] = {};
        const int r1 = min(a.M, (chunk + 1) * GB_ROWS);
#pragma unroll 4
        for (int r = chunk * GB_ROWS + rr; r < r1; r += 8) {
            if (c >= a.N) break;
            float v[8];
            const __nv_bfloat16 *p = a.g + r * a.ldg + c;
            if (vec && c + 8 <= a.N) load8<__nv_bfloat16, true>(p, 8, v);
            else load8<__nv_bfloat16, false>(p, a.N - c, v);
            if (a.g16) store8<__nv_bfloat16, true>(a.g16 + (size_t)r * a.pn + c, 8, v);
#pragma unroll
            for (int k = 0; k < 8; k++) s[k] = __fadd_rn(s[k], v[k]);
        }
        if (!a.part) continue;
#pragma unroll
        for (int k = 0; k < 8; k++) red[rr][cg + k] = s[k];
        __syncthreads();
        float t = red[0][threadIdx.x];
        for (int w = 1; w < 8; w++) t = __fadd_rn(t, red[w][threadIdx.x]);
        const int n = c - cg + (int)threadIdx.x;
        if (n < a.N) a.part[(size_t)chunk * a.N + n] = t;
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// the two products
// ---------------------------------------------------------------------------
constexpr int BW_BK = 64;  // reduction indices per stage

template <int CG, int BN>
struct BwLayout {
    static constexpr uint32_t A_BYTES = F4_BM * BW_BK * 2;
    static constexpr uint32_t B_BYTES = BN / CG * BW_BK * 2;
    static constexpr uint32_t STAGE = A_BYTES + B_BYTES;
    static constexpr uint32_t STG = F4_EPI_WARPS * 2 * F4_BLK;
    static constexpr int FIT = (int)((227 * 1024 - 1024 - STG - 512) / STAGE);
    static constexpr int STAGES = FIT > 8 ? 8 : FIT;
    static constexpr uint32_t OFF_STG = STAGES * STAGE;
    static constexpr uint32_t OFF_BARS = OFF_STG + STG;
    static constexpr int NBARS = 2 * STAGES + 5;
    static constexpr uint32_t OFF_MISC = OFF_BARS + NBARS * 8;
    static constexpr size_t SMEM = 1024 + OFF_MISC + 16;
    static constexpr int COLS = pow2_cols(2 * BN);
    static_assert(NBARS * 8 + 16 <= 512, "barriers fit");
};

// one of the products: rows x cols outputs, sums over red indices
struct BwProduct {
    int rows, cols, red, a_mn;  // a_mn: A is stored [red][rows] (gW), else [rows][red]
    F4Out out;
    // straight-through mask: the float original and the scales of its packed form
    const void *orig;
    long ldo;
    int otype;
    Fp4Args q;
};
struct BwArgs {
    BwProduct p[2];
    int n;               // products
    const float *part;   // partial column sums of G [chunks][N], or null
    float *gb;
    int chunks, N;
};

// MN-major operand tile as TMA leaves it: boxes of 64 (M or N) x 64 (reduction),
// rows of 128 bytes, 128-byte swizzle; 8-row groups 1024 bytes apart (stride
// offset), boxes 8192 bytes apart (leading offset)
__device__ __forceinline__ uint64_t mn128_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)(8192 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
           ((uint64_t)2 << 61);
}

// kind::f16, D fp32, A and B bf16, B MN-major
__host__ __device__ constexpr uint32_t bw_idesc(int m, int n, bool a_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((a_mn ? 1u : 0u) << 15) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// bit i: element (row, col + i) of the original lies within the range of its block
template <bool NV>
MNMT_DEV uint32_t inside32(const BwProduct &p, int row, int col) {
    if (!p.orig) return 0xFFFFFFFFu;
    const uint8_t *sp = p.q.scales + fp4_scale_at(row, col / fp4_block(NV), fp4_tiles_k(p.cols, NV));
    const float r0 = fp4_scale_of<NV>(sp[0], p.q.g).r, r1 = NV && col + 16 < p.cols ? fp4_scale_of<NV>(sp[1], p.q.g).r : r0;
    uint32_t m = 0;
    auto gather = [&](auto t) {
        using T = decltype(t);
        const T *src = static_cast<const T *>(p.orig) + row * p.ldo + col;
        const bool vec = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if (col + 8 * j >= p.cols) break;
            float v[8];
            if (vec && col + 8 * j + 8 <= p.cols) load8<T, true>(src + 8 * j, 8, v);
            else load8<T, false>(src + 8 * j, p.cols - col - 8 * j, v);
#pragma unroll
            for (int k = 0; k < 8; k++) m |= (uint32_t)(fabsf(__fmul_rn(v[k], j < 2 ? r0 : r1)) <= 6.0f) << (8 * j + k);
        }
    };
    if (p.otype == MNMT_F32) gather(float{});
    else if (p.otype == MNMT_BF16) gather(__nv_bfloat16{});
    else gather(__half{});
    return m;
}

// Persistent, 320 threads per CTA: warp 0 lane 0 loads tiles by TMA, warp 1 lane
// 0 issues MMAs into two TMEM accumulators, warps 2..9 drain them.  Tiles of
// product 0 come before those of product 1.
template <int CG, int BN, bool NV>
__global__ void __launch_bounds__(F4_THREADS, 1)
    fp4_backward_gemm(const __grid_constant__ CUtensorMap tmA0, const __grid_constant__ CUtensorMap tmB0, const __grid_constant__ CUtensorMap tmY0,
                      const __grid_constant__ CUtensorMap tmA1, const __grid_constant__ CUtensorMap tmB1, const __grid_constant__ CUtensorMap tmY1,
                      const __grid_constant__ BwArgs a, int *status) {
    pdl_grid_wait();
    using L = BwLayout<CG, BN>;
    constexpr int STAGES = L::STAGES, BOXES = BN / CG / 64;

    extern __shared__ uint8_t bw_raw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(bw_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t bars = s_addr(sm + L::OFF_BARS);
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
    auto accf_bar = [&](int b) { return bars + 8u * (2 * STAGES + b); };
    auto acce_bar = [&](int b) { return bars + 8u * (2 * STAGES + 2 + b); };
    const uint32_t done_bar = bars + 8u * (2 * STAGES + 4);
    uint32_t *misc = reinterpret_cast<uint32_t *>(sm + L::OFF_MISC);  // [0] tmem base, [1] abort, [2] consumed
    volatile uint32_t *abort_flag = misc + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank = 0;
    if constexpr (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int unit = (int)blockIdx.x / CG, units = (int)gridDim.x / CG;
    auto mt = [&](int i) { return (a.p[i].rows + CG * F4_BM - 1) / (CG * F4_BM); };
    auto nt = [&](int i) { return (a.p[i].cols + BN - 1) / BN; };
    const long t0 = (long)mt(0) * nt(0), tiles = t0 + (a.n > 1 ? (long)mt(1) * nt(1) : 0);
    // product and corner of a tile: the dimension of fewer tiles runs fastest
    struct At {
        int p, m, n;
    };
    auto at = [&](long t) {
        At r;
        r.p = t >= t0;
        if (r.p) t -= t0;
        const int m = mt(r.p), n = nt(r.p);
        r.m = (int)(m <= n ? t % m : t / n) * CG * F4_BM;
        r.n = (int)(m <= n ? t / m : t % n) * BN;
        return r;
    };

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; s++) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(accf_bar(b), 1);
            mbar_init(acce_bar(b), CG * F4_EPI_WARPS);
        }
        mbar_init(done_bar, 1);
        misc[1] = 0;
        misc[2] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            tmem_alloc<L::COLS>(s_addr(misc));
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s_addr(misc)), "r"(L::COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
        tc_fence_before();
    }
    if constexpr (CG == 2) asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = misc[0];

    uint32_t issued = 0;
    if (warp == 0 && lane == 0) {
        // ---- TMA producer ----
        uint32_t it = 0;
        bool failed = false;
        const uint32_t ring = s_addr(sm);
        for (long tile = unit; tile < tiles && !failed && !*abort_flag; tile += units) {
            const At t = at(tile);
            const CUtensorMap *ta = t.p ? &tmA1 : &tmA0, *tb = t.p ? &tmB1 : &tmB0;
            const int m0 = t.m + (int)rank * F4_BM, n0 = t.n + (int)rank * (BN / CG), nkb = (a.p[t.p].red + BW_BK - 1) / BW_BK;
            const bool a_mn = a.p[t.p].a_mn;
            for (int kb = 0; kb < nkb; kb++, it++) {
                const int s = (int)(it % STAGES);
                if (it >= STAGES && !mbar_wait(empty_bar(s), (it / STAGES - 1) & 1)) {
                    *abort_flag = 1;
                    set_status(status, MNMT_ETIMEOUT);
                    failed = true;
                    break;
                }
                if (rank == 0) mbar_expect_tx(full_bar(s), CG * L::STAGE);
                const uint32_t bar = CG == 1 ? full_bar(s) : t2_mapa(full_bar(s), 0), base = ring + s * L::STAGE;
                if (a_mn) {
                    f4_load<CG>(base, ta, m0, kb * BW_BK, bar);
                    f4_load<CG>(base + 8192, ta, m0 + 64, kb * BW_BK, bar);
                } else {
                    f4_load<CG>(base, ta, kb * BW_BK, m0, bar);
                }
#pragma unroll
                for (int j = 0; j < BOXES; j++) f4_load<CG>(base + L::A_BYTES + j * 8192, tb, n0 + 64 * j, kb * BW_BK, bar);
                issued = it + 1;
            }
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---- MMA issuer ----
        uint32_t it = 0, lt = 0;
        bool failed = false;
        const uint32_t ring = s_addr(sm);
        const uint64_t b_desc = mn128_desc(ring + L::A_BYTES);
        for (long tile = unit; tile < tiles && !failed; tile += units, lt++) {
            const int buf = (int)(lt & 1), p = tile >= t0;
            if (lt >= 2 && !mbar_wait(acce_bar(buf), (lt / 2 - 1) & 1)) {
                failed = true;
                break;
            }
            tc_fence_after();
            const uint32_t d = tbase + (uint32_t)(buf * BN);
            const bool a_mn = a.p[p].a_mn;
            const uint64_t a_desc = a_mn ? mn128_desc(ring) : sw128_desc(ring);
            const uint64_t a_step = a_mn ? 2048 >> 4 : 32 >> 4;  // 16 reduction indices
            const uint32_t idesc = bw_idesc(CG * F4_BM, BN, a_mn);
            const int nkb = (a.p[p].red + BW_BK - 1) / BW_BK;
            for (int kb = 0; kb < nkb; kb++, it++) {
                const int s = (int)(it % STAGES);
                if (!mbar_wait(full_bar(s), (it / STAGES) & 1)) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                const uint64_t off = (uint64_t)((s * L::STAGE) >> 4);
#pragma unroll
                for (int k = 0; k < BW_BK / 16; k++) {
                    const uint64_t ad = a_desc + off + a_step * k, bd = b_desc + off + (uint64_t)(k * (2048 >> 4));
                    if constexpr (CG == 1) mma_f16(d, ad, bd, idesc, (uint32_t)(kb | k));
                    else t2_mma(d, ad, bd, idesc, (uint32_t)(kb | k));
                }
                f4_commit<CG>(empty_bar(s));
            }
            if (!failed) f4_commit<CG>(accf_bar(buf));
        }
        if (failed) {
            *abort_flag = 1;
            set_status(status, MNMT_ETIMEOUT);
        }
        pdl_allow_next();
        misc[2] = it;  // k-blocks whose copies this thread saw land
        f4_commit<CG>(done_bar);
    } else if (warp == 1 && lane == 0) {
        pdl_allow_next();  // the leader's trigger decides
    } else if (warp >= 2) {
        // ---- epilogue ----
        constexpr int NB = BN / 64;
        const int ew = warp - 2, q = warp & 3, cw = (BN / 2) * (ew >> 2);
        if (a.gb)  // the bias gradient, always in the same order
            for (long n = (long)blockIdx.x * F4_EPI_WARPS * 32 + ew * 32 + lane; n < a.N; n += (long)gridDim.x * F4_EPI_WARPS * 32) {
                float s = 0.0f;
#pragma unroll 8
                for (int c = 0; c < a.chunks; c++) s = __fadd_rn(s, a.part[(size_t)c * a.N + n]);
                a.gb[n] = s;
            }
        uint8_t *stg = sm + L::OFF_STG + ew * 2 * F4_BLK;
        uint32_t lt = 0, blocks = 0;
        for (long tile = unit; tile < tiles; tile += units, lt++) {
            const int buf = (int)(lt & 1);
            const At t = at(tile);
            const BwProduct &p = a.p[t.p];
            const CUtensorMap *ty = t.p ? &tmY1 : &tmY0;
            const int row0 = t.m + (int)rank * F4_BM + 32 * q, col0 = t.n + cw;
            uint32_t in[NB];
#pragma unroll
            for (int b = 0; b < NB; b++) in[b] = row0 + lane < p.rows && col0 + 32 * b < p.cols ? inside32<NV>(p, row0 + lane, col0 + 32 * b) : 0;
            bool ok = *abort_flag == 0 && mbar_wait(accf_bar(buf), (lt >> 1) & 1);
            if (!ok && *abort_flag == 0) {
                *abort_flag = 1;
                set_status(status, MNMT_ETIMEOUT);
            }
            tc_fence_after();
            ok = __all_sync(0xFFFFFFFFu, ok && *abort_flag == 0);
            const uint32_t taddr = tbase + ((uint32_t)(32 * q) << 16) + (uint32_t)(buf * BN + cw);
            const bool mine = ok && row0 < p.rows;
#pragma unroll
            for (int b = 0; b < NB; b++) {
                float v[32];
                if (mine && col0 + 32 * b < p.cols) {
                    uint32_t r[32];
                    tmem_ld32(taddr + 32 * b, r);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; i++) v[i] = (in[b] >> i) & 1u ? __fmul_rn(__uint_as_float(r[i]), p.out.alpha) : 0.0f;
                }
                if (b == NB - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (CG == 1) mbar_arrive(acce_bar(buf));
                        else t2_arrive_remote(t2_mapa(acce_bar(buf), 0));
                    }
                }
                if (mine && col0 + 32 * b < p.cols) f4_store_block(p.out, ty, stg, blocks, v, row0, col0 + 32 * b, p.rows, p.cols);
            }
        }
        if (lane == 0) t2_store_wait();
    }

    // ---- teardown: every MMA and copy has completed before a CTA ends ----
    __syncthreads();
    if (warp == 0 && lane == 0 && rank == 0 && *abort_flag)
        for (uint32_t it = misc[2]; it < issued; it++) mbar_wait(full_bar((int)(it % STAGES)), (it / STAGES) & 1);
    if (warp == 1) {
        if (lane == 0) mbar_wait(done_bar, 0);
        __syncwarp();
        tc_fence_after();
    }
    if constexpr (CG == 2) asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    if (warp == 1) {
        if constexpr (CG == 1) tmem_free<L::COLS>(tbase);
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tbase), "r"(L::COLS) : "memory");
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
int g_bw_pairs = 0;

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
int up8(int n) { return (n + 7) & ~7; }

bool encode_bf16(CUtensorMap *tm, const void *p, int cols, int rows, long ld, int box_rows) {
    return encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, p, cols, rows, (cuuint64_t)ld * 2, 64, box_rows, CU_TENSOR_MAP_SWIZZLE_128B, true);
}

template <int CG, int BN, bool NV>
cudaError_t bw_init() {
    cudaError_t err = cudaFuncSetAttribute(fp4_backward_gemm<CG, BN, NV>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)BwLayout<CG, BN>::SMEM);
    if (err != cudaSuccess || CG == 1) return err;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = f4_config(CG, 64, BwLayout<CG, BN>::SMEM, nullptr, attr);
    int n = 0;
    err = cudaOccupancyMaxActiveClusters(&n, fp4_backward_gemm<CG, BN, NV>, &cfg);
    if (err == cudaSuccess && (g_bw_pairs == 0 || n < g_bw_pairs)) g_bw_pairs = n;
    return err;
}

template <int CG, int BN, bool NV>
cudaError_t bw_launch(const CUtensorMap (&tm)[6], const BwArgs &a, int *status, cudaStream_t st) {
    long tiles = 0;
    for (int i = 0; i < a.n; i++) tiles += (long)fp4_div_up(a.p[i].rows, CG * F4_BM) * fp4_div_up(a.p[i].cols, BN);
    if (tiles == 0) tiles = 1;  // the bias gradient alone
    const long fit = CG == 2 ? g_bw_pairs : device_sm_count();
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = f4_config(CG, (int)(tiles < fit ? tiles : fit), BwLayout<CG, BN>::SMEM, st, attr);
    return cudaLaunchKernelEx(&cfg, fp4_backward_gemm<CG, BN, NV>, tm[0], tm[1], tm[2], tm[3], tm[4], tm[5], a, status);
}

// scratch: W and X in bf16, a copy of G, partial column sums
struct Scratch {
    size_t w, x, g, part, bytes;
    int pk, pn;
};
Scratch scratch(int M, int N, int K) {
    Scratch s;
    s.pk = up8(K), s.pn = up8(N);
    s.w = 0;
    s.x = up16((size_t)N * s.pk * 2);
    s.g = s.x + up16((size_t)M * s.pk * 2);
    s.part = s.g + up16((size_t)M * s.pn * 2);
    s.bytes = s.part + up16((size_t)fp4_div_up(M, GB_ROWS) * N * 4) + 16;
    return s;
}

}  // namespace

cudaError_t fp4_backward_init() {
    cudaError_t err = bw_init<2, 256, false>();
    if (err == cudaSuccess) err = bw_init<2, 256, true>();
    if (err == cudaSuccess) err = bw_init<1, 64, false>();
    if (err == cudaSuccess) err = bw_init<1, 64, true>();
    return err;
}

size_t fp4_backward_workspace(int M, int N, int K) { return scratch(M, N, K).bytes; }

cudaError_t launch_fp4_linear_backward(const Fp4BackwardArgs &b, cudaStream_t st) {
    const int M = b.x.rows, N = b.w.rows, K = b.x.cols;
    cudaError_t err = cudaSuccess;
    if (M == 0 || N == 0) {  // sums over nothing
        if (b.gx) err = cudaMemset2DAsync(b.gx, (size_t)b.ldgx * (b.xdtype == MNMT_F32 ? 4 : 2), 0, (size_t)K * (b.xdtype == MNMT_F32 ? 4 : 2), M, st);
        if (b.gw && err == cudaSuccess) err = cudaMemset2DAsync(b.gw, (size_t)b.ldgw * 4, 0, (size_t)K * 4, N, st);
        if (b.gb && err == cudaSuccess) err = cudaMemsetAsync(b.gb, 0, (size_t)N * 4, st);
        return err;
    }
    if (!b.gx && !b.gw && !b.gb) return cudaSuccess;
    const Scratch s = scratch(M, N, K);
    uint8_t *ws = static_cast<uint8_t *>(b.workspace);
    const bool products = b.gx || b.gw;
    const bool copy = products && ((reinterpret_cast<uintptr_t>(b.g) & 15) || b.ldg % 8);
    PrepArgs p;
    p.w = b.w, p.x = b.x;
    p.g = static_cast<const __nv_bfloat16 *>(b.g), p.ldg = b.ldg;
    p.w16 = b.gx ? reinterpret_cast<__nv_bfloat16 *>(ws + s.w) : nullptr;
    p.x16 = b.gw ? reinterpret_cast<__nv_bfloat16 *>(ws + s.x) : nullptr;
    p.g16 = copy ? reinterpret_cast<__nv_bfloat16 *>(ws + s.g) : nullptr;
    p.part = b.gb ? reinterpret_cast<float *>(ws + s.part) : nullptr;
    p.M = M, p.N = N, p.K = K, p.pk = s.pk, p.pn = s.pn;
    // blocks in proportion to the bytes each part moves, eight per SM at most
    const long groups = fp4_div_up(K, 32), strips = (long)fp4_div_up(N, 256) * fp4_div_up(M, GB_ROWS), cap = 4L * device_sm_count();
    auto part = [&](long blocks) { return (int)(blocks < cap ? blocks : cap); };
    p.bw = p.w16 ? part((N * groups + 255) / 256) : 0;
    p.bx = p.x16 ? part((M * groups + 255) / 256) : 0;
    const int bg = p.g16 || p.part ? part(strips) : 0;
    launch_pdl(b.nv ? fp4_backward_prepare<true> : fp4_backward_prepare<false>, p.bw + p.bx + bg, 256, 0, st, p);
    if ((err = cudaGetLastError()) != cudaSuccess) return err;

    BwArgs a;
    a.n = 0;
    a.part = p.part, a.gb = b.gb, a.chunks = fp4_div_up(M, GB_ROWS), a.N = N;
    CUtensorMap tm[6];
    memset(tm, 0, sizeof(tm));
    const void *g = copy ? static_cast<const void *>(p.g16) : b.g;
    const long ldg = copy ? s.pn : b.ldg;
    long blocks64 = 0, pairs = 0;
    auto add = [&](bool input) {
        BwProduct &r = a.p[a.n];
        r.rows = input ? M : N, r.cols = K, r.red = input ? N : M, r.a_mn = !input;
        r.out = input ? F4Out{b.gx, b.ldgx, b.xdtype, 0, 0, b.nv ? b.w.g : 1.0f, nullptr} : F4Out{b.gw, b.ldgw, MNMT_F32, 0, 0, b.nv ? b.x.g : 1.0f, nullptr};
        r.orig = input ? b.xo : b.wo, r.ldo = input ? b.ldx : b.ldw, r.otype = input ? b.xdtype : b.wdtype;
        r.q = input ? b.x : b.w;
        CUtensorMap *t = tm + 3 * a.n;
        encode_out(t + 2, r.out, r.rows, r.cols);
        blocks64 += (long)fp4_div_up(r.rows, F4_BM) * fp4_div_up(K, 64);
        pairs += (long)fp4_div_up(r.rows, 2 * F4_BM) * fp4_div_up(K, 256);
        a.n++;
        return encode_bf16(t, g, N, M, ldg, input ? F4_BM : 64) && encode_bf16(t + 1, input ? p.w16 : p.x16, K, input ? N : M, s.pk, 64);
    };
    // the longer reduction first: its tiles take longest
    const bool input_first = N >= M;
    for (int i = 0; i < 2; i++) {
        const bool input = (i == 0) == input_first;
        if ((input ? b.gx != nullptr : b.gw != nullptr) && !add(input)) return cudaErrorInvalidValue;
    }
    if (a.n == 0) a.p[0] = BwProduct{};
    const bool small = blocks64 <= 2L * device_sm_count();
    if (small) return b.nv ? bw_launch<1, 64, true>(tm, a, b.status, st) : bw_launch<1, 64, false>(tm, a, b.status, st);
    return b.nv ? bw_launch<2, 256, true>(tm, a, b.status, st) : bw_launch<2, 256, false>(tm, a, b.status, st);
}

}  // namespace mnmt
