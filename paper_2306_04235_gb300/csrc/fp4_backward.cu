// fp4_backward.cu -- gradients of the linear on microscaled 4-bit floating-point
// operands (include/mnmt.h, mnmt_fp4_linear_backward).
//
//   gX[m][k] = in_x alpha_w sum_n G[m][n] W[n][k]
//   gW[n][k] = in_w alpha_x sum_m G[m][n] X[m][k],   gb[n] = sum_m G[m][n]
// The output gradients stay bf16, so both products run on tcgen05 kind::f16: a
// code times its block scale (a power of two, or an E4M3 number) has at most six
// significant bits and is exact in bf16, products are exact in fp32.
//
// fp4_backward_prepare (memory): W and X decoded to bf16 in their stored order, the
// straight-through masks as bits, a copy of G where TMA cannot read it (rows not
// 16-byte aligned), tickets zeroed.
// fp4_backward_gemm, both products in one persistent launch (tensor cores): the
// reduction index is the row of a stored operand, so the MMAs read W, X and (for
// gW) G "MN-major" from tiles as they lie in memory: no transposed copies.  The
// epilogue warps apply masks and store (masks from the float
// originals there, a row per lane, waited for memory: gX of 16384 x 512 x 2048 130
// us, 65 with bits); two warps sum the bias gradient meanwhile.  16384 x 8192 x 2048:
// 594 us, 1.85 PFLOP/s; with preparation 635, in a row 650 to 700 under the power cap,
// against 565 at the measured rate of bf16 (645 at the sustained one).
// fp4_backward_finish: where the reduction of a product was split (few tiles, long
// sums), adds the parts' sums in their order and applies masks (memory; 512 x 2048 x
// 2048 27 to 30 us in all, 46 x 1024 x 256 9.3 to 9.8: three and two short launches).
#include <type_traits>

#include "fp4.cuh"
#include "fp4_tile.cuh"
#include "train.h"

namespace mnmt {
namespace {

__host__ __device__ constexpr int up32(int n) { return (n + 31) / 32 * 32; }

// what is made of a packed matrix: its values in bf16 (without the tensor scale),
// rows pk apart, and a bit per element, set where the float original lies within
// the range of its block, rows of mp bytes; each may be null
struct PrepMatrix {
    Fp4Args q;
    __nv_bfloat16 *values;
    uint8_t *mask;
    const void *orig;
    long ldo;
    int otype, blocks;
};
struct PrepArgs {
    PrepMatrix m[2];
    const __nv_bfloat16 *g;
    long ldg;
    __nv_bfloat16 *g16;  // may be null
    int *tickets;
    int n_tickets, M, N, pk, mp, pn;
};

// A thread's groups of eight columns, every step-th one of all rows', without
// divisions after the first (with one per group the whole call took 27.9 us at
// 512 x 2048 x 2048, without 27.0).
struct GroupWalk {
    int row, group, groups, dr, dg;
    MNMT_DEV GroupWalk(int first, int step, int n) : groups(n) {
        row = first / n, group = first % n;
        dr = step / n, dg = step % n;
    }
    MNMT_DEV void next() {
        row += dr, group += dg;
        if (group >= groups) group -= groups, row++;
    }
};

template <bool NV, typename T>
MNMT_DEV void prepare_rows(const PrepMatrix &m, int pk, int mp, int block) {
    const int tiles_k = fp4_tiles_k(m.q.cols, NV);
    const size_t pitch = fp4_pitch(m.q.cols);
    const T *orig = static_cast<const T *>(m.orig);
    const bool vec = ((reinterpret_cast<uintptr_t>(orig) | (uintptr_t)m.ldo * sizeof(T)) & 15) == 0;
#pragma unroll 2
    for (GroupWalk w(block * 256 + threadIdx.x, m.blocks * 256, pk / 8); w.row < m.q.rows; w.next()) {
        const int row = w.row, c = 8 * w.group;
        const uint32_t byte = m.q.scales[fp4_scale_at(row, c / fp4_block(NV), tiles_k)];
        if (m.values) {
            const uint32_t codes = *reinterpret_cast<const uint32_t *>(m.q.codes + row * pitch + (c >> 1));
            const float S = fp4_scale_of<NV>(byte, 1.0f).S;
            float v[8];
#pragma unroll
            for (int b = 0; b < 4; b++) {
                const float2 f = fp4_float2((codes >> (8 * b)) & 0xFFu);
                v[2 * b] = __fmul_rn(f.x, S), v[2 * b + 1] = __fmul_rn(f.y, S);
            }
            store8<__nv_bfloat16, true>(m.values + (size_t)row * pk + c, 8, v);
        }
        if (m.mask) {
            const float r = fp4_scale_of<NV>(byte, m.q.g).r;
            const T *src = orig + row * m.ldo + c;
            float v[8];
            if (vec && c + 8 <= m.q.cols) load8<T, true>(src, 8, v);
            else load8<T, false>(src, m.q.cols - c, v);
            uint32_t in = 0;
#pragma unroll
            for (int k = 0; k < 8; k++) in |= (uint32_t)(fabsf(__fmul_rn(v[k], r)) <= 6.0f) << k;
            m.mask[(size_t)row * mp + (c >> 3)] = (uint8_t)in;
        }
    }
}

template <bool NV>
__global__ void __launch_bounds__(256) fp4_backward_prepare(PrepArgs a) {
    pdl_grid_wait();
    pdl_allow_next();  // the products' kernel sets itself up meanwhile
    int block = blockIdx.x;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const PrepMatrix &m = a.m[i];
        if (block < m.blocks) {
            if (m.otype == MNMT_F32) prepare_rows<NV, float>(m, a.pk, a.mp, block);
            else if (m.otype == MNMT_BF16) prepare_rows<NV, __nv_bfloat16>(m, a.pk, a.mp, block);
            else prepare_rows<NV, __half>(m, a.pk, a.mp, block);
            return;
        }
        block -= m.blocks;
    }
    const int first = block * 256 + threadIdx.x, step = ((int)gridDim.x - a.m[0].blocks - a.m[1].blocks) * 256;
    for (int i = first; i < a.n_tickets; i += step) a.tickets[i] = 0;
    if (!a.g16) return;
    for (GroupWalk w(first, step, a.pn / 8); w.row < a.M; w.next()) {
        const long r = w.row;
        const int c = 8 * w.group;
        float v[8];
        load8<__nv_bfloat16, false>(a.g + r * a.ldg + c, a.N - c, v);
        store8<__nv_bfloat16, true>(a.g16 + (size_t)r * a.pn + c, 8, v);
    }
}

// ---------------------------------------------------------------------------
// the two products
// ---------------------------------------------------------------------------
constexpr int BW_BK = 64;  // reduction indices per stage
// The tensor core's fp32 accumulator drops bits at every MMA (its relative error
// grows by about 3e-8 per MMA of 16 terms, always towards zero: 3e-5 measured
// after 16384 terms).  Results are therefore accumulated there over a number of terms
// and added up in registers: fp32 over 1024 (16384 terms: 5e-7 off), 16-bit ones, whose
// rounding is 2^-9 or 2^-12, over 8192 (2^-16).
constexpr int BW_CHUNK = 16, BW_CHUNK16 = 128;  // stages
constexpr int BW_TILE = 12;  // what an item takes beside its stages, in stages
constexpr int BW_EPI_WARPS = 8, BW_GB_WARPS = 2, BW_THREADS = 64 + 32 * (BW_EPI_WARPS + BW_GB_WARPS);
constexpr int GB_COLS = 256, GB_FLIGHT = 16;  // columns of G that a warp sums at a time, rows that it loads at a time
constexpr int GB_JOIN = 512;  // blocks' sums added in fp32, above that in 64 bits (for all: 1 us of every call)

template <int CG, int BN>
struct BwLayout {
    static constexpr uint32_t A_BYTES = F4_BM * BW_BK * 2;
    static constexpr uint32_t B_BYTES = BN / CG * BW_BK * 2;
    static constexpr uint32_t STAGE = A_BYTES + B_BYTES;
    static constexpr uint32_t STG = BW_EPI_WARPS * 4096;  // a warp's two blocks of 2 KB
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
    int chunk;                  // stages per accumulator
    int parts, len;             // parts of the reduction, stages of a part
    F4Out out;                  // parts > 1: fp32 sums [parts][rows][ldy], without masks
    const uint8_t *mask;        // straight-through bits, rows of mp bytes, or null
    int mp;
};
struct BwArgs {
    BwProduct p[2];
    int n;  // products
    // bias gradient: G (readable up to column gcols), partial column sums
    // [blocks of rows][N], done per 256 columns; gb may be null
    const __nv_bfloat16 *g;
    long ldg;
    int gcols, gb_rows;  // rows: that a warp sums at a time
    float *gb, *gb_part;
    int *gb_tickets;
    int M, N;
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

// The bias gradient by warps w of n: gb_rows x 256 columns at a time, eight columns
// per lane; the warp that finishes the last row block of 256 columns adds the
// blocks' sums in their order.  A term passes through at most 512 + 512 additions in
// fp32, whatever M is.
__device__ __noinline__ void bias_gradient(const BwArgs &a, int w, int n) {
    const int lane = threadIdx.x & 31;
    const int strips = fp4_div_up(a.N, GB_COLS), blocks = fp4_div_up(a.M, a.gb_rows);
    const bool vec = (reinterpret_cast<uintptr_t>(a.g) & 15) == 0 && a.ldg % 8 == 0;
    for (long i = w; i < (long)strips * blocks; i += n) {
        const int block = (int)(i / strips), strip = (int)(i - (long)block * strips), c = strip * GB_COLS + 8 * lane;
        const int r0 = block * a.gb_rows, r1 = min(a.M, r0 + a.gb_rows);
        float s[8] = {};
        if (c < a.N) {
            const __nv_bfloat16 *p = a.g + c;
            if (vec && c + 8 <= a.gcols) {
                auto add = [&](int r, int n) {
                    uint4 w[GB_FLIGHT];
#pragma unroll
                    for (int u = 0; u < GB_FLIGHT; u++)
                        w[u] = u < n ? *reinterpret_cast<const uint4 *>(p + (r + u) * a.ldg) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < GB_FLIGHT; u++) {
                        const uint32_t x[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            s[2 * k] = __fadd_rn(s[2 * k], __uint_as_float(x[k] << 16));
                            s[2 * k + 1] = __fadd_rn(s[2 * k + 1], __uint_as_float(x[k] & 0xFFFF0000u));
                        }
                    }
                };
                int r = r0;
                for (; r + GB_FLIGHT <= r1; r += GB_FLIGHT) add(r, GB_FLIGHT);
                if (r < r1) add(r, r1 - r);
            } else {
#pragma unroll 4
                for (int r = r0; r < r1; r++) {
                    float v[8];
                    load8<__nv_bfloat16, false>(p + r * a.ldg, a.N - c, v);
#pragma unroll
                    for (int k = 0; k < 8; k++) s[k] = __fadd_rn(s[k], v[k]);
                }
            }
        }
        if (blocks > 1) {
            float *out = a.gb_part + (size_t)block * strips * GB_COLS + c;
            reinterpret_cast<float4 *>(out)[0] = make_float4(s[0], s[1], s[2], s[3]);
            reinterpret_cast<float4 *>(out)[1] = make_float4(s[4], s[5], s[6], s[7]);
            __threadfence();
            __syncwarp();
            int old = 0;
            if (lane == 0) old = atomicAdd(a.gb_tickets + strip, 1);
            if (__shfl_sync(0xFFFFFFFFu, old, 0) != blocks - 1) continue;
            __threadfence();
            const float4 *in = reinterpret_cast<const float4 *>(a.gb_part + c);
            double sum[8] = {};
            for (int b0 = 0; b0 < blocks; b0 += GB_JOIN) {
                const int b1 = min(blocks, b0 + GB_JOIN);
                float4 lo = make_float4(0.0f, 0.0f, 0.0f, 0.0f), hi = lo;
#pragma unroll 8
                for (int b = b0; b < b1; b++) {
                    const float4 x = __ldcg(in + (size_t)b * strips * (GB_COLS / 4)), y = __ldcg(in + (size_t)b * strips * (GB_COLS / 4) + 1);
                    lo.x = __fadd_rn(lo.x, x.x), lo.y = __fadd_rn(lo.y, x.y), lo.z = __fadd_rn(lo.z, x.z), lo.w = __fadd_rn(lo.w, x.w);
                    hi.x = __fadd_rn(hi.x, y.x), hi.y = __fadd_rn(hi.y, y.y), hi.z = __fadd_rn(hi.z, y.z), hi.w = __fadd_rn(hi.w, y.w);
                }
                s[0] = lo.x, s[1] = lo.y, s[2] = lo.z, s[3] = lo.w, s[4] = hi.x, s[5] = hi.y, s[6] = hi.z, s[7] = hi.w;
                if (blocks <= GB_JOIN) break;
#pragma unroll
                for (int k = 0; k < 8; k++) sum[k] += s[k];
            }
            if (blocks > GB_JOIN)
#pragma unroll
                for (int k = 0; k < 8; k++) s[k] = (float)sum[k];
        }
#pragma unroll
        for (int k = 0; k < 8; k++)
            if (c + k < a.N) a.gb[c + k] = s[k];
    }
}

// Persistent, 384 threads per CTA: warp 0 lane 0 loads tiles by TMA, warp 1 lane
// 0 issues MMAs into two TMEM accumulators, warps 2..9 drain them, warps 10 and
// 11 sum the bias gradient.  An item is a part of a tile.
template <int CG, int BN>
__global__ void __launch_bounds__(BW_THREADS, 1)
    fp4_backward_gemm(const __grid_constant__ CUtensorMap tmA0, const __grid_constant__ CUtensorMap tmB0, const __grid_constant__ CUtensorMap tmY0,
                      const __grid_constant__ CUtensorMap tmA1, const __grid_constant__ CUtensorMap tmB1, const __grid_constant__ CUtensorMap tmY1,
                      const __grid_constant__ BwArgs a, int *status) {
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
    const long n0 = (long)mt(0) * nt(0) * a.p[0].parts, n1 = a.n > 1 ? (long)mt(1) * nt(1) * a.p[1].parts : 0;
    // A unit (CTA or pair) takes every units-th item of product 0; the units that
    // then have one item less take as many more of product 1 as fit that item's
    // time, then all of them take turns.
    const int heavy = (int)(n0 % units);
    const long extra = heavy ? (long)(units - heavy) * ((a.p[0].len + BW_TILE) / (a.p[1].len + BW_TILE)) : 0;
    struct Range {
        long first, step, end;
    };
    auto range = [&](int phase) {
        if (phase == 0) return Range{unit, units, n0};
        if (phase == 1) return Range{unit >= heavy ? unit - heavy : n1, units - heavy, extra < n1 ? extra : n1};
        return Range{extra + (unit >= heavy ? unit - heavy : units - heavy + unit), units, n1};
    };
    // tile, part and corner of an item: the dimension of fewer tiles runs fastest
    struct At {
        int p, m, n, k0, k1;
    };
    auto at = [&](int phase, long item) {
        At r;
        r.p = phase > 0;
        const BwProduct &p = a.p[r.p];
        const long tile = item / p.parts;
        r.k0 = (int)(item - tile * p.parts) * p.len;
        r.k1 = min((p.red + BW_BK - 1) / BW_BK, r.k0 + p.len);
        const int m = mt(r.p), n = nt(r.p);
        r.m = (int)(m <= n ? tile % m : tile / n) * CG * F4_BM;
        r.n = (int)(m <= n ? tile / m : tile % n) * BN;
        return r;
    };

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; s++) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(accf_bar(b), 1);
            mbar_init(acce_bar(b), CG * BW_EPI_WARPS);
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
    pdl_grid_wait();  // nothing before this reads or writes global memory

    uint32_t issued = 0;
    if (warp == 0 && lane == 0) {
        // ---- TMA producer ----
        uint32_t it = 0;
        bool failed = false;
        const uint32_t ring = s_addr(sm);
        for (int phase = 0; phase < 3; phase++) {
            const Range r = range(phase);
            for (long item = r.first; item < r.end && !failed && !*abort_flag; item += r.step) {
                const At t = at(phase, item);
                const CUtensorMap *ta = t.p ? &tmA1 : &tmA0, *tb = t.p ? &tmB1 : &tmB0;
                const int m0 = t.m + (int)rank * F4_BM, n0 = t.n + (int)rank * (BN / CG);
                const bool a_mn = a.p[t.p].a_mn;
                for (int kb = t.k0; kb < t.k1; kb++, it++) {
                    const int s = (int)(it % STAGES);
                    if (it >= STAGES && !f4_wait(empty_bar(s), (it / STAGES - 1) & 1)) {
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
        }
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---- MMA issuer ----
        uint32_t it = 0, lt = 0;  // k-blocks and accumulators so far
        bool failed = false;
        const uint32_t ring = s_addr(sm);
        const uint64_t b_desc = mn128_desc(ring + L::A_BYTES);
        for (int phase = 0; phase < 3; phase++) {
            const Range r = range(phase);
            const bool a_mn = a.p[phase > 0].a_mn;
            const uint64_t a_desc = a_mn ? mn128_desc(ring) : sw128_desc(ring);
            const uint64_t a_step = a_mn ? 2048 >> 4 : 32 >> 4;  // 16 reduction indices
            const uint32_t idesc = bw_idesc(CG * F4_BM, BN, a_mn);
            const int chunk = a.p[phase > 0].chunk;
            for (long item = r.first; item < r.end && !failed; item += r.step) {
                const At t = at(phase, item);
                for (int k0 = t.k0; k0 < t.k1 && !failed; k0 += chunk, lt++) {
                    const int buf = (int)(lt & 1), k1 = min(t.k1, k0 + chunk);
                    if (lt >= 2 && !f4_wait(acce_bar(buf), (lt / 2 - 1) & 1)) {
                        failed = true;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t d = tbase + (uint32_t)(buf * BN);
                    for (int kb = k0; kb < k1; kb++, it++) {
                        const int s = (int)(it % STAGES);
                        if (!f4_wait(full_bar(s), (it / STAGES) & 1)) {
                            failed = true;
                            break;
                        }
                        tc_fence_after();
                        const uint64_t off = (uint64_t)((s * L::STAGE) >> 4);
#pragma unroll
                        for (int k = 0; k < BW_BK / 16; k++) {
                            const uint64_t ad = a_desc + off + a_step * k, bd = b_desc + off + (uint64_t)(k * (2048 >> 4));
                            if constexpr (CG == 1) mma_f16(d, ad, bd, idesc, (uint32_t)((kb - k0) | k));
                            else t2_mma(d, ad, bd, idesc, (uint32_t)((kb - k0) | k));
                        }
                        f4_commit<CG>(empty_bar(s));
                    }
                    if (!failed) f4_commit<CG>(accf_bar(buf));
                }
            }
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
    } else if (warp >= 2 + BW_EPI_WARPS || a.n == 0) {
        const int w = a.n == 0 ? BW_EPI_WARPS + BW_GB_WARPS : BW_GB_WARPS, first = 2 + BW_EPI_WARPS + BW_GB_WARPS - w;
        if (a.gb && warp >= first) bias_gradient(a, (int)blockIdx.x * w + warp - first, (int)gridDim.x * w);
    } else if (warp >= 2) {
        // ---- epilogue ----
        constexpr int NB = BN / 64;
        const int ew = warp - 2, q = warp & 3, cw = (BN / 2) * (ew >> 2);
        uint8_t *stg = sm + L::OFF_STG + ew * 4096;
        uint32_t lt = 0, sent = 0;
        for (int phase = 0; phase < 3; phase++) {
            const Range rg = range(phase);
            const BwProduct &p = a.p[phase > 0];
            if (!p.out.tma) {
                // f4_store_block writes the staging blocks without asking, and stores by TMA
                // of the product before may still be reading them
                if (lane == 0) t2_store_wait_read<0>();
                __syncwarp();
            }
            for (long item = rg.first; item < rg.end; item += rg.step) {
                const At t = at(phase, item);
                const int row0 = t.m + (int)rank * F4_BM + 32 * q, col0 = t.n + cw;
                uint32_t in[NB];
#pragma unroll
                for (int b = 0; b < NB; b++) in[b] = 0xFFFFFFFFu;
                if (p.mask && row0 + lane < p.rows) {
                    const uint8_t *src = p.mask + (size_t)(row0 + lane) * p.mp + (col0 >> 3);
                    if constexpr (NB == 4) {
                        if (col0 < p.cols) {
                            const uint4 w = *reinterpret_cast<const uint4 *>(src);
                            in[0] = w.x, in[1] = w.y, in[2] = w.z, in[3] = w.w;
                        }
                    } else {
#pragma unroll
                        for (int b = 0; b < NB; b++)
                            if (col0 + 32 * b < p.cols) in[b] = reinterpret_cast<const uint32_t *>(src)[b];
                    }
                }
                float acc[NB][32];
#pragma unroll
                for (int b = 0; b < NB; b++)
#pragma unroll
                    for (int i = 0; i < 32; i++) acc[b][i] = 0.0f;
                bool ok = true;
                for (int k0 = t.k0; k0 < t.k1; k0 += p.chunk, lt++) {
                    const int buf = (int)(lt & 1);
                    ok = *abort_flag == 0 && f4_wait(accf_bar(buf), (lt >> 1) & 1);
                    if (!ok && *abort_flag == 0) {
                        *abort_flag = 1;
                        set_status(status, MNMT_ETIMEOUT);
                    }
                    tc_fence_after();
                    ok = __all_sync(0xFFFFFFFFu, ok && *abort_flag == 0);
                    const uint32_t taddr = tbase + ((uint32_t)(32 * q) << 16) + (uint32_t)(buf * BN + cw);
#pragma unroll
                    for (int b = 0; b < NB; b++) {
                        if (!ok || row0 >= p.rows) break;
                        uint32_t r[32];
                        tmem_ld32(taddr + 32 * b, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; i++) acc[b][i] = __fadd_rn(acc[b][i], __uint_as_float(r[i]));
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) f4_release<CG>(acce_bar(buf));
                }
                if (!ok || row0 >= p.rows) continue;
                // parts of a split product: 32 rows and more apart, all by TMA
                const int part0 = p.parts > 1 ? t.k0 / p.len * up32(p.rows) : 0;
#pragma unroll
                for (int b = 0; b < NB; b++) {
                    if (col0 + 32 * b >= p.cols) continue;
#pragma unroll
                    for (int i = 0; i < 32; i++) acc[b][i] = (in[b] >> i) & 1u ? __fmul_rn(acc[b][i], p.out.alpha) : 0.0f;
                    if (p.out.tma) f4_send_block<64, 2>(p.out, phase ? &tmY1 : &tmY0, stg, sent, acc[b], part0 + row0, col0 + 32 * b, p.cols);
                    else f4_store_block<4096, false>(p.out, stg, acc[b], row0, col0 + 32 * b, p.rows, p.cols);
                }
            }
        }
        if (lane == 0) t2_store_wait();
    }

    // ---- teardown: every MMA and copy has completed before a CTA ends ----
    __syncthreads();
    if (warp == 0 && lane == 0 && rank == 0 && *abort_flag)
        for (uint32_t it = misc[2]; it < issued; it++) f4_wait(full_bar((int)(it % STAGES)), (it / STAGES) & 1);
    if (warp == 1) {
        if (lane == 0) f4_wait(done_bar, 0);
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
// the parts of split products
// ---------------------------------------------------------------------------
struct FinishProduct {
    const float *sums;  // [parts][rows in whole 32][ld]
    int parts, rows, cols, ld, blocks;
    F4Out out;
    const uint8_t *mask;
    int mp;
};
struct FinishArgs {
    FinishProduct p[2];
};

// eight columns of a row per thread and step
__global__ void __launch_bounds__(256) fp4_backward_finish(FinishArgs a) {
    pdl_grid_wait();
    const bool second = (int)blockIdx.x >= a.p[0].blocks;
    const FinishProduct &p = a.p[second];
    const long part = (long)up32(p.rows) * p.ld;
    const int first = ((int)blockIdx.x - (second ? a.p[0].blocks : 0)) * 256 + threadIdx.x;
    for (GroupWalk w(first, p.blocks * 256, fp4_div_up(p.cols, 8)); w.row < p.rows; w.next()) {
        const int row = w.row, c = 8 * w.group, n = p.cols - c;
        const float *src = p.sums + (long)row * p.ld + c;
        float s[8] = {};
#pragma unroll 4
        for (int k = 0; k < p.parts; k++) {
            float v[8];
            load8<float, true>(src + k * part, 8, v);  // rows are padded to eight columns
#pragma unroll
            for (int j = 0; j < 8; j++) s[j] = __fadd_rn(s[j], v[j]);
        }
        const uint32_t in = p.mask ? p.mask[(size_t)row * p.mp + (c >> 3)] : 0xFFu;
#pragma unroll
        for (int j = 0; j < 8; j++) s[j] = (in >> j) & 1u ? __fmul_rn(s[j], p.out.alpha) : 0.0f;
        auto put = [&](auto t) {
            using T = decltype(t);
            T *o = static_cast<T *>(p.out.y) + row * p.out.ldy + c;
            if (p.out.al && n >= 8) store8<T, true>(o, 8, s);
            else store8<T, false>(o, n, s);
        };
        if (p.out.type == MNMT_F32) put(float{});
        else if (p.out.type == MNMT_BF16) put(__nv_bfloat16{});
        else put(__half{});
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
int g_bw_pairs = 0;

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
int up8(int n) { return (n + 7) & ~7; }

bool encode_bf16(CUtensorMap *tm, const void *p, int cols, int rows, long ld, int box_rows) {
    return encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, p, cols, rows, (cuuint64_t)ld * 2, 64, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int CG, int BN>
cudaError_t bw_init() {
    cudaError_t err = cudaFuncSetAttribute(fp4_backward_gemm<CG, BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)BwLayout<CG, BN>::SMEM);
    if (err != cudaSuccess || CG == 1) return err;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = f4_config(CG, 64, BW_THREADS, BwLayout<CG, BN>::SMEM, nullptr, attr);
    int n = 0;
    err = cudaOccupancyMaxActiveClusters(&n, fp4_backward_gemm<CG, BN>, &cfg);
    if (err == cudaSuccess && (g_bw_pairs == 0 || n < g_bw_pairs)) g_bw_pairs = n;
    return err;
}

// Tiles and parts of the two products (index 0: gX, 1: gW), by sizes alone (the
// workspace's size is asked for before any device is set up): for 152 SMs.
struct Plan {
    bool pair;
    int units;
    int parts[2], len[2];  // of the reduction; stages of a part
    long tiles[2], items;
};
Plan plan(int M, int N, int K, bool gx, bool gw) {
    Plan best = {};
    const int rows[2] = {M, N}, red[2] = {N, M};
    const bool want[2] = {gx, gw};
    for (int pair = 1; pair >= 0; pair--) {
        Plan p = {};
        p.pair = pair;
        p.units = pair ? 76 : 152;
        const int least = pair ? 8 : 16;  // stages of a part, at least: finishing split sums is one more launch
        double work = 0.0;
        for (int i = 0; i < 2; i++) {
            if (!want[i]) continue;
            p.tiles[i] = (long)fp4_div_up(rows[i], pair ? 2 * F4_BM : F4_BM) * fp4_div_up(K, pair ? 256 : 64);
            work += (double)p.tiles[i] * (fp4_div_up(red[i], BW_BK) + BW_TILE);
        }
        const double share = work / p.units;  // of a unit, in stages
        const bool few = p.tiles[0] + p.tiles[1] < p.units;
        for (int i = 0; i < 2; i++) {
            // a reduction longer than a unit's share is split into parts of about that
            const int nkb = fp4_div_up(red[i], BW_BK);
            const double len = share - BW_TILE > least ? share - BW_TILE : least;
            double parts = want[i] && nkb > len ? nkb / len + (few ? 0.0 : 0.99) : 1.0;
            if (parts > 64.0) parts = 64.0;
            if (p.tiles[i] * parts > p.units) parts = (double)p.units / p.tiles[i];  // no second round of parts
            p.parts[i] = parts < 1.0 ? 1 : (int)parts;
            p.len[i] = fp4_div_up(nkb, p.parts[i]);
            p.parts[i] = fp4_div_up(nkb, p.len[i]);
            p.items += p.tiles[i] * p.parts[i];
        }
        best = p;
        // us, pairs / single CTAs: 512 x 2048 x 2048 (share 26) 29.4 / 27.3, 4096 x 2048 x 512
        // (35) 29.1 / 44.4, 2048^3 (74) 40.5 / 76.9, 46 x 1024 x 256 (1) 14.5 / 9.7
        if (pair && share >= 30) break;
    }
    return best;
}
size_t partial_bytes(const Plan &p, int i, int rows, int K) { return p.parts[i] > 1 ? (size_t)p.parts[i] * up32(rows) * up8(K) * 4 : 0; }

// Rows of G that a warp sums at a time.  It waits for memory once per GB_FLIGHT rows,
// the last warp of 256 columns then once per eight partial sums: about sqrt(2 M)
// rows make that shortest, more where the warps have more to do (two per SM beside the
// products, ten without), at most 512 (sums of fp32).  With 128 rows for all, eight at a time: 1001 x 771 x 389 25.8 us (so: 14.4),
// 16384 x 2048 x 512 83.8 (63.3).
int gb_rows(int M, int N, bool products) {
    if (M <= 64) return 64;  // nothing to join
    const int per = 152 * (BW_GB_WARPS + (products ? 0 : BW_EPI_WARPS)) / fp4_div_up(N, GB_COLS);
    int r = fp4_div_up(fp4_div_up(M, per > 1 ? per : 1), GB_FLIGHT) * GB_FLIGHT;
    while ((long)r * r < 2L * M) r += GB_FLIGHT;
    return r < 512 ? r : 512;
}

// scratch: W and X in bf16, their masks, a copy of G, sums of the bias gradient, of split products, tickets
struct Scratch {
    size_t w, x, mw, mx, g, gb, partial, tickets, bytes;
    int pk, mp, pn, strips;
};
Scratch scratch(int M, int N, int K) {
    Scratch s;
    s.pk = up8(K), s.mp = (int)up16(fp4_div_up(K, 8)), s.pn = up8(N), s.strips = fp4_div_up(N, GB_COLS);
    s.w = 0;
    s.x = up16((size_t)N * s.pk * 2);
    s.mw = s.x + up16((size_t)M * s.pk * 2);
    s.mx = s.mw + (size_t)N * s.mp;
    s.g = s.mx + (size_t)M * s.mp;
    s.gb = s.g + up16((size_t)M * s.pn * 2);
    s.partial = s.gb + (size_t)fp4_div_up(M, gb_rows(M, N, false)) * s.strips * GB_COLS * 4;
    size_t most = 0;
    for (int w = 1; w < 4; w++) {
        const Plan p = plan(M, N, K, w & 1, w & 2);
        const size_t n = partial_bytes(p, 0, M, K) + partial_bytes(p, 1, N, K);
        if (n > most) most = n;
    }
    s.tickets = s.partial + most;
    s.bytes = s.tickets + up16((size_t)s.strips * 4) + 16;
    return s;
}

template <int CG, int BN>
cudaError_t bw_launch(const CUtensorMap (&tm)[6], const BwArgs &a, long items, int *status, cudaStream_t st) {
    const long fit = CG == 2 ? g_bw_pairs : device_sm_count();
    // the bias gradient's warps take the whole GPU where the products do not
    const long gb = a.gb ? (long)fp4_div_up(a.N, GB_COLS) * fp4_div_up(a.M, a.gb_rows) / (CG * BW_GB_WARPS) : 0;
    if (items < gb) items = gb;
    if (items < 1) items = 1;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = f4_config(CG, (int)(items < fit ? items : fit), BW_THREADS, BwLayout<CG, BN>::SMEM, st, attr);
    return cudaLaunchKernelEx(&cfg, fp4_backward_gemm<CG, BN>, tm[0], tm[1], tm[2], tm[3], tm[4], tm[5], a, status);
}

}  // namespace

cudaError_t fp4_backward_init() {
    cudaError_t err = bw_init<2, 256>();
    if (err == cudaSuccess) err = bw_init<1, 64>();
    return err;
}

size_t fp4_backward_workspace(int M, int N, int K) {
    // sums over nothing use none and have no plan; the call still wants a buffer
    return M == 0 || N == 0 ? 16 : scratch(M, N, K).bytes;
}

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
    const Plan pl = plan(M, N, K, b.gx, b.gw);
    uint8_t *ws = static_cast<uint8_t *>(b.workspace);
    int *tickets = reinterpret_cast<int *>(ws + s.tickets);
    const bool products = b.gx || b.gw;
    const bool copy = products && ((reinterpret_cast<uintptr_t>(b.g) & 15) || b.ldg % 8);
    PrepArgs p;
    memset(&p, 0, sizeof(p));
    p.m[0].q = b.w, p.m[1].q = b.x;
    if (b.gx) p.m[0].values = reinterpret_cast<__nv_bfloat16 *>(ws + s.w);
    if (b.gw) p.m[1].values = reinterpret_cast<__nv_bfloat16 *>(ws + s.x);
    if (b.gw && b.wo) p.m[0].mask = ws + s.mw, p.m[0].orig = b.wo, p.m[0].ldo = b.ldw, p.m[0].otype = b.wdtype;
    if (b.gx && b.xo) p.m[1].mask = ws + s.mx, p.m[1].orig = b.xo, p.m[1].ldo = b.ldx, p.m[1].otype = b.xdtype;
    p.g = static_cast<const __nv_bfloat16 *>(b.g), p.ldg = b.ldg;
    p.g16 = copy ? reinterpret_cast<__nv_bfloat16 *>(ws + s.g) : nullptr;
    p.tickets = tickets, p.n_tickets = s.strips;
    p.M = M, p.N = N, p.pk = s.pk, p.mp = s.mp, p.pn = s.pn;
    const long cap = 8L * device_sm_count();
    auto blocks = [&](long threads) { return (int)((threads + 255) / 256 < cap ? (threads + 255) / 256 : cap); };
    for (PrepMatrix &m : p.m) m.blocks = m.values || m.mask ? blocks((long)m.q.rows * s.pk / 8) : 0;
    const int rest = copy ? blocks((long)M * s.pn / 8) : 1;
    launch_pdl(b.nv ? fp4_backward_prepare<true> : fp4_backward_prepare<false>, p.m[0].blocks + p.m[1].blocks + rest, 256, 0, st, p);
    if ((err = cudaGetLastError()) != cudaSuccess) return err;

    BwArgs a;
    memset(&a, 0, sizeof(a));
    a.M = M, a.N = N;
    a.g = copy ? p.g16 : p.g, a.ldg = copy ? s.pn : b.ldg, a.gcols = copy ? s.pn : N, a.gb_rows = gb_rows(M, N, products);
    a.gb = b.gb, a.gb_part = reinterpret_cast<float *>(ws + s.gb), a.gb_tickets = tickets;
    a.p[0].parts = a.p[1].parts = 1;
    CUtensorMap tm[6];
    memset(tm, 0, sizeof(tm));
    FinishArgs f;
    memset(&f, 0, sizeof(f));
    int split = 0;
    uint8_t *partial = ws + s.partial;
    // the longer part first
    const bool input_first = pl.len[0] >= pl.len[1];
    for (int i = 0; i < 2; i++) {
        const bool input = (i == 0) == input_first;
        if (input ? !b.gx : !b.gw) continue;
        BwProduct &r = a.p[a.n];
        CUtensorMap *t = tm + 3 * a.n;
        a.n++;
        r.rows = input ? M : N, r.cols = K, r.red = input ? N : M, r.a_mn = !input;
        r.out = input ? F4Out{b.gx, b.ldgx, b.xdtype, 0, 0, 0, b.nv ? b.w.g : 1.0f, nullptr} : F4Out{b.gw, b.ldgw, MNMT_F32, 0, 0, 0, b.nv ? b.x.g : 1.0f, nullptr};
        r.out.al = out_alignment(r.out.y, r.out.ldy, r.out.type);
        r.mask = p.m[input].mask, r.mp = s.mp;
        r.parts = pl.parts[!input], r.len = pl.len[!input];
        if (r.parts > 1) {
            FinishProduct &q = f.p[split++];
            q.sums = reinterpret_cast<const float *>(partial);
            q.parts = r.parts, q.rows = r.rows, q.cols = K, q.ld = s.pk;
            q.out = r.out, q.mask = r.mask, q.mp = s.mp;
            const long n = ((long)r.rows * fp4_div_up(K, 8) + 255) / 256, most = 8L * device_sm_count();
            q.blocks = (int)(n < most ? n : most);
            r.out = F4Out{partial, s.pk, MNMT_F32, out_alignment(partial, s.pk, MNMT_F32), 0, 0, 1.0f, nullptr};
            r.mask = nullptr;
            partial += partial_bytes(pl, !input, r.rows, K);
        }
        r.chunk = r.out.type == MNMT_F32 ? BW_CHUNK : BW_CHUNK16;
        const int width = r.parts > 1 ? s.pk : K;
        r.out.tma = tma_output(r.out, width);
        if (r.out.tma && !encode_out<64>(t + 2, r.out, r.parts > 1 ? r.parts * up32(r.rows) : r.rows, width)) return cudaErrorInvalidValue;
        if (!encode_bf16(t, a.g, N, M, a.ldg, input ? F4_BM : 64) || !encode_bf16(t + 1, p.m[!input].values, K, input ? N : M, s.pk, 64))
            return cudaErrorInvalidValue;
    }

    err = pl.pair ? bw_launch<2, 256>(tm, a, pl.items, b.status, st) : bw_launch<1, 64>(tm, a, pl.items, b.status, st);
    if (err != cudaSuccess || !split) return err;
    launch_pdl(fp4_backward_finish, f.p[0].blocks + f.p[1].blocks, 256, 0, st, f);
    return cudaGetLastError();
}

}  // namespace mnmt
