// fp4_tc.cu -- product of two microscaled 4-bit floating-point matrices on the
// fifth-generation tensor cores (mnmt_fp4_linear):
//   y[m][n] = act(alpha sum_k X[m][k] W[n][k] + bias[n]).
//
// tcgen05.mma kind::mxf4 / mxf4nvf4 multiplies packed E2M1 codes and applies the
// block scales itself: 64 codes of K per instruction, scales in TMEM, sums in
// fp32.  So the kernel moves the codes as they are stored (128-byte-swizzled TMA
// tiles of 256 codes) and the scales as they are stored: a 512-byte tile of 128
// rows x 4 blocks goes to four TMEM columns with one tcgen05.cp.
//
// Persistent, 10 to 18 warps per CTA:
//   warp 0          TMA producer: codes and scales of a k-block of 256 into a ring;
//   warp 1          copies a k-block's scales to TMEM (copies and MMAs of one issuer
//                   run in the order of issue; two sets of columns by turns all the
//                   same, so that no copy touches what the k-block before it reads:
//                   waiting for those MMAs instead costs 8192^3 192 us), issues its
//                   four MMAs, frees the slot;
//   the others      drain a finished accumulator (TMEM holds two; long sums take
//                   several), apply alpha, bias and ReLU, round, and store by TMA or
//                   from registers.
// CG = 2: a pair of CTAs computes 256 x 192 tiles, each CTA half of the rows of
// both operands; CG = 1: 128 x 128 or 128 x 64 tiles for smaller grids.
// Measured to bf16, back to back: 8192^3 MX 152 us (7.2 PFLOP/s), NV 173; 16384 x 8192 x
// 2048 MX 93 us (5.9), NV 104 (after a flush of L2 160, 177, 98, 110).  With K of 2048 a
// tile's drain stands against eight k-blocks only (tensor pipe active 59 %); small grids
// are bound by their start.
// Every wait is bounded; one that runs out records MNMT_ETIMEOUT in *status, and
// the CTA stops issuing work, waits (bounded) for what it has in flight, frees
// its TMEM and returns.
#include <type_traits>

#include "fp4.cuh"
#include "fp4_tile.cuh"
#include "mbarrier.cuh"
#include "routes.h"
#include "tcgen05.cuh"
#include "train.h"

namespace mnmt {
namespace {

constexpr int F4_BK = 256;  // codes per k-block: 128 bytes
// The tensor core's fp32 accumulator truncates at every MMA of 64 terms (NV, terms of one
// sign: 6e-8 of the sum lost after 4096 terms, 5.5e-7 after 8192, 2.5e-6 after 16384,
// 8.6e-5 after 262144).  fp32 results therefore leave it every 8192 terms and are added
// up in registers, 16-bit ones, whose rounding is 2^-9 or 2^-12, every 65536 (2e-5).
// (Every 4096 took 8192^3 to fp32 from 173 us to 182, 2100 x 8192 x 8192 from 59 to 65.)
constexpr int F4_CHUNK = 32, F4_CHUNK16 = 256;  // k-blocks

template <int CG, int BN, bool NV>
struct F4Layout {
    static constexpr int T = NV ? 4 : 2;                // scale tiles along a k-block
    static constexpr int R = BN > 128 ? 2 : 1;          // row tiles of W's scales that a tile touches
    static constexpr uint32_t A_BYTES = F4_BM * 128;
    static constexpr uint32_t B_BYTES = BN / CG * 128;
    static constexpr uint32_t OFF_SFA = A_BYTES + B_BYTES, OFF_SFB = OFF_SFA + T * 512;
    static constexpr uint32_t STAGE = OFF_SFB + R * T * 512;
    static constexpr int EPI = BN == 192 ? 12 : BN / 8, CW = 4 * BN / EPI;  // epilogue warps, columns of each (its 32 rows)
    static constexpr int THREADS = 64 + 32 * EPI;
    static constexpr uint32_t BLK = CG == 1 ? 4096 : 2048;  // a warp's staging block
    static constexpr uint32_t OFF_AFTER = EPI * (BLK + CW * 4) + 512;  // staging, bias, barriers
    static constexpr int FIT = (int)((227 * 1024 - 1024 - OFF_AFTER) / STAGE);
    static constexpr int STAGES = FIT > 8 ? 8 : FIT;
    static constexpr uint32_t OFF_STG = STAGES * STAGE;
    static constexpr uint32_t OFF_COLS = OFF_STG + EPI * BLK;  // [EPI][CW] fp32
    static constexpr uint32_t OFF_BARS = OFF_COLS + EPI * CW * 4;
    static constexpr int NBARS = 2 * STAGES + 5;  // full, empty, acc_full[2], acc_empty[2], done
    static constexpr uint32_t OFF_MISC = OFF_BARS + NBARS * 8;
    static constexpr size_t SMEM = 1024 + OFF_MISC + 16;
    static constexpr int COL_SFA = 2 * BN, COL_SFB = COL_SFA + 4 * T, SF = 4 * T + 4 * R * T;  // TMEM columns; two sets of scales
    static constexpr int COLS = COL_SFA + 2 * SF <= 256 ? 256 : 512;
    static_assert(COL_SFA + 2 * SF <= 512, "TMEM holds 512 columns");
    static_assert(STAGE % 1024 == 0, "swizzled tiles start on 1024 bytes");
    static_assert(OFF_MISC + 16 - OFF_STG <= OFF_AFTER, "barriers fit");
};

// instruction descriptor of the block-scaled kinds: E2M1 operands, both K-major,
// scales UE8M0 or UE4M3, K = 64; id: which bytes of a scale word apply
__host__ __device__ constexpr uint32_t f4_idesc(int m, int n, bool nv, int id) {
    return ((uint32_t)id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((nv ? 0u : 1u) << 23) | ((uint32_t)(m >> 7) << 27) |
           ((uint32_t)id << 29);
}

// a 512-byte scale tile: no swizzle, 8-row groups of 128 bytes
__device__ __forceinline__ uint64_t f4_scale_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)8 << 16) | ((uint64_t)8 << 32) | ((uint64_t)1 << 46);
}

template <int CG, bool NV>
__device__ __forceinline__ void f4_mma_on(uint32_t on, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                          uint32_t accumulate) {
#define F4_MMA(G, KIND)                                                                                            \
    asm volatile(                                                                                                  \
        "{\n\t.reg .pred p, q;\n\t"                                                                                \
        "setp.ne.b32 p, %4, 0;\n\t"                                                                                \
        "setp.ne.b32 q, %7, 0;\n\t"                                                                                \
        "@q tcgen05.mma.cta_group::" G ".kind::" KIND " [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::"r"(d),           \
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb), "r"(on)                                   \
        : "memory")
    if constexpr (CG == 1 && NV) F4_MMA("1", "mxf4nvf4.block_scale.scale_vec::4X");
    else if constexpr (CG == 1) F4_MMA("1", "mxf4.block_scale.scale_vec::2X");
    else if constexpr (NV) F4_MMA("2", "mxf4nvf4.block_scale.scale_vec::4X");
    else F4_MMA("2", "mxf4.block_scale.scale_vec::2X");
#undef F4_MMA
}

// scale tile -> four TMEM columns, repeated in the four lane quarters (of both CTAs of a pair)
template <int CG>
__device__ __forceinline__ void f4_copy_scales_on(uint32_t on, uint32_t taddr, uint64_t desc) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr),
                     "l"(desc), "r"(on)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr),
                     "l"(desc), "r"(on)
                     : "memory");
}

// how a tile is stored, F4_BY_TMA where f4_launch says so, else from registers;
// pairs know it when they are compiled (for the registers: 16384 x 8192 x 2048
// back to back 92.5 us, 94.8 with both)
enum { F4_EITHER, F4_BY_TMA, F4_BY_LANES };

// LONG: a sum takes several accumulators, chunk k-blocks each (compiled apart: pairs have
// no registers left for it)
template <int CG, int BN, bool NV, int ST, bool LONG>
__global__ void __launch_bounds__((F4Layout<CG, BN, NV>::THREADS), 1)
    fp4_gemm(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmSA,
             const __grid_constant__ CUtensorMap tmSB, const __grid_constant__ CUtensorMap tmY, F4Out o, int M, int N, int K, int chunk, int *status) {
    using L = F4Layout<CG, BN, NV>;
    constexpr int STAGES = L::STAGES, T = L::T, R = L::R;

    extern __shared__ uint8_t f4_raw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(f4_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t bars = s_addr(sm + L::OFF_BARS);
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
    auto accf_bar = [&](int b) { return bars + 8u * (2 * STAGES + b); };
    auto acce_bar = [&](int b) { return bars + 8u * (2 * STAGES + 2 + b); };
    const uint32_t done_bar = bars + 8u * (2 * STAGES + 4);
    uint32_t *misc = reinterpret_cast<uint32_t *>(sm + L::OFF_MISC);  // [0] tmem base, [1] abort, [2] consumed
    volatile uint32_t *abort_flag = misc + 1;

    const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    uint32_t rank = 0;
    if constexpr (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int unit = (int)blockIdx.x / CG, units = (int)gridDim.x / CG;
    const int mt = (M + CG * F4_BM - 1) / (CG * F4_BM), nt = (N + BN - 1) / BN;
    const int steps = (K + 63) / 64, full = steps / 4, nkb = (K + F4_BK - 1) / F4_BK, tiles_k = fp4_tiles_k(K, NV);

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; s++) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; b++) {
            mbar_init(accf_bar(b), 1);
            mbar_init(acce_bar(b), CG * L::EPI);
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
    // barriers and accumulators are set up, in both CTAs of a pair
    if constexpr (CG == 2) asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = misc[0];
    pdl_grid_wait();  // nothing before this reads or writes global memory

    uint32_t issued = 0;
    if (warp == 0) {
        // ---- TMA producer: this CTA's rows of all its tiles ----
        const uint32_t on = elect_one();
        uint32_t s = 0, phase = 1;  // slot, and the parity its release completes
        bool failed = false;
        const uint32_t ring = s_addr(sm), lead = CG == 1 ? bars : t2_mapa(bars, 0);
        for (F4Walk w(mt, nt, unit, units); w.more() && !failed && !*abort_flag; w.next()) {
            const int m0 = w.m() * CG * F4_BM + (int)rank * F4_BM, nb = w.n() * BN, n0 = nb + (int)rank * (BN / CG);
            // scale tiles of the rows' tile rows (tiles past the row's end belong
            // to k-steps that are not issued)
            int sa = (m0 >> 7) * tiles_k, sb = (nb >> 7) * tiles_k;
            for (int kb = 0; kb < nkb; kb++) {
                if (!f4_wait(empty_bar(s), phase)) {  // a fresh barrier passes
                    *abort_flag = 1;
                    set_status(status, MNMT_ETIMEOUT);
                    failed = true;
                    break;
                }
                // the leader's barrier takes the bytes of both CTAs of a pair
                expect_tx_on(on && rank == 0, full_bar(s), CG * L::STAGE);
                const uint32_t bar = lead + 8u * s, base = ring + s * L::STAGE;
                f4_load_on<CG>(on, base, &tmA, kb * 128, m0, bar);
                f4_load_on<CG>(on, base + L::A_BYTES, &tmB, kb * 128, n0, bar);
                f4_load_on<CG>(on, base + L::OFF_SFA, &tmSA, 0, sa, bar);
#pragma unroll
                for (int r = 0; r < R; r++) f4_load_on<CG>(on, base + L::OFF_SFB + r * T * 512, &tmSB, 0, sb + r * tiles_k, bar);
                sa += T, sb += T;
                issued++;
                if (++s == STAGES) s = 0, phase ^= 1;
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ---- scales to TMEM and MMAs ----
        const uint32_t on = elect_one();
        uint32_t s = 0, phase = 0, lt = 0, seen = 0;
        bool failed = false;
        const uint32_t ring = s_addr(sm);
        const uint64_t a_desc = sw128_desc(ring), b_desc = sw128_desc(ring + L::A_BYTES);
        const uint64_t sa_desc = f4_scale_desc(ring + L::OFF_SFA), sb_desc = f4_scale_desc(ring + L::OFF_SFB);
        // Through a shuffle: every lane has the same value, and says so.  (Operands that
        // the compiler cannot see to be uniform, or a test per MMA for the last k-block,
        // cost more than the MMA: 8192^3 191 -> 157 us.)
        const uint32_t base = __shfl_sync(0xFFFFFFFFu, tbase, 0), sfa = base + L::COL_SFA, cfb = base + L::COL_SFB;
        for (F4Walk w(mt, nt, unit, units); w.more() && !failed; w.next()) {
            // scale columns of the tile's first row of W: every other tile of 64 or 192 columns
            // starts in the middle of a row tile, two columns on
            const uint32_t sfb = __shfl_sync(0xFFFFFFFFu, cfb + ((uint32_t)(w.n() * BN & 127) >> 5), 0);
            int k0 = 0;
            do {
                const uint32_t buf = lt & 1, d = base + buf * BN;
                const int k1 = LONG ? min(nkb, k0 + chunk) : nkb;
                if (lt >= 2 && !f4_wait(acce_bar(buf), (lt / 2 - 1) & 1)) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                for (int kb = k0; kb < k1; kb++) {
                    if (!f4_wait(full_bar(s), phase)) {
                        failed = true;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t off = (uint64_t)((s * L::STAGE) >> 4);
                    const uint32_t set = (seen & 1) * L::SF;
#pragma unroll
                    for (int t = 0; t < T; t++) {
                        f4_copy_scales_on<CG>(on, sfa + set + 4 * t, sa_desc + off + (uint64_t)(t * 32));
#pragma unroll
                        for (int r = 0; r < R; r++) f4_copy_scales_on<CG>(on, cfb + set + 4 * (R * t + r), sb_desc + off + (uint64_t)((r * T + t) * 32));
                    }
                    auto mma = [&](int k) {
                        const int t = NV ? k : k >> 1, id = NV ? 0 : 2 * (k & 1);
                        f4_mma_on<CG, NV>(on, d, a_desc + off + (uint64_t)(2 * k), b_desc + off + (uint64_t)(2 * k), f4_idesc(CG * F4_BM, BN, NV, id),
                                          sfa + set + 4 * t, sfb + set + 4 * R * t, (uint32_t)((kb - k0) | k));
                    };
                    if (kb < full) {
                        mma(0), mma(1), mma(2), mma(3);
                    } else {
                        mma(0);
                        if (steps - 4 * kb > 1) mma(1);
                        if (steps - 4 * kb > 2) mma(2);
                    }
                    f4_commit_on<CG>(on, empty_bar(s));
                    seen++;
                    if (++s == STAGES) s = 0, phase ^= 1;
                }
                if (!failed) f4_commit_on<CG>(on, accf_bar(buf));
                k0 = k1, lt++;
            } while (LONG && k0 < nkb && !failed);
        }
        if (failed) {
            *abort_flag = 1;
            set_status(status, MNMT_ETIMEOUT);
        }
        pdl_allow_next();  // every MMA of this CTA (pair) is issued
        misc[2] = seen;    // k-blocks whose copies this warp saw land
        f4_commit_on<CG>(on, done_bar);
    } else if (warp == 1) {
        pdl_allow_next();  // the leader's trigger decides
    } else if (warp >= 2) {
        // ---- epilogue: warp ew takes 32 of this CTA's rows, CW columns of the tile ----
        constexpr int CW = L::CW, NB = CW / 32;
        const int ew = warp - 2, q = warp & 3, cw = CW * (ew >> 2);
        uint8_t *stg = sm + L::OFF_STG + ew * L::BLK;
        float *bias = reinterpret_cast<float *>(sm + L::OFF_COLS) + ew * CW;
        const unsigned long long alpha = f4_two(o.alpha, o.alpha);
        uint32_t lt = 0, sent = 0;
        float next[NB];  // a lane's bias columns of the tile to come
        F4Walk w(mt, nt, unit, units);
        auto fetch_bias = [&]() {
#pragma unroll
            for (int b = 0; b < NB; b++) {
                const int n = w.n() * BN + cw + 32 * b + lane;
                next[b] = o.bias && w.more() && n < N ? o.bias[n] : 0.0f;
            }
        };
        fetch_bias();
        while (w.more()) {
            const int row0 = w.m() * CG * F4_BM + (int)rank * F4_BM + 32 * q, col0 = w.n() * BN + cw;
            __syncwarp();
#pragma unroll
            for (int b = 0; b < NB; b++) bias[32 * b + lane] = next[b];
            w.next();
            fetch_bias();
            bool ok;
            uint32_t r[NB][32];
            int k0 = 0;
            do {
                const int buf = (int)(lt & 1);
                ok = *abort_flag == 0 && f4_wait(accf_bar(buf), (lt >> 1) & 1);
                if (!ok && *abort_flag == 0) {
                    *abort_flag = 1;
                    set_status(status, MNMT_ETIMEOUT);
                }
                tc_fence_after();
                ok = __all_sync(0xFFFFFFFFu, ok && *abort_flag == 0);
                const uint32_t taddr = tbase + ((uint32_t)(32 * q) << 16) + (uint32_t)(buf * BN + cw);
                if (!LONG || k0 == 0) {
#pragma unroll
                    for (int b = 0; b < NB; b++) tmem_ld32(taddr + 32 * b, r[b]);
                    tmem_wait_ld();
                } else {
#pragma unroll
                    for (int b = 0; b < 2 * NB; b++) {
                        uint32_t more[16];
                        tmem_ld16(taddr + 16 * b, more);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; i++) {
                            uint32_t &sum = r[b >> 1][16 * (b & 1) + i];
                            sum = __float_as_uint(__fadd_rn(__uint_as_float(sum), __uint_as_float(more[i])));
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) f4_release<CG>(acce_bar(buf));  // this warp is done with the accumulator buffer
                k0 += chunk, lt++;
            } while (LONG && k0 < nkb);
            if (!ok || row0 >= M) continue;
#pragma unroll
            for (int b = 0; b < NB; b++) {
                if (col0 + 32 * b >= N) break;
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 c = *reinterpret_cast<const float4 *>(bias + 32 * b + i);
                    unsigned long long x = f4_two(__uint_as_float(r[b][i]), __uint_as_float(r[b][i + 1]));
                    unsigned long long y = f4_two(__uint_as_float(r[b][i + 2]), __uint_as_float(r[b][i + 3]));
                    if (NV) x = f4_mul2(x, alpha), y = f4_mul2(y, alpha);
                    f4_untwo(f4_add2(x, f4_two(c.x, c.y)), v[i], v[i + 1]);
                    f4_untwo(f4_add2(y, f4_two(c.z, c.w)), v[i + 2], v[i + 3]);
                }
                if (o.relu)
#pragma unroll
                    for (int i = 0; i < 32; i++) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(v[i]));
                const int col = col0 + 32 * b;
                if (ST == F4_BY_TMA || (ST == F4_EITHER && o.tma)) f4_send_block<L::BLK / 32, 1>(o, &tmY, stg, sent, v, row0, col, N);
                else if (ST == F4_BY_LANES && o.al && col + 32 <= N) f4_store_rows(o, v, row0, col, M);
                else f4_store_block<L::BLK, CG == 2>(o, stg, v, row0, col, M, N);
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
// host side
// ---------------------------------------------------------------------------
int g_f4_pairs = 0;  // CTA pairs that fit at once

bool encode_codes(CUtensorMap *tm, const Fp4Args &q, int box_rows) {
    const size_t pitch = fp4_pitch(q.cols);
    return encode(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, q.codes, pitch, q.rows, pitch, 128, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}
// the scale tiles as a matrix of 128 words each
bool encode_scales(CUtensorMap *tm, const Fp4Args &q, bool nv) {
    const size_t n = fp4_scale_bytes(q.rows, q.cols, nv) / 512;
    return encode(tm, CU_TENSOR_MAP_DATA_TYPE_UINT32, q.scales, 128, n, 512, 128, nv ? 4 : 2, CU_TENSOR_MAP_SWIZZLE_NONE);
}

template <int CG, int BN, bool NV, int ST = F4_EITHER, bool LONG = false>
cudaError_t f4_init() {
    cudaError_t err = cudaFuncSetAttribute(fp4_gemm<CG, BN, NV, ST, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)F4Layout<CG, BN, NV>::SMEM);
    if (err != cudaSuccess || CG == 1) return err;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = f4_config(CG, 64, F4Layout<CG, BN, NV>::THREADS, F4Layout<CG, BN, NV>::SMEM, nullptr, attr);
    int n = 0;
    err = cudaOccupancyMaxActiveClusters(&n, fp4_gemm<CG, BN, NV, ST, LONG>, &cfg);
    if (err == cudaSuccess && (g_f4_pairs == 0 || n < g_f4_pairs)) g_f4_pairs = n;
    return err;
}

template <int CG, int BN, bool NV>
cudaError_t f4_launch(const Fp4Args &x, const Fp4Args &w, const F4Out &out, int *status, cudaStream_t st) {
    const int M = x.rows, N = w.rows, K = x.cols;
    CUtensorMap ta, tb, tsa, tsb, ty;
    if (!encode_codes(&ta, x, F4_BM) || !encode_codes(&tb, w, BN / CG) || !encode_scales(&tsa, x, NV) || !encode_scales(&tsb, w, NV))
        return cudaErrorInvalidValue;
    // Stores by TMA: a store of 32 bytes per lane takes 61 passes through the L1 data
    // pipe, which bounds small tiles (us, from registers / TMA: 512 x 32000 x 512 to
    // fp32 19.3 / 15.0; pairs, 16384 x 8192, K = 256 76 / 52, 2048 101 / 95), but pairs
    // of long K are bound by the MMAs (8192^3 152 / 155, to fp32 164 / 176).
    F4Out o = out;
    o.tma = tma_output(o, N) && (CG == 1 || K <= 4096);
    ty = ta;
    if (o.tma && !encode_out<F4Layout<CG, BN, NV>::BLK / 32>(&ty, o, M, N)) return cudaErrorInvalidValue;
    const long tiles = (long)((M + CG * F4_BM - 1) / (CG * F4_BM)) * ((N + BN - 1) / BN);
    const long fit = CG == 2 ? g_f4_pairs : device_sm_count();
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = f4_config(CG, (int)(tiles < fit ? tiles : fit), F4Layout<CG, BN, NV>::THREADS, F4Layout<CG, BN, NV>::SMEM, st, attr);
    const int chunk = o.type == MNMT_F32 ? F4_CHUNK : F4_CHUNK16;
    const bool more = K > chunk * F4_BK;
    auto launch = [&](auto st_kind, auto is_long) {
        return cudaLaunchKernelEx(&cfg, fp4_gemm<CG, BN, NV, decltype(st_kind)::value, decltype(is_long)::value>, ta, tb, tsa, tsb, ty, o, M, N, K, chunk, status);
    };
    using Either = std::integral_constant<int, F4_EITHER>;
    using Lanes = std::integral_constant<int, F4_BY_LANES>;
    if constexpr (CG == 1) return more ? launch(Either{}, std::true_type{}) : launch(Either{}, std::false_type{});
    else if (o.tma) return launch(std::integral_constant<int, F4_BY_TMA>{}, std::false_type{});  // K <= 4096
    else return more ? launch(Lanes{}, std::true_type{}) : launch(Lanes{}, std::false_type{});
}

}  // namespace

template <bool NV>
static cudaError_t init_all() {
    cudaError_t err = f4_init<2, 192, NV, F4_BY_TMA>();
    if (err == cudaSuccess) err = f4_init<2, 192, NV, F4_BY_LANES>();
    if (err == cudaSuccess) err = f4_init<2, 192, NV, F4_BY_LANES, true>();
    if (err == cudaSuccess) err = f4_init<1, 128, NV>();
    if (err == cudaSuccess) err = f4_init<1, 128, NV, F4_EITHER, true>();
    if (err == cudaSuccess) err = f4_init<1, 64, NV>();
    if (err == cudaSuccess) err = f4_init<1, 64, NV, F4_EITHER, true>();
    return err;
}
cudaError_t fp4_init() {
    const cudaError_t err = init_all<false>();
    return err == cudaSuccess ? init_all<true>() : err;
}

cudaError_t launch_fp4_product(const Fp4Args &x, const Fp4Args &w, bool nv, float alpha, const float *bias, int relu, void *y, int ydtype,
                               long ldy, int *status, cudaStream_t st) {
    const F4Out o{y, ldy, ydtype, out_alignment(y, ldy, ydtype), 0, relu, alpha, bias};
    auto go = [&](auto n) {
        constexpr bool NV = decltype(n)::value;
        switch (route_fp4_tiles(x.rows, w.rows, x.cols, device_sm_count())) {
            case FP4_64: return f4_launch<1, 64, NV>(x, w, o, status, st);
            case FP4_128: return f4_launch<1, 128, NV>(x, w, o, status, st);
            default: return f4_launch<2, 192, NV>(x, w, o, status, st);
        }
    };
    return nv ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace mnmt
