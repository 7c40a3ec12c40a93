// seq_attn_backward.cu -- gradients of attention over sequences (seq_attn.cuh), in two
// kernels, each of which computes the scores again and adds up in TMEM, in a fixed order:
//   dq:      128 query rows of a head walk the keys that they see:
//            S = Q K^T, dP = G V^T, dS = P (dP - D), dQ += dS K; D = sum g o on the way in
//   dk, dv:  128 key rows of a key head walk the queries that see them, head by head:
//            S^T = K Q^T, dP^T = V G^T, dV += P^T G, dK += dS^T Q
// (seven products instead of the five of one kernel that adds to dQ from everywhere,
// whose sums would depend on the order of arrival).
// One CTA per SM (tiles of 128 walked rows) or two (heads up to 64, tiles of 64: sentences, which share tiles, leave less of
// them empty, 67 -> 48 us for the batch below), eight warps of two threads per row.  P and dS go to TMEM in the
// operands' type, as the A operand of the second products.  While the threads work on
// one of S and dP the tensor core is on the products that follow the other:
//   dk, dv:  dV(j), S(j+1) once P(j) is written, dK(j), dP(j+1) once dS(j) is
//   dq:      S(j+1), dP(j+1) once S(j), dP(j) are in registers, dQ(j) once dS(j) is written
// Where tiles of keys are few and their walks long (shared key heads), a cluster of up to
// eight CTAs divides a walk's steps and adds up its sums through distributed shared memory.
// fp16 holds little below 2^-14, so P and dS go to TMEM times powers of two, which their exponents take in and results
// lose again: P of dv 2^15; dS in dq, per row, and in dk, per walk, as the largest |g| that it meets comes to 16..32 if it is smaller (where
// |dP| then reaches 65504, sums are infinite and are computed again).  Unscaled, 2048 keys with g of 1e-3 left dq of heads of 64 off by
// 2.7e-3 of its norm, 5.1e-4 so (its own rounding 4.7e-4).
// A walk goes backwards from the last row that is seen, as in the forward pass, and rows
// whose result is not finite are computed again over their own queries or keys alone.
//
// Bound by: long walks, the tensor core, fed in turns with the threads (8192 rows of 16 heads of 128 on 4 key heads, not
// causal 1190 to 1210 us: 1.14 PFLOP/s of the formula's five products, 1.59 of the seven; pipe active 53 % in dq, 69 % in dk, dv,
// 4096 causal rows); sentences, a chain of latencies in front of 2 to 3 tiles a CTA (128 x 20..128 rows of 8 heads
// of 64, causal 39.6 us for 11 us of bytes; several heads a CTA, one after another, as the forward pass takes them, measured the
// same: the CTA beside it fills the starts as well).
#include "seq_tile.cuh"

namespace mnmt {
namespace {

constexpr int BW_THREADS = 320;  // eight warps on the elements, a TMA warp, an MMA warp

__device__ __forceinline__ void elements_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// A thread's W / 2 columns (of a row's W) from TMEM
template <int W>
__device__ __forceinline__ void load_half(uint32_t taddr, uint32_t (&r)[W / 64][32]) {
#pragma unroll
    for (int b = 0; b < W / 64; b++) tmem_ld32(taddr + 32 * b, r[b]);
    tmem_wait_ld();
}

// Columns c0 .. c1 - 1 of a row's sums of all CTAs of a cluster, added in the order of the CTAs, times f and
// stored to row o; at: this CTA's sums of the row.  live: 0 for a row that has none.  Whether one is not finite.
template <bool BF>
__device__ __forceinline__ bool sq_join(uint32_t at, int c0, int c1, int ctas, float live, float f, bool in, void *o, int dh) {
    bool odd = false;
#pragma unroll 2
    for (int col = c0; col < c1; col += 8) {
        float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int r = 0; r < ctas; r++) {
            const uint32_t from = t2_mapa(at + (col / 4) * (SQ_ROWS * 16), r);
            const float4 y = sq_remote(from), z = sq_remote(from + SQ_ROWS * 16);
            v[0] += y.x, v[1] += y.y, v[2] += y.z, v[3] += y.w, v[4] += z.x, v[5] += z.y, v[6] += z.z, v[7] += z.w;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (live == 0.0f) v[i] = 0.0f;
            odd |= !(fabsf(v[i]) < INFINITY);
            v[i] *= f;
        }
        if (in) sq_store<BF>(o, col, dh, v);
    }
    return odd;
}

// sum of eight products of 16-bit elements
template <typename T>
__device__ __forceinline__ float dot8(const uint4 &x, const uint4 &y) {
    const uint32_t a[4] = {x.x, x.y, x.z, x.w}, b[4] = {y.x, y.y, y.z, y.w};
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (std::is_same_v<T, __half>) {
            const float2 u = __half22float2(*reinterpret_cast<const __half2 *>(&a[i])), v = __half22float2(*reinterpret_cast<const __half2 *>(&b[i]));
            s = fmaf(u.x, v.x, fmaf(u.y, v.y, s));
        } else {
            s = fmaf(__uint_as_float(a[i] << 16), __uint_as_float(b[i] << 16),
                     fmaf(__uint_as_float(a[i] & 0xFFFF0000u), __uint_as_float(b[i] & 0xFFFF0000u), s));
        }
    }
    return s;
}

// log2 of the power that takes a largest |g| of `top` to 16..32 (larger ones, 0 and what is not finite: as it is; a power below 1 would
// take small dS to steps above 2^-24)
__device__ __forceinline__ int gain_of(float top) { return top > 0.0f ? max(0, 4 - ((int)(__float_as_uint(top) >> 23) - 127)) : 0; }
constexpr int GAIN_ROWS = 32;      // query rows of a largest |g| that the dq kernel leaves
constexpr float P_GAIN = 15.0f;    // log2 of the power of P in dk, dv
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 .. 127

// --------------------------------------------------------------------------- dq
template <int DH, int W>
struct DqLayout {
    // a stage of K more than of V: it is held until dQ of its tile, and its successor needs a microsecond to come
    // (two stages: the MMA warp waited 1300 cycles a tile for K)
    static constexpr int VS = DH == 64 ? 3 : 2, KS = VS + 1, QT = sq_bytes<DH>(), TILE = sq_bytes<DH, W>();
    static constexpr int OFF_G = QT, OFF_K = 2 * QT, OFF_V = OFF_K + KS * TILE, SMEM = OFF_V + VS * TILE + 1024;
    static_assert((KS + VS) * TILE >= 4 * SQ_INTS, "starts and lengths before keys and values");
    // columns of dP, dS, what it was rounded by, and dQ behind S
    static constexpr int T_DP = W, T_DS = 2 * W, T_DL = T_DS + W / 2, T_DQ = T_DL + W / 2, COLS = pow2_cols(T_DQ + DH);
};

// Rows of `again`, a lane's row each, computed again over their own keys; columns c0 .. c1 - 1 are stored
template <typename T>
__device__ __noinline__ void dq_again(const SeqAttn &a, uint32_t again, int row, int h, Span keys, float lse2, float D, float f, float c, int c0, int c1) {
    const int lane = threadIdx.x & 31, hk = h / a.group();
    for (; again; again &= again - 1) {
        const int src = __ffs(again) - 1, rr = __shfl_sync(0xFFFFFFFFu, row, src);
        const Span sp{__shfl_sync(0xFFFFFFFFu, keys.lo, src), __shfl_sync(0xFFFFFFFFu, keys.hi, src)};
        const float4 d = attn_row_dq(static_cast<const T *>(a.q.p) + rr * a.q.ld + h * a.q.hd, static_cast<const T *>(a.g.p) + rr * a.g.ld + h * a.g.hd,
                                     __shfl_sync(0xFFFFFFFFu, lse2, src), __shfl_sync(0xFFFFFFFFu, D, src), static_cast<const T *>(a.k.p) + hk * a.k.hd,
                                     a.k.ld, static_cast<const T *>(a.v.p) + hk * a.v.hd, a.v.ld, sp, a.dh, c);
        const float fs = __shfl_sync(0xFFFFFFFFu, f, src), v[4] = {d.x * fs, d.y * fs, d.z * fs, d.w * fs};
        if (4 * lane >= c0 && 4 * lane < c1 && 4 * lane < a.dh) store4(static_cast<T *>(a.dq.p) + rr * a.dq.ld + h * a.dq.hd + 4 * lane, v);
    }
}

// The first walk, for rows of sequences of few keys, over n tiles: the sum of dS with D from the rounded o; lo .. hi - 1: the
// row's keys as seen from a thread's columns of the first tile (none: hi <= lo).  16 columns at a time in a loop that stays one:
// its code lies between the start and the walk of every CTA, and four times as much of it cost those without such rows 1 %.
struct FirstWalk {
    float rest;
    bool ok;
};
template <int W>
__device__ __forceinline__ FirstWalk dq_first_walk(const SqWaits &wait, uint32_t sp_full, uint32_t sp_free, uint32_t scores, uint32_t weights, int lo, int hi,
                                                   int n, float c, float lse2, float D) {
    const unsigned long long c2 = f4_two(c, c), l2 = f4_two(-lse2, -lse2), d2 = f4_two(-D, -D);
    unsigned long long rest = f4_two(0.0f, 0.0f);
    for (int j = 0; j < n; j++, lo += W, hi += W) {
        if (!wait(sp_full, (uint32_t)j & 1)) return FirstWalk{0.0f, false};
        tc_fence_after();
        if (__any_sync(0xFFFFFFFFu, hi > 0 && lo < W / 2 && lo < hi)) {
#pragma unroll 1
            for (int b = 0; b < W / 2; b += 16) {
                uint32_t s[16], p[16];
                tmem_ld16(scores + b, s);
                tmem_ld16(weights + b, p);
                tmem_wait_ld();
                const uint32_t see = sq_bits(lo - b, hi - b);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    float x, y, u, v;
                    f4_untwo(sq_fma2(f4_two(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c2, l2), x, y);
                    const unsigned long long t = f4_add2(f4_two(__uint_as_float(p[2 * i]), __uint_as_float(p[2 * i + 1])), d2);
                    f4_untwo(f4_mul2(f4_two(exp2_fast(x), exp2_fast(y)), t), u, v);
                    rest = f4_add2(rest, f4_two((see >> (2 * i)) & 1u ? u : 0.0f, (see >> (2 * i + 1)) & 1u ? v : 0.0f));
                }
            }
        }
        tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(sp_free);
    }
    float ra, rb;
    f4_untwo(rest, ra, rb);
    return FirstWalk{ra + rb, true};
}

template <int DH, bool BF, int W>
__global__ void __launch_bounds__(BW_THREADS, 512 / DqLayout<DH, W>::COLS) seq_attn_dq_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tg,
                                                                    const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                                                                    const __grid_constant__ SeqAttn a, const float c, float *delta, float *tops, const int ctas) {
    using L = DqLayout<DH, W>;
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    // With bf16 and heads up to 64 dS goes in two parts, rounded and what that left, as the tensor core has room there (12 %
    // busy with sentences), and dk and dv take a D that the rows' sums correct: on the batch of sentences gradients were off by up to
    // 2.6e-3 of their norm, 2.4e-3 so (1.7e-3 is the results' own rounding), for 2 of 40 us.
    constexpr bool FINE = BF && DH == 64;
    constexpr int KS = L::KS, VS = L::VS;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[2 * KS + 2 * VS + 6];
    __shared__ uint32_t tslot;
    __shared__ int failed, span[4][4];
    __shared__ float dots[SQ_ROWS];
    __shared__ uint16_t g_top[BF ? 1 : SQ_ROWS];  // largest |g| of a row
    __shared__ uint8_t odd_rows[2][SQ_ROWS];
    const uint32_t sm = (s_addr(raw) + 1023u) & ~1023u, bar0 = s_addr(bars);
    uint8_t *smp = raw + (sm - s_addr(raw));
    const auto k_full = [&](int s) { return bar0 + 8 * s; };
    const auto k_free = [&](int s) { return bar0 + 8 * (KS + s); };
    const auto v_full = [&](int s) { return bar0 + 8 * (2 * KS + s); };
    const auto v_free = [&](int s) { return bar0 + 8 * (2 * KS + VS + s); };
    const uint32_t q_full = bar0 + 8 * (2 * KS + 2 * VS), sp_full = q_full + 8, sp_free = q_full + 16, ds_full = q_full + 24, ds_free = q_full + 32,
                   dq_full = q_full + 40;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int share = (int)blockIdx.x % ctas, unit = (int)blockIdx.x / ctas, h = unit % a.hq, hk = h / a.group();
    const int tile = (int)gridDim.x / ctas / a.hq - 1 - unit / a.hq;
    const int half = warp >> 2, rt = (int)threadIdx.x & 127, row = tile * SQ_ROWS + rt;
    if (threadIdx.x == 0) {
        for (int s = 0; s < KS; s++) mbar_init(k_full(s), 1), mbar_init(k_free(s), 1);
        for (int s = 0; s < VS; s++) mbar_init(v_full(s), 1), mbar_init(v_free(s), 1);
        mbar_init(q_full, 2), mbar_init(sp_full, 1), mbar_init(sp_free, 8), mbar_init(ds_full, 8), mbar_init(ds_free, 1), mbar_init(dq_full, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) tmem_alloc<L::COLS>(s_addr(&tslot));
    pdl_grid_wait();
    // D of the tile's rows, 16 a warp, DH / 8 lanes a row; the loads are in flight while the starts come
    constexpr int PC = DH / 8, NR = 16 * PC / 32;  // 16-byte pieces of a row, rows of a lane
    uint4 ov[NR], gv[NR];
    if (warp < 8) {
        const int c = 8 * (lane % PC);
#pragma unroll
        for (int i = 0; i < NR; i++) {
            const int r = tile * SQ_ROWS + 16 * warp + i * (32 / PC) + lane / PC;
            const bool on = r < a.q_rows && c < a.dh;
            ov[i] = on ? *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.o.p) + r * a.o.ld + h * a.o.hd + c) : make_uint4(0, 0, 0, 0);
            gv[i] = on ? *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.g.p) + r * a.g.ld + h * a.g.hd + c) : make_uint4(0, 0, 0, 0);
        }
    }
    const SeqAttn ix = seq_shared(a, reinterpret_cast<int *>(smp + L::OFF_K), BW_THREADS);  // where keys and values come later
    Span keys{0, 0};
    bool in = false, few = false;
    if (warp < 8) {
        keys = keys_of_lane(ix, row - lane, in, few);
        const bool some = keys.hi > keys.lo;
        few &= some;
        const int lo = __reduce_min_sync(0xFFFFFFFFu, some ? keys.lo : 0x7FFFFFFF), hi = __reduce_max_sync(0xFFFFFFFFu, some ? keys.hi : 0);
        const int few_lo = __reduce_min_sync(0xFFFFFFFFu, few ? keys.lo : 0x7FFFFFFF), few_hi = __reduce_max_sync(0xFFFFFFFFu, few ? keys.hi : 0);
        if (lane == 0 && half == 0) span[0][warp] = lo, span[1][warp] = hi, span[2][warp] = few_lo, span[3][warp] = few_hi;
#pragma unroll
        for (int i = 0; i < NR; i++) {
            float dot = dot8<T>(ov[i], gv[i]);
#pragma unroll
            for (int o = PC / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
            if (lane % PC == 0) dots[16 * warp + i * (32 / PC) + lane / PC] = dot;
            if constexpr (!BF) {
                const auto abs2 = [](uint32_t x) { return __habs2(*reinterpret_cast<const __half2 *>(&x)); };
                __half2 t = __hmax2(__hmax2(abs2(gv[i].x), abs2(gv[i].y)), __hmax2(abs2(gv[i].z), abs2(gv[i].w)));
#pragma unroll
                for (int o = PC / 2; o > 0; o >>= 1) t = __hmax2(t, __shfl_xor_sync(0xFFFFFFFFu, t, o));
                if (lane % PC == 0) g_top[16 * warp + i * (32 / PC) + lane / PC] = __half_as_ushort(__hmax(__low2half(t), __high2half(t)));
            }
        }
    }
    sq_before_copies();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tS = tslot, tP = tS + L::T_DP, tD = tS + L::T_DS, tL = tS + L::T_DL, tO = tS + L::T_DQ;
    const int first = min(min(span[0][0], span[0][1]), min(span[0][2], span[0][3])), end = max(max(span[1][0], span[1][1]), max(span[1][2], span[1][3]));
    // this CTA's tiles, nt of them from t0 on
    const int all_t = end > first ? (end - first + W - 1) / W : 0, t0 = (int)((long)all_t * share / ctas), nt = (int)((long)all_t * (share + 1) / ctas) - t0;
    // Where a sequence's rows see few keys (10 on average or fewer), D from the rounded o is off by what weighs most in dq and dk
    // (sequences of 2 or 3: 3.7e-3 of dq's norm, 1.7e-3 its own rounding; of 10: 2.4e-3; of 40: 2.0e-3).  The tiles that hold
    // such rows' keys, n1 of them from f0 on, are walked before the others for the sum of dS, which is zero but for that; where a
    // cluster shares the rows, by each of its CTAs.  (Up to 16 keys: 128 x 20..128 causal rows of 8 heads of 64 40.8 us, so 39.1.)
    const int few_lo = min(min(span[2][0], span[2][1]), min(span[2][2], span[2][3])), few_hi = max(max(span[3][0], span[3][1]), max(span[3][2], span[3][3]));
    const int f0 = (end - few_hi) / W, n1 = few_hi > few_lo ? (end - few_lo - 1) / W - f0 + 1 : 0, n = n1 + nt;  // steps of both walks
    const SqWaits wait{&failed, a.status};

    if (warp == 8) {
        if (lane == 0 && n) {
            sq_load<DH>(sm, &tq, h, tile * SQ_ROWS, q_full);
            sq_load<DH>(sm + L::OFF_G, &tg, h, tile * SQ_ROWS, q_full);
            int jk = 0, jv = 0;  // loads issued
            const auto at = [&](int j) { return end - W * ((j < n1 ? f0 + j : t0 + j - n1) + 1); };  // rows of step j's tile
            // K(0), then V(j) and K(j + KS - VS) by turns: each waits for what the tensor core is done with first
            for (; jv < n; jv++) {
                if (jv >= VS && !wait.one(v_free(jv % VS), (uint32_t)(jv / VS - 1) & 1)) break;
                for (; jk <= jv; jk++) sq_load<DH, W>(sm + L::OFF_K + jk % KS * L::TILE, &tk, hk, at(jk), k_full(jk % KS));  // the first
                sq_load<DH, W>(sm + L::OFF_V + jv % VS * L::TILE, &tv, hk, at(jv), v_full(jv % VS));
                for (; jk < n && jk <= jv + KS - VS; jk++) {
                    if (jk >= KS && !wait.one(k_free(jk % KS), (uint32_t)(jk / KS - 1) & 1)) break;
                    sq_load<DH, W>(sm + L::OFF_K + jk % KS * L::TILE, &tk, hk, at(jk), k_full(jk % KS));
                }
                if (failed) {
                    jv++;
                    break;
                }
            }
            if (failed) {  // copies in flight land before the block ends
                wait.one(q_full, 0);
                for (int i = max(0, jk - KS); i < jk; i++) wait.one(k_full(i % KS), (uint32_t)(i / KS) & 1);
                for (int i = max(0, jv - VS); i < jv; i++) wait.one(v_full(i % VS), (uint32_t)(i / VS) & 1);
            }
        }
    } else if (warp == 9) {
        if (n) {
            const uint32_t on = elect_one();
            const uint64_t qd = sq_k(sm), gd = sq_k(sm + L::OFF_G), kd = sq_k(sm + L::OFF_K), vd = sq_k(sm + L::OFF_V), kt = sq_mn<W>(sm + L::OFF_K);
            bool ok = wait(q_full, 0);
            for (int j = 0; j <= n && ok; j++) {
                if (j < n) {  // S(j), dP(j)
                    const int s = j % KS, sv = j % VS;
                    const uint64_t koff = (uint64_t)(s * (L::TILE >> 4)), voff = (uint64_t)(sv * (L::TILE >> 4));
                    if (j && !(ok = wait(sp_free, (uint32_t)(j - 1) & 1))) break;
                    if (!(ok = wait(k_full(s), (uint32_t)(j / KS) & 1))) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < DH / 16; k++) sq_mma(on, tS, qd + sq_k_step(k), kd + koff + sq_k_step<W>(k), sq_idesc(W, BF, false), k > 0);
                    if (!(ok = wait(v_full(sv), (uint32_t)(j / VS) & 1))) break;
                    tc_fence_after();
#pragma unroll
                    for (int k = 0; k < DH / 16; k++) sq_mma(on, tP, gd + sq_k_step(k), vd + voff + sq_k_step<W>(k), sq_idesc(W, BF, false), k > 0);
                    f4_commit_on<1>(on, v_free(sv));
                    f4_commit_on<1>(on, sp_full);
                    if (j < n1) f4_commit_on<1>(on, k_free(s));
                }
                if (j > n1) {  // dQ(j - 1)
                    const int i = j - 1 - n1, s = (j - 1) % KS;
                    if (!(ok = wait(ds_full, (uint32_t)i & 1))) break;
                    tc_fence_after();
                    const uint64_t b = kt + (uint64_t)(s * (L::TILE >> 4));
#pragma unroll
                    for (int k = 0; k < W / 16; k++) sq_mma_ta(on, tO, tD + 8 * k, b + sq_mn_step(k), sq_idesc(DH, BF, true), (uint32_t)(i | k));
                    if constexpr (FINE) {
#pragma unroll
                        for (int k = 0; k < W / 16; k++) sq_mma_ta(on, tO, tL + 8 * k, b + sq_mn_step(k), sq_idesc(DH, BF, true), 1);
                    }
                    f4_commit_on<1>(on, k_free(s));
                    f4_commit_on<1>(on, ds_free);
                }
            }
            f4_commit_on<1>(on, dq_full);
            wait(dq_full, 0);
        }
        pdl_allow_next();
    } else {
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const bool none = keys.hi <= keys.lo;
        float D = dots[rt];
        bool ok = true;
        if (n1) {
            const int at = end - W * (f0 + 1) + W / 2 * half;
            const FirstWalk x = dq_first_walk<W>(wait, sp_full, sp_free, tS + lanes + W / 2 * half, tP + lanes + W / 2 * half, few ? keys.lo - at : 0,
                                                 few ? keys.hi - at : 0, n1, c, none ? 0.0f : a.lse[(long)h * a.q_rows + row] * LOG2E, D);
            ok = x.ok;
            // a row's two halves (every warp comes here, whether its waits were in vain or not)
            elements_sync();
            if (half) dots[rt] = x.rest;
            elements_sync();
            if (!half) dots[rt] = D + (x.rest + dots[rt]);
            elements_sync();
            D = dots[rt];
        }
        const long at_row = (long)h * a.q_rows + row;
        if (!FINE && in && half == 0 && share == 0) delta[at_row] = D;
        int gain = 0;  // log2 of what dS is multiplied by
        if constexpr (!BF) {
            const float top = __half2float(__ushort_as_half(g_top[rt]));
            gain = gain_of(top);
            if (half == 0 && share == 0) {
                const uint32_t most = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(in && !none && top < INFINITY ? top : 0.0f));
                if (lane == 0 && row < a.q_rows) tops[(long)h * ((a.q_rows + GAIN_ROWS - 1) / GAIN_ROWS) + row / GAIN_ROWS] = __uint_as_float(most);
            }
        }
        unsigned long long rest = f4_two(0.0f, 0.0f);  // sum of dS
        const float lse2 = none ? 0.0f : a.lse[at_row] * LOG2E;
        const float l = (float)gain - lse2;
        const unsigned long long c2 = f4_two(c, c), l2 = f4_two(l, l), d2 = f4_two(-D, -D);
        for (int j = 0; j < nt && ok; j++) {
            if (!(ok = wait(sp_full, (uint32_t)(n1 + j) & 1))) break;
            tc_fence_after();
            const int at = end - W * (t0 + j + 1) + W / 2 * half, lo = keys.lo - at, hi = keys.hi - at;
            const bool all = __all_sync(0xFFFFFFFFu, lo <= 0 && hi >= W / 2), some = __any_sync(0xFFFFFFFFu, hi > 0 && lo < W / 2);
            // (a value where there is none to read, or the registers count as used from one turn of the loop to the next:
            // up to 160 bytes of spills, 8 so; 3 x 2500..4095 rows of 16 heads of 128 400 us, 387 at the time)
            uint32_t s[W / 64][32] = {}, p[W / 64][32] = {};
            if (some) {
#pragma unroll
                for (int b = 0; b < W / 64; b++) {
                    tmem_ld32(tS + lanes + W / 2 * half + 32 * b, s[b]);
                    tmem_ld32(tP + lanes + W / 2 * half + 32 * b, p[b]);
                }
                tmem_wait_ld();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(sp_free);
            if (j && !(ok = wait(ds_free, (uint32_t)(j - 1) & 1))) break;
            // dS of the 32 b columns: without the masks where the warp's rows see all of them
            const auto ds = [&](auto whole) {
#pragma unroll
                for (int b = 0; b < W / 64; b++) {
                    const uint32_t see = sq_bits(lo - 32 * b, hi - 32 * b);
#pragma unroll
                    for (int i0 = 0; i0 < 16; i0 += 8) {
                        uint32_t w[8];
                        [[maybe_unused]] uint32_t wl[8];
#pragma unroll
                        for (int k = 0; k < 8; k++) {
                            const int i = i0 + k;
                            float x, y, u, v;
                            f4_untwo(sq_fma2(f4_two(__uint_as_float(s[b][2 * i]), __uint_as_float(s[b][2 * i + 1])), c2, l2), x, y);
                            const unsigned long long t = f4_add2(f4_two(__uint_as_float(p[b][2 * i]), __uint_as_float(p[b][2 * i + 1])), d2);
                            f4_untwo(f4_mul2(f4_two(exp2_fast(x), exp2_fast(y)), t), u, v);
                            if (!decltype(whole)::value) u = (see >> (2 * i)) & 1u ? u : 0.0f, v = (see >> (2 * i + 1)) & 1u ? v : 0.0f;
                            w[k] = sq_pack<BF>(u, v);
                            if constexpr (FINE) {
                                rest = f4_add2(rest, f4_two(u, v));
                                wl[k] = sq_pack<BF>(u - __uint_as_float(w[k] << 16), v - __uint_as_float(w[k] & 0xFFFF0000u));
                            }
                        }
                        tmem_st8(tD + lanes + W / 4 * half + 16 * b + i0, w);
                        if constexpr (FINE) tmem_st8(tL + lanes + W / 4 * half + 16 * b + i0, wl);
                    }
                }
            };
            if (all) {
                ds(std::true_type{});
            } else if (some) {
                ds(std::false_type{});
            } else {
                const uint32_t zeros[16] = {};
#pragma unroll
                for (int b = 0; b < W / 64; b++) {
                    tmem_st16(tD + lanes + W / 4 * half + 16 * b, zeros);
                    if constexpr (FINE) tmem_st16(tL + lanes + W / 4 * half + 16 * b, zeros);
                }
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full);
        }
        if (n) ok = wait(dq_full, 0) && ok;
        tc_fence_after();
        float *rests = reinterpret_cast<float *>(smp + L::OFF_K);  // where keys were, of a row's two halves
        if (FINE) {
            // A row's dS add up to zero but for what D is off by (o is rounded): D + that is what dk and dv take.  (Where a
            // cluster shares the row, its CTAs' sums are added below.)
            float ra, rb;
            f4_untwo(rest, ra, rb);
            elements_sync();
            if (ctas > 1) rests[2 * rt + half] = ra + rb;
            else if (half) dots[rt] = ra + rb;
            elements_sync();
            if (ctas == 1 && in && half == 0) delta[at_row] = none ? D : D + (ra + rb + dots[rt]);
        }
        // a query's only key has the weight 1 and dS = 0, where dP - D would leave what their two sums are rounded by (0, not
        // nothing: what is not a number stays so)
        const float f = keys.hi - keys.lo == 1 ? 0.0f : a.scale, fo = BF ? f : f * pow2(-gain);
        bool odd = false;
        int c0 = 0, c1 = DH;  // the columns that this CTA stores
        if (ctas == 1 && ok) {
            uint32_t out[DH / 4];
#pragma unroll
            for (int b = 0; b < DH / 64; b++) {
                uint32_t w[32] = {};
                if (nt) tmem_ld32(tO + lanes + half * (DH / 2) + 32 * b, w);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const float x = nt && !none ? __uint_as_float(w[2 * i]) : 0.0f, y = nt && !none ? __uint_as_float(w[2 * i + 1]) : 0.0f;
                    odd |= !(fabsf(x) < INFINITY) || !(fabsf(y) < INFINITY);
                    out[16 * b + i] = sq_pack<BF>(x * fo, y * fo);
                }
            }
            // the queries have been multiplied: their rows are free
            sq_store_rows<DH / 2>(smp + warp * (32 * DH), out, static_cast<uint16_t *>(a.dq.p) + (long)(row - lane) * a.dq.ld + h * a.dq.hd + half * (DH / 2),
                                  a.dq.ld, __ballot_sync(0xFFFFFFFFu, in), a.dh - half * (DH / 2));
        } else if (ctas > 1) {
            // sums of this CTA's tiles to shared memory, where queries and gradients were: four columns of a row side by side
            float4 *sums = reinterpret_cast<float4 *>(smp) + rt, *mine = sums + half * (DH / 8) * SQ_ROWS;
#pragma unroll
            for (int b = 0; b < DH / 64; b++) {
                uint32_t w[32] = {};
                if (nt) tmem_ld32(tO + lanes + half * (DH / 2) + 32 * b, w);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; i++)
                    mine[(8 * b + i) * SQ_ROWS] = nt ? make_float4(__uint_as_float(w[4 * i]), __uint_as_float(w[4 * i + 1]), __uint_as_float(w[4 * i + 2]),
                                                                  __uint_as_float(w[4 * i + 3]))
                                                    : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            __syncwarp();
            sq_cluster_sync();
            if (FINE && share == 0 && half == 0) {
                float r = 0.0f;
                for (int i = 0; i < ctas; i++) {
                    const float2 x = sq_remote2(t2_mapa(s_addr(rests + 2 * rt), i));
                    r += x.x + x.y;
                }
                if (in) delta[at_row] = none ? D : D + r;
            }
            // every CTA of the cluster adds up a share of the columns, in the order of the CTAs
            c0 = DH / ctas * share, c1 = c0 + DH / ctas;
            if (ok && half == 0)
                odd = sq_join<BF>(s_addr(sums), c0, c1, ctas, none ? 0.0f : 1.0f, fo, in, static_cast<T *>(a.dq.p) + row * a.dq.ld + h * a.dq.hd, a.dh);
        }
        odd_rows[half][rt] = odd;
        elements_sync();
        odd = ok && in && (odd_rows[0][rt] || odd_rows[1][rt]);
        // the rows of a warp and its partner by turns
        const uint32_t again = __ballot_sync(0xFFFFFFFFu, odd && (rt & 1) == half);
        if (again) dq_again<T>(a, again, row, h, keys, lse2, D, f, c, c0, c1);
    }
    if (ctas > 1) {
        __syncwarp();
        if (warp >= 8) sq_cluster_sync();
        sq_cluster_sync();  // no CTA leaves while others read its sums
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) tmem_free<L::COLS>(tslot);
}

// --------------------------------------------------------------------------- dk, dv
template <int DH, int W>
struct DkvLayout {
    // a stage of Q more than of G: it is held until dK of its tile, which comes last
    static constexpr int GS = DH == 64 ? 3 : 2, QS = GS + 1, KT = sq_bytes<DH>(), TILE = sq_bytes<DH, W>(), NUM = 8 * W;
    // K and V, stages of Q and G, two of -lse log2 e and -D of W queries, barriers and the rest (no room for more with heads of 128)
    static constexpr int OFF_V = KT, OFF_Q = 2 * KT, OFF_G = OFF_Q + QS * TILE, OFF_N = OFF_G + GS * TILE, OFF_R = OFF_N + 2 * NUM;
    static constexpr int SMEM = OFF_R + 8 * (2 * QS + 2 * GS + 10) + 48 + 2 * SQ_ROWS;
    static_assert((QS + GS) * TILE >= 4 * SQ_INTS, "starts and lengths before queries");
    static constexpr int T_DP = W, T_DV = 2 * W, T_DK = 2 * W + DH, COLS = pow2_cols(2 * W + 2 * DH);
    static_assert(OFF_N >= 2 * SQ_ROWS * DH * 4, "a CTA's sums for its cluster");
};

// As dq_again, dk and dv over the queries of all heads of key head hk
template <typename T>
__device__ __noinline__ void dkv_again(const SeqAttn &a, uint32_t again, int row, int hk, Span qs, float fk, float c, const float *delta, int c0, int c1) {
    const int lane = threadIdx.x & 31;
    for (; again; again &= again - 1) {
        const int src = __ffs(again) - 1, rr = __shfl_sync(0xFFFFFFFFu, row, src);
        const Span sp{__shfl_sync(0xFFFFFFFFu, qs.lo, src), __shfl_sync(0xFFFFFFFFu, qs.hi, src)};
        float dk[4] = {0.0f, 0.0f, 0.0f, 0.0f}, dv[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int h = hk * a.group(); h < (hk + 1) * a.group(); h++)
            attn_row_dkv(static_cast<const T *>(a.k.p) + rr * a.k.ld + hk * a.k.hd, static_cast<const T *>(a.v.p) + rr * a.v.ld + hk * a.v.hd,
                         static_cast<const T *>(a.q.p) + h * a.q.hd, a.q.ld, static_cast<const T *>(a.g.p) + h * a.g.hd, a.g.ld,
                         a.lse + (long)h * a.q_rows, delta + (long)h * a.q_rows, sp, a.dh, c, dk, dv);
#pragma unroll
        for (int i = 0; i < 4; i++) dk[i] *= __shfl_sync(0xFFFFFFFFu, fk, src);
        if (4 * lane >= c0 && 4 * lane < c1 && 4 * lane < a.dh) {
            store4(static_cast<T *>(a.dk.p) + rr * a.dk.ld + hk * a.dk.hd + 4 * lane, dk);
            store4(static_cast<T *>(a.dv.p) + rr * a.dv.ld + hk * a.dv.hd + 4 * lane, dv);
        }
    }
}

template <int DH, bool BF, int W>
__global__ void __launch_bounds__(BW_THREADS, 512 / DkvLayout<DH, W>::COLS) seq_attn_dkv_kernel(const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                                                                     const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tg,
                                                                     const __grid_constant__ SeqAttn a, const float c, const float *delta, const float *tops, const int ctas) {
    using L = DkvLayout<DH, W>;
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    constexpr int QS = L::QS, GS = L::GS;
    extern __shared__ __align__(1024) uint8_t smp[];  // nothing else is in shared memory
    const uint32_t sm = s_addr(smp), bar0 = sm + L::OFF_R;
    int *rest = reinterpret_cast<int *>(smp + L::OFF_R + 8 * (2 * QS + 2 * GS + 10));
    uint32_t &tslot = *reinterpret_cast<uint32_t *>(rest);
    int &failed = rest[1], *span_lo = rest + 2, *span_hi = rest + 6;
    volatile int &gain = rest[10];  // log2 of what dS is multiplied by, from the first numbers of queries on
    uint8_t *odd_rows = reinterpret_cast<uint8_t *>(rest + 12);
    const auto q_full = [&](int s) { return bar0 + 8 * s; };
    const auto q_free = [&](int s) { return bar0 + 8 * (QS + s); };
    const auto g_full = [&](int s) { return bar0 + 8 * (2 * QS + s); };
    const auto g_free = [&](int s) { return bar0 + 8 * (2 * QS + GS + s); };
    const uint32_t kv_full = bar0 + 8 * (2 * QS + 2 * GS), s_full = kv_full + 8, dp_full = kv_full + 16, p_full = kv_full + 24, ds_full = kv_full + 32,
                   out_full = kv_full + 40, n_full = kv_full + 48, n_free = kv_full + 64;  // the last: two each
    if (sm & 1023u) {  // alike in all threads of all CTAs
        if (threadIdx.x == 0) set_status(a.status, MNMT_ECUDA);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int share = (int)blockIdx.x % ctas, unit = (int)blockIdx.x / ctas, hk = unit % a.hkv, tile = unit / a.hkv;
    const int h0 = hk * a.group(), heads = a.group();
    const int half = warp >> 2, rt = (int)threadIdx.x & 127, row = tile * SQ_ROWS + rt;
    if (threadIdx.x == 0) {
        for (int s = 0; s < QS; s++) mbar_init(q_full(s), 1), mbar_init(q_free(s), 1);
        for (int s = 0; s < GS; s++) mbar_init(g_full(s), 1), mbar_init(g_free(s), 1);
        mbar_init(n_full, 1), mbar_init(n_full + 8, 1), mbar_init(n_free, 8), mbar_init(n_free + 8, 8);
        mbar_init(kv_full, 2), mbar_init(s_full, 1), mbar_init(dp_full, 1), mbar_init(p_full, 8), mbar_init(ds_full, 8), mbar_init(out_full, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) tmem_alloc<L::COLS>(s_addr(&tslot));
    pdl_grid_wait();
    const SeqAttn ix = seq_shared(a, reinterpret_cast<int *>(smp + L::OFF_Q), BW_THREADS);  // where queries come later
    Span qs{0, 0};
    bool in = false, one = false;
    if (warp < 8) {
        qs = queries_of_lane(ix, row - lane, in, one);
        const bool some = qs.hi > qs.lo;
        const int lo = __reduce_min_sync(0xFFFFFFFFu, some ? qs.lo : 0x7FFFFFFF), hi = __reduce_max_sync(0xFFFFFFFFu, some ? qs.hi : 0);
        if (lane == 0 && half == 0) span_lo[warp] = lo, span_hi[warp] = hi;
    }
    sq_before_copies();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tS = tslot, tP = tS + L::T_DP, tV = tS + L::T_DV, tK = tS + L::T_DK;
    const int first = min(min(span_lo[0], span_lo[1]), min(span_lo[2], span_lo[3])), end = max(max(span_hi[0], span_hi[1]), max(span_hi[2], span_hi[3]));
    const int nt = end > first ? (end - first + W - 1) / W : 0;  // tiles of one head
    // this CTA's steps of the walk over all heads: n of them from step0 on
    const int step0 = (int)((long)nt * heads * share / ctas), n = (int)((long)nt * heads * (share + 1) / ctas) - step0;
    const int head0 = nt ? step0 / nt : 0, t0 = step0 - head0 * nt;
    const SqWaits wait{&failed, a.status};

    if (warp == 8) {
        // From the largest |g| of the rows and heads of the whole walk, whoever shares it.  (The first head's first are on their
        // way from the start: most sentences have no others.)
        const int per = (a.q_rows + GAIN_ROWS - 1) / GAIN_ROWS, tops0 = first / GAIN_ROWS, n_tops = nt ? (end - 1) / GAIN_ROWS - tops0 + 1 : 0;
        const uint32_t *top_of = reinterpret_cast<const uint32_t *>(tops) + (long)h0 * per + tops0;
        [[maybe_unused]] const uint32_t top0 = !BF && lane < n_tops ? top_of[lane] : 0;
        [[maybe_unused]] const auto find_gain = [&] {
            uint32_t top = top0;
            for (int i = lane; i < n_tops; i += 32)
#pragma unroll 4
                for (int h = i < 32 ? 1 : 0; h < heads; h++) top = max(top, top_of[(long)h * per + i]);
            const int e = gain_of(__uint_as_float(__reduce_max_sync(0xFFFFFFFFu, top)));
            if (lane == 0) gain = e;
            return e;
        };
        if (!BF && nt && !n) find_gain();  // no step of the walk, but a share of the columns
        if (n) {
            if (lane == 0) {
                sq_load<DH>(sm, &tk, hk, tile * SQ_ROWS, kv_full);
                sq_load<DH>(sm + L::OFF_V, &tv, hk, tile * SQ_ROWS, kv_full);
            }
            // Q(0), then G(j), Q(j + QS - GS) and the numbers of tile j's queries by turns
            int jq = 0, jg = 0, hq = h0 + head0, tq_ = t0, hg = hq, tg_ = t0;
            [[maybe_unused]] float lift = 1.0f;
            bool ok = true;
            const auto next_q = [&] {
                const int s = jq % QS;
                if (jq >= QS) ok = wait(q_free(s), (uint32_t)(jq / QS - 1) & 1);
                if (!ok) return;
                if (lane == 0) sq_load<DH, W>(sm + L::OFF_Q + s * L::TILE, &tq, hq, end - W * (tq_ + 1), q_full(s));
                if (++tq_ == nt) tq_ = 0, hq++;
                jq++;
            };
            next_q();
            while (ok && jg < n) {
                const int s = jg % GS, at = end - W * (tg_ + 1);
                if (jg >= GS) ok = wait(g_free(s), (uint32_t)(jg / GS - 1) & 1);
                if (!ok) break;
                if (lane == 0) sq_load<DH, W>(sm + L::OFF_G + s * L::TILE, &tg, hg, at, g_full(s));
                // -lse log2 e and -D
                float x[2][W / 32];
#pragma unroll
                for (int i = 0; i < W / 32; i++) {
                    const int r = at + 32 * i + lane;
                    const bool on = r >= 0 && r < a.q_rows;
                    x[0][i] = on ? -LOG2E * __ldg(a.lse + (long)hg * a.q_rows + r) : 0.0f;
                    x[1][i] = on ? -delta[(long)hg * a.q_rows + r] : 0.0f;
                }
                if (++tg_ == nt) tg_ = 0, hg++;
                const int b = jg & 1, turn = jg >> 1;
                jg++;
                while (ok && jq < n && jq < jg + QS - GS) next_q();
                if (ok && turn) ok = wait(n_free + 8 * b, (uint32_t)(turn - 1) & 1);
                if (!ok) break;
                if constexpr (!BF) {  // P and dS times their powers (here: the numbers have had time to come)
                    if (jg == 1) lift = pow2(find_gain() - (int)P_GAIN);
#pragma unroll
                    for (int i = 0; i < W / 32; i++) x[0][i] += P_GAIN, x[1][i] *= lift;
                }
                float *num = reinterpret_cast<float *>(smp + L::OFF_N + b * L::NUM);
#pragma unroll
                for (int i = 0; i < W / 32; i++) num[32 * i + lane] = x[0][i], num[W + 32 * i + lane] = x[1][i];
                __syncwarp();
                if (lane == 0) mbar_arrive(n_full + 8 * b);
            }
            if (wait.given_up()) {  // copies in flight land before the block ends
                wait(kv_full, 0);
                for (int i = max(0, jq - QS); i < jq; i++) wait(q_full(i % QS), (uint32_t)(i / QS) & 1);
                for (int i = max(0, jg - GS); i < jg; i++) wait(g_full(i % GS), (uint32_t)(i / GS) & 1);
            }
        }
    } else if (warp == 9) {
        if (n) {
            const uint32_t on = elect_one();
            const uint64_t kd = sq_k(sm), vd = sq_k(sm + L::OFF_V), qd = sq_k(sm + L::OFF_Q), gd = sq_k(sm + L::OFF_G);
            const uint64_t qt = sq_mn<W>(sm + L::OFF_Q), gt = sq_mn<W>(sm + L::OFF_G);
            const auto scores = [&](int j) {  // S^T(j)
                const int s = j % QS;
                if (!wait(q_full(s), (uint32_t)(j / QS) & 1)) return false;
                tc_fence_after();
                const uint64_t b = qd + (uint64_t)(s * (L::TILE >> 4));
#pragma unroll
                for (int k = 0; k < DH / 16; k++) sq_mma(on, tS, kd + sq_k_step(k), b + sq_k_step<W>(k), sq_idesc(W, BF, false), k > 0);
                f4_commit_on<1>(on, s_full);
                return true;
            };
            const auto weights = [&](int j) {  // dP^T(j)
                const int s = j % GS;
                if (!wait(g_full(s), (uint32_t)(j / GS) & 1)) return false;
                tc_fence_after();
                const uint64_t b = gd + (uint64_t)(s * (L::TILE >> 4));
#pragma unroll
                for (int k = 0; k < DH / 16; k++) sq_mma(on, tP, vd + sq_k_step(k), b + sq_k_step<W>(k), sq_idesc(W, BF, false), k > 0);
                f4_commit_on<1>(on, dp_full);
                return true;
            };
            bool ok = wait(kv_full, 0) && scores(0) && weights(0);
            for (int j = 0; j < n && ok; j++) {
                const int sq = j % QS, sg = j % GS;
                const uint64_t qoff = (uint64_t)(sq * (L::TILE >> 4)), goff = (uint64_t)(sg * (L::TILE >> 4));
                if (!(ok = wait(p_full, (uint32_t)j & 1))) break;
                tc_fence_after();
                // a row's two threads write W / 4 columns each, W / 2 apart
#pragma unroll
                for (int k = 0; k < W / 16; k++)
                    sq_mma_ta(on, tV, tS + 8 * (k % (W / 32)) + W / 2 * (k / (W / 32)), gt + goff + sq_mn_step(k), sq_idesc(DH, BF, true), (uint32_t)(j | k));
                f4_commit_on<1>(on, g_free(sg));
                if (j + 1 < n && !(ok = scores(j + 1))) break;
                if (!(ok = wait(ds_full, (uint32_t)j & 1))) break;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < W / 16; k++)
                    sq_mma_ta(on, tK, tP + 8 * (k % (W / 32)) + W / 2 * (k / (W / 32)), qt + qoff + sq_mn_step(k), sq_idesc(DH, BF, true), (uint32_t)(j | k));
                f4_commit_on<1>(on, q_free(sq));
                if (j + 1 < n && !(ok = weights(j + 1))) break;
            }
            f4_commit_on<1>(on, out_full);
            wait(out_full, 0);
        }
        pdl_allow_next();
    } else {
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const unsigned long long c2 = f4_two(c, c);
        bool ok = true;
        for (int j = 0, t = t0; j < n; j++) {
            const int at = end - W * (t + 1) + W / 2 * half, lo = qs.lo - at, hi = qs.hi - at;
            if (++t == nt) t = 0;
            const float4 *num = reinterpret_cast<const float4 *>(smp + L::OFF_N + (j & 1) * L::NUM) + W / 8 * half;
            const bool all = __all_sync(0xFFFFFFFFu, lo <= 0 && hi >= W / 2), some = __any_sync(0xFFFFFFFFu, hi > 0 && lo < W / 2);
            if (!(ok = wait(s_full, (uint32_t)j & 1) && wait(n_full + 8 * (j & 1), (uint32_t)(j >> 1) & 1))) break;
            tc_fence_after();
            // Two passes over a thread's columns, P and dS, without the masks where the warp's rows see all of them
            uint32_t r[W / 64][32] = {};  // as in the dq kernel
            const uint32_t zeros[16] = {};
            const auto weights = [&](auto whole) {
                load_half<W>(tS + lanes + W / 2 * half, r);
#pragma unroll
                for (int b = 0; b < W / 64; b++) {
                    const uint32_t see = sq_bits(lo - 32 * b, hi - 32 * b);
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const float4 x = num[8 * b + i];
                        float p[4];
                        f4_untwo(sq_fma2(f4_two(__uint_as_float(r[b][4 * i]), __uint_as_float(r[b][4 * i + 1])), c2, f4_two(x.x, x.y)), p[0], p[1]);
                        f4_untwo(sq_fma2(f4_two(__uint_as_float(r[b][4 * i + 2]), __uint_as_float(r[b][4 * i + 3])), c2, f4_two(x.z, x.w)), p[2], p[3]);
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            p[e] = exp2_fast(p[e]);
                            if (!decltype(whole)::value) p[e] = (see >> (4 * i + e)) & 1u ? p[e] : 0.0f;
                            r[b][4 * i + e] = __float_as_uint(p[e]);
                        }
                        w[2 * i] = sq_pack<BF>(p[0], p[1]), w[2 * i + 1] = sq_pack<BF>(p[2], p[3]);
                    }
                    tmem_st16(tS + lanes + W / 2 * half + 16 * b, w);
                }
            };
            const auto gradients = [&](auto whole) {
                [[maybe_unused]] const float lift = BF ? 1.0f : pow2(gain - (int)P_GAIN);
                [[maybe_unused]] const unsigned long long lift2 = f4_two(lift, lift);
                const auto less_d = [&](unsigned long long dp, unsigned long long d) { return BF ? f4_add2(dp, d) : sq_fma2(dp, lift2, d); };
                uint32_t q[W / 64][32];
                load_half<W>(tP + lanes + W / 2 * half, q);
#pragma unroll
                for (int b = 0; b < W / 64; b++) {
                    const uint32_t see = sq_bits(lo - 32 * b, hi - 32 * b);
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const float4 x = num[W / 4 + 8 * b + i];
                        float d[4];
                        f4_untwo(f4_mul2(f4_two(__uint_as_float(r[b][4 * i]), __uint_as_float(r[b][4 * i + 1])),
                                         less_d(f4_two(__uint_as_float(q[b][4 * i]), __uint_as_float(q[b][4 * i + 1])), f4_two(x.x, x.y))),
                                 d[0], d[1]);
                        f4_untwo(f4_mul2(f4_two(__uint_as_float(r[b][4 * i + 2]), __uint_as_float(r[b][4 * i + 3])),
                                         less_d(f4_two(__uint_as_float(q[b][4 * i + 2]), __uint_as_float(q[b][4 * i + 3])), f4_two(x.z, x.w))),
                                 d[2], d[3]);
                        if (!decltype(whole)::value) {
#pragma unroll
                            for (int e = 0; e < 4; e++) d[e] = (see >> (4 * i + e)) & 1u ? d[e] : 0.0f;
                        }
                        w[2 * i] = sq_pack<BF>(d[0], d[1]), w[2 * i + 1] = sq_pack<BF>(d[2], d[3]);
                    }
                    tmem_st16(tP + lanes + W / 2 * half + 16 * b, w);
                }
            };
            const auto written = [&](uint32_t bar) {
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar);
            };
            if (all) {
                weights(std::true_type{});
            } else if (some) {
                weights(std::false_type{});
            } else {
#pragma unroll
                for (int b = 0; b < W / 64; b++) tmem_st16(tS + lanes + W / 2 * half + 16 * b, zeros);
            }
            written(p_full);
            if (!(ok = wait(dp_full, (uint32_t)j & 1))) break;
            tc_fence_after();
            if (all) {
                gradients(std::true_type{});
            } else if (some) {
                gradients(std::false_type{});
            } else {
#pragma unroll
                for (int b = 0; b < W / 64; b++) tmem_st16(tP + lanes + W / 2 * half + 16 * b, zeros);
            }
            written(ds_full);
            if (lane == 0) mbar_arrive(n_free + 8 * (j & 1));
        }
        if (n) ok = wait(out_full, 0) && ok;
        tc_fence_after();
        // a row's two threads: dv, dk
        const HeadRows &x = half ? a.dk : a.dv;
        const float fk = one ? 0.0f : a.scale;  // as in the dq kernel
        const auto factor = [&] { return half ? BF || !nt ? fk : fk * pow2(-gain) : BF ? 1.0f : pow2(-(int)P_GAIN); };
        T *o = static_cast<T *>(x.p) + row * x.ld + hk * x.hd;
        bool odd = false;
        int c0 = 0, c1 = DH;  // the columns that this CTA stores
        if (ctas == 1) {
            if (ok) {
                const float f = factor();
                uint32_t out[DH / 2];
#pragma unroll
                for (int b = 0; b < DH / 32; b++) {
                    uint32_t w[32] = {};
                    if (n) tmem_ld32((half ? tK : tV) + lanes + 32 * b, w);
                    tmem_wait_ld();
                    const bool any = n && qs.hi > qs.lo;
#pragma unroll
                    for (int i = 0; i < 16; i++) {
                        const float y = any ? __uint_as_float(w[2 * i]) : 0.0f, z = any ? __uint_as_float(w[2 * i + 1]) : 0.0f;
                        odd |= !(fabsf(y) < INFINITY) || !(fabsf(z) < INFINITY);
                        out[16 * b + i] = sq_pack<BF>(y * f, z * f);
                    }
                }
                // the keys and values have been multiplied: their rows are free
                sq_store_rows<DH>(smp + warp * (64 * DH), out, reinterpret_cast<uint16_t *>(o) - lane * x.ld, x.ld, __ballot_sync(0xFFFFFFFFu, in), a.dh);
            }
        } else {
            // sums of this CTA's steps to shared memory, where the tiles were: four columns of a row side by side
            float4 *mine = reinterpret_cast<float4 *>(smp) + half * (DH / 4) * SQ_ROWS + rt;
#pragma unroll
            for (int b = 0; b < DH / 32; b++) {
                uint32_t w[32] = {};
                if (n) tmem_ld32((half ? tK : tV) + lanes + 32 * b, w);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; i++)
                    mine[(8 * b + i) * SQ_ROWS] = n ? make_float4(__uint_as_float(w[4 * i]), __uint_as_float(w[4 * i + 1]), __uint_as_float(w[4 * i + 2]),
                                                                  __uint_as_float(w[4 * i + 3]))
                                                    : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            __syncwarp();
            sq_cluster_sync();
            // every CTA of the cluster adds up a share of the columns, in the order of the CTAs
            c0 = DH / ctas * share, c1 = c0 + DH / ctas;
            if (ok) odd = sq_join<BF>(s_addr(mine), c0, c1, ctas, qs.hi > qs.lo ? 1.0f : 0.0f, factor(), in, o, a.dh);
        }
        odd_rows[half * SQ_ROWS + rt] = odd;
        elements_sync();
        odd = ok && in && (odd_rows[rt] || odd_rows[SQ_ROWS + rt]);
        const uint32_t again = __ballot_sync(0xFFFFFFFFu, odd && (rt & 1) == half);
        if (again) dkv_again<T>(a, again, row, hk, qs, fk, c, delta, c0, c1);
    }
    if (ctas > 1) {
        if (warp >= 8) {
            __syncwarp();
            sq_cluster_sync();
        }
        __syncwarp();
        sq_cluster_sync();  // no CTA leaves while others read its sums
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) tmem_free<L::COLS>(tslot);
}

// Where there are no queries or no keys at all, gradients of rows in sequences are zero.
template <typename T>
__global__ void __launch_bounds__(256) seq_attn_zero_kernel(SeqAttn a) {
    pdl_grid_wait();
    const long w = ((long)blockIdx.x * 256 + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    bool in, one, few;
    if (a.k_rows == 0) {
        if (w >= a.q_rows) return;
        keys_of_query(a, (int)w, last_with_rows(a.q_len, seq_of(a.q_start, a.n_seqs, (int)w)), in, few);
        for (int h = 0; in && 4 * lane < a.dh && h < a.hq; h++) store4(static_cast<T *>(a.dq.p) + w * a.dq.ld + h * a.dq.hd + 4 * lane, z);
    } else {
        if (w >= a.k_rows) return;
        queries_of_key(a, (int)w, last_with_rows(a.k_len, seq_of(a.k_start, a.n_seqs, (int)w)), in, one);
        for (int h = 0; in && 4 * lane < a.dh && h < a.hkv; h++) {
            store4(static_cast<T *>(a.dk.p) + w * a.dk.ld + h * a.dk.hd + 4 * lane, z);
            store4(static_cast<T *>(a.dv.p) + w * a.dv.ld + h * a.dv.hd + 4 * lane, z);
        }
    }
}

// CTAs that share the walks of `units` tiles, `slots` of them on the card at a time: one to eight, by a model of the time in us
// fitted to measured calls (1 to 8 sequences of 46 to 8192 rows, heads of 64 and 128, one to 16 heads a key head).  A CTA
// takes 8 us beside its steps, a cluster as many more as it has CTAs; a step of 64 takes 0.95 where two CTAs share an SM, one of
// 128 alone 1.45.  In one round the longest walk counts; in more, the sum of the work and half of the longest walk.
// (At the time of the fit: 4096 causal rows of 8 heads of 64: two CTAs 90 us, one 110; 2048 rows of 16 heads of 128 on 2 key heads: four 103,
// two 147, eight 146; 2048 rows of 8 heads of 128: one 58, two 63, four 83.  These take 95, 76 and 49 now, by the choices that it makes.
// Rows in memory over sequences stand for their lengths: a long sequence among many short ones is walked as they are.)
int walk_ctas(long units, long slots, double longest, double mean, int w) {
    const double step = w == 64 ? 0.95 : 1.45;
    int best = 1;
    double least = 0.0;
    for (int p = 1; p <= 8 && (p == 1 || longest >= 2.0 * p); p *= 2) {
        const double beside = 8.0 + (p > 1 ? p : 0), chain = beside + longest / p * step, n = (double)units * p;
        const double t = n <= slots ? chain : (n * beside + units * mean * step) / slots + chain / 2;
        if (p == 1 || t < least) best = p, least = t;
    }
    return best;
}
// steps of a walk over rows of n sequences, at most and on average
int dkv_ctas(long tiles, const SeqAttn &a, int w, int blocks) {
    const double steps = ((double)a.q_rows / ((double)a.n_seqs * w) + 1) * a.group();
    return walk_ctas(tiles * a.hkv, 152L * blocks, steps, a.causal ? steps / 2 : steps, w);
}
int dq_ctas(long tiles, const SeqAttn &a, int w, int blocks) {
    const double steps = (double)a.k_rows / ((double)a.n_seqs * w) + 1;
    return walk_ctas(tiles * a.hq, 152L * blocks, steps, a.causal ? steps / 2 : steps, w);
}

template <int DH, bool BF, int W>
cudaError_t tile_backward(const SeqAttn &a, cudaStream_t st) {
    // whole tiles of the rows that stay, tiles of W rows of those that are walked
    CUtensorMap tq, tk, tv, tg, wq, wk, wv, wg;
    if (!sq_map(&tq, a.q, a.q_rows, a.hq, a.dh, SQ_ROWS) || !sq_map(&tg, a.g, a.q_rows, a.hq, a.dh, SQ_ROWS) ||
        !sq_map(&tk, a.k, a.k_rows, a.hkv, a.dh, SQ_ROWS) || !sq_map(&tv, a.v, a.k_rows, a.hkv, a.dh, SQ_ROWS))
        return cudaErrorInvalidValue;
    if (W == SQ_ROWS) {
        wq = tq, wk = tk, wv = tv, wg = tg;
    } else if (!sq_map(&wq, a.q, a.q_rows, a.hq, a.dh, W) || !sq_map(&wg, a.g, a.q_rows, a.hq, a.dh, W) || !sq_map(&wk, a.k, a.k_rows, a.hkv, a.dh, W) ||
               !sq_map(&wv, a.v, a.k_rows, a.hkv, a.dh, W)) {
        return cudaErrorInvalidValue;
    }
    float *delta = static_cast<float *>(a.workspace), *tops = delta + (size_t)a.hq * a.q_rows;
    const float c = a.scale * LOG2E;
    const unsigned qt = (unsigned)((a.q_rows + SQ_ROWS - 1) / SQ_ROWS), kt = (unsigned)((a.k_rows + SQ_ROWS - 1) / SQ_ROWS);
    const int cq = dq_ctas(qt, a, W, 512 / DqLayout<DH, W>::COLS);
    const cudaError_t e = sq_launch(seq_attn_dq_kernel<DH, BF, W>, qt * a.hq * cq, cq, BW_THREADS, DqLayout<DH, W>::SMEM, st, tq, tg, wk, wv, a, c, delta, tops, cq);
    if (e != cudaSuccess) return e;
    const int ctas = dkv_ctas(kt, a, W, 512 / DkvLayout<DH, W>::COLS);
    return sq_launch(seq_attn_dkv_kernel<DH, BF, W>, kt * a.hkv * ctas, ctas, BW_THREADS, DkvLayout<DH, W>::SMEM, st, tk, tv, wq, wg, a, c,
                     (const float *)delta, (const float *)tops, ctas);
}

template <int DH, bool BF, int W>
cudaError_t tile_init() {
    const cudaError_t e = cudaFuncSetAttribute(seq_attn_dq_kernel<DH, BF, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, DqLayout<DH, W>::SMEM);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(seq_attn_dkv_kernel<DH, BF, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, DkvLayout<DH, W>::SMEM);
}

}  // namespace

cudaError_t seq_attn_backward_init() {
    cudaError_t e = tile_init<64, true, 64>();
    if (e == cudaSuccess) e = tile_init<64, false, 64>();
    if (e == cudaSuccess) e = tile_init<128, true, 128>();
    if (e == cudaSuccess) e = tile_init<128, false, 128>();
    return e;
}

// D of every row and head; fp16: and the largest |g| of every GAIN_ROWS rows and head
size_t seq_attn_backward_workspace(const SeqAttn &a) {
    const size_t n = a.q_rows, tops = a.dtype == MNMT_F16 ? (n + GAIN_ROWS - 1) / GAIN_ROWS : 0;
    return ((size_t)a.hq * (n + tops) * 4 + 31) / 16 * 16;
}

cudaError_t launch_seq_attn_backward(const SeqAttn &a, cudaStream_t st) {
    const bool bf = a.dtype == MNMT_BF16;
    if (a.q_rows == 0 || a.k_rows == 0)
        return launch_pdl(bf ? seq_attn_zero_kernel<__nv_bfloat16> : seq_attn_zero_kernel<__half>, (unsigned)((a.q_rows + a.k_rows + 7) / 8), 256, 0, st, a);
    if (a.dh > 64) return bf ? tile_backward<128, true, 128>(a, st) : tile_backward<128, false, 128>(a, st);
    return bf ? tile_backward<64, true, 64>(a, st) : tile_backward<64, false, 64>(a, st);
}

}  // namespace mnmt
