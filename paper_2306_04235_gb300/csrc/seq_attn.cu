// seq_attn.cu -- attention over sequences, forward (seq_attn.cuh).
//
// A CTA takes 128 query rows of one head, whatever sequences they belong to (tiles of a
// sequence each would leave half of their rows empty at 90 rows a sentence): the keys that
// a row sees are an interval of key rows, and the tile walks 64 keys at a time through the
// union of its rows' intervals, from its end backwards, so that no tile reaches past the
// last key that a row sees (what lies there, unwritten rows for instance, would meet zero
// weights, and zero times NaN is NaN).
//   S = Q K^T (TMEM), one thread per row: P = 2^(c s - m), c = scale log2 e, with the
//   running maximum m and sum l; P over S in TMEM, in the operands' type; O += P V.
// m is moved, and O scaled, only where a score exceeds it by 2^8 (the sum and the
// result carry the same factor, so any m near the maximum serves).  For fp16 m is 7 less, so that
// weights reach 2^15: those below 2^-25 of the largest would leave O but not l (32767 keys at 2^-25.2
// of one: o 8.5e-4 low, 4e-6 so, of which one step is 4.9e-4).
// Two CTAs per SM; three tiles of scores in TMEM (heads up to 64; two above), so that the
// tensor core is tiles ahead of the threads that take powers: tiles of 128 keys with one
// buffer waited 1750 of 3200 cycles a tile for it, before MMAs were issued by a converged warp
// (sq_mma); under a branch on the lane the issue of a tile took 1250 cycles and set the pace (2 x
// 6000..8192 rows of 16 heads of 128 352 us, 309 then).  Tiles of 128 keys were not measured again since.
// Where O of a row is not finite though its sum is, an infinity or a NaN of a key
// that the row does not see may have come in: such rows are computed again over
// their own keys alone (attn_row).
//
// Bound by: heads of 128, the tensor core and its operands (8192 rows of 16 heads, 4 key
// heads, causal 191 us, 1.43 PFLOP/s, pipe active 63 %: S of 64 keys reads 6 KB of shared memory
// for 32 cycles of products, and 168 registers leave no more CTAs); heads of 64, issue (0.84 PFLOP/s; 8192 rows of 8 heads, not causal, 163 us);
// short sequences, a chain of latencies (128 targets of 20..160 rows against 20..128 keys, 8 heads of 64: 19 us for
// 6.5 us of bytes: start 1, starts 0.6, search 0.6, first tile 1.4, 0.7 a tile, 1.8 the end of a head).
#include "seq_tile.cuh"

namespace mnmt {
namespace {

constexpr int FW_THREADS = 192;  // four softmax warps, a TMA warp, an MMA warp
constexpr int KT = 64;           // keys of a tile
template <int DH>
struct FwLayout {
    // tiles of keys and values, of queries
    static constexpr int STAGES = DH == 64 ? 4 : 2, QS = DH == 64 ? 2 : 1, QT = sq_bytes<DH>(), TILE = sq_bytes<DH, KT>();
    static constexpr int OFF_K = QS * QT, OFF_V = OFF_K + STAGES * TILE, SMEM = OFF_V + STAGES * TILE + 1024;
    static_assert(2 * STAGES * TILE >= 4 * SQ_INTS, "starts and lengths before keys and values");
    static_assert(OFF_V + STAGES * TILE >= SQ_ROWS * (DH * 4 + 8), "a CTA's sums for its cluster");
    // tiles of scores in TMEM, columns of O behind them; CTAs per SM
    static constexpr int BUFS = DH == 64 ? 3 : 2, T_O = BUFS * KT, COLS = pow2_cols(T_O + DH), BLOCKS = 512 / COLS;
};
constexpr float FW_SLACK = 8.0f;  // how far, in powers of two, a score may exceed m and its type's lift

// 32 scores of a row from TMEM, -inf where the row does not see the key (see: bits of the 32)
__device__ __forceinline__ void hide(uint32_t (&r)[32], uint32_t see) {
#pragma unroll
    for (int i = 0; i < 32; i++) r[i] = (see >> i) & 1u ? r[i] : 0xFF800000u;
}
__device__ __forceinline__ void max32(const uint32_t (&r)[32], float (&mx)[4]) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) mx[i / 2 & 3] = fmaxf(fmaxf(mx[i / 2 & 3], __uint_as_float(r[i])), __uint_as_float(r[i + 1]));
}
// their weights 2^(c s - m), packed; sums in ls
template <bool BF>
__device__ __forceinline__ void weigh(const uint32_t (&r)[32], unsigned long long c2, unsigned long long m2, unsigned long long &ls, uint32_t (&p)[16]) {
#pragma unroll
    for (int i = 0; i < 16; i++) {
        float x, y;
        f4_untwo(sq_fma2(f4_two(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), c2, m2), x, y);
        x = exp2_fast(x), y = exp2_fast(y);
        ls = f4_add2(ls, f4_two(x, y));
        p[i] = sq_pack<BF>(x, y);
    }
}

// Rows of `again`, a lane's row each, computed again over their own keys; columns c0 .. c1 - 1 are stored
template <typename T>
__device__ __noinline__ void forward_again(const SeqAttn &a, uint32_t again, int row, int h, Span keys, float c, int c0, int c1) {
    const int lane = threadIdx.x & 31, hk = h / a.group();
    for (; again; again &= again - 1) {
        const int src = __ffs(again) - 1, rr = __shfl_sync(0xFFFFFFFFu, row, src);
        const Span s{__shfl_sync(0xFFFFFFFFu, keys.lo, src), __shfl_sync(0xFFFFFFFFu, keys.hi, src)};
        const RowSum x = attn_row(static_cast<const T *>(a.q.p) + rr * a.q.ld + h * a.q.hd, static_cast<const T *>(a.k.p) + hk * a.k.hd, a.k.ld,
                                  static_cast<const T *>(a.v.p) + hk * a.v.hd, a.v.ld, s, a.dh, c);
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = x.acc[i] / x.l;
        if (4 * lane >= c0 && 4 * lane < c1 && 4 * lane < a.dh) store4(static_cast<T *>(a.o.p) + rr * a.o.ld + h * a.o.hd + 4 * lane, v);
    }
}

// The end of a CTA whose cluster divides a head's walk: its softmax warps meet the others' here once
template <int DH, bool BF>
__device__ __noinline__ void forward_join(const SeqAttn &a, uint8_t *smp, int ctas, int share, int row, int h0, bool in, Span keys, float c, float m, float l,
                                          bool ok, uint32_t tO, int nt) {
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    const bool none = keys.hi <= keys.lo;
    // This CTA's sums, four columns of a row side by side, and its m and l, where queries and keys were
    float4 *mine = reinterpret_cast<float4 *>(smp) + threadIdx.x;
    float2 *ml = reinterpret_cast<float2 *>(smp + SQ_ROWS * DH * 4) + threadIdx.x;
#pragma unroll
    for (int b = 0; b < DH / 32; b++) {
        uint32_t w[32];
        if (nt) tmem_ld32(tO + 32 * b, w);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 8; i++)
            mine[(8 * b + i) * SQ_ROWS] = nt ? make_float4(__uint_as_float(w[4 * i]), __uint_as_float(w[4 * i + 1]), __uint_as_float(w[4 * i + 2]),
                                                           __uint_as_float(w[4 * i + 3]))
                                             : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    *ml = make_float2(m, l);
    __syncwarp();
    sq_cluster_sync();
    // every CTA joins a share of the columns, in the order of the CTAs
    const int c0 = DH / ctas * share, c1 = c0 + DH / ctas;
    const uint32_t at = s_addr(mine), at_ml = s_addr(ml);
    float w[8], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; r++) {
        if (r >= ctas) continue;
        const float2 x = sq_remote2(t2_mapa(at_ml, r));
        top = fmaxf(top, x.x);
        w[r] = x.x;
    }
    const float mu = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int r = 0; r < 8; r++) {
        if (r >= ctas) continue;
        w[r] = exp2_fast(w[r] - mu);
        sum = fmaf(sq_remote2(t2_mapa(at_ml, r)).y, w[r], sum);
    }
    const float inv = none ? 0.0f : 1.0f / sum;
    bool odd = false;
    if (ok) {
        T *o = static_cast<T *>(a.o.p) + row * a.o.ld + h0 * a.o.hd;
#pragma unroll 1
        for (int col = c0; col < c1; col += 8) {
            float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int r = 0; r < 8; r++) {
                if (r >= ctas) continue;
                const uint32_t from = t2_mapa(at + (col / 4) * (SQ_ROWS * 16), r);
                const float4 y = sq_remote(from), z = sq_remote(from + SQ_ROWS * 16);
                v[0] = fmaf(y.x, w[r], v[0]), v[1] = fmaf(y.y, w[r], v[1]), v[2] = fmaf(y.z, w[r], v[2]), v[3] = fmaf(y.w, w[r], v[3]);
                v[4] = fmaf(z.x, w[r], v[4]), v[5] = fmaf(z.y, w[r], v[5]), v[6] = fmaf(z.z, w[r], v[6]), v[7] = fmaf(z.w, w[r], v[7]);
            }
#pragma unroll
            for (int i = 0; i < 8; i++) {
                odd |= !(fabsf(v[i]) < INFINITY);
                v[i] = none ? 0.0f : v[i] * inv;
            }
            if (in) sq_store<BF>(o, col, a.dh, v);
        }
        if (in && a.lse && share == 0) a.lse[(long)h0 * a.q_rows + row] = none ? -INFINITY : row_lse(top, sum);
    }
    __syncwarp();
    forward_again<T>(a, __ballot_sync(0xFFFFFFFFu, ok && in && !none && odd && fabsf(sum) < INFINITY), row, h0, keys, c, c0, c1);
}

// MANY: a CTA takes several heads one after another; else one, whose walk a cluster may divide
template <int DH, bool BF, bool MANY>
__global__ void __launch_bounds__(FW_THREADS, FwLayout<DH>::BLOCKS)
    seq_attn_forward_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                            const __grid_constant__ SeqAttn a, const float c, const int several) {
    const int heads = MANY ? several : 1, ctas = MANY ? 1 : several;
    using L = FwLayout<DH>;
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    constexpr int ST = L::STAGES, BUFS = L::BUFS, QS = L::QS;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[4 * ST + 2 * QS + 5 + 2 * BUFS];
    __shared__ uint32_t tslot;
    __shared__ int failed, span[2][4];
    const uint32_t sm = (s_addr(raw) + 1023u) & ~1023u, bar0 = s_addr(bars);
    uint8_t *smp = raw + (sm - s_addr(raw));
    const auto k_full = [&](int s) { return bar0 + 8 * s; };
    const auto k_free = [&](int s) { return bar0 + 8 * (ST + s); };
    const auto v_full = [&](int s) { return bar0 + 8 * (2 * ST + s); };
    const auto v_free = [&](int s) { return bar0 + 8 * (3 * ST + s); };
    const auto q_full = [&](int s) { return bar0 + 8 * (4 * ST + s); };
    const auto q_free = [&](int s) { return bar0 + 8 * (4 * ST + QS + s); };
    const uint32_t o_full = bar0 + 8 * (4 * ST + 2 * QS), o_free = o_full + 8, pv_done = o_full + 16, done = o_full + 32, s_full = o_full + 40,
                   p_full = s_full + 8 * BUFS;  // two of pv_done by turns, BUFS of s_full and p_full (a warp may be a tile ahead)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // heads h0 .. h0 + nh - 1 of a tile of rows, the last rows (causal: the longest walks) first
    // (ctas > 1: a cluster divides the walk of one head)
    const int groups = (a.hq + heads - 1) / heads, share = (int)blockIdx.x % ctas, unit = (int)blockIdx.x / ctas;
    const int h0 = unit % groups * heads, nh = MANY ? min(heads, a.hq - h0) : 1;
    const int tile = (int)gridDim.x / ctas / groups - 1 - unit / groups, row = tile * SQ_ROWS + (int)threadIdx.x;
    if (threadIdx.x == 128) {
        for (int s = 0; s < ST; s++) mbar_init(k_full(s), 1), mbar_init(k_free(s), 1), mbar_init(v_full(s), 1), mbar_init(v_free(s), 1);
        for (int s = 0; s < QS; s++) mbar_init(q_full(s), 1), mbar_init(q_free(s), 4);
        for (int b = 0; b < BUFS; b++) mbar_init(s_full + 8 * b, 1), mbar_init(p_full + 8 * b, 4);
        mbar_init(o_full, 1), mbar_init(o_free, 4), mbar_init(pv_done, 1), mbar_init(pv_done + 8, 1), mbar_init(done, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) tmem_alloc<L::COLS>(s_addr(&tslot));
    pdl_grid_wait();
    const SeqAttn ix = seq_shared(a, reinterpret_cast<int *>(smp + L::OFF_K), FW_THREADS);  // where keys and values come later
    Span keys{0, 0};
    bool in = false, few;
    if (warp < 4) {
        keys = keys_of_lane(ix, row - lane, in, few);
        const bool some = keys.hi > keys.lo;
        const int lo = __reduce_min_sync(0xFFFFFFFFu, some ? keys.lo : 0x7FFFFFFF), hi = __reduce_max_sync(0xFFFFFFFFu, some ? keys.hi : 0);
        if (lane == 0) span[0][warp] = lo, span[1][warp] = hi;
    }
    sq_before_copies();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tS = tslot, tO = tslot + L::T_O;  // P(j) takes the first half of S(j)'s columns
    const int first = min(min(span[0][0], span[0][1]), min(span[0][2], span[0][3])), end = max(max(span[1][0], span[1][1]), max(span[1][2], span[1][3]));
    // this CTA's tiles of a head, nt of them from t0 on; of all heads
    const int all_t = end > first ? (end - first + KT - 1) / KT : 0, t0 = (int)((long)all_t * share / ctas), nt = (int)((long)all_t * (share + 1) / ctas) - t0;
    const int n = nt * nh;
    const SqWaits wait{&failed, a.status};

    if (warp == 4) {
        if (lane == 0) {
            int j = 0, nq = 1;  // tiles of keys and values, and tiles of queries, whose copies were issued
            sq_load<DH>(sm, &tq, h0, tile * SQ_ROWS, q_full(0));
            bool ok = true;
            for (int it = 0; it < nh && nt && ok; it++) {
                const int hk = (h0 + it) / a.group();
                for (int t = 0; t < nt && ok; t++, j++) {
                    const int s = j % ST, at = end - KT * (t0 + t + 1);
                    const uint32_t ph = (uint32_t)(j / ST - 1) & 1;
                    if (j >= ST && !(ok = wait.one(k_free(s), ph))) break;
                    sq_load<DH, KT>(sm + L::OFF_K + s * L::TILE, &tk, hk, at, k_full(s));
                    if (j >= ST && !(ok = wait.one(v_free(s), ph))) {
                        wait.one(k_full(s), (uint32_t)(j / ST) & 1);  // in flight
                        break;
                    }
                    sq_load<DH, KT>(sm + L::OFF_V + s * L::TILE, &tv, hk, at, v_full(s));
                    // the next head's queries, once the results of the head that had their place are stored
                    if (t == min(1, nt - 1) && QS > 1 && nq < nh) {
                        if (nq >= QS && !(ok = wait.one(q_free(nq % QS), (uint32_t)(nq / QS - 1) & 1))) continue;
                        sq_load<DH>(sm + nq % QS * L::QT, &tq, h0 + nq, tile * SQ_ROWS, q_full(nq % QS));
                        nq++;
                    }
                }
                if (QS == 1 && ok && nq < nh) {
                    if (!(ok = wait.one(q_free(0), (uint32_t)it & 1))) break;
                    sq_load<DH>(sm, &tq, h0 + nq, tile * SQ_ROWS, q_full(0));
                    nq++;
                }
            }
            if (failed || nt == 0) {  // copies in flight land before the block ends
                for (int i = max(0, nq - QS); i < nq; i++) wait.one(q_full(i % QS), (uint32_t)(i / QS) & 1);
                for (int i = max(0, j - ST); i < j; i++) wait.one(k_full(i % ST), (uint32_t)(i / ST) & 1), wait.one(v_full(i % ST), (uint32_t)(i / ST) & 1);
            }
        }
    } else if (warp == 5) {
        if (nt) {
            const uint32_t on = elect_one();
            const uint64_t qd = sq_k(sm), kd = sq_k(sm + L::OFF_K), vd = sq_mn<KT>(sm + L::OFF_V);
            int next = 0, nit = 0, nst = 0;  // the next scores: number, head and tile of it
            const auto scores = [&] {
                const int s = next % ST;
                if ((MANY ? nst : next) == 0 && !wait(q_full(nit % QS), (uint32_t)(nit / QS) & 1)) return false;
                if (!wait(k_full(s), (uint32_t)(next / ST) & 1)) return false;
                tc_fence_after();
                const uint64_t a = qd + (uint64_t)(nit % QS * (L::QT >> 4)), b = kd + (uint64_t)(s * (L::TILE >> 4));
                const uint32_t d = tS + next % BUFS * KT;
#pragma unroll
                for (int k = 0; k < DH / 16; k++) sq_mma(on, d, a + sq_k_step(k), b + sq_k_step<KT>(k), sq_idesc(KT, BF, false), k > 0);
                f4_commit_on<1>(on, k_free(s));
                f4_commit_on<1>(on, s_full + 8 * (next % BUFS));
                next++;
                if (MANY && ++nst == nt) nst = 0, nit++;
                return true;
            };
            bool ok = true;
            if constexpr (MANY) {
                for (int it = 0, j = 0; it < nh && ok; it++)
                    for (int t = 0; t < nt && ok; t++, j++) {
                        // Scores up to BUFS tiles ahead (MMAs keep their order: P(j - 1), whose place S(j + BUFS - 1) takes, has been
                        // read).  The next head's only if its queries are there: they may wait for what this head has yet to do.
                        while (ok && next < n && next < j + BUFS &&
                               (next == j || nst > 0 || (nit <= it + QS - 1 && __all_sync(0xFFFFFFFFu, mbar_test(q_full(nit % QS), (uint32_t)(nit / QS) & 1)))))
                            ok = scores();
                        if (ok && t == 0 && it > 0) ok = wait(o_free, (uint32_t)(it - 1) & 1);  // the last head's O has been read
                        const int s = j % ST;
                        if (!ok || !(ok = wait(p_full + 8 * (j % BUFS), (uint32_t)(j / BUFS) & 1) && wait(v_full(s), (uint32_t)(j / ST) & 1))) break;
                        tc_fence_after();
                        const uint64_t b = vd + (uint64_t)(s * (L::TILE >> 4));
                        const uint32_t p = tS + j % BUFS * KT;
#pragma unroll
                        for (int k = 0; k < KT / 16; k++) sq_mma_ta(on, tO, p + 8 * k, b + sq_mn_step(k), sq_idesc(DH, BF, true), (uint32_t)(t | k));
                        f4_commit_on<1>(on, v_free(s));
                        f4_commit_on<1>(on, pv_done + 8 * (j & 1));
                        if (t == nt - 1) f4_commit_on<1>(on, o_full);
                    }
            } else {
                // one head: no question of whose queries are there (asked before every tile, 8192 rows of 8 heads of 64 took 179 us, 163 so)
                for (int j = 0; j < BUFS && j < nt && ok; j++) ok = scores();
                for (int j = 0; j < nt && ok; j++) {
                    const int s = j % ST;
                    if (!(ok = wait(p_full + 8 * (j % BUFS), (uint32_t)(j / BUFS) & 1) && wait(v_full(s), (uint32_t)(j / ST) & 1))) break;
                    tc_fence_after();
                    const uint64_t b = vd + (uint64_t)(s * (L::TILE >> 4));
                    const uint32_t p = tS + j % BUFS * KT;
#pragma unroll
                    for (int k = 0; k < KT / 16; k++) sq_mma_ta(on, tO, p + 8 * k, b + sq_mn_step(k), sq_idesc(DH, BF, true), (uint32_t)(j | k));
                    f4_commit_on<1>(on, v_free(s));
                    f4_commit_on<1>(on, pv_done + 8 * (j & 1));
                    if (j + BUFS < nt && !(ok = scores())) break;  // MMAs keep their order: P(j) has been read
                }
                f4_commit_on<1>(on, o_full);
            }
            f4_commit_on<1>(on, done);
            wait(done, 0);
        }
        pdl_allow_next();
    } else {
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        bool ok = true;
        float m = -INFINITY, l = 0.0f;  // m: of c s, less the lift
        const bool none = keys.hi <= keys.lo;  // no key: zeros; a sum of nothing but zeros is not a number, as 0 / 0
        for (int it = 0, j = 0; it < nh && ok; it++) {
            const int h = h0 + it;
            m = -INFINITY, l = 0.0f;
            for (int t = 0; t < nt; t++, j++) {
                if (!(ok = wait(s_full + 8 * (j % BUFS), (uint32_t)(j / BUFS) & 1))) break;
                tc_fence_after();
                const uint32_t tP = tS + j % BUFS * KT + lanes;
                const int at = end - KT * (t0 + t + 1), lo = keys.lo - at, hi = keys.hi - at;
                const bool all = __all_sync(0xFFFFFFFFu, lo <= 0 && hi >= KT);
                const auto p_ready = [&] {
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + 8 * (j % BUFS));
                };
                if (!__any_sync(0xFFFFFFFFu, hi > 0 && lo < KT)) {  // no row of the warp sees a key of the tile
                    const uint32_t zeros[16] = {};
#pragma unroll
                    for (int b = 0; b < KT / 32; b++) tmem_st16(tP + 16 * b, zeros);
                    p_ready();
                    continue;
                }
                uint32_t r[KT / 32][32];
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int b = 0; b < KT / 32; b++) tmem_ld32(tP + 32 * b, r[b]);
                tmem_wait_ld();
                if (!all) {
#pragma unroll
                    for (int b = 0; b < KT / 32; b++) hide(r[b], sq_bits(lo - 32 * b, hi - 32 * b));
                }
#pragma unroll
                for (int b = 0; b < KT / 32; b++) max32(r[b], mx);
                const float top = c * fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                // the first scores, or scores that 2^8 does not hold
                constexpr float LIFT = weight_lift<BF>();
                if (__any_sync(0xFFFFFFFFu, top > m + (LIFT + FW_SLACK))) {
                    const float mn = top > m + (LIFT + FW_SLACK) ? top - LIFT : m;
                    const float f = m == -INFINITY ? 1.0f : exp2_fast(m - mn);  // nothing was added yet: 0 stays 0
                    m = mn;
                    l *= f;
                    if (t > 0 && __any_sync(0xFFFFFFFFu, f != 1.0f)) {
                        // P V up to the tile before is in O.  (Not every turn is waited for: those two before are over, as S(j)
                        // was multiplied after them.)
                        if (!(ok = wait(pv_done + 8 * ((j - 1) & 1), (uint32_t)((j - 1) >> 1) & 1))) break;
                        tc_fence_after();
#pragma unroll
                        for (int b = 0; b < DH / 16; b++) {
                            uint32_t o[16];
                            tmem_ld16(tO + lanes + 16 * b, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; i++) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_st16(tO + lanes + 16 * b, o);
                        }
                    }
                }
                const float mu = m == -INFINITY ? 0.0f : m;  // no score yet: 2^-inf
                const unsigned long long c2 = f4_two(c, c), m2 = f4_two(-mu, -mu);
                unsigned long long ls = f4_two(0.0f, 0.0f);
#pragma unroll
                for (int b = 0; b < KT / 32; b++) {
                    uint32_t p[16];
                    weigh<BF>(r[b], c2, m2, ls, p);
                    tmem_st16(tP + 16 * b, p);  // over scores that were read
                }
                float la, lb;
                f4_untwo(ls, la, lb);
                l += la + lb;
                p_ready();
            }
            if (ok) ok = nt ? wait(o_full, (uint32_t)it & 1) : wait(q_full(0), 0);
            if (!ok) break;
            tc_fence_after();
            if (!MANY && ctas > 1) break;  // one head, joined below
            const float inv = none ? 0.0f : 1.0f / l;
            uint32_t out[DH / 2];
            const unsigned long long i2 = f4_two(inv, inv), z2 = f4_two(0.0f, 0.0f);
            unsigned long long nans = z2;  // sums of 0 x: not zero where an x is not finite
#pragma unroll
            for (int b = 0; b < DH / 32; b++) {
                uint32_t w[32];
                if (nt) tmem_ld32(tO + lanes + 32 * b, w);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const unsigned long long x = nt ? f4_two(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])) : z2;
                    float u, v;
                    nans = sq_fma2(x, z2, nans);
                    f4_untwo(f4_mul2(x, i2), u, v);
                    out[16 * b + i] = none ? 0u : sq_pack<BF>(u, v);
                }
            }
            float na, nb;
            f4_untwo(nans, na, nb);
            const bool odd = !(na + nb == 0.0f);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free);
            // the queries have been multiplied: their rows are free
            sq_store_rows<DH>(smp + it % QS * L::QT + warp * (64 * DH), out, static_cast<uint16_t *>(a.o.p) + (long)(row - lane) * a.o.ld + h * a.o.hd, a.o.ld,
                              __ballot_sync(0xFFFFFFFFu, in), a.dh);
            sq_before_copies();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_free(it % QS));
            if (in && a.lse) a.lse[(long)h * a.q_rows + row] = none ? -INFINITY : row_lse(m, l);
            const uint32_t again = __ballot_sync(0xFFFFFFFFu, in && !none && odd && fabsf(l) < INFINITY);
            if (again) forward_again<T>(a, again, row, h, keys, c, 0, DH);
        }
        if (!MANY && ctas > 1) forward_join<DH, BF>(a, smp, ctas, share, row, h0, in, keys, c, m, l, ok, tO + lanes, nt);
    }
    if (!MANY && ctas > 1) {
        __syncwarp();
        if (warp >= 4) sq_cluster_sync();
        sq_cluster_sync();  // no CTA leaves while others read its sums
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) tmem_free<L::COLS>(tslot);
}

// The give-up of SqWaits, for mnmt_wait_timeout_selftest: a warp half of whose lanes would see
// their phase end, one none of whose lanes do, and one whose lanes all do, which the others' giving up does not touch.
__global__ void __launch_bounds__(96) seq_wait_selftest_kernel(int *status) {
    __shared__ __align__(8) uint64_t bars[2];
    __shared__ int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t never = s_addr(bars), ended = never + 8;
    if (threadIdx.x == 0) {
        mbar_init(never, 1), mbar_init(ended, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        mbar_arrive(ended);
    }
    __syncthreads();
    const SqWaits wait{&failed, status};
    const bool ok = wait(warp == 2 || (warp == 0 && lane < 16) ? ended : never, 0);
    const uint32_t all = __ballot_sync(0xFFFFFFFFu, ok);
    if (lane == 0 && (all != (warp == 2 ? 0xFFFFFFFFu : 0u) || wait.one(never, 0) || !wait.one(ended, 0) || !failed)) atomicExch(status, MNMT_ECUDA);
}

// Where there are no keys at all, rows of sequences are zeros.
template <typename T>
__global__ void __launch_bounds__(256) seq_attn_zero_kernel(SeqAttn a) {
    pdl_grid_wait();
    const long w = ((long)blockIdx.x * 256 + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    bool in, few;
    if (w >= a.q_rows) return;
    keys_of_query(a, (int)w, last_with_rows(a.q_len, seq_of(a.q_start, a.n_seqs, (int)w)), in, few);
    if (!in) return;
    const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int h = 0; h < a.hq; h++) {
        if (4 * lane < a.dh) store4(static_cast<T *>(a.o.p) + w * a.o.ld + h * a.o.hd + 4 * lane, z);
        if (lane == 0 && a.lse) a.lse[(long)h * a.q_rows + w] = -INFINITY;
    }
}

// Heads that a CTA takes one after another: many short sequences, whose lookups and starts then
// count once for several heads
int forward_heads(long items, const SeqAttn &a) {
    const long keys = a.n_seqs ? a.k_rows / a.n_seqs : 0, h = (items + 2 * 152 - 1) / (2 * 152);
    return keys >= 256 ? 1 : (int)(h < 4 ? h : 4);
}
// CTAs that share the walk of a head: few tiles of rows, each with four tiles of keys at least.  Causal walks, which differ
// in length, gain until there are two CTAs for every SM (4096 rows of 8 heads 44 -> 35 us at the time, 34 now), others until there is
// one (64 rows on 8192 keys of 8 heads 80 -> 16, 14 now; 2048 rows not causal 24 -> 26, so alone, 20 now).  (Rows in memory over
// sequences stand for their lengths, here and in forward_heads: a long sequence among many short ones is walked as they are.)
int forward_ctas(long items, const SeqAttn &a) {
    const long keys = a.n_seqs ? a.k_rows / a.n_seqs : 0;
    int p = 1;
    while (p < 8 && items * p < (a.causal ? 2 * 152 : 76) && keys >= 4L * KT * 2 * p) p *= 2;
    return p;
}

template <int DH, bool BF>
cudaError_t tile_forward(const SeqAttn &a, cudaStream_t st) {
    CUtensorMap tq, tk, tv;
    if (!sq_map(&tq, a.q, a.q_rows, a.hq, a.dh, SQ_ROWS) || !sq_map(&tk, a.k, a.k_rows, a.hkv, a.dh, KT) || !sq_map(&tv, a.v, a.k_rows, a.hkv, a.dh, KT))
        return cudaErrorInvalidValue;
    const int tiles = (a.q_rows + SQ_ROWS - 1) / SQ_ROWS, heads = forward_heads((long)tiles * a.hq, a), ctas = forward_ctas((long)tiles * a.hq, a);
    const unsigned grid = (unsigned)tiles * (unsigned)((a.hq + heads - 1) / heads) * (unsigned)ctas;  // heads: short sequences, ctas: long ones
    if (heads > 1) return sq_launch(seq_attn_forward_kernel<DH, BF, true>, grid, 1, FW_THREADS, FwLayout<DH>::SMEM, st, tq, tk, tv, a, a.scale * LOG2E, heads);
    return sq_launch(seq_attn_forward_kernel<DH, BF, false>, grid, ctas, FW_THREADS, FwLayout<DH>::SMEM, st, tq, tk, tv, a, a.scale * LOG2E, ctas);
}

template <int DH, bool BF>
cudaError_t tile_init() {
    const cudaError_t e = cudaFuncSetAttribute(seq_attn_forward_kernel<DH, BF, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwLayout<DH>::SMEM);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(seq_attn_forward_kernel<DH, BF, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwLayout<DH>::SMEM);
}

}  // namespace

cudaError_t seq_attn_init() {
    cudaError_t e = tile_init<64, true>();
    if (e == cudaSuccess) e = tile_init<64, false>();
    if (e == cudaSuccess) e = tile_init<128, true>();
    if (e == cudaSuccess) e = tile_init<128, false>();
    return e;
}

cudaError_t launch_seq_wait_selftest(int *status, cudaStream_t st) {
    seq_wait_selftest_kernel<<<1, 96, 0, st>>>(status);
    return cudaGetLastError();
}

size_t seq_attn_forward_workspace(const SeqAttn &) { return 16; }

cudaError_t launch_seq_attn_forward(const SeqAttn &a, cudaStream_t st) {
    const bool bf = a.dtype == MNMT_BF16;
    if (a.k_rows == 0) return launch_pdl(bf ? seq_attn_zero_kernel<__nv_bfloat16> : seq_attn_zero_kernel<__half>, (unsigned)((a.q_rows + 7) / 8), 256, 0, st, a);
    if (a.dh <= 64) return bf ? tile_forward<64, true>(a, st) : tile_forward<64, false>(a, st);
    return bf ? tile_forward<128, true>(a, st) : tile_forward<128, false>(a, st);
}

}  // namespace mnmt
