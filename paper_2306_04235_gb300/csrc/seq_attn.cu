// seq_attn.cu -- attention over sequences, forward (seq_attn.cuh).
//
// A CTA takes 128 query rows of one head, whatever sequences they belong to: the
// keys that a row sees are an interval of key rows, and the tile walks 128 keys at
// a time through the union of its rows' intervals, from its end backwards, so that
// no tile reaches past the last key that a row sees (what lies there, unwritten
// rows for instance, would meet zero weights, and zero times NaN is NaN).
//   S = Q K^T (TMEM), one thread per row: P = 2^(c s - m), c = scale log2 e, with the
//   running maximum m and sum l; P over S in TMEM, in the operands' type; O += P V.
// m is moved, and O scaled, only where a score exceeds it by 2^8 (the sum and the
// result carry the same factor, so any m near the maximum serves).
// Two CTAs per SM, so that the tensor core works for one while the other's threads
// take powers.
// Where O of a row is not finite though its sum is, an infinity or a NaN of a key
// that the row does not see may have come in: such rows are computed again over
// their own keys alone (attn_row).
#include "seq_tile.cuh"

namespace mnmt {
namespace {

constexpr int FW_THREADS = 192;  // four softmax warps, a TMA warp, an MMA warp
// KT: keys of a tile; BLOCKS: CTAs per SM
template <int DH, int KT>
struct FwLayout {
    static constexpr int STAGES = 2, QT = sq_bytes<DH>(), TILE = sq_bytes<DH, KT>();
    static constexpr int OFF_K = QT, OFF_V = OFF_K + STAGES * TILE, SMEM = OFF_V + STAGES * TILE + 1024;
    static constexpr bool APART = DH + KT > 128;  // P beside S
    static constexpr int T_P = APART ? KT : 0, T_O = KT + (APART ? KT / 2 : 0), COLS = pow2_cols(T_O + DH), BLOCKS = 512 / COLS;
};
constexpr float FW_SLACK = 8.0f;  // how far, in powers of two, a score may exceed m

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

template <int DH, bool BF, int KT>
__global__ void __launch_bounds__(FW_THREADS, FwLayout<DH, KT>::BLOCKS)
    seq_attn_forward_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                            const SeqAttn a, const float c) {
    using L = FwLayout<DH, KT>;
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    constexpr int ST = L::STAGES;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[4 * ST + 6];
    __shared__ uint32_t tslot;
    __shared__ int failed, span[2][4];
    const uint32_t sm = (s_addr(raw) + 1023u) & ~1023u, bar0 = s_addr(bars);
    uint8_t *smp = raw + (sm - s_addr(raw));
    const auto k_full = [&](int s) { return bar0 + 8 * s; };
    const auto k_free = [&](int s) { return bar0 + 8 * (ST + s); };
    const auto v_full = [&](int s) { return bar0 + 8 * (2 * ST + s); };
    const auto v_free = [&](int s) { return bar0 + 8 * (3 * ST + s); };
    const uint32_t q_full = bar0 + 8 * (4 * ST), s_full = q_full + 8, p_full = q_full + 16, o_full = q_full + 24, s_read = q_full + 32,
                   pv_done = q_full + 40;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = blockIdx.x % a.hq, tile = (int)(gridDim.x / a.hq) - 1 - (int)(blockIdx.x / a.hq);  // the last rows (causal: the longest) first
    const int row = tile * SQ_ROWS + (int)threadIdx.x;
    if (threadIdx.x == 128) {
        for (int s = 0; s < ST; s++) mbar_init(k_full(s), 1), mbar_init(k_free(s), 1), mbar_init(v_full(s), 1), mbar_init(v_free(s), 1);
        mbar_init(q_full, 1), mbar_init(s_full, 1), mbar_init(p_full, 4), mbar_init(o_full, 1), mbar_init(s_read, 4),
            mbar_init(pv_done, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) tmem_alloc<L::COLS>(s_addr(&tslot));
    pdl_grid_wait();
    if (threadIdx.x == 128) sq_load<DH>(sm, &tq, h, tile * SQ_ROWS, q_full);
    Span keys{0, 0};
    bool in = false;
    if (warp < 4) {
        keys = keys_of_lane(a, row - lane, in);
        const bool some = keys.hi > keys.lo;
        const int lo = __reduce_min_sync(0xFFFFFFFFu, some ? keys.lo : 0x7FFFFFFF), hi = __reduce_max_sync(0xFFFFFFFFu, some ? keys.hi : 0);
        if (lane == 0) span[0][warp] = lo, span[1][warp] = hi;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tS = tslot, tP = tslot + L::T_P, tO = tslot + L::T_O;
    const int first = min(min(span[0][0], span[0][1]), min(span[0][2], span[0][3])), end = max(max(span[1][0], span[1][1]), max(span[1][2], span[1][3]));
    const int nt = end > first ? (end - first + KT - 1) / KT : 0;
    const SqWaits wait{&failed, a.status};

    if (warp == 4) {
        if (lane == 0) {
            const int hk = h / a.group();
            int j = 0;
            for (; j < nt; j++) {
                const int s = j % ST, at = end - KT * (j + 1);
                const uint32_t ph = (uint32_t)(j / ST - 1) & 1;
                if (j >= ST && !wait(k_free(s), ph)) break;
                sq_load<DH, KT>(sm + L::OFF_K + s * L::TILE, &tk, hk, at, k_full(s));
                if (j >= ST && !wait(v_free(s), ph)) {
                    wait(k_full(s), (uint32_t)(j / ST) & 1);  // in flight
                    break;
                }
                sq_load<DH, KT>(sm + L::OFF_V + s * L::TILE, &tv, hk, at, v_full(s));
            }
            if (failed || nt == 0) {  // copies in flight land before the block ends
                wait(q_full, 0);
                for (int i = max(0, j - ST); i < j; i++) wait(k_full(i % ST), (uint32_t)(i / ST) & 1), wait(v_full(i % ST), (uint32_t)(i / ST) & 1);
            }
        }
    } else if (warp == 5) {
        if (lane == 0 && nt) {
            const auto scores = [&](int j) {  // S(j)
                const int s = j % ST;
                if (!wait(k_full(s), (uint32_t)(j / ST) & 1)) return false;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < DH / 16; k++)
                    mma_f16(tS, sq_k(sm, k), sq_k<KT>(sm + L::OFF_K + s * L::TILE, k), sq_idesc(KT, BF, false), k > 0);
                mma_commit(k_free(s));
                mma_commit(s_full);
                return true;
            };
            bool ok = wait(q_full, 0) && scores(0);
            for (int j = 0; j < nt && ok; j++) {
                const int s = j % ST;
                if (L::APART && j + 1 < nt && !(ok = wait(s_read, (uint32_t)j & 1) && scores(j + 1))) break;
                if (!(ok = wait(p_full, (uint32_t)j & 1) && wait(v_full(s), (uint32_t)(j / ST) & 1))) break;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < KT / 16; k++)
                    mma_f16_ta(tO, tP + 8 * k, sq_mn<KT>(sm + L::OFF_V + s * L::TILE, k), sq_idesc(DH, BF, true), (uint32_t)(j | k));
                mma_commit(v_free(s));
                if (L::APART) mma_commit(pv_done);
                if (!L::APART && j + 1 < nt && !(ok = scores(j + 1))) break;  // MMAs keep their order: P(j) has been read
            }
            mma_commit(o_full);
            wait(o_full, 0);
        }
        pdl_allow_next();
    } else {
        constexpr bool HOLD = L::APART;  // registers for a row of scores; else they are read twice
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        float m = -INFINITY, l = 0.0f;  // m: of c s
        bool ok = true;
        for (int j = 0; j < nt; j++) {
            if (!(ok = wait(s_full, (uint32_t)j & 1))) break;
            tc_fence_after();
            const int at = end - KT * (j + 1), lo = keys.lo - at, hi = keys.hi - at;
            const bool all = __all_sync(0xFFFFFFFFu, lo <= 0 && hi >= KT);
            // the products of P(j - 1) are in O, and P is free (over S: S(j) came after them)
            const auto last_done = [&] { return !L::APART || j == 0 || wait(pv_done, (uint32_t)(j - 1) & 1); };
            const auto p_ready = [&] {
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full);
            };
            if (!__any_sync(0xFFFFFFFFu, hi > 0 && lo < KT)) {  // no row of the warp sees a key of the tile
                if (L::APART && lane == 0) mbar_arrive(s_read);
                if (!(ok = last_done())) break;
                const uint32_t zeros[16] = {};
#pragma unroll
                for (int b = 0; b < KT / 32; b++) tmem_st16(tP + lanes + 16 * b, zeros);
                p_ready();
                continue;
            }
            uint32_t r[HOLD ? KT / 32 : 1][32];
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if constexpr (HOLD) {
#pragma unroll
                for (int b = 0; b < KT / 32; b++) tmem_ld32(tS + lanes + 32 * b, r[b]);
                tmem_wait_ld();
                if (L::APART) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(s_read);
                }
                if (!all) {
#pragma unroll
                    for (int b = 0; b < KT / 32; b++) hide(r[b], sq_bits(lo - 32 * b, hi - 32 * b));
                }
#pragma unroll
                for (int b = 0; b < KT / 32; b++) max32(r[b], mx);
            } else {
#pragma unroll
                for (int b = 0; b < KT / 32; b++) {
                    tmem_ld32(tS + lanes + 32 * b, r[0]);
                    tmem_wait_ld();
                    if (!all) hide(r[0], sq_bits(lo - 32 * b, hi - 32 * b));
                    max32(r[0], mx);
                }
            }
            const float top = c * fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
            if (!(ok = last_done())) break;
            tc_fence_after();
            // the first scores, or scores that 2^8 does not hold
            if (__any_sync(0xFFFFFFFFu, top > m + FW_SLACK)) {
                const float mn = top > m + FW_SLACK ? top : m;
                const float f = m == -INFINITY ? 1.0f : exp2_fast(m - mn);  // nothing was added yet: 0 stays 0
                m = mn;
                l *= f;
                if (j > 0 && __any_sync(0xFFFFFFFFu, f != 1.0f)) {
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
                if constexpr (HOLD) {
                    weigh<BF>(r[b], c2, m2, ls, p);
                } else {
                    tmem_ld32(tS + lanes + 32 * b, r[0]);
                    tmem_wait_ld();
                    if (!all) hide(r[0], sq_bits(lo - 32 * b, hi - 32 * b));
                    weigh<BF>(r[0], c2, m2, ls, p);
                }
                tmem_st16(tP + lanes + 16 * b, p);  // over S: scores that were read
            }
            float la, lb;
            f4_untwo(ls, la, lb);
            l += la + lb;
            p_ready();
        }
        ok = wait(nt ? o_full : q_full, 0) && ok;
        tc_fence_after();
        // no tile and no key: zeros; a sum of nothing but zeros is not a number, as 0 / 0
        const bool none = keys.hi <= keys.lo;
        const float inv = none ? 0.0f : 1.0f / l;
        bool odd = false;
        if (ok) {
            uint32_t out[DH / 2];
#pragma unroll
            for (int b = 0; b < DH / 32; b++) {
                uint32_t w[32];
                if (nt) tmem_ld32(tO + lanes + 32 * b, w);
                tmem_wait_ld();
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; i++) {
                    const float x = nt ? __uint_as_float(w[i]) : 0.0f;
                    odd |= !(fabsf(x) < INFINITY);
                    v[i] = none ? 0.0f : x * inv;
                }
#pragma unroll
                for (int i = 0; i < 16; i++) out[16 * b + i] = sq_pack<BF>(v[2 * i], v[2 * i + 1]);
            }
            // the queries have been multiplied: their rows are free
            sq_store_rows<DH>(smp + warp * (64 * DH), out, static_cast<uint16_t *>(a.o.p) + (long)(row - lane) * a.o.ld + h * a.o.hd, a.o.ld,
                              __ballot_sync(0xFFFFFFFFu, in), a.dh);
            if (in && a.lse) a.lse[(long)h * a.q_rows + row] = none ? -INFINITY : row_lse(m, l);
            const int hk = h / a.group();
            for (uint32_t again = __ballot_sync(0xFFFFFFFFu, in && !none && odd && fabsf(l) < INFINITY); again; again &= again - 1) {
                const int src = __ffs(again) - 1, rr = __shfl_sync(0xFFFFFFFFu, row, src);
                const Span s{__shfl_sync(0xFFFFFFFFu, keys.lo, src), __shfl_sync(0xFFFFFFFFu, keys.hi, src)};
                const RowSum x = attn_row(static_cast<const T *>(a.q.p) + rr * a.q.ld + h * a.q.hd, static_cast<const T *>(a.k.p) + hk * a.k.hd, a.k.ld,
                                          static_cast<const T *>(a.v.p) + hk * a.v.hd, a.v.ld, s, a.dh, c);
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] = x.acc[i] / x.l;
                if (4 * lane < a.dh) store4(static_cast<T *>(a.o.p) + rr * a.o.ld + h * a.o.hd + 4 * lane, v);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) tmem_free<L::COLS>(tslot);
}

// Where there are no keys at all, rows of sequences are zeros.
template <typename T>
__global__ void __launch_bounds__(256) seq_attn_zero_kernel(SeqAttn a) {
    pdl_grid_wait();
    const long w = ((long)blockIdx.x * 256 + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    bool in;
    if (w >= a.q_rows) return;
    keys_of_query(a, (int)w, seq_of(a.q_start, a.n_seqs, (int)w), in);
    if (!in) return;
    const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int h = 0; h < a.hq; h++) {
        if (4 * lane < a.dh) store4(static_cast<T *>(a.o.p) + w * a.o.ld + h * a.o.hd + 4 * lane, z);
        if (lane == 0 && a.lse) a.lse[(long)h * a.q_rows + w] = -INFINITY;
    }
}

template <int DH, bool BF, int KT>
cudaError_t tile_forward(const SeqAttn &a, cudaStream_t st) {
    CUtensorMap tq, tk, tv;
    if (!sq_map(&tq, a.q, a.q_rows, a.hq, a.dh, SQ_ROWS) || !sq_map(&tk, a.k, a.k_rows, a.hkv, a.dh, KT) || !sq_map(&tv, a.v, a.k_rows, a.hkv, a.dh, KT))
        return cudaErrorInvalidValue;
    const unsigned grid = (unsigned)((a.q_rows + SQ_ROWS - 1) / SQ_ROWS) * (unsigned)a.hq;
    return launch_pdl(seq_attn_forward_kernel<DH, BF, KT>, grid, FW_THREADS, FwLayout<DH, KT>::SMEM, st, tq, tk, tv, a, a.scale * LOG2E);
}

template <int DH, int KT>
cudaError_t tile_init() {
    const cudaError_t e = cudaFuncSetAttribute(seq_attn_forward_kernel<DH, true, KT>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwLayout<DH, KT>::SMEM);
    return e != cudaSuccess ? e
                            : cudaFuncSetAttribute(seq_attn_forward_kernel<DH, false, KT>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwLayout<DH, KT>::SMEM);
}

}  // namespace

cudaError_t seq_attn_init() {
    cudaError_t e = tile_init<64, 64>();
    if (e == cudaSuccess) e = tile_init<64, 128>();
    if (e == cudaSuccess) e = tile_init<128, 64>();
    return e;
}

size_t seq_attn_forward_workspace(const SeqAttn &) { return 16; }

cudaError_t launch_seq_attn_forward(const SeqAttn &a, cudaStream_t st) {
    const bool bf = a.dtype == MNMT_BF16;
    if (a.k_rows == 0) return launch_pdl(bf ? seq_attn_zero_kernel<__nv_bfloat16> : seq_attn_zero_kernel<__half>, (unsigned)((a.q_rows + 7) / 8), 256, 0, st, a);
    if (a.dh > 64) return bf ? tile_forward<128, true, 64>(a, st) : tile_forward<128, false, 64>(a, st);
    // Tiles of 64 keys, four CTAs per SM, where sequences are short: 64 x 200 rows of 8 heads 25 us (128 keys: 29),
    // one of 46 rows 5.3 (5.9).  Not where CTAs are few (4 x 512: 13.8, 128 keys 10.9) or walks long (8192
    // causal rows 186, 112: all CTAs are on the card at once, and SMs with long walks are waited for).
    const long keys = a.n_seqs ? a.k_rows / a.n_seqs : 0, ctas = (a.q_rows + SQ_ROWS - 1L) / SQ_ROWS * a.hq;
    if (keys <= 64 || (keys < 1024 && ctas > 2 * 152)) return bf ? tile_forward<64, true, 64>(a, st) : tile_forward<64, false, 64>(a, st);
    return bf ? tile_forward<64, true, 128>(a, st) : tile_forward<64, false, 128>(a, st);
}

}  // namespace mnmt
