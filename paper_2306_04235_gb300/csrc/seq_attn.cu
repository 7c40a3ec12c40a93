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
constexpr int KT = 64;           // keys of a tile
// BUFS: tiles of scores in TMEM; BLOCKS: CTAs per SM
template <int DH>
struct FwLayout {
    static constexpr int STAGES = DH == 64 ? 4 : 2, QT = sq_bytes<DH>(), TILE = sq_bytes<DH, KT>();
    static constexpr int OFF_K = QT, OFF_V = OFF_K + STAGES * TILE, SMEM = OFF_V + STAGES * TILE + 1024;
    static_assert(2 * STAGES * TILE >= 4 * SQ_INTS, "starts and lengths before keys and values");
    static constexpr int BUFS = DH == 64 ? 3 : 2, T_O = BUFS * KT, COLS = pow2_cols(T_O + DH), BLOCKS = 512 / COLS;
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

template <int DH, bool BF>
__global__ void __launch_bounds__(FW_THREADS, FwLayout<DH>::BLOCKS)
    seq_attn_forward_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                            const SeqAttn a, const float c) {
    using L = FwLayout<DH>;
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    constexpr int ST = L::STAGES, BUFS = L::BUFS;
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[4 * ST + 4 + 2 * BUFS];
    __shared__ uint32_t tslot;
    __shared__ int failed, span[2][4];
    const uint32_t sm = (s_addr(raw) + 1023u) & ~1023u, bar0 = s_addr(bars);
    uint8_t *smp = raw + (sm - s_addr(raw));
    const auto k_full = [&](int s) { return bar0 + 8 * s; };
    const auto k_free = [&](int s) { return bar0 + 8 * (ST + s); };
    const auto v_full = [&](int s) { return bar0 + 8 * (2 * ST + s); };
    const auto v_free = [&](int s) { return bar0 + 8 * (3 * ST + s); };
    const uint32_t q_full = bar0 + 8 * (4 * ST), o_full = q_full + 8, pv_done = q_full + 16, s_full = q_full + 32,
                   p_full = s_full + 8 * BUFS;  // two of pv_done by turns, BUFS of s_full and p_full (a warp may be a tile ahead)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = blockIdx.x % a.hq, tile = (int)(gridDim.x / a.hq) - 1 - (int)(blockIdx.x / a.hq);  // the last rows (causal: the longest) first
    const int row = tile * SQ_ROWS + (int)threadIdx.x;
    if (threadIdx.x == 128) {
        for (int s = 0; s < ST; s++) mbar_init(k_full(s), 1), mbar_init(k_free(s), 1), mbar_init(v_full(s), 1), mbar_init(v_free(s), 1);
        for (int b = 0; b < BUFS; b++) mbar_init(s_full + 8 * b, 1), mbar_init(p_full + 8 * b, 4);
        mbar_init(q_full, 1), mbar_init(o_full, 1), mbar_init(pv_done, 1), mbar_init(pv_done + 8, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) tmem_alloc<L::COLS>(s_addr(&tslot));
    pdl_grid_wait();
    if (threadIdx.x == 128) sq_load<DH>(sm, &tq, h, tile * SQ_ROWS, q_full);
    const SeqAttn ix = seq_shared(a, reinterpret_cast<int *>(smp + L::OFF_K), FW_THREADS);  // where keys and values come later
    Span keys{0, 0};
    bool in = false;
    if (warp < 4) {
        keys = keys_of_query(ix, row, in);
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
        if (nt) {
            const uint32_t on = elect_one();
            const uint64_t qd = sq_k(sm), kd = sq_k(sm + L::OFF_K), vd = sq_mn<KT>(sm + L::OFF_V);
            const auto scores = [&](int j) {  // S(j)
                const int s = j % ST;
                if (!wait(k_full(s), (uint32_t)(j / ST) & 1)) return false;
                tc_fence_after();
                const uint64_t b = kd + (uint64_t)(s * (L::TILE >> 4));
                const uint32_t d = tS + j % BUFS * KT;
#pragma unroll
                for (int k = 0; k < DH / 16; k++) sq_mma(on, d, qd + sq_k_step(k), b + sq_k_step<KT>(k), sq_idesc(KT, BF, false), k > 0);
                f4_commit_on<1>(on, k_free(s));
                f4_commit_on<1>(on, s_full + 8 * (j % BUFS));
                return true;
            };
            bool ok = wait(q_full, 0);
            for (int j = 0; j < BUFS && j < nt && ok; j++) ok = scores(j);
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
                if (j + BUFS < nt && !(ok = scores(j + BUFS))) break;  // MMAs keep their order: P(j) has been read
            }
            f4_commit_on<1>(on, o_full);
            wait(o_full, 0);
        }
        pdl_allow_next();
    } else {
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        float m = -INFINITY, l = 0.0f;  // m: of c s
        bool ok = true;
        for (int j = 0; j < nt; j++) {
            if (!(ok = wait(s_full + 8 * (j % BUFS), (uint32_t)(j / BUFS) & 1))) break;
            tc_fence_after();
            const uint32_t tP = tS + j % BUFS * KT + lanes;
            const int at = end - KT * (j + 1), lo = keys.lo - at, hi = keys.hi - at;
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
            if (__any_sync(0xFFFFFFFFu, top > m + FW_SLACK)) {
                const float mn = top > m + FW_SLACK ? top : m;
                const float f = m == -INFINITY ? 1.0f : exp2_fast(m - mn);  // nothing was added yet: 0 stays 0
                m = mn;
                l *= f;
                if (j > 0 && __any_sync(0xFFFFFFFFu, f != 1.0f)) {
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
    keys_of_query(a, (int)w, in);
    if (!in) return;
    const float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int h = 0; h < a.hq; h++) {
        if (4 * lane < a.dh) store4(static_cast<T *>(a.o.p) + w * a.o.ld + h * a.o.hd + 4 * lane, z);
        if (lane == 0 && a.lse) a.lse[(long)h * a.q_rows + w] = -INFINITY;
    }
}

template <int DH, bool BF>
cudaError_t tile_forward(const SeqAttn &a, cudaStream_t st) {
    CUtensorMap tq, tk, tv;
    if (!sq_map(&tq, a.q, a.q_rows, a.hq, a.dh, SQ_ROWS) || !sq_map(&tk, a.k, a.k_rows, a.hkv, a.dh, KT) || !sq_map(&tv, a.v, a.k_rows, a.hkv, a.dh, KT))
        return cudaErrorInvalidValue;
    const unsigned grid = (unsigned)((a.q_rows + SQ_ROWS - 1) / SQ_ROWS) * (unsigned)a.hq;
    return launch_pdl(seq_attn_forward_kernel<DH, BF>, grid, FW_THREADS, FwLayout<DH>::SMEM, st, tq, tk, tv, a, a.scale * LOG2E);
}

template <int DH, bool BF>
cudaError_t tile_init() {
    return cudaFuncSetAttribute(seq_attn_forward_kernel<DH, BF>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwLayout<DH>::SMEM);
}

}  // namespace

cudaError_t seq_attn_init() {
    cudaError_t e = tile_init<64, true>();
    if (e == cudaSuccess) e = tile_init<64, false>();
    if (e == cudaSuccess) e = tile_init<128, true>();
    if (e == cudaSuccess) e = tile_init<128, false>();
    return e;
}

size_t seq_attn_forward_workspace(const SeqAttn &) { return 16; }

cudaError_t launch_seq_attn_forward(const SeqAttn &a, cudaStream_t st) {
    const bool bf = a.dtype == MNMT_BF16;
    if (a.k_rows == 0) return launch_pdl(bf ? seq_attn_zero_kernel<__nv_bfloat16> : seq_attn_zero_kernel<__half>, (unsigned)((a.q_rows + 7) / 8), 256, 0, st, a);
    if (a.dh <= 64) return bf ? tile_forward<64, true>(a, st) : tile_forward<64, false>(a, st);
    return bf ? tile_forward<128, true>(a, st) : tile_forward<128, false>(a, st);
}

}  // namespace mnmt
