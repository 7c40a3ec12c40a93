// seq_attn.cuh -- softmax attention over sequences whose rows lie one after
// another (include/mnmt.h, mnmt_attention_forward / _backward / _token): the
// shapes its kernels share and the plain loops over one row's own keys.
//
//   s_ij = scale q_i . k_j,  P_ij = exp(s_ij - lse_i),  o_i = sum_j P_ij v_j
//   lse_i = log sum_j exp(s_ij)
//   D_i = do_i . o_i,  dS_ij = P_ij (do_i . v_j - D_i)
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij do_i
//
// The keys that a query sees are one interval of key rows, and the queries that
// see a key one interval of query rows; a mask is a pair of row numbers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "fp4.cuh"
#include "train.h"

namespace mnmt {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Span {
    int lo, hi;  // rows lo .. hi - 1; empty where hi <= lo
};

// the sequence that row may belong to: the last of n that starts at or before it, -1 if none
MNMT_DEV int seq_of(const int *start, int n, int row) {
    int lo = 0, hi = n;  // starts before lo are <= row, from hi on > row
#pragma unroll 1
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= row) lo = mid + 1;
        else hi = mid;
    }
    return lo - 1;
}

// rows of sequence b, whatever the arrays hold within 0 .. rows
MNMT_DEV Span seq_rows(const int *start, const int *len, int b, int rows) {
    const int s = start[b];
    const long e = len ? (long)s + max(len[b], 0) : (long)start[b + 1];
    Span r;
    r.lo = min(max(s, 0), rows);
    r.hi = (int)(e < r.lo ? r.lo : e > rows ? rows : e);
    return r;
}

// b, or the last sequence before it that has rows where it has none (with lengths given, a sequence without rows may start at or
// among another's; 0 if there is none).  Whole warps, 256 lengths at a look: rows behind the last sequence of a batch with room for
// more go back over all that are not used (128 sentences in a batch for 1000, forward: step by step 64 us, so 20).
MNMT_DEV int last_with_rows(const int *len, int b) {
    if (!len) return b;
    const int lane = threadIdx.x & 31;
    bool need = b > 0 && len[b] <= 0;
    for (uint32_t todo; (todo = __ballot_sync(0xFFFFFFFFu, need)) != 0;) {
        const int from = __shfl_sync(0xFFFFFFFFu, b, __ffs(todo) - 1);
        int x = from, at = -1;  // no rows from x to from
        while (x > 0 && at < 0) {
            bool some[8];
#pragma unroll
            for (int i = 0; i < 8; i++) some[i] = len[max(x - 1 - 32 * i - lane, 0)] > 0 && x - 1 - 32 * i - lane >= 0;
#pragma unroll
            for (int i = 7; i >= 0; i--) {
                const uint32_t m = __ballot_sync(0xFFFFFFFFu, some[i]);
                if (m) at = x - 32 * i - __ffs(m);
            }
            x -= 256;
        }
        at = max(at, 0);
        if (need && b <= from && b > at) b = at, need = false;
    }
    return b;
}

// the keys that query row sees (b: as last_with_rows after seq_of; in: whether it belongs to a sequence at all; few: whether the rows of its
// sequence that see a key see 10 of them or fewer on average)
MNMT_DEV Span keys_of_query(const SeqAttn &a, int row, int b, bool &in, bool &few) {
    in = few = false;
    if (b < 0) return Span{0, 0};
    const Span q = seq_rows(a.q_start, a.q_len, b, a.q_rows);
    if (row >= q.hi) return Span{0, 0};
    in = true;
    Span k = seq_rows(a.k_start, a.k_len, b, a.k_rows);
    const int nk = k.hi - k.lo;
    few = nk <= 20 && 2 * nk - (a.causal ? min(q.hi - q.lo, nk) - 1 : 0) <= 20;
    if (a.causal) k.hi = min(k.hi, k.hi - (q.hi - 1 - row));  // the last query sees all keys
    if (k.hi < k.lo) k.hi = k.lo;
    return k;
}

// the queries that see key row (one: they see no other key)
MNMT_DEV Span queries_of_key(const SeqAttn &a, int row, int b, bool &in, bool &one) {
    in = one = false;
    if (b < 0) return Span{0, 0};
    const Span k = seq_rows(a.k_start, a.k_len, b, a.k_rows);
    if (row >= k.hi) return Span{0, 0};
    in = true;
    one = k.hi - k.lo == 1;
    Span q = seq_rows(a.q_start, a.q_len, b, a.q_rows);
    if (a.causal) q.lo = max(q.lo, q.hi - (k.hi - row));
    if (q.hi < q.lo) q.hi = q.lo;
    return q;
}

// The starts and lengths of up to SQ_SEQS sequences in shared memory (buf: SQ_INTS words), so
// that finding a row's sequence waits for global memory once: every step of a search there
// took 0.7 us, the search of a block 2.4 to 2.8.  More sequences are looked up where they are.
// All threads of the block; ends with a barrier.
constexpr int SQ_SEQS = 1024, SQ_INTS = 4 * (SQ_SEQS + 1);
MNMT_DEV SeqAttn seq_shared(const SeqAttn &a, int *buf, int threads) {
    SeqAttn s = a;
    if (a.n_seqs <= SQ_SEQS) {
        const int nq = a.n_seqs + (a.q_len ? 0 : 1), nk = a.n_seqs + (a.k_len ? 0 : 1);
        int *qs = buf, *ql = qs + SQ_SEQS + 1, *ks = ql + SQ_SEQS + 1, *kl = ks + SQ_SEQS + 1;
        for (int i = threadIdx.x; i <= a.n_seqs; i += threads) {
            if (i < nq) qs[i] = a.q_start[i];
            if (i < nk) ks[i] = a.k_start[i];
            if (a.q_len && i < a.n_seqs) ql[i] = a.q_len[i];
            if (a.k_len && i < a.n_seqs) kl[i] = a.k_len[i];
        }
        s.q_start = qs, s.k_start = ks;
        s.q_len = a.q_len ? ql : nullptr, s.k_len = a.k_len ? kl : nullptr;
    }
    __syncthreads();
    return s;
}
// The sequences of 32 rows, row0 + lane, by a whole warp.  Of up to 1024 starts the first row
// takes two comparisons (every 32nd start, then 32 of them); the rows behind it count the
// starts among them, as bits of a word.  More starts, or sequences without rows, are searched
// lane by lane.  Few instructions count here: they run once a block, from a cold cache (with
// searches by shuffles 1.2 us).
MNMT_DEV int seq_of_lane(const int *start, int n, int row0) {
    const int lane = threadIdx.x & 31;
    if (n <= SQ_SEQS) {
        const auto at = [&](int i) { return i < n ? start[i] : 0x7FFFFFFF; };
        const int block = 32 * max(0, __popc(__ballot_sync(0xFFFFFFFFu, at(32 * lane) <= row0)) - 1);  // starts 0, 32, .. that are <= row0
        const int lo = block + __popc(__ballot_sync(0xFFFFFFFFu, at(block + lane) <= row0));
        const int d = at(lo + lane) - row0;  // > 0: the next 32 starts
        const uint32_t among = __reduce_or_sync(0xFFFFFFFFu, d < 32 ? 1u << d : 0u);
        if (__popc(among) == __popc(__ballot_sync(0xFFFFFFFFu, d < 32))) return lo - 1 + __popc(among & (0xFFFFFFFFu >> (31 - lane)));
    }
    return seq_of(start, n, row0 + lane);
}

// the keys that query row0 + lane sees, and the queries that see key row0 + lane; whole warps
MNMT_DEV Span keys_of_lane(const SeqAttn &a, int row0, bool &in, bool &few) {
    const int row = row0 + (threadIdx.x & 31), b = row0 < a.q_rows ? last_with_rows(a.q_len, seq_of_lane(a.q_start, a.n_seqs, row0)) : -1;
    return keys_of_query(a, row, row < a.q_rows ? b : -1, in, few);
}
MNMT_DEV Span queries_of_lane(const SeqAttn &a, int row0, bool &in, bool &one) {
    const int row = row0 + (threadIdx.x & 31), b = row0 < a.k_rows ? last_with_rows(a.k_len, seq_of_lane(a.k_start, a.n_seqs, row0)) : -1;
    return queries_of_key(a, row, row < a.k_rows ? b : -1, in, one);
}

MNMT_DEV float warp_sum_f(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// How far below a row's largest score its weights' reference lies, in powers of two: fp16 weights are
// taken 2^7 larger, as far as 65504 allows beside a slack of 2^8, and reach as much further down.
template <bool BF>
__host__ __device__ constexpr float weight_lift() { return BF ? 0.0f : 7.0f; }

// 2^x to within 2 ulp, 0 below -126
MNMT_DEV float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// dot product of dh elements (a multiple of 8) of two rows on 16 bytes
template <typename T>
MNMT_DEV float row_dot(const T *x, const T *y, int dh) {
    float s = 0.0f;
    for (int c = 0; c < dh; c += 8) {
        float u[8], v[8];
        load8<T, true>(x + c, 8, u);
        load8<T, true>(y + c, 8, v);
#pragma unroll
        for (int i = 0; i < 8; i++) s = fmaf(u[i], v[i], s);
    }
    return s;
}

// four elements of a row, 8-byte aligned
template <typename T>
MNMT_DEV void load4(const T *p, float (&v)[4]) {
    const uint2 w = *reinterpret_cast<const uint2 *>(p);
    if constexpr (std::is_same_v<T, __half>) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&w.x)), b = __half22float2(*reinterpret_cast<const __half2 *>(&w.y));
        v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
    } else {
        v[0] = __uint_as_float(w.x << 16), v[1] = __uint_as_float(w.x & 0xFFFF0000u);
        v[2] = __uint_as_float(w.y << 16), v[3] = __uint_as_float(w.y & 0xFFFF0000u);
    }
}
template <typename T>
MNMT_DEV void store4(T *p, const float (&v)[4]) {
    uint2 w;
    T *t = reinterpret_cast<T *>(&w);
#pragma unroll
    for (int i = 0; i < 4; i++) t[i] = from_f32<T>(v[i]);
    *reinterpret_cast<uint2 *>(p) = w;
}

// One query row by a warp: lane l holds elements 4 l .. 4 l + 3 of the sum (dh <= 128).
// m: the largest score times log2 e, l: sum of 2^(s - m), over keys k.lo .. k.hi - 1.
struct RowSum {
    float m, l, acc[4];
};
template <typename T>
__device__ __noinline__ RowSum attn_row(const T *q, const T *k, long ldk, const T *v, long ldv, Span s, int dh, float c) {
    const int lane = threadIdx.x & 31;
    RowSum r{-INFINITY, 0.0f, {0.0f, 0.0f, 0.0f, 0.0f}};
    for (int j0 = s.lo; j0 < s.hi; j0 += 32) {
        const int j = j0 + lane;
        const bool on = j < s.hi;
        const float x = on ? row_dot(q, k + j * ldk, dh) * c : -INFINITY;
        const float mn = fmaxf(r.m, warp_max_f(x)), mu = mn == -INFINITY ? 0.0f : mn;
        const float p = on ? exp2_fast(x - mu) : 0.0f, alpha = exp2_fast(r.m - mu);
        r.m = mn;
        r.l = fmaf(r.l, alpha, warp_sum_f(p));
#pragma unroll
        for (int i = 0; i < 4; i++) r.acc[i] *= alpha;
        const int n = min(32, s.hi - j0);
        for (int t = 0; t < n; t++) {
            const float pt = __shfl_sync(0xFFFFFFFFu, p, t);
            if (4 * lane < dh) {
                float w[4];
                load4(v + (j0 + t) * ldv + 4 * lane, w);
#pragma unroll
                for (int i = 0; i < 4; i++) r.acc[i] = fmaf(pt, w[i], r.acc[i]);
            }
        }
    }
    return r;
}
// log-sum-exp of a row
MNMT_DEV float row_lse(float m, float l) { return fmaf(m, LN2, logf(l)); }

// dq of one query row (without the scale): lane l holds elements 4 l .. 4 l + 3
template <typename T>
__device__ __noinline__ float4 attn_row_dq(const T *q, const T *g, float lse2, float delta, const T *k, long ldk, const T *v, long ldv, Span s, int dh,
                                           float c) {
    const int lane = threadIdx.x & 31;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int j0 = s.lo; j0 < s.hi; j0 += 32) {
        const int j = j0 + lane;
        float ds = 0.0f;
        if (j < s.hi) {
            const float p = exp2_fast(fmaf(row_dot(q, k + j * ldk, dh), c, -lse2));
            ds = p * (row_dot(g, v + j * ldv, dh) - delta);
        }
        const int n = min(32, s.hi - j0);
        for (int t = 0; t < n; t++) {
            const float d = __shfl_sync(0xFFFFFFFFu, ds, t);
            if (4 * lane < dh) {
                float w[4];
                load4(k + (j0 + t) * ldk + 4 * lane, w);
#pragma unroll
                for (int i = 0; i < 4; i++) acc[i] = fmaf(d, w[i], acc[i]);
            }
        }
    }
    return make_float4(acc[0], acc[1], acc[2], acc[3]);
}

// dk (without the scale) and dv of one key row from one query head, added to dk and dv
template <typename T>
__device__ __noinline__ void attn_row_dkv(const T *k, const T *v, const T *q, long ldq, const T *g, long ldg, const float *lse, const float *delta, Span s,
                                          int dh, float c, float (&dk)[4], float (&dv)[4]) {
    const int lane = threadIdx.x & 31;
    for (int i0 = s.lo; i0 < s.hi; i0 += 32) {
        const int i = i0 + lane;
        float p = 0.0f, ds = 0.0f;
        if (i < s.hi) {
            p = exp2_fast(fmaf(row_dot(q + i * ldq, k, dh), c, -lse[i] * LOG2E));
            ds = p * (row_dot(g + i * ldg, v, dh) - delta[i]);
        }
        const int n = min(32, s.hi - i0);
        for (int t = 0; t < n; t++) {
            const float pt = __shfl_sync(0xFFFFFFFFu, p, t), dt = __shfl_sync(0xFFFFFFFFu, ds, t);
            if (4 * lane < dh) {
                float w[4], u[4];
                load4(q + (i0 + t) * ldq + 4 * lane, w);
                load4(g + (i0 + t) * ldg + 4 * lane, u);
#pragma unroll
                for (int e = 0; e < 4; e++) dk[e] = fmaf(dt, w[e], dk[e]), dv[e] = fmaf(pt, u[e], dv[e]);
            }
        }
    }
}

}  // namespace mnmt
