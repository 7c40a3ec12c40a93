// seq_attn_token.cu -- attention of one query per sequence against a cache
// (include/mnmt.h, mnmt_attention_token): bound by the bytes of keys and values.
//
// A warp works alone on a run of keys of one (sequence, key head): the up to 16 query
// heads that share them are the 16 rows of an mma.sync tile (a product of 16 rows is
// never bound by the tensor core, so the instruction that needs no tensor memory
// serves).  Keys and values come 16 bytes a lane by cp.async into the warp's own ring,
// three stages of 8 KB; rows past the run's end are filled with zeros, so that nothing
// behind a cache's filled part is read.
//   S = Q K^T, P = 2^(c S - m), O += P V with the running maximum m and sum l.
// Few long sequences (units = sequences x key heads x groups of 16 heads below two
// per warp of the card): all tiles of all units are cut into equal runs, one per warp,
// whatever unit they belong to; units that were cut are joined by a second kernel in
// the order of their runs.  Many: a warp per unit, one launch, however long a single unit is.
// 12 sequences of 9000..32768 keys of 4 heads of 128: 93 us, 5.9 TB/s (86 % of measured), of which the join 9; 512 of 80..160
// keys of 8 heads of 64: 24.6 us, 5.2 TB/s (3.4 rounds of warps); 4 of 30..34 keys: 3.2 us, a launch.  Bound by bytes in
// flight: 192 KB of rings per SM; rings of half the stages and twice the warps were no faster (23.7 and 94 us).
#include "seq_attn.cuh"

namespace mnmt {
namespace {

constexpr int TK_WARPS = 4, TK_STAGES = 3, TK_STAGE = 8192;  // bytes of a stage: keys, then values
constexpr int TK_SMEM = TK_WARPS * TK_STAGES * TK_STAGE;
constexpr int TK_BLOCKS = 2;          // per SM
constexpr int TK_GRID = 152 * TK_BLOCKS;  // blocks that cut units (a constant: sizes of workspaces are asked for without a device)
constexpr int TK_MIN_RUN = 4;         // tiles of a run at least
constexpr int TK_SPLIT_ROWS = 512;    // key rows in memory from which a cut is worth a second launch
constexpr float TK_SLACK = 8.0f;      // how far, in powers of two, a score may exceed m and its type's lift (weight_lift)
template <int DH>
__host__ __device__ constexpr int tk_keys() { return TK_STAGE / (4 * DH); }  // keys of a tile

// What a run leaves of a unit that was cut: [rows][DH] sums, then m and l of each row
template <int DH>
__host__ __device__ constexpr size_t tk_slot(int rows) { return (size_t)rows * (DH + 2); }

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
template <bool BF>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (BF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool BF>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    if constexpr (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// unit u: sequence b, key head hk, query heads from h on, n of them
struct Unit {
    int b, hk, h, n;
};
__device__ __forceinline__ Unit unit_of(const SeqAttn &a, int chunks, long u) {
    const int per = a.hkv * chunks, r = (int)(u % per), i = r % chunks;
    Unit x;
    x.b = (int)(u / per), x.hk = r / chunks, x.h = x.hk * a.group() + 16 * i, x.n = min(16, a.group() - 16 * i);
    return x;
}

// The 16 rows of a warp's tile after keys k.lo .. k.hi - 1: lane t of four holds columns
// 8 i + 2 t, + 1 of rows lane / 4 (o[i][0..1]) and lane / 4 + 8 (o[i][2..3])
template <int DH>
struct RunSum {
    float o[DH / 8][4], m[2], l[2];
};

template <int DH, bool BF>
__device__ __forceinline__ void run_keys(const SeqAttn &a, const Unit &u, Span keys, float c, uint32_t ring, RunSum<DH> &r) {
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    constexpr int KT = tk_keys<DH>(), CH = DH / 8, V_OFF = TK_STAGE / 2;  // keys of a tile, 16-byte pieces of a row
    const int lane = threadIdx.x & 31, t = lane & 3;
    const int nt = (keys.hi - keys.lo + KT - 1) / KT;
    // a lane copies piece `pc` of rows pr, pr + 32 / CH, ... ; pieces are stored at piece ^ (row % 8)
    const int pc = lane % CH, pr = lane / CH;
    const T *kp = static_cast<const T *>(a.k.p) + u.hk * a.k.hd + 8 * pc, *vp = static_cast<const T *>(a.v.p) + u.hk * a.v.hd + 8 * pc;
    const auto load = [&](int i) {
        if (i < nt && 8 * pc < a.dh) {
            const uint32_t st = ring + (i % TK_STAGES) * TK_STAGE;
            const int k0 = keys.lo + i * KT;
#pragma unroll
            for (int x = 0; x < KT * CH / 32; x++) {
                const int rr = pr + x * (32 / CH), key = k0 + rr;
                const bool on = key < keys.hi;
                const uint32_t at = st + rr * (DH * 2) + 16 * ((pc & ~7) | ((pc ^ rr) & 7));
                cp16(at, kp + (on ? key * a.k.ld : 0), on);
                cp16(at + V_OFF, vp + (on ? key * a.v.ld : 0), on);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < TK_STAGES - 1; i++) load(i);
    // the queries as an A operand
    uint32_t q[DH / 16][4];
    {
        const T *qp = static_cast<const T *>(a.q.p) + u.b * a.q.ld + u.h * a.q.hd;
#pragma unroll
        for (int k = 0; k < DH / 16; k++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int row = (lane >> 2) + 8 * (e & 1), col = 16 * k + 2 * t + 8 * (e >> 1);
                q[k][e] = row < u.n && col < a.dh ? *reinterpret_cast<const uint32_t *>(qp + row * a.q.hd + col) : 0u;
            }
    }
#pragma unroll
    for (int i = 0; i < DH / 8; i++)
#pragma unroll
        for (int e = 0; e < 4; e++) r.o[i][e] = 0.0f;
    r.m[0] = r.m[1] = -INFINITY, r.l[0] = r.l[1] = 0.0f;
    for (int i = 0; i < nt; i++) {
        load(i + TK_STAGES - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(TK_STAGES - 1) : "memory");
        __syncwarp();
        const uint32_t st = ring + (i % TK_STAGES) * TK_STAGE;
        float s[KT / 8][4];
#pragma unroll
        for (int j = 0; j < KT / 8; j++) {
#pragma unroll
            for (int e = 0; e < 4; e++) s[j][e] = 0.0f;
            const int rr = 8 * j + (lane & 7);
#pragma unroll
            for (int k = 0; k < DH / 16; k += 2) {
                const int p = 2 * k + (lane >> 3);
                uint32_t b[4];
                ldsm4(st + rr * (DH * 2) + 16 * ((p & ~7) | ((p ^ rr) & 7)), b);
                mma16<BF>(s[j], q[k], b[0], b[1]);
                mma16<BF>(s[j], q[k + 1], b[2], b[3]);
            }
        }
        const int left = keys.hi - (keys.lo + i * KT);
        if (left < KT) {
#pragma unroll
            for (int j = 0; j < KT / 8; j++)
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (8 * j + 2 * t + (e & 1) >= left) s[j][e] = -INFINITY;
        }
#pragma unroll
        for (int x = 0; x < 2; x++) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < KT / 8; j++) top = fmaxf(top, fmaxf(s[j][2 * x], s[j][2 * x + 1]));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = c * fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            constexpr float LIFT = weight_lift<BF>();
            if (__any_sync(0xFFFFFFFFu, top > r.m[x] + (LIFT + TK_SLACK))) {
                const float mn = top > r.m[x] + (LIFT + TK_SLACK) ? top - LIFT : r.m[x], f = r.m[x] == -INFINITY ? 1.0f : exp2_fast(r.m[x] - mn);
                r.m[x] = mn;
                r.l[x] *= f;
#pragma unroll
                for (int n = 0; n < DH / 8; n++) r.o[n][2 * x] *= f, r.o[n][2 * x + 1] *= f;
            }
            const float mu = r.m[x] == -INFINITY ? 0.0f : r.m[x];
#pragma unroll
            for (int j = 0; j < KT / 8; j++) {
                s[j][2 * x] = exp2_fast(fmaf(s[j][2 * x], c, -mu));
                s[j][2 * x + 1] = exp2_fast(fmaf(s[j][2 * x + 1], c, -mu));
                r.l[x] += s[j][2 * x] + s[j][2 * x + 1];
            }
        }
        uint32_t p[KT / 16][4];
#pragma unroll
        for (int k = 0; k < KT / 16; k++)
#pragma unroll
            for (int e = 0; e < 4; e++) p[k][e] = pack2<BF>(s[2 * k + (e >> 1)][2 * (e & 1)], s[2 * k + (e >> 1)][2 * (e & 1) + 1]);
        // A tile's products from zero, then added: the tensor core truncates what it adds, which over a long walk
        // made sums small (65536 keys 4e-4 of o, 2^20 keys 7e-3; so 1e-6).
#pragma unroll
        for (int n = 0; n < DH / 8; n += 2) {
            const int x = n + (lane >> 4);
            float y[2][4] = {};
#pragma unroll
            for (int k = 0; k < KT / 16; k++) {
                const int rr = 16 * k + (lane & 15);
                uint32_t b[4];
                ldsm4_t(st + V_OFF + rr * (DH * 2) + 16 * ((x & ~7) | ((x ^ rr) & 7)), b);
                mma16<BF>(y[0], p[k], b[0], b[1]);
                mma16<BF>(y[1], p[k], b[2], b[3]);
            }
#pragma unroll
            for (int e = 0; e < 4; e++) r.o[n][e] += y[0][e], r.o[n + 1][e] += y[1][e];
        }
        __syncwarp();  // the stage has been read
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
    for (int x = 0; x < 2; x++) {
        r.l[x] += __shfl_xor_sync(0xFFFFFFFFu, r.l[x], 1);
        r.l[x] += __shfl_xor_sync(0xFFFFFFFFu, r.l[x], 2);
    }
}

// results of a whole unit
template <int DH, bool BF>
__device__ __forceinline__ void run_out(const SeqAttn &a, const Unit &u, bool none, const RunSum<DH> &r) {
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    const int lane = threadIdx.x & 31, t = lane & 3;
#pragma unroll
    for (int x = 0; x < 2; x++) {
        const int row = (lane >> 2) + 8 * x;
        if (row >= u.n) continue;
        const float inv = none ? 0.0f : 1.0f / r.l[x];
        T *o = static_cast<T *>(a.o.p) + u.b * a.o.ld + (u.h + row) * a.o.hd + 2 * t;
#pragma unroll
        for (int n = 0; n < DH / 8; n++)
            if (8 * n < a.dh) *reinterpret_cast<uint32_t *>(o + 8 * n) = none ? 0u : pack2<BF>(r.o[n][2 * x] * inv, r.o[n][2 * x + 1] * inv);
        if (t == 0 && a.lse) a.lse[(long)(u.h + row) * a.q_rows + u.b] = none ? -INFINITY : row_lse(r.m[x], r.l[x]);
    }
}

// Pieces of 2^piece keys before each sequence's, in units of one head: pre[0 .. n_seqs].  All threads of the block.
__device__ __forceinline__ void tile_prefix(const SeqAttn &a, int piece, int *pre) {
    __shared__ int sums[32];
    const int n = a.n_seqs, per = (n + (int)blockDim.x - 1) / (int)blockDim.x, from = (int)threadIdx.x * per, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = 0;
    for (int b = from; b < min(n, from + per); b++) {
        const Span k = seq_rows(a.k_start, a.k_len, b, a.k_rows);
        const int t = (k.hi - k.lo + (1 << piece) - 1) >> piece;
        pre[b + 1] = t;
        s += t;
    }
    int x = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    for (int w = 0; w < warp; w++) x += sums[w];
    x -= s;
    if (threadIdx.x == 0) pre[0] = 0;
    for (int b = from; b < min(n, from + per); b++) x += pre[b + 1], pre[b + 1] = x;
    __syncthreads();
}

// tiles of a run when `total` tiles are cut for at most `warps` warps
__device__ __forceinline__ long run_tiles(long total, int warps) { return max((long)TK_MIN_RUN, (total + warps - 1) / warps); }

template <int DH, bool BF>
__global__ void __launch_bounds__(32 * TK_WARPS, TK_BLOCKS) seq_attn_token_kernel(const SeqAttn a, const float c, const int chunks, const int split) {  // split: log2 of a piece's keys, 0: whole units
    extern __shared__ __align__(128) uint8_t ring_all[];
    pdl_grid_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ring_all) + warp * TK_STAGES * TK_STAGE;
    if (a.dh < DH) {  // pieces behind the head's elements stay zero
        for (int i = lane; i < TK_STAGES * TK_STAGE / 16; i += 32)
            reinterpret_cast<uint4 *>(ring_all + warp * TK_STAGES * TK_STAGE)[i] = make_uint4(0, 0, 0, 0);
        __syncwarp();
    }
    const long w = (long)blockIdx.x * TK_WARPS + warp;
    RunSum<DH> r;
    if (!split) {
        if (w < (long)a.n_seqs * a.hkv * chunks) {
            const Unit u = unit_of(a, chunks, w);
            const Span k = seq_rows(a.k_start, a.k_len, u.b, a.k_rows);
            run_keys<DH, BF>(a, u, k, c, ring, r);
            run_out<DH, BF>(a, u, k.hi <= k.lo, r);
        }
        pdl_allow_next();
        return;
    }
    int *pre = reinterpret_cast<int *>(ring_all + TK_SMEM);
    tile_prefix(a, split, pre);
    const int per = a.hkv * chunks, rows = min(16, a.group());
    int *pre_out = reinterpret_cast<int *>(static_cast<float *>(a.workspace) + 2 * (size_t)TK_GRID * TK_WARPS * tk_slot<DH>(rows));
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b <= a.n_seqs; b += 32 * TK_WARPS) pre_out[b] = pre[b];
    const long total = (long)pre[a.n_seqs] * per, run = run_tiles(total, (int)gridDim.x * TK_WARPS), t0 = w * run, t1 = min(total, t0 + run);
    float *slot = static_cast<float *>(a.workspace) + 2 * w * tk_slot<DH>(rows);
    for (long t = t0; t < t1;) {
        // the sequence that has tile t: the last whose tiles start at or before it and that has any
        int lo = 0, hi = a.n_seqs;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if ((long)pre[mid + 1] * per <= t) lo = mid + 1;
            else hi = mid;
        }
        const int nb = pre[lo + 1] - pre[lo], x = (int)((t - (long)pre[lo] * per) / nb);
        const long ut = (long)pre[lo] * per + (long)x * nb, ue = ut + nb;  // the unit's tiles
        const Unit u = unit_of(a, chunks, (long)lo * per + x);
        const Span k = seq_rows(a.k_start, a.k_len, u.b, a.k_rows);
        const long te = min(t1, ue);
        const Span part{k.lo + (int)((t - ut) << split), (int)min((long)k.hi, k.lo + ((te - ut) << split))};
        run_keys<DH, BF>(a, u, part, c, ring, r);
        if (t == ut && te == ue) {
            run_out<DH, BF>(a, u, false, r);
        } else {
            float *o = slot + (t == t0 ? 0 : tk_slot<DH>(rows));  // a run's first unit, or its last
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const int row = (lane >> 2) + 8 * e;
                if (row >= u.n) continue;
#pragma unroll
                for (int n = 0; n < DH / 8; n++) *reinterpret_cast<float2 *>(o + row * DH + 8 * n + 2 * (lane & 3)) = make_float2(r.o[n][2 * e], r.o[n][2 * e + 1]);
                if ((lane & 3) == 0) *reinterpret_cast<float2 *>(o + rows * DH + 2 * row) = make_float2(r.m[e], r.l[e]);
            }
        }
        t = te;
    }
    pdl_allow_next();
}

// A block per unit, row and COLS columns: the runs of a unit that was cut, an equal part of them a warp,
// added in their order; zeros where there is no key.  pre: as the first kernel left it.
template <int DH, bool BF, int TJ_WARPS, int COLS>
__global__ void __launch_bounds__(32 * TJ_WARPS) seq_attn_token_join_kernel(const SeqAttn a, const int chunks, const int warps, const int *pre) {
    using T = std::conditional_t<BF, __nv_bfloat16, __half>;
    constexpr int E = COLS / 32, CB = DH / COLS;  // columns of a lane, blocks of a row
    __shared__ float sums[TJ_WARPS][COLS + 1], tops[TJ_WARPS];
    pdl_grid_wait();
    const int per = a.hkv * chunks, rows = min(16, a.group()), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long un = blockIdx.x / (rows * CB);
    const int row = (int)(blockIdx.x / CB % rows), c0 = (int)(blockIdx.x % CB) * COLS, col = c0 + (int)threadIdx.x;
    const bool mine = (int)threadIdx.x < COLS && col < a.dh;
    const Unit u = unit_of(a, chunks, un);
    if (row >= u.n) return;
    const int p0 = pre[u.b], nb = pre[u.b + 1] - p0;
    const long total = (long)pre[a.n_seqs] * per, run = run_tiles(total, warps);
    const long ut = (long)p0 * per + (un - (long)u.b * per) * nb, ue = ut + nb;
    T *o = static_cast<T *>(a.o.p) + u.b * a.o.ld + (u.h + row) * a.o.hd;
    float *lse = a.lse ? a.lse + (long)(u.h + row) * a.q_rows + u.b : nullptr;
    if (nb == 0) {
        if (mine) o[col] = from_f32<T>(0.0f);
        if (col == 0 && lse) *lse = -INFINITY;
        return;
    }
    const long wa = ut / run, wb = (ue - 1) / run;
    if (wa == wb) return;
    const float *ws = static_cast<const float *>(a.workspace);
    const size_t size = tk_slot<DH>(rows);
    const auto part = [&](long x) { return ws + (2 * x + (x == wa && x * run < ut ? 1 : 0)) * size; };
    // the largest maximum, then the sums
    const long share = (wb - wa + TJ_WARPS) / TJ_WARPS, xa = wa + warp * share, xb = min(wb, xa + share - 1);
    float m = -INFINITY;
    for (long x = xa + lane; x <= xb; x += 32) m = fmaxf(m, part(x)[rows * DH + 2 * row]);
    m = warp_max_f(m);
    if (lane == 0) tops[warp] = m;
    __syncthreads();
    for (int w = 0; w < TJ_WARPS; w++) m = fmaxf(m, tops[w]);
    const float mu = m == -INFINITY ? 0.0f : m;
    float l = 0.0f, acc[E];
#pragma unroll
    for (int i = 0; i < E; i++) acc[i] = 0.0f;
#pragma unroll 8
    for (long x = xa; x <= xb; x++) {
        const float *p = part(x);
        const float2 ml = *reinterpret_cast<const float2 *>(p + rows * DH + 2 * row);
        const float f = exp2_fast(ml.x - mu);
        l = fmaf(ml.y, f, l);
#pragma unroll
        for (int i = 0; i < E; i++) acc[i] = fmaf(p[row * DH + c0 + 32 * i + lane], f, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < E; i++) sums[warp][32 * i + lane] = acc[i];
    if (lane == 0) sums[warp][COLS] = l;
    __syncthreads();
    l = 0.0f;
    for (int w = 0; w < TJ_WARPS; w++) l += sums[w][COLS];
    if (mine) {
        float x = 0.0f;
        for (int w = 0; w < TJ_WARPS; w++) x += sums[w][threadIdx.x];
        o[col] = from_f32<T>(x / l);
    }
    if (col == 0 && lse) *lse = row_lse(m, l);
}

int token_chunks(const SeqAttn &a) { return (a.group() + 15) / 16; }
// cut units into runs: too few to fill the card, and long enough to be worth it
bool token_split(const SeqAttn &a) {
    return (long)a.n_seqs * a.hkv * token_chunks(a) < 2L * TK_GRID * TK_WARPS && a.k_rows >= TK_SPLIT_ROWS;
}

// log2 of the keys of a piece that a unit is cut into: a tile, but as many as keep the number of all sequences' pieces within 31
// bits, however many of them share a long cache's rows
template <int DH>
int token_piece(const SeqAttn &a) {
    int piece = 4;
    while (1 << piece < tk_keys<DH>() || a.n_seqs * (((long)a.k_rows >> piece) + 1) > 0x7FFFFFFFL) piece++;
    return piece;
}

template <int DH, bool BF>
cudaError_t token(const SeqAttn &a, cudaStream_t st) {
    const int chunks = token_chunks(a), split = token_split(a);
    const long units = (long)a.n_seqs * a.hkv * chunks;
    const float c = a.scale * LOG2E;
    if (!split) return launch_pdl(seq_attn_token_kernel<DH, BF>, (unsigned)((units + TK_WARPS - 1) / TK_WARPS), 32 * TK_WARPS, TK_SMEM, st, a, c, chunks, 0);
    const int blocks = TK_GRID;
    const size_t pre = ((size_t)a.n_seqs + 1) * 4;
    const cudaError_t e = launch_pdl(seq_attn_token_kernel<DH, BF>, blocks, 32 * TK_WARPS, TK_SMEM + pre, st, a, c, chunks, token_piece<DH>(a));
    if (e != cudaSuccess) return e;
    const int rows = a.group() < 16 ? a.group() : 16;
    const int *left = reinterpret_cast<const int *>(static_cast<const float *>(a.workspace) + 2 * (size_t)TK_GRID * TK_WARPS * tk_slot<DH>(rows));
    // A unit of hundreds of runs: sixteen warps for 32 columns (32768 keys of 2 x 128: 15 us, four warps a row 46).  Else
    // four a row, as most blocks have little to do.
    const auto join = [&](auto w, auto cols) {
        constexpr int WARPS = decltype(w)::value, COLS = decltype(cols)::value;
        return launch_pdl(seq_attn_token_join_kernel<DH, BF, WARPS, COLS>, (unsigned)(units * rows * (DH / COLS)), 32 * WARPS, 0, st, a, chunks,
                          blocks * TK_WARPS, left);
    };
    return units <= 32 ? join(std::integral_constant<int, 16>{}, std::integral_constant<int, 32>{})
                       : join(std::integral_constant<int, 4>{}, std::integral_constant<int, DH>{});
}

template <int DH, bool BF>
cudaError_t token_init() {
    // the ring, and the pieces before each of fewer than 2 TK_GRID TK_WARPS sequences
    return cudaFuncSetAttribute(seq_attn_token_kernel<DH, BF>, cudaFuncAttributeMaxDynamicSharedMemorySize, TK_SMEM + 15 * 1024);
}

}  // namespace

cudaError_t seq_attn_token_init() {
    cudaError_t e = token_init<64, true>();
    if (e == cudaSuccess) e = token_init<64, false>();
    if (e == cudaSuccess) e = token_init<128, true>();
    if (e == cudaSuccess) e = token_init<128, false>();
    return e;
}

size_t seq_attn_token_workspace(const SeqAttn &a) {
    if (!token_split(a)) return 16;
    const int rows = a.group() < 16 ? a.group() : 16;
    return 2 * (size_t)TK_GRID * TK_WARPS * (a.dh <= 64 ? tk_slot<64>(rows) : tk_slot<128>(rows)) * 4 + ((size_t)a.n_seqs + 1) * 4;
}

cudaError_t launch_seq_attn_token(const SeqAttn &a, cudaStream_t st) {
    const bool bf = a.dtype == MNMT_BF16;
    if (a.dh <= 64) return bf ? token<64, true>(a, st) : token<64, false>(a, st);
    return bf ? token<128, true>(a, st) : token<128, false>(a, st);
}

}  // namespace mnmt
