// embed_rows.cu -- lookup of token rows of a floating-point table, and the table's
// gradient (include/mnmt.h, mnmt_embed).
//
//   out[t] = fl(fl(scale E[id_t]) + PE[pos_t]);  gE[v] = scale sum over id_t = v of g_t
// The lookup is one pass over the rows of out (16384 x 2048 fp32 33 us: 8.3 TB/s counted with every row read once, as
// frequent rows come from L2).  The gradient is dense, so most of its bytes are zeros:
// 16384 tokens of 2048 bf16 into 32000 fp32 rows take 78 us for 48 us of bytes: zeros 45 (4.3 TB/s, beside the sort's 19), sums 22
// (6.2 TB/s), joins 8; 46 tokens into 8000 x 256 4.9 us in one launch.  Sums in the tokens' order, whatever the launch:
// no atomic's order enters a result.
#include "row_pass.cuh"
#include "train.h"

namespace mnmt {
namespace {

// out[t] = fl(fl(scale E[id]) + PE[pos]): one pass over the rows of out
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) embed_rows_kernel(EmbedRowsArgs a, int alt, int alp, int alo, int lr) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    constexpr int E = row_elements(VEC);
    for (Walk<E> w(a.T, a.d, lr); w.more(); w.next()) {
        const RowAt p = w.at();
        const bool in = p.row < a.T;
        const int id = in ? a.ids[p.row] : 0, pos = in && a.pe ? a.pos ? a.pos[p.row] : (int)p.row : 0;
        const bool ok = in && id >= 0 && id < a.V && (!a.pe || (pos >= 0 && pos < a.P));
        if (in && !ok) set_status(a.status, MNMT_EINVAL);
        Raw<T, E> rt;
        Raw<float, E> rp;
        fetch<T, VEC>(static_cast<const T *>(a.table) + (ok ? id * a.ld : 0), w, p, a.d, ok, alt, rt);
        if (a.pe) fetch<float, VEC>(a.pe + (ok ? pos * a.ldpe : 0), w, p, a.d, ok, alp, rp);
        float v[E];
        settle<T, VEC>(rt, w, alt, buf, v);
#pragma unroll
        for (int k = 0; k < E; k++) v[k] = __fmul_rn(v[k], a.scale);
        if (a.pe) {
            float s[E];
            settle<float, VEC>(rp, w, alp, buf, s);
#pragma unroll
            for (int k = 0; k < E; k++) v[k] = __fadd_rn(v[k], s[k]);
        }
        if (!ok) {
#pragma unroll
            for (int k = 0; k < E; k++) v[k] = 0.0f;
        }
        put<O, VEC>(static_cast<O *>(a.out) + p.row * a.ldo, w, p, a.d, in, alo, buf, v);
    }
}

// --------------------------------------------------------------------------- the table's gradient
constexpr int EB_COLS = 256;  // columns of a warp: eight a lane

// A lane's eight of the warp's columns from c0 on: side by side where rows are 16-byte
// aligned (VEC), else 32 apart, so that lanes next to each other load what is.
template <bool VEC>
struct LaneCols {
    int c0, d;
    MNMT_DEV int at(int k) const { return VEC ? c0 + 8 * (threadIdx.x & 31) + k : c0 + 32 * k + (threadIdx.x & 31); }
    template <typename T>
    MNMT_DEV void load(const T *row, float (&v)[8]) const {
        if (VEC && at(0) + 8 <= d) {
            load8<T, true>(row + at(0), 8, v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] = at(k) < d ? to_f32(row[at(k)]) : 0.0f;
        }
    }
    // the same as words, to be converted when they are added
    template <typename T>
    MNMT_DEV void fetch8(const T *row, Raw<T, 8> &r) const {
        constexpr int NW = sizeof(T) * 2;
        if (VEC && at(0) + 8 <= d) {
#pragma unroll
            for (int i = 0; i < NW / 4; i++) {
                const uint4 v = reinterpret_cast<const uint4 *>(row + at(0))[i];
                r.w[4 * i] = v.x, r.w[4 * i + 1] = v.y, r.w[4 * i + 2] = v.z, r.w[4 * i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NW; i++) r.w[i] = 0;
#pragma unroll
            for (int k = 0; k < 8; k++)
                if (at(k) < d) r.w[k * NW / 8] |= bits_of(row[at(k)]) << (sizeof(T) == 2 ? 16 * (k & 1) : 0);
        }
    }
    template <typename O>
    MNMT_DEV void store(O *row, const float (&v)[8]) const {
        if (VEC && at(0) + 8 <= d) {
            store8<O, true>(row + at(0), 8, v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; k++)
                if (at(k) < d) row[at(k)] = from_f32<O>(v[k]);
        }
    }
    // the row of a token's gradient from the sum of its g (wide: rows start on 32 bytes)
    template <typename O>
    MNMT_DEV void finish(O *row, float (&s)[8], float scale, bool accumulate, bool wide) const {
        float old[8];
        if (accumulate) load(row, old);
#pragma unroll
        for (int k = 0; k < 8; k++) {
            s[k] = __fmul_rn(s[k], scale);
            if (accumulate) s[k] = __fadd_rn(old[k], s[k]);
        }
        if (VEC && sizeof(O) == 4 && wide && at(0) + 8 <= d) {
            uint32_t w[8];
#pragma unroll
            for (int k = 0; k < 8; k++) w[k] = __float_as_uint(s[k]);
            st32(row + at(0), w);
            return;
        }
        store(row, s);
    }
};

// s += the rows of g that lanes of `mask` hold the numbers of, in lane order, several in flight
template <typename T, bool VEC>
MNMT_DEV void add_rows(const T *g, long ld, int t, uint32_t mask, const LaneCols<VEC> &cols, float (&s)[8]) {
    constexpr int N = 8;
    while (mask) {
        float v[N][8];
        bool on[N];
#pragma unroll
        for (int i = 0; i < N; i++) {
            on[i] = mask != 0;
            const int row = __shfl_sync(0xFFFFFFFFu, t, on[i] ? __ffs(mask) - 1 : 0);
            if (on[i]) cols.load(g + row * ld, v[i]);
            mask &= mask - 1;
        }
#pragma unroll
        for (int i = 0; i < N; i++)
            if (on[i]) {
#pragma unroll
                for (int k = 0; k < 8; k++) s[k] += v[i][k];
            }
    }
}

// Few tokens, one launch.  Block (x, y) has the rows of the table that are x modulo the
// number of row sets (frequent tokens have low numbers: they spread over the blocks) and
// 256 columns.  Each warp looks through its eighth of the tokens and lists those of the
// block's rows; rows that many tokens name are added up by all warps, each over its own
// list, the others by a warp each over all lists: in the tokens' order both.
constexpr int EF_TOKENS = 4096, EF_ROWS = 4096;  // at most: tokens, rows of a block
constexpr int EF_MANY = 32;                      // tokens of a row from which all warps work on it
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256) embed_few_kernel(EmbedRowsArgs a) {
    __shared__ uint16_t list[EF_TOKENS], slot[EF_TOKENS];
    __shared__ uint32_t count[EF_ROWS / 2];  // of two rows each
    __shared__ int found[8], many[EF_TOKENS / EF_MANY + 1], n_many;
    __shared__ float part[8][EB_COLS];
    pdl_grid_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sets = gridDim.x, x = blockIdx.x;
    const int rows = (a.V - x + sets - 1) / sets;
    const LaneCols<VEC> cols{(int)blockIdx.y * EB_COLS, a.d};
    const T *g = static_cast<const T *>(a.table);
    O *out = static_cast<O *>(a.out);
    for (int i = threadIdx.x; i < (rows + 1) / 2; i += 256) count[i] = 0;
    if (threadIdx.x == 0) n_many = 0;
    __syncthreads();
    const int per = (a.T + 7) / 8, t0 = warp * per, t1 = min(a.T, t0 + per);
    int n = 0;
    for (int t = t0; t < t1; t += 32) {
        const int id = t + lane < t1 ? a.ids[t + lane] : -1;
        const bool bad = t + lane < t1 && (id < 0 || id >= a.V);
        if (bad && x == 0 && blockIdx.y == 0) set_status(a.status, MNMT_EINVAL);
        const bool mine = id >= 0 && id < a.V && id != a.pad_id && id % sets == x;
        const uint32_t m = __ballot_sync(0xFFFFFFFFu, mine);
        if (mine) {
            const int at = t0 + n + __popc(m & ((1u << lane) - 1u)), r = id / sets;
            list[at] = (uint16_t)(t + lane), slot[at] = (uint16_t)r;
            atomicAdd(&count[r >> 1], r & 1 ? 65536u : 1u);
        }
        n += __popc(m);
    }
    if (lane == 0) found[warp] = n;
    __syncthreads();
    const auto of = [&](int r) { return (count[r >> 1] >> (r & 1 ? 16 : 0)) & 0xFFFFu; };
    // a warp's list: s += its tokens of row r
    const auto add_list = [&](int w, int r, float(&s)[8]) {
        const int first = w * per, end = first + found[w];
        for (int i = first; i < end; i += 32) {
            const bool on = i + lane < end && slot[i + lane] == r;
            add_rows<T, VEC>(g, a.ld, on ? list[i + lane] : 0, __ballot_sync(0xFFFFFFFFu, on), cols, s);
        }
    };
    for (int r = warp; r < rows; r += 8) {
        const int c = of(r);
        if (c >= EF_MANY) {
            if (lane == 0) many[atomicAdd(&n_many, 1)] = r;  // in any order: each row's sum is its own
        } else if (c || !a.accumulate) {
            float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
            if (c)
                for (int w = 0; w < 8; w++) add_list(w, r, s);
            cols.finish(out + ((long)r * sets + x) * a.ldo, s, a.scale, a.accumulate, a.wide);
        }
    }
    __syncthreads();
    for (int i = 0; i < n_many; i++) {
        float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        add_list(warp, many[i], s);
#pragma unroll
        for (int k = 0; k < 8; k++) part[warp][32 * k + lane] = s[k];
        __syncthreads();
        if (warp == 0) {
            for (int w = 1; w < 8; w++)
#pragma unroll
                for (int k = 0; k < 8; k++) s[k] += part[w][32 * k + lane];
            cols.finish(out + ((long)many[i] * sets + x) * a.ldo, s, a.scale, a.accumulate, a.wide);
        }
        __syncthreads();
    }
}

// Many tokens: sorted by their number (stable), in chunks of 32 a warp adds up; rows
// whose tokens lie in several chunks are joined from the chunks' sums.
struct SortBufs {
    int *key[2], *idx[2];
};

// Stable sort of the tokens by one cluster, eight bits a pass: counts per warp, an
// exclusive sum over (digit, CTA, warp), then every token to its place.  Tokens
// without a gradient take the number V, behind all others.
constexpr int ES_THREADS = 1024, ES_WARPS = 32, ES_CLUSTER = 8;
MNMT_DEV void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__global__ void __launch_bounds__(ES_THREADS) embed_sort_kernel(const int *ids, int T, int V, int pad_id, int passes, SortBufs b, int *status) {
    __shared__ int cnt[ES_WARPS][256], tot[256], base[256], wsum[8];
    pdl_grid_wait();
    pdl_allow_next();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = threadIdx.x;
    const int ctas = gridDim.x, rank = blockIdx.x;  // the grid is one cluster
    const long per = ((long)T + ctas * ES_WARPS * 32 - 1) / (ctas * ES_WARPS * 32) * 32;  // tokens of a warp
    const long first = (rank * ES_WARPS + warp) * per, end = min((long)T, first + per);
    for (int pass = 0; pass < passes; pass++) {
        const int *key = b.key[(pass & 1) ^ 1], *idx = b.idx[(pass & 1) ^ 1];
        int *okey = b.key[pass & 1], *oidx = b.idx[pass & 1];
        const auto load = [&](long t, bool report) {
            if (pass) return t < end ? key[t] : 0;
            const int id = t < end ? ids[t] : 0;
            const bool bad = id < 0 || id >= V;
            if (bad && report) set_status(status, MNMT_EINVAL);
            return bad || id == pad_id ? V : id;
        };
        const int shift = 8 * pass;
        for (int i = d; i < ES_WARPS * 256; i += ES_THREADS) cnt[i >> 8][i & 255] = 0;
        __syncthreads();
        for (long t = first; t < end; t += 32) {
            const uint32_t live = __ballot_sync(0xFFFFFFFFu, t + lane < end);
            const int dig = t + lane < end ? (load(t + lane, true) >> shift) & 255 : 256;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, dig) & live;
            if (dig < 256 && lane == __ffs(same) - 1) cnt[warp][dig] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        if (d < 256) {
            int s = 0;
            for (int w = 0; w < ES_WARPS; w++) {
                const int c = cnt[w][d];
                cnt[w][d] = s;
                s += c;
            }
            tot[d] = s;
        }
        cluster_sync_all();
        int before = 0, all = 0, x = 0;
        if (d < 256) {
            const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&tot[d]);
#pragma unroll 8
            for (int c = 0; c < ctas; c++) {
                uint32_t at;
                int v;
                asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(mine), "r"(c));
                asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at));
                if (c < rank) before += v;
                all += v;
            }
            x = all;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
                if (lane >= o) x += y;
            }
            if (lane == 31) wsum[warp] = x;
        }
        __syncthreads();
        if (d < 256) {
            for (int w = 0; w < warp; w++) x += wsum[w];
            base[d] = x - all + before;
        }
        __syncthreads();
        for (long t = first; t < end; t += 32) {
            const bool on = t + lane < end;
            const uint32_t live = __ballot_sync(0xFFFFFFFFu, on);
            const int k = load(t + lane, false), dig = on ? (k >> shift) & 255 : 256;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, dig) & live;
            if (on) {
                const int to = base[dig] + cnt[warp][dig] + __popc(same & ((1u << lane) - 1u));
                okey[to] = k, oidx[to] = pass ? idx[t + lane] : (int)(t + lane);
            }
            __syncwarp();
            if (on && lane == __ffs(same) - 1) cnt[warp][dig] += __popc(same);
            __syncwarp();
        }
        cluster_sync_all();  // every token is in its place, every CTA's counts have been read
    }
}

// Rows that no token names are zero.  Needs the ids alone: runs beside the sort, which lets it
// start only when what was in the stream before is done; alone (no tokens), it waits for that itself.
// A block has the rows that are its number modulo the blocks (those of frequent tokens have low numbers).
constexpr int EZ_BITS = 1 << 16, EZ_THREADS = 256, EZ_SETS = 4 * 152;
template <typename O>
__global__ void __launch_bounds__(EZ_THREADS) embed_zero_kernel(EmbedRowsArgs a, bool vec) {
    __shared__ uint32_t named[EZ_BITS / 32];
    if (a.T == 0) pdl_grid_wait();
    pdl_allow_next();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, x = blockIdx.x;
    const int rows = x < a.V ? (a.V - x + EZ_SETS - 1) / EZ_SETS : 0;
    const long whole = vec ? (long)a.d * sizeof(O) / 16 : 0;  // 16-byte pieces of a row
    const int quads = (reinterpret_cast<uintptr_t>(a.ids) & 15) ? 0 : a.T / 4;
    for (int f = 0; f < rows; f += EZ_BITS) {
        const int n = min(EZ_BITS, rows - f);
        __syncthreads();
        for (int i = threadIdx.x; i < (n + 31) / 32; i += EZ_THREADS) named[i] = 0;
        __syncthreads();
        const auto name = [&](int id) {
            const int r = id / EZ_SETS - f;
            if (id >= 0 && id < a.V && id != a.pad_id && id % EZ_SETS == x && r >= 0 && r < n) atomicOr(&named[r >> 5], 1u << (r & 31));
        };
#pragma unroll 8
        for (int i = threadIdx.x; i < quads; i += EZ_THREADS) {
            const int4 q = reinterpret_cast<const int4 *>(a.ids)[i];
            name(q.x), name(q.y), name(q.z), name(q.w);
        }
        for (int t = 4 * quads + threadIdx.x; t < a.T; t += EZ_THREADS) name(a.ids[t]);
        __syncthreads();
        for (int r = warp; r < n; r += EZ_THREADS / 32)
            if (!((named[r >> 5] >> (r & 31)) & 1u)) {
                O *row = static_cast<O *>(a.out) + ((long)(f + r) * EZ_SETS + x) * a.ldo;
                for (long i = lane; i < whole; i += 32) reinterpret_cast<uint4 *>(row)[i] = make_uint4(0, 0, 0, 0);
                for (long i = whole * (16 / sizeof(O)) + lane; i < a.d; i += 32) row[i] = from_f32<O>(0.0f);
            }
    }
    pdl_grid_wait();  // the sort's end is this kernel's too
}

// A warp per chunk of 32 sorted tokens and 256 columns.  A row whose tokens all lie in
// the chunk is finished here; the sum of one that came from the chunk before, or goes on
// into the next, is left in slot 2 chunk (it starts at the chunk's first token) or + 1.
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256) embed_sum_kernel(EmbedRowsArgs a, const int *key, const int *idx, float *parts) {
    pdl_grid_wait();
    const int lane = threadIdx.x & 31, cb = (a.d + EB_COLS - 1) / EB_COLS;
    const long w = ((long)blockIdx.x * 256 + threadIdx.x) >> 5, chunk = w / cb, p0 = 32 * chunk;
    if (p0 >= a.T) return;
    const LaneCols<VEC> cols{(int)(w % cb) * EB_COLS, a.d};
    const bool on = p0 + lane < a.T;
    const int k = on ? key[p0 + lane] : a.V, t = on ? idx[p0 + lane] : 0;
    const int prev = p0 ? key[p0 - 1] : -1, next = p0 + 32 < a.T ? key[p0 + 32] : a.V;
    const int left = __shfl_up_sync(0xFFFFFFFFu, k, 1);
    const uint32_t heads = __ballot_sync(0xFFFFFFFFu, lane > 0 && k != left);  // first tokens of further rows
    const T *g = static_cast<const T *>(a.table);
    float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    int from = 0;
    const auto flush = [&](int to) {  // tokens from .. to - 1 are one row's
        const int v = __shfl_sync(0xFFFFFFFFu, k, from);
        if (v < a.V) {
            if ((from > 0 || prev != v) && (to < 32 || next != v)) {
                cols.finish(static_cast<O *>(a.out) + (long)v * a.ldo, s, a.scale, a.accumulate, a.wide);
            } else {
                float *p = parts + (2 * chunk + (from > 0)) * (long)(cb * EB_COLS) + cols.c0;
                reinterpret_cast<float4 *>(p)[2 * lane] = make_float4(s[0], s[1], s[2], s[3]);
                reinterpret_cast<float4 *>(p)[2 * lane + 1] = make_float4(s[4], s[5], s[6], s[7]);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e++) s[e] = 0.0f;
        from = to;
    };
    for (int i0 = 0; i0 < 32; i0 += 8) {  // eight rows in flight, whosever they are
        Raw<T, 8> v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const bool some = __shfl_sync(0xFFFFFFFFu, k, i0 + i) < a.V;
            const long row = __shfl_sync(0xFFFFFFFFu, t, i0 + i);
            if (some) {
                cols.fetch8(g + row * a.ld, v[i]);
            } else {
#pragma unroll
                for (uint32_t &w : v[i].w) w = 0;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if ((heads >> (i0 + i)) & 1u) flush(i0 + i);
#pragma unroll
            for (int e = 0; e < 8; e++) s[e] += raw_at(v[i], e);
        }
    }
    flush(32);
}

// A block per 8 chunks and 256 columns: the rows that begin in one of the chunks and go on
// into the next, a warp each; those of many chunks by all warps, an eighth of them each.
constexpr int EJ_MANY = 16;
template <typename O, bool VEC>
__global__ void __launch_bounds__(256) embed_join_kernel(EmbedRowsArgs a, const int *key, const float *parts) {
    __shared__ float part[8][EB_COLS];
    __shared__ long chunks[8];
    pdl_grid_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cb = (a.d + EB_COLS - 1) / EB_COLS;
    const long chunk = (long)(blockIdx.x / cb) * 8 + warp, q0 = 32 * chunk;
    const LaneCols<VEC> cols{(int)(blockIdx.x % cb) * EB_COLS, a.d};
    // the warp's chunk: its last row, whether that goes on and whether it began here
    int row = a.V;
    bool from_first = false, begins = false;
    if (q0 + 32 < a.T) {
        const int first = key[q0], next = key[q0 + 32], prev = q0 ? key[q0 - 1] : -1;
        row = key[q0 + 31];
        from_first = first == row;
        begins = row < a.V && next == row && !(from_first && prev == row);
    }
    long n = 0;  // its chunks: 32 at a time, those that end with it
    if (begins) {
        long last = chunk;
        for (;;) {
            const long c = last + 1 + lane;
            const uint32_t full = __ballot_sync(0xFFFFFFFFu, 32 * c + 31 < a.T && key[32 * c + 31] == row);
            const int m = full == 0xFFFFFFFFu ? 32 : __ffs(~full) - 1;
            last += m;
            if (m < 32) break;
        }
        if (32 * (last + 1) < a.T && key[32 * (last + 1)] == row) last++;
        n = last - chunk + 1;
    }
    // the sums of chunks c0 .. c1 - 1 of a row that begins in chunk c
    const auto add = [&](long c, bool whole, long c0, long c1, float(&s)[8]) {
#pragma unroll 8
        for (long i = c0; i < c1; i++) {
            const float4 *p = reinterpret_cast<const float4 *>(parts + (2 * i + (i == c && !whole)) * (long)(cb * EB_COLS) + cols.c0);
            const float4 x = p[2 * lane], y = p[2 * lane + 1];
            s[0] += x.x, s[1] += x.y, s[2] += x.z, s[3] += x.w, s[4] += y.x, s[5] += y.y, s[6] += y.z, s[7] += y.w;
        }
    };
    if (n && n < EJ_MANY) {
        float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        add(chunk, from_first, chunk, chunk + n, s);
        cols.finish(static_cast<O *>(a.out) + (long)row * a.ldo, s, a.scale, a.accumulate, a.wide);
    }
    if (lane == 0) chunks[warp] = n < EJ_MANY ? 0 : from_first ? n : -n;
    __syncthreads();
    for (int w = 0; w < 8; w++) {
        if (chunks[w] == 0) continue;  // alike in all threads
        const long c = chunk - warp + w, m = chunks[w] < 0 ? -chunks[w] : chunks[w], per = (m + 7) / 8;
        float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        add(c, chunks[w] > 0, min(c + m, c + warp * per), min(c + m, c + (warp + 1) * per), s);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; k++) part[warp][32 * k + lane] = s[k];
        __syncthreads();
        if (warp == w) {
#pragma unroll
            for (int k = 0; k < 8; k++) s[k] = part[0][32 * k + lane];
            for (int x = 1; x < 8; x++)
#pragma unroll
                for (int k = 0; k < 8; k++) s[k] += part[x][32 * k + lane];
            cols.finish(static_cast<O *>(a.out) + (long)row * a.ldo, s, a.scale, a.accumulate, a.wide);
        }
    }
}

template <typename F>
void by_types(int dtype, int otype, F &&f) {
    auto with = [&](auto t) {
        if (otype == MNMT_F32) f(t, float{});
        else if (otype == MNMT_BF16) f(t, __nv_bfloat16{});
        else f(t, __half{});
    };
    if (dtype == MNMT_F32) with(float{});
    else if (dtype == MNMT_BF16) with(__nv_bfloat16{});
    else with(__half{});
}

}  // namespace

cudaError_t launch_embed_rows(const EmbedRowsArgs &a, cudaStream_t st) {
    by_types(a.dtype, a.otype, [&](auto t, auto o) {
        using T = decltype(t);
        using O = decltype(o);
        const int at = row_alignment(static_cast<const T *>(a.table), a.ld), ap = a.pe ? row_alignment(a.pe, a.ldpe) : 2;
        const int ao = row_alignment(static_cast<const O *>(a.out), a.ldo);
        const bool vec = at == 2 && ap == 2 && ao == 2;
        launch_pdl(vec ? embed_rows_kernel<T, O, true> : embed_rows_kernel<T, O, false>, row_grid(a.T, a.d, vec, device_sm_count()), 256, 0, st, a, at, ap,
                   ao, row_lanes(a.d, vec));
    });
    return cudaGetLastError();
}

namespace {
// row sets of embed_few_kernel: four blocks per SM over all columns, no more than rows
int few_sets(int V, int d) {
    const int cb = (d + EB_COLS - 1) / EB_COLS, sets = (4 * 152 + cb - 1) / cb;
    return sets < V ? sets : V;
}
bool few_tokens(int T, int V, int d) { return T <= EF_TOKENS && (V + few_sets(V, d) - 1) / few_sets(V, d) <= EF_ROWS && (d + EB_COLS - 1) / EB_COLS <= 65535; }
size_t sort_ints(int T) { return ((size_t)T + 3) / 4 * 4; }
size_t sum_parts(int T, int d) { return 2 * (((size_t)T + 31) / 32) * ((size_t)(d + EB_COLS - 1) / EB_COLS * EB_COLS); }
}  // namespace

size_t embed_rows_backward_workspace(int T, int V, int d) {
    return T == 0 || few_tokens(T, V, d) ? 16 : 16 * sort_ints(T) + 4 * sum_parts(T, d);
}

cudaError_t launch_embed_rows_backward(const EmbedRowsArgs &args, cudaStream_t st) {
    cudaError_t err = cudaSuccess;
    EmbedRowsArgs a = args;
    by_types(a.dtype, a.otype, [&](auto t, auto o) {
        using T = decltype(t);
        using O = decltype(o);
        const bool vec = row_alignment(static_cast<const T *>(a.table), a.T ? a.ld : 0) && row_alignment(static_cast<const O *>(a.out), a.ldo);
        const unsigned cb = (unsigned)((a.d + EB_COLS - 1) / EB_COLS);
        a.wide = row_alignment(static_cast<const O *>(a.out), a.ldo) == 2;
        if (few_tokens(a.T, a.V, a.d)) {
            err = launch_pdl(vec ? embed_few_kernel<T, O, true> : embed_few_kernel<T, O, false>, dim3((unsigned)few_sets(a.V, a.d), cb), 256, 0, st, a);
            return;
        }
        const bool ovec = row_alignment(static_cast<const O *>(a.out), a.ldo) > 0;
        if (a.T == 0) {  // nothing to sort or add; a table of that size is zeroed by as many blocks as beside the sort
            if (!a.accumulate) err = launch_pdl(embed_zero_kernel<O>, EZ_SETS, EZ_THREADS, 0, st, a, ovec);
            return;
        }
        const long chunks = ((long)a.T + 31) / 32;
        if (chunks * cb > 0x7FFFFFFFL) {
            err = cudaErrorInvalidValue;
            return;
        }
        SortBufs b;
        int *p = static_cast<int *>(a.workspace);
        for (int i = 0; i < 2; i++) b.key[i] = p + 2 * i * sort_ints(a.T), b.idx[i] = b.key[i] + sort_ints(a.T);
        float *parts = reinterpret_cast<float *>(p + 4 * sort_ints(a.T));
        int passes = 1;
        while (passes < 4 && (a.V >> (8 * passes)) != 0) passes++;
        cudaLaunchConfig_t cfg = {};
        int ctas = 1;
        while (ctas < ES_CLUSTER && a.T > 1024 * ctas) ctas *= 2;
        cfg.gridDim = dim3(ctas);
        cfg.blockDim = dim3(ES_THREADS);
        cfg.stream = st;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)ctas, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(st, &cs) != cudaSuccess) cs = cudaStreamCaptureStatusNone;
        cfg.attrs = attr;
        cfg.numAttrs = cs == cudaStreamCaptureStatusActive ? 1 : 2;
        if ((err = cudaLaunchKernelEx(&cfg, embed_sort_kernel, a.ids, a.T, a.V, a.pad_id, passes, b, a.status)) != cudaSuccess) return;
        if (!a.accumulate && (err = launch_pdl(embed_zero_kernel<O>, EZ_SETS, EZ_THREADS, 0, st, a, ovec)) != cudaSuccess) return;
        const int *key = b.key[(passes - 1) & 1], *idx = b.idx[(passes - 1) & 1];
        err = launch_pdl(vec ? embed_sum_kernel<T, O, true> : embed_sum_kernel<T, O, false>, (unsigned)((chunks * cb + 7) / 8), 256, 0, st, a, key, idx, parts);
        if (err == cudaSuccess)
            err = launch_pdl(vec ? embed_join_kernel<O, true> : embed_join_kernel<O, false>, (unsigned)((chunks + 7) / 8 * cb), 256, 0, st, a, key, (const float *)parts);
    });
    return err;
}

}  // namespace mnmt
