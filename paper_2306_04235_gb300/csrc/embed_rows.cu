// embed_rows.cu -- lookup of token rows of a floating-point table, and the table's
// gradient (include/mnmt.h, mnmt_embed).
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

// A warp per row of the table: all tokens that name it, in their order.
template <typename T, typename O>
__global__ void __launch_bounds__(256) embed_rows_backward_kernel(EmbedRowsArgs a) {
    pdl_grid_wait();
    const int lane = threadIdx.x & 31;
    const long id = ((long)blockIdx.x * 256 + threadIdx.x) >> 5;
    if (id == 0 && a.status)
        for (int t = lane; t < a.T; t += 32)
            if (a.ids[t] < 0 || a.ids[t] >= a.V) set_status(a.status, MNMT_EINVAL);
    if (id >= a.V) return;
    O *out = static_cast<O *>(a.out) + id * a.ldo;
    const T *g = static_cast<const T *>(a.table);
    for (int c0 = 0; c0 < a.d; c0 += 256) {
        float s[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        for (int t0 = 0; t0 < a.T; t0 += 32) {
            uint32_t m = __ballot_sync(0xFFFFFFFFu, t0 + lane < a.T && a.ids[t0 + lane] == id && id != a.pad_id);
            for (; m; m &= m - 1) {
                const T *row = g + (t0 + __ffs(m) - 1) * a.ld;
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (c0 + 32 * k + lane < a.d) s[k] += to_f32(row[c0 + 32 * k + lane]);
            }
        }
#pragma unroll
        for (int k = 0; k < 8; k++) {
            const int c = c0 + 32 * k + lane;
            if (c < a.d) out[c] = from_f32<O>(__fadd_rn(a.accumulate ? to_f32(out[c]) : 0.0f, __fmul_rn(s[k], a.scale)));
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

size_t embed_rows_backward_workspace(int, int, int) { return 16; }

cudaError_t launch_embed_rows_backward(const EmbedRowsArgs &a, cudaStream_t st) {
    by_types(a.dtype, a.otype, [&](auto t, auto o) {
        launch_pdl(embed_rows_backward_kernel<decltype(t), decltype(o)>, (unsigned)((a.V + 7) / 8), 256, 0, st, a);
    });
    return cudaGetLastError();
}

}  // namespace mnmt
