// seq_attn.cu -- attention over sequences, forward (seq_attn.cuh): a warp per
// query row and head, one pass over the keys with the running maximum and sum.
#include "seq_attn.cuh"

namespace mnmt {
namespace {

template <typename T>
__global__ void __launch_bounds__(256) seq_attn_rows_kernel(SeqAttn a, float c, bool token) {
    pdl_grid_wait();
    const long w = ((long)blockIdx.x * 256 + threadIdx.x) >> 5;
    if (w >= (long)a.q_rows * a.hq) return;
    const int row = (int)(w / a.hq), h = (int)(w % a.hq), hk = h / a.group(), lane = threadIdx.x & 31;
    bool in = true;
    const Span s = token ? seq_rows(a.k_start, a.k_len, row, a.k_rows) : keys_of_query(a, row, in);
    if (!in) return;
    const RowSum r = attn_row(static_cast<const T *>(a.q.p) + row * a.q.ld + h * a.q.hd, static_cast<const T *>(a.k.p) + hk * a.k.hd, a.k.ld,
                              static_cast<const T *>(a.v.p) + hk * a.v.hd, a.v.ld, s, a.dh, c);
    const bool none = s.hi <= s.lo;
    const float inv = none ? 0.0f : 1.0f / r.l;
    float o[4];
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = r.acc[i] * inv;
    if (4 * lane < a.dh) store4(static_cast<T *>(a.o.p) + row * a.o.ld + h * a.o.hd + 4 * lane, o);
    if (lane == 0 && a.lse) a.lse[(long)h * a.q_rows + row] = none ? -INFINITY : row_lse(r.m, r.l);
}

cudaError_t rows_forward(const SeqAttn &a, bool token, cudaStream_t st) {
    const long blocks = ((long)a.q_rows * a.hq + 7) / 8;
    const float c = a.scale * LOG2E;
    return launch_pdl(a.dtype == MNMT_BF16 ? seq_attn_rows_kernel<__nv_bfloat16> : seq_attn_rows_kernel<__half>, (unsigned)blocks, 256, 0, st, a, c, token);
}

}  // namespace

size_t seq_attn_forward_workspace(const SeqAttn &) { return 16; }
size_t seq_attn_token_workspace(const SeqAttn &) { return 16; }

cudaError_t launch_seq_attn_forward(const SeqAttn &a, cudaStream_t st) { return rows_forward(a, false, st); }
cudaError_t launch_seq_attn_token(const SeqAttn &a, cudaStream_t st) { return rows_forward(a, true, st); }

}  // namespace mnmt
