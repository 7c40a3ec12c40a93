// seq_attn_backward.cu -- gradients of attention over sequences (seq_attn.cuh): D,
// then a warp per query row for dq and a warp per key row for dk and dv.
#include "seq_attn.cuh"

namespace mnmt {
namespace {

template <typename T>
__global__ void __launch_bounds__(256) seq_attn_delta_kernel(SeqAttn a, float *delta) {
    pdl_grid_wait();
    const long w = (long)blockIdx.x * 256 + threadIdx.x;
    if (w >= (long)a.q_rows * a.hq) return;
    const int row = (int)(w / a.hq), h = (int)(w % a.hq);
    delta[(long)h * a.q_rows + row] =
        row_dot(static_cast<const T *>(a.o.p) + row * a.o.ld + h * a.o.hd, static_cast<const T *>(a.g.p) + row * a.g.ld + h * a.g.hd, a.dh);
}

template <typename T>
__global__ void __launch_bounds__(256) seq_attn_dq_rows_kernel(SeqAttn a, float c, const float *delta) {
    pdl_grid_wait();
    const long w = ((long)blockIdx.x * 256 + threadIdx.x) >> 5;
    if (w >= (long)a.q_rows * a.hq) return;
    const int row = (int)(w / a.hq), h = (int)(w % a.hq), hk = h / a.group(), lane = threadIdx.x & 31;
    bool in;
    const Span s = keys_of_query(a, row, in);
    if (!in) return;
    const long at = (long)h * a.q_rows + row;
    const float4 d = attn_row_dq(static_cast<const T *>(a.q.p) + row * a.q.ld + h * a.q.hd, static_cast<const T *>(a.g.p) + row * a.g.ld + h * a.g.hd,
                                 a.lse[at] * LOG2E, delta[at], static_cast<const T *>(a.k.p) + hk * a.k.hd, a.k.ld,
                                 static_cast<const T *>(a.v.p) + hk * a.v.hd, a.v.ld, s, a.dh, c);
    const float o[4] = {d.x * a.scale, d.y * a.scale, d.z * a.scale, d.w * a.scale};
    if (4 * lane < a.dh) store4(static_cast<T *>(a.dq.p) + row * a.dq.ld + h * a.dq.hd + 4 * lane, o);
}

template <typename T>
__global__ void __launch_bounds__(256) seq_attn_dkv_rows_kernel(SeqAttn a, float c, const float *delta) {
    pdl_grid_wait();
    const long w = ((long)blockIdx.x * 256 + threadIdx.x) >> 5;
    if (w >= (long)a.k_rows * a.hkv) return;
    const int row = (int)(w / a.hkv), hk = (int)(w % a.hkv), lane = threadIdx.x & 31;
    bool in;
    const Span s = queries_of_key(a, row, in);
    if (!in) return;
    float dk[4] = {0.0f, 0.0f, 0.0f, 0.0f}, dv[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int h = hk * a.group(); h < (hk + 1) * a.group(); h++)
        attn_row_dkv(static_cast<const T *>(a.k.p) + row * a.k.ld + hk * a.k.hd, static_cast<const T *>(a.v.p) + row * a.v.ld + hk * a.v.hd,
                     static_cast<const T *>(a.q.p) + h * a.q.hd, a.q.ld, static_cast<const T *>(a.g.p) + h * a.g.hd, a.g.ld,
                     a.lse + (long)h * a.q_rows, delta + (long)h * a.q_rows, s, a.dh, c, dk, dv);
#pragma unroll
    for (int i = 0; i < 4; i++) dk[i] *= a.scale;
    if (4 * lane < a.dh) {
        store4(static_cast<T *>(a.dk.p) + row * a.dk.ld + hk * a.dk.hd + 4 * lane, dk);
        store4(static_cast<T *>(a.dv.p) + row * a.dv.ld + hk * a.dv.hd + 4 * lane, dv);
    }
}

template <typename T>
cudaError_t backward(const SeqAttn &a, cudaStream_t st) {
    float *delta = static_cast<float *>(a.workspace);
    const float c = a.scale * LOG2E;
    const long q = (long)a.q_rows * a.hq, k = (long)a.k_rows * a.hkv;
    if (q) {
        launch_pdl(seq_attn_delta_kernel<T>, (unsigned)((q + 255) / 256), 256, 0, st, a, delta);
        launch_pdl(seq_attn_dq_rows_kernel<T>, (unsigned)((q + 7) / 8), 256, 0, st, a, c, (const float *)delta);
    }
    if (k) launch_pdl(seq_attn_dkv_rows_kernel<T>, (unsigned)((k + 7) / 8), 256, 0, st, a, c, (const float *)delta);
    return cudaGetLastError();
}

}  // namespace

size_t seq_attn_backward_workspace(const SeqAttn &a) { return ((size_t)a.hq * a.q_rows * 4 + 31) / 16 * 16; }

cudaError_t launch_seq_attn_backward(const SeqAttn &a, cudaStream_t st) {
    return a.dtype == MNMT_BF16 ? backward<__nv_bfloat16>(a, st) : backward<__half>(a, st);
}

}  // namespace mnmt
