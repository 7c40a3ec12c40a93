// train.h -- launches of the operators on microscaled 4-bit floating point (fp4.cuh),
// of dropout, of attention over sequences (seq_attn.cuh) and of the embedding.
#pragma once

#include "internal.h"

namespace mnmt {

// one-time set-up on the current device; MNMT_OK or an error code (recorded)
int ensure_device();

struct Fp4Args;
cudaError_t launch_fp4_quantize(const void *x, int dtype, long ldx, const Fp4Args &q, bool nv, void *values, long ldv,
                                cudaStream_t st);
cudaError_t launch_fp4_dequantize(const Fp4Args &q, bool nv, void *values, int dtype, long ldv, cudaStream_t st);
cudaError_t launch_fp4_quantize_backward(const void *x, int dtype, long ldx, const void *g, long ldg, void *gx, long ldgx,
                                         int rows, int cols, bool nv, float tg, float inv6g, cudaStream_t st);
cudaError_t launch_fp4_product(const Fp4Args &x, const Fp4Args &w, bool nv, float alpha, const float *bias, int relu,
                               void *y, int ydtype, long ldy, int *status, cudaStream_t st);
// a few rows: quantisation (x non-null) and product in one launch
cudaError_t launch_fp4_small(const Fp4Args &x, const Fp4Args &w, bool nv, const void *xp, int xdtype, long ldx, float alpha,
                             const float *bias, int relu, void *y, int ydtype, long ldy, cudaStream_t st);
cudaError_t fp4_init();  // set-up of the product kernels on the current device
cudaError_t fp4_backward_init();
size_t fp4_backward_workspace(int M, int N, int K);

constexpr int DROPOUT_PARTIALS = MNMT_DROPOUT_WORKSPACE / 8;  // blocks of a backward pass, at most
struct DropoutArgs {
    const void *x, *r, *g;  // g: backward
    long ldx, ldr, ldg;
    int dtype, otype;       // of x and gx; of r, out, g and gr
    float gamma, scale;
    uint32_t thr;           // keep a field of 16 bits >= thr
    int relu, M, d;
    uint64_t seed, offset;
    void *out, *gx, *gr;
    long ldo, ldgx, ldgr;
    float *ggamma;
    void *workspace;
    // what a backward pass reads beside g: x where ReLU decides about gx, r for the gain (their types are given then only)
    const void *backward_x() const { return relu && gx ? x : nullptr; }
    const void *backward_r() const { return ggamma ? r : nullptr; }
};
cudaError_t launch_dropout(const DropoutArgs &a, cudaStream_t st);
cudaError_t launch_dropout_backward(const DropoutArgs &a, cudaStream_t st);

// element (row, head, e) of an attention operand is at p + row * ld + head * hd + e
struct HeadRows {
    void *p;
    long ld, hd;
};
// attention over sequences (seq_attn.cuh); sequence b has query rows from q_start[b] on, q_len[b] of them
// (q_len null: up to q_start[b + 1]), keys alike
struct SeqAttn {
    int n_seqs, q_rows, k_rows, hq, hkv, dh, dtype, causal;
    float scale;
    const int *q_start, *q_len, *k_start, *k_len;
    HeadRows q, k, v, o;
    float *lse;  // [hq][q_rows], natural logarithm
    HeadRows g, dq, dk, dv;  // backward: output gradient, results
    void *workspace;
    int *status;
    __host__ __device__ int group() const { return hq / hkv; }
};
cudaError_t seq_attn_init();  // set-up of the kernels on the current device
cudaError_t seq_attn_backward_init();
cudaError_t seq_attn_token_init();
cudaError_t launch_seq_wait_selftest(int *status, cudaStream_t st);
size_t seq_attn_forward_workspace(const SeqAttn &a);
size_t seq_attn_backward_workspace(const SeqAttn &a);
size_t seq_attn_token_workspace(const SeqAttn &a);
cudaError_t launch_seq_attn_forward(const SeqAttn &a, cudaStream_t st);
cudaError_t launch_seq_attn_backward(const SeqAttn &a, cudaStream_t st);
cudaError_t launch_seq_attn_token(const SeqAttn &a, cudaStream_t st);

struct EmbedRowsArgs {
    const int32_t *ids, *pos;  // [T]; pos null: row t is position t
    int T, V, d, P;
    const void *table;         // backward: the gradient of the rows [T][d]
    int dtype;
    long ld;
    float scale;
    const float *pe;           // null: none
    long ldpe;
    void *out;                 // backward: the gradient of the table [V][d]
    int otype;
    long ldo;
    int pad_id, accumulate;    // backward
    int wide;                  // backward: rows of out start on 32 bytes
    void *workspace;
    int *status;
};
cudaError_t launch_embed_rows(const EmbedRowsArgs &a, cudaStream_t st);
cudaError_t launch_embed_rows_backward(const EmbedRowsArgs &a, cudaStream_t st);
size_t embed_rows_backward_workspace(int T, int V, int d);

}  // namespace mnmt
