// train.h -- launches of the operators on microscaled 4-bit floating point (fp4.cuh)
// and of dropout.
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

}  // namespace mnmt
