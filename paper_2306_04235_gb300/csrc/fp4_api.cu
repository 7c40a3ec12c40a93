// fp4_api.cu -- entry points of the 4-bit floating-point operators and of
// dropout: argument checks, then the launchers.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>

#include "fp4.cuh"
#include "routes.h"
#include "train.h"

using namespace mnmt;

namespace {

constexpr int32_t MAX_DIM = 1 << 30;

int fail(int code, const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return set_error(code, buf);
}

int done(cudaError_t e, const char *call) {
    return e == cudaSuccess ? MNMT_OK : fail(MNMT_ECUDA, "%s: %s", call, cudaGetErrorString(e));
}

int type_size(int32_t dtype) { return dtype == MNMT_F32 ? 4 : dtype == MNMT_BF16 || dtype == MNMT_F16 ? 2 : 0; }
bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// a matrix argument: p non-null and aligned to its elements, ld wide enough
bool matrix_ok(const void *p, int32_t dtype, int64_t ld, int32_t cols) {
    const int e = type_size(dtype);
    return e && p && aligned(p, e) && ld >= cols && ld <= ((int64_t)1 << 40);
}

// Whether `out` may be written while `in` is read: apart, or in place with one row
// stride.  With two, a warp would write over rows that others have yet to read.
bool in_place_ok(const void *out, int64_t ldo, const void *in, int64_t ldi, int32_t rows) { return out != in || !out || ldo == ldi || rows <= 1; }

// one-time set-up of the product kernels, apart from the library's own so that
// programs that only translate do not load them
int fp4_ready() {
    if (int rc = ensure_device()) return rc;
    static std::mutex mu;
    static bool ready[64] = {false};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return fail(MNMT_ECUDA, "fp4: no usable current device");
    std::lock_guard<std::mutex> lk(mu);
    if (!ready[dev]) {
        cudaError_t e = fp4_init();
        if (e == cudaSuccess) e = fp4_backward_init();
        if (e != cudaSuccess) return fail(MNMT_ECUDA, "fp4 kernel set-up failed: %s", cudaGetErrorString(e));
        ready[dev] = true;
    }
    return MNMT_OK;
}

// 0 if q's sizes and format are valid (and, with buffers, its pointers)
int check_fp4(const char *call, const mnmt_fp4 *q, bool buffers) {
    if (!q) return fail(MNMT_EINVAL, "%s: null matrix", call);
    if (q->rows < 0 || q->cols < 1 || q->rows > MAX_DIM || q->cols > MAX_DIM)
        return fail(MNMT_EINVAL, "%s: bad size %d x %d", call, q->rows, q->cols);
    if (q->format != MNMT_FP4_MX && q->format != MNMT_FP4_NV) return fail(MNMT_EINVAL, "%s: unknown format %d", call, q->format);
    if (q->format == MNMT_FP4_NV && !(q->tensor_scale >= 0x1p-100f && q->tensor_scale <= 0x1p100f))
        return fail(MNMT_EINVAL, "%s: tensor scale %g outside [2^-100, 2^100]", call, q->tensor_scale);
    if (buffers && q->rows > 0 && (!q->codes || !q->scales)) return fail(MNMT_EINVAL, "%s: null codes or scales", call);
    if (!aligned(q->codes, 16) || !aligned(q->scales, 16)) return fail(MNMT_EINVAL, "%s: codes and scales must be 16-byte aligned", call);
    return MNMT_OK;
}

bool is_nv(const mnmt_fp4 *q) { return q->format == MNMT_FP4_NV; }

Fp4Args args_of(const mnmt_fp4 *q) {
    Fp4Args a;
    a.codes = q->codes;
    a.scales = q->scales;
    a.rows = q->rows;
    a.cols = q->cols;
    a.g = is_nv(q) ? q->tensor_scale : 1.0f;
    const float six = 6.0f * a.g;
    a.inv6g = 1.0f / six;
    return a;
}

// threshold and factor of a drop probability
bool drop_args(DropoutArgs &a, float p) {
    if (!(p >= 0.0f && p <= 1.0f)) return false;
    a.thr = (uint32_t)std::nearbyint(p * 65536.0f);
    a.scale = a.thr < 65536u ? 65536.0f / (float)(65536u - a.thr) : 0.0f;
    return true;
}

}  // namespace

extern "C" size_t mnmt_fp4_pitch(int32_t cols) { return cols < 1 ? 0 : fp4_pitch(cols); }

extern "C" size_t mnmt_fp4_scale_bytes(int32_t rows, int32_t cols, int32_t format) {
    return rows < 1 || cols < 1 ? 0 : fp4_scale_bytes(rows, cols, format == MNMT_FP4_NV);
}

extern "C" int mnmt_fp4_quantize(const mnmt_fp4 *q, const void *x, int32_t dtype, int64_t ldx, void *values, int64_t ldv, void *cuda_stream) {
    int rc = ensure_device();
    if (rc) return rc;
    if ((rc = check_fp4("fp4_quantize", q, false))) return rc;
    if (!type_size(dtype)) return fail(MNMT_EINVAL, "fp4_quantize: unknown type %d", dtype);
    if (q->rows == 0) return MNMT_OK;
    if (!q->codes != !q->scales || (!q->codes && !values)) return fail(MNMT_EINVAL, "fp4_quantize: codes and scales, values or all three");
    if (!matrix_ok(x, dtype, ldx, q->cols) || (values && !matrix_ok(values, dtype, ldv, q->cols)))
        return fail(MNMT_EINVAL, "fp4_quantize: bad pointer or row stride");
    if (!in_place_ok(values, ldv, x, ldx, q->rows)) return fail(MNMT_EINVAL, "fp4_quantize: in place needs one row stride");
    return done(launch_fp4_quantize(x, dtype, ldx, args_of(q), is_nv(q), values, ldv, static_cast<cudaStream_t>(cuda_stream)), "fp4_quantize");
}

extern "C" int mnmt_fp4_dequantize(const mnmt_fp4 *q, void *values, int32_t dtype, int64_t ldv, void *cuda_stream) {
    int rc = ensure_device();
    if (rc) return rc;
    if ((rc = check_fp4("fp4_dequantize", q, true))) return rc;
    if (!type_size(dtype)) return fail(MNMT_EINVAL, "fp4_dequantize: unknown type %d", dtype);
    if (q->rows == 0) return MNMT_OK;
    if (!matrix_ok(values, dtype, ldv, q->cols)) return fail(MNMT_EINVAL, "fp4_dequantize: bad pointer or row stride");
    return done(launch_fp4_dequantize(args_of(q), is_nv(q), values, dtype, ldv, static_cast<cudaStream_t>(cuda_stream)), "fp4_dequantize");
}

extern "C" int mnmt_fp4_quantize_backward(const mnmt_fp4 *q, const void *x, int32_t dtype, int64_t ldx, const void *g, int64_t ldg, void *gx,
                                          int64_t ldgx, void *cuda_stream) {
    int rc = ensure_device();
    if (rc) return rc;
    if ((rc = check_fp4("fp4_quantize_backward", q, false))) return rc;
    if (!type_size(dtype)) return fail(MNMT_EINVAL, "fp4_quantize_backward: unknown type %d", dtype);
    if (q->rows == 0) return MNMT_OK;
    if (!matrix_ok(x, dtype, ldx, q->cols) || !matrix_ok(g, dtype, ldg, q->cols) || !matrix_ok(gx, dtype, ldgx, q->cols))
        return fail(MNMT_EINVAL, "fp4_quantize_backward: bad pointer or row stride");
    if (!in_place_ok(gx, ldgx, x, ldx, q->rows) || !in_place_ok(gx, ldgx, g, ldg, q->rows))
        return fail(MNMT_EINVAL, "fp4_quantize_backward: in place needs one row stride");
    const Fp4Args a = args_of(q);
    return done(launch_fp4_quantize_backward(x, dtype, ldx, g, ldg, gx, ldgx, q->rows, q->cols, is_nv(q), a.g, a.inv6g,
                                             static_cast<cudaStream_t>(cuda_stream)),
                "fp4_quantize_backward");
}

extern "C" int mnmt_fp4_linear(const mnmt_fp4 *xq, const mnmt_fp4 *w, const void *x, int32_t xdtype, int64_t ldx, const float *bias, int32_t relu,
                               void *y, int32_t ydtype, int64_t ldy, int32_t *status, void *cuda_stream) {
    int rc = fp4_ready();
    if (rc) return rc;
    if ((rc = check_fp4("fp4_linear", xq, true)) || (rc = check_fp4("fp4_linear", w, true))) return rc;
    if (xq->cols != w->cols || xq->format != w->format) return fail(MNMT_EINVAL, "fp4_linear: operands of different depth or format");
    if (!type_size(ydtype) || (x && !type_size(xdtype))) return fail(MNMT_EINVAL, "fp4_linear: unknown type");
    if (xq->rows == 0) return MNMT_OK;
    if (x && !matrix_ok(x, xdtype, ldx, xq->cols)) return fail(MNMT_EINVAL, "fp4_linear: bad input pointer or row stride");
    if (w->rows > 0 && !matrix_ok(y, ydtype, ldy, w->rows)) return fail(MNMT_EINVAL, "fp4_linear: bad output pointer or row stride");
    if (!aligned(bias, 4) || !aligned(status, 4)) return fail(MNMT_EINVAL, "fp4_linear: bias and status must be 4-byte aligned");
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const Fp4Args a = args_of(xq), b = args_of(w);
    if (w->rows > 0 && route_fp4_small(a.rows, b.rows, a.cols))
        return done(launch_fp4_small(a, b, is_nv(w), x, xdtype, ldx, a.g * b.g, bias, relu != 0, y, ydtype, ldy, st), "fp4_linear");
    if (x) {
        cudaError_t e = launch_fp4_quantize(x, xdtype, ldx, a, is_nv(xq), nullptr, 0, st);
        if (e != cudaSuccess) return done(e, "fp4_linear");
    }
    if (w->rows == 0) return MNMT_OK;
    return done(launch_fp4_product(a, b, is_nv(w), a.g * b.g, bias, relu != 0, y, ydtype, ldy, status, st), "fp4_linear");
}

extern "C" size_t mnmt_fp4_linear_backward_workspace(int32_t M, int32_t N, int32_t K) {
    return M < 0 || N < 0 || K < 1 || M > MAX_DIM || N > MAX_DIM || K > MAX_DIM ? 0 : fp4_backward_workspace(M, N, K);
}

extern "C" int mnmt_fp4_linear_backward(const mnmt_fp4 *xq, const mnmt_fp4 *wq, const void *G, int64_t ldg, const void *x, int32_t xdtype,
                                        int64_t ldx, const void *w, int32_t wdtype, int64_t ldw, void *workspace, void *gx, int64_t ldgx,
                                        float *gw, int64_t ldgw, float *gb, int32_t *status, void *cuda_stream) {
    int rc = fp4_ready();
    if (rc) return rc;
    if ((rc = check_fp4("fp4_linear_backward", xq, true)) || (rc = check_fp4("fp4_linear_backward", wq, true))) return rc;
    const int M = xq->rows, N = wq->rows, K = xq->cols;
    if (K != wq->cols || xq->format != wq->format) return fail(MNMT_EINVAL, "fp4_linear_backward: operands of different depth or format");
    if ((M > 0 && N > 0 && !matrix_ok(G, MNMT_BF16, ldg, N)) || (M > 0 && (x || gx) && !type_size(xdtype)) ||
        (N > 0 && w && !type_size(wdtype)) || (M > 0 && x && !matrix_ok(x, xdtype, ldx, K)) || (N > 0 && w && !matrix_ok(w, wdtype, ldw, K)) ||
        (M > 0 && gx && !matrix_ok(gx, xdtype, ldgx, K)) || (N > 0 && gw && !matrix_ok(gw, MNMT_F32, ldgw, K)))
        return fail(MNMT_EINVAL, "fp4_linear_backward: bad type, pointer or row stride");
    if (!workspace || !aligned(workspace, 16)) return fail(MNMT_EINVAL, "fp4_linear_backward: workspace must be given, 16-byte aligned");
    if (!aligned(gb, 4) || !aligned(status, 4)) return fail(MNMT_EINVAL, "fp4_linear_backward: gb and status must be 4-byte aligned");
    Fp4BackwardArgs a;
    a.x = args_of(xq);
    a.w = args_of(wq);
    a.nv = is_nv(xq);
    a.g = G;
    a.ldg = ldg;
    a.xo = x;
    a.wo = w;
    a.ldx = ldx;
    a.ldw = ldw;
    a.xdtype = x || gx ? xdtype : MNMT_F32;
    a.wdtype = w ? wdtype : MNMT_F32;
    a.workspace = workspace;
    a.gx = M > 0 ? gx : nullptr;
    a.ldgx = ldgx;
    a.gw = N > 0 ? gw : nullptr;
    a.ldgw = ldgw;
    a.gb = N > 0 ? gb : nullptr;
    a.status = status;
    return done(launch_fp4_linear_backward(a, static_cast<cudaStream_t>(cuda_stream)), "fp4_linear_backward");
}

extern "C" int mnmt_dropout(const void *x, int32_t dtype, int64_t ldx, const void *r, int64_t ldr, float gamma, float p, uint64_t seed,
                            uint64_t offset, int32_t relu, int32_t M, int32_t d, void *out, int32_t otype, int64_t ldo, void *cuda_stream) {
    int rc = ensure_device();
    if (rc) return rc;
    DropoutArgs a;
    std::memset(&a, 0, sizeof(a));
    if (M < 0 || d < 1 || M > MAX_DIM || d > MAX_DIM || !type_size(dtype) || !type_size(otype))
        return fail(MNMT_EINVAL, "dropout: bad size %d x %d or type", M, d);
    if (!drop_args(a, p)) return fail(MNMT_EINVAL, "dropout: probability %g outside [0, 1]", p);
    if (M == 0) return MNMT_OK;
    if (!matrix_ok(x, dtype, ldx, d) || !matrix_ok(out, otype, ldo, d) || (r && !matrix_ok(r, otype, ldr, d)))
        return fail(MNMT_EINVAL, "dropout: bad pointer or row stride");
    if ((out == x && (dtype != otype || ldo != ldx)) || !in_place_ok(out, ldo, r, ldr, M))
        return fail(MNMT_EINVAL, "dropout: in place needs one type and stride");
    a.x = x, a.ldx = ldx, a.dtype = dtype;
    a.r = r, a.ldr = ldr, a.gamma = gamma;
    a.out = out, a.ldo = ldo, a.otype = otype;
    a.seed = seed, a.offset = offset, a.relu = relu != 0, a.M = M, a.d = d;
    return done(launch_dropout(a, static_cast<cudaStream_t>(cuda_stream)), "dropout");
}

extern "C" int mnmt_dropout_backward(const void *g, int32_t otype, int64_t ldg, const void *x, int32_t dtype, int64_t ldx, const void *r,
                                     int64_t ldr, float gamma, float p, uint64_t seed, uint64_t offset, int32_t relu, int32_t M, int32_t d,
                                     void *gx, int64_t ldgx, void *gr, int64_t ldgr, float *ggamma, void *workspace, void *cuda_stream) {
    int rc = ensure_device();
    if (rc) return rc;
    DropoutArgs a;
    std::memset(&a, 0, sizeof(a));
    if (M < 0 || d < 1 || M > MAX_DIM || d > MAX_DIM || !type_size(otype) || ((gx || (relu && x)) && !type_size(dtype)))
        return fail(MNMT_EINVAL, "dropout_backward: bad size %d x %d or type", M, d);
    if (!drop_args(a, p)) return fail(MNMT_EINVAL, "dropout_backward: probability %g outside [0, 1]", p);
    if (!gx && !gr && !ggamma) return fail(MNMT_EINVAL, "dropout_backward: no output");
    if (M > 0 && (!matrix_ok(g, otype, ldg, d) || (gx && !matrix_ok(gx, dtype, ldgx, d)) || (gx && relu && !matrix_ok(x, dtype, ldx, d)) ||
                  (gr && !matrix_ok(gr, otype, ldgr, d)) || (ggamma && !matrix_ok(r, otype, ldr, d))))
        return fail(MNMT_EINVAL, "dropout_backward: bad pointer or row stride");
    if (ggamma && (!aligned(ggamma, 4) || !workspace || !aligned(workspace, 8)))
        return fail(MNMT_EINVAL, "dropout_backward: ggamma needs an 8-byte aligned workspace");
    if (gx && gx == gr) return fail(MNMT_EINVAL, "dropout_backward: gx and gr are one buffer");
    if ((M > 0 && gx && gx == g && (dtype != otype || ldgx != ldg)) || (relu && !in_place_ok(gx, ldgx, x, ldx, M)) ||
        !in_place_ok(gr, ldgr, g, ldg, M))
        return fail(MNMT_EINVAL, "dropout_backward: in place needs one type and stride");
    a.g = g, a.ldg = ldg, a.otype = otype;
    a.x = x, a.ldx = ldx, a.dtype = gx ? dtype : MNMT_F32;
    a.r = r, a.ldr = ldr, a.gamma = gamma;
    a.seed = seed, a.offset = offset, a.relu = relu != 0, a.M = M, a.d = d;
    a.gx = gx, a.ldgx = ldgx, a.gr = gr, a.ldgr = ldgr, a.ggamma = ggamma, a.workspace = workspace;
    return done(launch_dropout_backward(a, static_cast<cudaStream_t>(cuda_stream)), "dropout_backward");
}
