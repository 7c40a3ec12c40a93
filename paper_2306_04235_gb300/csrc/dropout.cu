// dropout.cu -- dropout from a counter-based generator, forward and backward
// (include/mnmt.h, mnmt_dropout).  No mask is stored: the backward pass draws
// the numbers of the forward pass again.
//
//   out = fl(fl(gamma r) + D(act(x))),  D(v) = keep ? fl(v s) : 0
//   gx = keep and act'(x) ? fl(g s) : 0,  gr = fl(gamma g),  ggamma = sum g r
// Generator: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", SC 2011), counter {column / 8, row, offset},
// key = seed: 128 bits, a 16-bit field for each of eight neighbouring columns.
// 16 bits, not 32, because ten rounds per four elements would take as long as
// the elements' bytes; the keep probability is then a multiple of 2^-16.
// Bound by memory where elements are wide (16384 x 2048 bf16 onto an fp32 residual
// 55 us, 6.1 TB/s), by latency where they are narrow (one step of a warp in flight:
// 16384 x 2048 bf16 to bf16 30 to 33 us, 4.0 to 4.5 TB/s, issue 56 %; backward with ReLU 47)
// or start anywhere (backward of 5003 x 1001 fp16 with all gradients 20 us, 3.9 TB/s).
#include <type_traits>

#include "fp4.cuh"
#include "row_pass.cuh"
#include "train.h"

namespace mnmt {
namespace {

struct Philox {
    uint32_t k0, k1;
    uint32_t o0, o1;  // the offset: counter words 2 and 3
    MNMT_DEV uint4 operator()(uint32_t c0, uint32_t c1) const {
        uint32_t a = c0, b = c1, c = o0, d = o1, x = k0, y = k1;
#pragma unroll
        for (int i = 0; i < 10; i++) {
            const unsigned long long p = (unsigned long long)0xD2511F53u * a, q = (unsigned long long)0xCD9E8D57u * c;
            a = (uint32_t)(q >> 32) ^ b ^ x;
            b = (uint32_t)q;
            c = (uint32_t)(p >> 32) ^ d ^ y;
            d = (uint32_t)p;
            x += 0x9E3779B9u;
            y += 0xBB67AE85u;
        }
        return make_uint4(a, b, c, d);
    }
};

// bit i: element i of the eight is kept
MNMT_DEV uint32_t keep8(const uint4 w, uint32_t thr) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t k = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        k |= (uint32_t)((u[i] & 0xFFFFu) >= thr) << (2 * i);
        k |= (uint32_t)((u[i] >> 16) >= thr) << (2 * i + 1);
    }
    return k;
}

// the E elements of a lane: one or two counters
template <int E>
MNMT_DEV uint32_t keep_lane(const Philox &ph, const RowAt &a, uint32_t thr) {
    const uint32_t g = (uint32_t)a.c >> 3, row = (uint32_t)a.row;
    uint32_t k = keep8(ph(g, row), thr);
    if constexpr (E == 16) k |= keep8(ph(g + 1, row), thr) << 8;
    return k;
}

// Steps of eight products that a lane's part of ggamma stays in fp32: a chain of 512
// additions whatever the matrix, and one in 64 bits for it.
constexpr int GAMMA_STEPS = 64;

// T: type of x and gx; O: type of out, r, g and gr
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) dropout_kernel(const T *x, long ldx, int alx, const O *r, long ldr, int alr, float gamma, uint32_t thr,
                                                                  float scale, Philox ph, int relu, int M, int d, O *out, long ldo, int alo, int lr) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    constexpr int E = row_elements(VEC);
    for (Walk<E> w(M, d, lr); w.more(); w.next()) {
        const RowAt a = w.at();
        const bool ok = a.row < M;
        Raw<T, E> rx;
        Raw<O, E> rr;
        fetch<T, VEC>(x + a.row * ldx, w, a, d, ok, alx, rx);
        if (r) fetch<O, VEC>(r + a.row * ldr, w, a, d, ok, alr, rr);
        const uint32_t keep = keep_lane<E>(ph, a, thr);
        float v[E];
        settle<T, VEC>(rx, w, alx, buf, v);
#pragma unroll
        for (int k = 0; k < E; k++) {
            const float y = relu && v[k] <= 0.0f ? 0.0f : v[k];  // a NaN stays
            v[k] = (keep >> k) & 1u ? __fmul_rn(y, scale) : 0.0f;
        }
        if (r) {
            float s[E];
            settle<O, VEC>(rr, w, alr, buf, s);
#pragma unroll
            for (int k = 0; k < E; k++) v[k] = __fadd_rn(__fmul_rn(gamma, s[k]), v[k]);
        }
        put<O, VEC>(out + a.row * ldo, w, a, d, ok, alo, buf, v);
    }
}

template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) dropout_backward_kernel(const O *g, long ldg, int alg, const T *x, long ldx, int alx, const O *r,
                                                                           long ldr, int alr, float gamma, uint32_t thr, float scale, Philox ph, int M,
                                                                           int d, T *gx, long ldgx, int algx, O *gr, long ldgr, int algr,
                                                                           double *partial, int lr) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    constexpr int E = 8;  // whatever the alignment, so that ggamma's sum has one order
    __shared__ double totals[256];  // a lane's sum but for the last steps (in shared memory for the registers)
    if (partial) totals[threadIdx.x] = 0.0;
    float sum = 0.0f;  // of at most GAMMA_STEPS steps
    int steps = GAMMA_STEPS;
    for (Walk<E> w(M, d, lr); w.more(); w.next()) {
        const RowAt a = w.at();
        const bool ok = a.row < M;
        Raw<O, E> rg, rr;
        Raw<T, E> rx;
        fetch<O, VEC>(g + a.row * ldg, w, a, d, ok, alg, rg);
        if (partial) fetch<O, VEC>(r + a.row * ldr, w, a, d, ok, alr, rr);
        if (x) fetch<T, VEC>(x + a.row * ldx, w, a, d, ok, alx, rx);
        uint32_t keep = gx ? keep_lane<E>(ph, a, thr) : 0;
        float u[E], v[E];
        settle<O, VEC>(rg, w, alg, buf, u);
        if (partial) {
            settle<O, VEC>(rr, w, alr, buf, v);
#pragma unroll
            for (int k = 0; k < E; k++) sum = __fmaf_rn(u[k], v[k], sum);
            if (--steps == 0) totals[threadIdx.x] += sum, sum = 0.0f, steps = GAMMA_STEPS;
        }
        if (gr) {
#pragma unroll
            for (int k = 0; k < E; k++) v[k] = __fmul_rn(gamma, u[k]);
            put<O, VEC>(gr + a.row * ldgr, w, a, d, ok, algr, buf, v);
        }
        if (gx) {
            if (x) {  // ReLU
                settle<T, VEC>(rx, w, alx, buf, v);
#pragma unroll
                for (int k = 0; k < E; k++) keep &= ~((uint32_t)!(v[k] > 0.0f) << k);
            }
#pragma unroll
            for (int k = 0; k < E; k++) u[k] = (keep >> k) & 1u ? __fmul_rn(u[k], scale) : 0.0f;
            put<T, VEC>(gx + a.row * ldgx, w, a, d, ok, algx, buf, u);
        }
    }
    if (partial) {
        // the block's sum, always in the same order
        __shared__ double red[8];
        double s = totals[threadIdx.x] + sum;
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
        __syncthreads();
        if (threadIdx.x == 0) {
            double t = 0.0;
            for (int w = 0; w < 8; w++) t += red[w];
            partial[blockIdx.x] = t;
        }
    }
}

// ggamma = the sum of n partial sums, in a fixed order
__global__ void __launch_bounds__(256) dropout_gamma_kernel(const double *partial, int n, float *ggamma) {
    pdl_grid_wait();
    __shared__ double red[256];
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) s += partial[i];
    red[threadIdx.x] = s;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
        if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) *ggamma = (float)red[0];
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

Philox generator(uint64_t seed, uint64_t offset) {
    return Philox{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)};
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs &a, cudaStream_t st) {
    by_types(a.dtype, a.otype, [&](auto t, auto o) {
        using T = decltype(t);
        using O = decltype(o);
        const T *x = static_cast<const T *>(a.x);
        const O *r = static_cast<const O *>(a.r);
        O *out = static_cast<O *>(a.out);
        const int ax = row_alignment(x, a.ldx), ar = r ? row_alignment(r, a.ldr) : 2, ao = row_alignment(out, a.ldo);
        const bool vec = ax == 2 && ar == 2 && ao == 2;
        launch_pdl(vec ? dropout_kernel<T, O, true> : dropout_kernel<T, O, false>, row_grid(a.M, a.d, vec, device_sm_count()), 256, 0, st, x, a.ldx,
                   ax, r, a.ldr, ar, a.gamma, a.thr, a.scale, generator(a.seed, a.offset), a.relu, a.M, a.d, out, a.ldo, ao,
                   row_lanes(a.d, vec));
    });
    return cudaGetLastError();
}

cudaError_t launch_dropout_backward(const DropoutArgs &a, cudaStream_t st) {
    by_types(a.dtype, a.otype, [&](auto t, auto o) {
        using T = decltype(t);
        using O = decltype(o);
        const O *g = static_cast<const O *>(a.g), *r = static_cast<const O *>(a.backward_r());
        const T *x = static_cast<const T *>(a.backward_x());
        T *gx = static_cast<T *>(a.gx);
        O *gr = static_cast<O *>(a.gr);
        double *partial = a.ggamma ? static_cast<double *>(a.workspace) : nullptr;
        const int ag = row_alignment(g, a.ldg), ax = x ? row_alignment(x, a.ldx) : 2, ar = r ? row_alignment(r, a.ldr) : 2;
        const int agx = gx ? row_alignment(gx, a.ldgx) : 2, agr = gr ? row_alignment(gr, a.ldgr) : 2;
        const bool vec = ag == 2 && ax == 2 && ar == 2 && agx == 2 && agr == 2;
        const int blocks = row_grid(a.M, a.d, false, device_sm_count()), grid = blocks < DROPOUT_PARTIALS ? blocks : DROPOUT_PARTIALS;
        launch_pdl(vec ? dropout_backward_kernel<T, O, true> : dropout_backward_kernel<T, O, false>, grid, 256, 0, st, g, a.ldg,
                   ag, x, a.ldx, ax, r, a.ldr, ar, a.gamma, a.thr, a.scale, generator(a.seed, a.offset), a.M, a.d, gx, a.ldgx, agx, gr, a.ldgr, agr,
                   partial, row_lanes(a.d, false));
        if (partial) launch_pdl(dropout_gamma_kernel, 1, 256, 0, st, (const double *)partial, grid, a.ggamma);
    });
    return cudaGetLastError();
}

}  // namespace mnmt
