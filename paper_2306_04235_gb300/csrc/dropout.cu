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
#include <type_traits>

#include "fp4.cuh"
#include "internal.h"

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

// T: type of x and gx; O: type of out, r, g and gr
template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) dropout_kernel(const T *x, long ldx, bool alx, const O *r, long ldr, bool alr, float gamma,
                                                                  uint32_t thr, float scale, Philox ph, int relu, int M, int d, O *out, long ldo,
                                                                  bool alo) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    constexpr int U = 2;  // chunks in flight
    for (Walk w(d); w.row < M;) {
        Raw8<T> rx[U];
        Raw8<O> rr[U];
        long row[U];
        int c0[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            row[u] = w.row, c0[u] = w.chunk * ROW_CHUNK;
            if (row[u] < M) {
                fetch8<T, VEC>(x + row[u] * ldx, c0[u], d, alx, rx[u]);
                if (r) fetch8<O, VEC>(r + row[u] * ldr, c0[u], d, alr, rr[u]);
            }
            w.next();
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (row[u] >= M) break;
            const uint32_t keep = keep8(ph((uint32_t)(c0[u] >> 3) + (threadIdx.x & 31), (uint32_t)row[u]), thr);
            float v[8], s[8];
            settle8<T, VEC>(rx[u], alx, buf, v);
            if (r) settle8<O, VEC>(rr[u], alr, buf, s);
#pragma unroll
            for (int k = 0; k < 8; k++) {
                float y = relu && v[k] <= 0.0f ? 0.0f : v[k];  // a NaN stays
                y = (keep >> k) & 1u ? __fmul_rn(y, scale) : 0.0f;
                v[k] = r ? __fadd_rn(__fmul_rn(gamma, s[k]), y) : y;
            }
            put8<O, VEC>(out + row[u] * ldo, c0[u], d, alo, buf, v);
        }
    }
}

template <typename T, typename O, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) dropout_backward_kernel(const O *g, long ldg, bool alg, const T *x, long ldx, bool alx, const O *r,
                                                                           long ldr, bool alr, float gamma, uint32_t thr, float scale, Philox ph, int M,
                                                                           int d, T *gx, long ldgx, bool algx, O *gr, long ldgr, bool algr,
                                                                           double *partial) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    float sum = 0.0f;
    for (Walk w(d); w.row < M; w.next()) {
        const int c0 = w.chunk * ROW_CHUNK;
        Raw8<O> rg, rr;
        Raw8<T> rx;
        fetch8<O, VEC>(g + w.row * ldg, c0, d, alg, rg);
        if (partial) fetch8<O, VEC>(r + w.row * ldr, c0, d, alr, rr);
        if (x) fetch8<T, VEC>(x + w.row * ldx, c0, d, alx, rx);
        uint32_t keep = gx ? keep8(ph((uint32_t)(c0 >> 3) + (threadIdx.x & 31), (uint32_t)w.row), thr) : 0;
        float u[8], v[8];
        settle8<O, VEC>(rg, alg, buf, u);
        if (partial) {
            settle8<O, VEC>(rr, alr, buf, v);
#pragma unroll
            for (int k = 0; k < 8; k++) sum = __fmaf_rn(u[k], v[k], sum);
        }
        if (gr) {
#pragma unroll
            for (int k = 0; k < 8; k++) v[k] = __fmul_rn(gamma, u[k]);
            put8<O, VEC>(gr + w.row * ldgr, c0, d, algr, buf, v);
        }
        if (gx) {
            if (x) {  // ReLU
                settle8<T, VEC>(rx, alx, buf, v);
#pragma unroll
                for (int k = 0; k < 8; k++) keep &= ~((uint32_t)!(v[k] > 0.0f) << k);
            }
#pragma unroll
            for (int k = 0; k < 8; k++) u[k] = (keep >> k) & 1u ? __fmul_rn(u[k], scale) : 0.0f;
            put8<T, VEC>(gx + w.row * ldgx, c0, d, algx, buf, u);
        }
    }
    if (partial) {
        // the block's sum, always in the same order
        __shared__ double red[8];
        double s = sum;
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
        const bool ax = row_aligned(x, a.ldx), ar = !r || row_aligned(r, a.ldr), ao = row_aligned(out, a.ldo);
        launch_pdl(ax && ar && ao ? dropout_kernel<T, O, true> : dropout_kernel<T, O, false>, row_grid(a.M, a.d, device_sm_count()), 256, 0, st, x, a.ldx,
                   ax, r, a.ldr, ar, a.gamma, a.thr, a.scale, generator(a.seed, a.offset), a.relu, a.M, a.d, out, a.ldo, ao);
    });
    return cudaGetLastError();
}

cudaError_t launch_dropout_backward(const DropoutArgs &a, cudaStream_t st) {
    by_types(a.dtype, a.otype, [&](auto t, auto o) {
        using T = decltype(t);
        using O = decltype(o);
        const O *g = static_cast<const O *>(a.g), *r = a.ggamma ? static_cast<const O *>(a.r) : nullptr;
        const T *x = a.relu ? static_cast<const T *>(a.x) : nullptr;
        T *gx = static_cast<T *>(a.gx);
        O *gr = static_cast<O *>(a.gr);
        double *partial = a.ggamma ? static_cast<double *>(a.workspace) : nullptr;
        const bool ag = row_aligned(g, a.ldg), ax = !x || row_aligned(x, a.ldx), ar = !r || row_aligned(r, a.ldr);
        const bool agx = !gx || row_aligned(gx, a.ldgx), agr = !gr || row_aligned(gr, a.ldgr);
        const int blocks = row_grid(a.M, a.d, device_sm_count()), grid = blocks < DROPOUT_PARTIALS ? blocks : DROPOUT_PARTIALS;
        launch_pdl(ag && ax && ar && agx && agr ? dropout_backward_kernel<T, O, true> : dropout_backward_kernel<T, O, false>, grid, 256, 0, st, g, a.ldg,
                   ag, x, a.ldx, ax, r, a.ldr, ar, a.gamma, a.thr, a.scale, generator(a.seed, a.offset), a.M, a.d, gx, a.ldgx, agx, gr, a.ldgr, agr,
                   partial);
        if (partial) launch_pdl(dropout_gamma_kernel, 1, 256, 0, st, (const double *)partial, grid, a.ggamma);
    });
    return cudaGetLastError();
}

}  // namespace mnmt
