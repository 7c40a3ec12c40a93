// fp4_linear.cu -- the linear on microscaled 4-bit floating-point operands and
// its gradients (include/mnmt.h, mnmt_fp4_linear, mnmt_fp4_linear_backward).
//
//   y = act(alpha sum_k X[m][k] W[n][k] + bias[n]),  X, W the codes times their
//   block scales, alpha the product of the tensor scales (NV; 1 for MX)
//   gX = in_x (alpha_w sum_n G[m][n] W[n][k]),  gW = in_w (alpha_x sum_m G[m][n] X[m][k]),
//   gb = sum_m G[m][n];  in_x, in_w: the element lies within its block's range
//
// A block of 256 threads computes a 64 x 64 tile of a product in fp32, both
// operands decoded into shared memory 16 reduction indices at a time.
#include <type_traits>

#include "fp4.cuh"
#include "internal.h"

namespace mnmt {
namespace {

constexpr int PT = 64, PK = 16;

// element (row, k) of a packed matrix, without the tensor scale
template <bool NV>
MNMT_DEV float fp4_at(const Fp4Args &q, int row, int k) {
    if (row >= q.rows || k >= q.cols) return 0.0f;
    const uint32_t byte = q.codes[(size_t)row * fp4_pitch(q.cols) + (k >> 1)];
    const float2 f = fp4_float2(byte);
    const Fp4Scale s = fp4_scale_of<NV>(q.scales[fp4_scale_at(row, k / fp4_block(NV), fp4_tiles_k(q.cols, NV))], 1.0f);
    return __fmul_rn(k & 1 ? f.y : f.x, s.S);
}

// acc[i][j] of rows i0 + ty + 16 i and columns j0 + tx + 16 j of sum_k a(i, k) b(j, k)
template <typename A, typename B>
MNMT_DEV void tile_product(float (&acc)[4][4], int K, A &&a, B &&b) {
    __shared__ float sa[PK][PT + 1], sb[PK][PT + 1];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int i0 = blockIdx.y * PT, j0 = blockIdx.x * PT;
    for (int k0 = 0; k0 < K; k0 += PK) {
        for (int t = threadIdx.x; t < PT * PK; t += 256) {
            sa[t % PK][t / PK] = k0 + t % PK < K ? a(i0 + t / PK, k0 + t % PK) : 0.0f;
            sb[t % PK][t / PK] = k0 + t % PK < K ? b(j0 + t / PK, k0 + t % PK) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PK; k++)
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = __fmaf_rn(sa[k][ty + 16 * i], sb[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
}

// whether fp32 x lies within the range of its block
template <bool NV>
MNMT_DEV bool fp4_inside(const Fp4Args &q, int row, int k, float x) {
    const Fp4Scale s = fp4_scale_of<NV>(q.scales[fp4_scale_at(row, k / fp4_block(NV), fp4_tiles_k(q.cols, NV))], q.g);
    return fabsf(__fmul_rn(x, s.r)) <= 6.0f;
}

// o[i][k] = inside ? alpha sum_j ... : 0.  INPUT: gX, i over rows of x, reduced
// over n; else gW, i over rows of w, reduced over m.  T: type of the original
// (mask) and of gX; R: type of the result.
template <bool NV, bool INPUT, typename T, typename R>
__global__ void __launch_bounds__(256) fp4_gradient_kernel(const __nv_bfloat16 *g, long ldg, int M, int N, Fp4Args other, Fp4Args own,
                                                           float alpha, const T *orig, long ldo, R *out, long ldout) {
    pdl_grid_wait();
    float acc[4][4] = {};
    if (INPUT)
        tile_product(acc, N, [&](int m, int n) { return m < M ? __bfloat162float(g[m * ldg + n]) : 0.0f; },
                     [&](int k, int n) { return fp4_at<NV>(other, n, k); });
    else
        tile_product(acc, M, [&](int n, int m) { return n < N ? __bfloat162float(g[m * ldg + n]) : 0.0f; },
                     [&](int k, int m) { return fp4_at<NV>(other, m, k); });
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) {
            const int r = blockIdx.y * PT + ty + 16 * i, k = blockIdx.x * PT + tx + 16 * j;
            if (r >= own.rows || k >= own.cols) continue;
            const bool in = !orig || fp4_inside<NV>(own, r, k, to_f32(orig[r * ldo + k]));
            out[r * ldout + k] = from_f32<R>(in ? __fmul_rn(alpha, acc[i][j]) : 0.0f);
        }
}

// gb[n] = sum over m of G[m][n]
__global__ void __launch_bounds__(256) fp4_bias_gradient_kernel(const __nv_bfloat16 *g, long ldg, int M, int N, float *gb) {
    pdl_grid_wait();
    __shared__ float red[8][32];
    const int n = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
    float s = 0.0f;
    if (n < N)
        for (int m = w; m < M; m += 8) s += __bfloat162float(g[m * ldg + n]);
    red[w][threadIdx.x & 31] = s;
    __syncthreads();
    if (w == 0 && n < N) {
        for (int i = 1; i < 8; i++) s += red[i][threadIdx.x & 31];
        gb[n] = s;
    }
}

template <typename F>
void by_type(int dtype, F &&f) {
    if (dtype == MNMT_F32) f(float{});
    else if (dtype == MNMT_BF16) f(__nv_bfloat16{});
    else f(__half{});
}

dim3 tiles(int rows, int cols) { return dim3((cols + PT - 1) / PT, (rows + PT - 1) / PT); }

}  // namespace

size_t fp4_backward_workspace(int, int, int) { return 16; }

cudaError_t launch_fp4_linear_backward(const Fp4BackwardArgs &a, cudaStream_t st) {
    const __nv_bfloat16 *g = static_cast<const __nv_bfloat16 *>(a.g);
    const int M = a.x.rows, N = a.w.rows, K = a.x.cols;
    if (a.gx)
        by_type(a.xdtype, [&](auto t) {
            using T = decltype(t);
            launch_pdl(a.nv ? fp4_gradient_kernel<true, true, T, T> : fp4_gradient_kernel<false, true, T, T>, tiles(M, K), 256, 0, st, g, a.ldg, M,
                       N, a.w, a.x, a.nv ? a.w.g : 1.0f, static_cast<const T *>(a.xo), a.ldx, static_cast<T *>(a.gx), a.ldgx);
        });
    if (a.gw)
        by_type(a.wdtype, [&](auto t) {
            using T = decltype(t);
            launch_pdl(a.nv ? fp4_gradient_kernel<true, false, T, float> : fp4_gradient_kernel<false, false, T, float>, tiles(N, K), 256, 0, st, g,
                       a.ldg, M, N, a.x, a.w, a.nv ? a.x.g : 1.0f, static_cast<const T *>(a.wo), a.ldw, a.gw, a.ldgw);
        });
    if (a.gb) launch_pdl(fp4_bias_gradient_kernel, (N + 31) / 32, 256, 0, st, g, a.ldg, M, N, a.gb);
    return cudaGetLastError();
}

}  // namespace mnmt
