// fp4.cu -- quantisation to microscaled 4-bit floating point, its inverse and
// its straight-through backward pass (include/mnmt.h, mnmt_fp4_*).
//
// Per block of 32 (MX) or 16 (NV) elements of a row, a = max |x|:
//   MX  e = max(floor(log2 a) - 2, -127), S = 2^e, r = 2^-e;
//   NV  s = E4M3(fl(a fl(1 / fl(6 g)))), S = fl(s g), r = fl(1 / S) (0 where S = 0);
//   q = E2M1(fl(x r)), value fl(q S), gradient |fl(x r)| <= 6 ? g : 0.
// All three are one pass over the data, bound by its bytes; a lane takes E = 16 or
// 8 elements of a row (row_pass.cuh), so a block is one, two or four neighbouring
// lanes.  16384 x 2048 bf16, codes and values: 27 us, 5.6 TB/s (codes alone 18, rows of
// 2047 69); the gradient of 8000 x 509 fp32 10 us, 4.8 TB/s.
#include <type_traits>

#include "fp4.cuh"
#include "row_pass.cuh"
#include "train.h"

namespace mnmt {
namespace {

// the largest magnitude of the lane's block as bits; a NaN stays one
template <bool NV, int E>
MNMT_DEV uint32_t block_amax(const float (&v)[E]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < E; i += 2)
        asm("{\n\t.reg .f32 a, b;\n\tabs.f32 a, %1;\n\tabs.f32 b, %2;\n\tmax.NaN.f32 %0, %0, a, b;\n\t}" : "+f"(m) : "f"(v[i]), "f"(v[i + 1]));
    uint32_t u = __float_as_uint(m);
#pragma unroll
    for (int o = 1; o < fp4_block(NV) / E; o *= 2) u = max(u, __shfl_xor_sync(0xFFFFFFFFu, u, o));
    return u;
}

// chunks in flight per warp
template <typename T>
constexpr int FLIGHT = sizeof(T) == 2 ? 2 : 1;

// codes and scales (q.codes, q.scales) and values, each where its pointer is given
template <typename T, bool NV, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) fp4_quantize_kernel(const T *x, long ldx, int alx, Fp4Args q, T *values, long ldv, int alv, int lr) {
    pdl_grid_wait();
    pdl_allow_next();  // a product that follows sets itself up meanwhile
    MNMT_ROW_BUF(buf, VEC);
    constexpr int E = row_elements(VEC), LPB = fp4_block(NV) / E, U = FLIGHT<T>;  // lanes per block
    const int lane = threadIdx.x & 31;
    const int tiles_k = fp4_tiles_k(q.cols, NV);
    const size_t pitch = fp4_pitch(q.cols);
    for (Walk<E> w(q.rows, q.cols, lr); w.more();) {
        Raw<T, E> raw[U];
        RowAt at[U];
        bool more[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            at[u] = w.at(), more[u] = w.more();
            if (more[u]) fetch<T, VEC>(x + at[u].row * ldx, w, at[u], q.cols, at[u].row < q.rows, alx, raw[u]);
            w.next();
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (!more[u]) break;
            const RowAt &a = at[u];
            const bool ok = a.row < q.rows;
            float v[E];
            settle<T, VEC>(raw[u], w, alx, buf, v);
            const Fp4Scale s = fp4_scale<NV>(block_amax<NV>(v), q.g, q.inv6g);
            const bool bad = !(s.S == s.S);
            uint32_t codes[E / 8];
#pragma unroll
            for (int h = 0; h < E / 8; h++) {
                uint32_t b[4];
#pragma unroll
                for (int i = 0; i < 4; i++) b[i] = fp4_code2(__fmul_rn(v[8 * h + 2 * i], s.r), __fmul_rn(v[8 * h + 2 * i + 1], s.r));
                codes[h] = bad ? 0u : __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
            }
            if (values) {
#pragma unroll
                for (int i = 0; i < E / 2; i++) {
                    const float2 f = fp4_float2((codes[i >> 2] >> (8 * (i & 3))) & 0xFFu);
                    v[2 * i] = __fmul_rn(f.x, s.S);
                    v[2 * i + 1] = __fmul_rn(f.y, s.S);
                }
                put<T, VEC>(values + a.row * ldv, w, a, q.cols, ok, alv, buf, v);
            }
            if (q.codes) {
                if (ok && (size_t)(a.c >> 1) < pitch) {
                    uint8_t *p = q.codes + a.row * pitch + (a.c >> 1);
                    if constexpr (E == 16) *reinterpret_cast<uint2 *>(p) = make_uint2(codes[0], codes[1]);
                    else *reinterpret_cast<uint32_t *>(p) = codes[0];
                }
                // the scales of four blocks, a word of a tile
                const int b = a.c / fp4_block(NV);
                uint32_t word = s.byte << (8 * (b & 3));
                word |= __shfl_xor_sync(0xFFFFFFFFu, word, LPB);
                word |= __shfl_xor_sync(0xFFFFFFFFu, word, 2 * LPB);
                if (ok && lane % (4 * LPB) == 0 && (b >> 2) < tiles_k)
                    *reinterpret_cast<uint32_t *>(q.scales + fp4_scale_at((int)a.row, b, tiles_k)) = word;
            }
        }
    }
    if (q.codes) {  // the last tiles' rows beyond the matrix
        const long pad = (long)(-(long)q.rows & 127) * tiles_k;
        for (long i = (long)blockIdx.x * blockDim.x + threadIdx.x; i < pad; i += (long)gridDim.x * blockDim.x)
            *reinterpret_cast<uint32_t *>(q.scales + fp4_scale_at(q.rows + (int)(i / tiles_k), 4 * (int)(i % tiles_k), tiles_k)) = 0;
    }
}

template <typename T, bool NV, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) fp4_dequantize_kernel(Fp4Args q, T *values, long ldv, int alv, int lr) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    constexpr int E = row_elements(VEC), U = FLIGHT<T>;
    const int tiles_k = fp4_tiles_k(q.cols, NV);
    const size_t pitch = fp4_pitch(q.cols);
    for (Walk<E> w(q.rows, q.cols, lr); w.more();) {
        RowAt at[U];
        bool more[U], ok[U];
        uint2 codes[U];
        uint32_t byte[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            at[u] = w.at(), more[u] = w.more(), ok[u] = at[u].row < q.rows;
            codes[u] = make_uint2(0, 0), byte[u] = 0;
            if (ok[u] && at[u].c < q.cols) {
                const uint8_t *p = q.codes + at[u].row * pitch + (at[u].c >> 1);
                if constexpr (E == 16) codes[u] = *reinterpret_cast<const uint2 *>(p);
                else codes[u].x = *reinterpret_cast<const uint32_t *>(p);
                byte[u] = q.scales[fp4_scale_at((int)at[u].row, at[u].c / fp4_block(NV), tiles_k)];
            }
            w.next();
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (!more[u]) break;
            const Fp4Scale s = fp4_scale_of<NV>(byte[u], q.g);
            float v[E];
#pragma unroll
            for (int i = 0; i < E / 2; i++) {
                const float2 f = fp4_float2(((i < 4 ? codes[u].x : codes[u].y) >> (8 * (i & 3))) & 0xFFu);
                v[2 * i] = __fmul_rn(f.x, s.S);
                v[2 * i + 1] = __fmul_rn(f.y, s.S);
            }
            put<T, VEC>(values + at[u].row * ldv, w, at[u], q.cols, ok[u], alv, buf, v);
        }
    }
}

template <typename T, bool NV, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) fp4_quantize_backward_kernel(const T *x, long ldx, int alx, const T *g, long ldg, int alg, T *gx,
                                                                                long ldgx, int algx, int rows, int cols, float tg, float inv6g, int lr) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    constexpr int E = row_elements(VEC);
    for (Walk<E> w(rows, cols, lr); w.more(); w.next()) {
        const RowAt a = w.at();
        const bool ok = a.row < rows;
        Raw<T, E> rx, rg;
        fetch<T, VEC>(x + a.row * ldx, w, a, cols, ok, alx, rx);
        fetch<T, VEC>(g + a.row * ldg, w, a, cols, ok, alg, rg);
        float v[E], d[E];
        settle<T, VEC>(rx, w, alx, buf, v);
        const Fp4Scale s = fp4_scale<NV>(block_amax<NV>(v), tg, inv6g);
        settle<T, VEC>(rg, w, alg, buf, d);
#pragma unroll
        for (int i = 0; i < E; i++) d[i] = fabsf(__fmul_rn(v[i], s.r)) <= 6.0f ? d[i] : 0.0f;
        put<T, VEC>(gx + a.row * ldgx, w, a, cols, ok, algx, buf, d);
    }
}

template <typename T, typename F>
void by_form(bool nv, bool vec, F &&f) {
    if (nv) vec ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
    else vec ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

}  // namespace

template <typename F>
static void by_type(int dtype, F &&f) {
    if (dtype == MNMT_F32) f(float{});
    else if (dtype == MNMT_BF16) f(__nv_bfloat16{});
    else f(__half{});
}

cudaError_t launch_fp4_quantize(const void *x, int dtype, long ldx, const Fp4Args &q, bool nv, void *values, long ldv, cudaStream_t st) {
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const T *xp = static_cast<const T *>(x);
        T *vp = static_cast<T *>(values);
        const int ax = row_alignment(xp, ldx), av = vp ? row_alignment(vp, ldv) : 2;
        by_form<T>(nv, ax == 2 && av == 2, [&](auto n, auto v) {
            launch_pdl(fp4_quantize_kernel<T, decltype(n)::value, decltype(v)::value>, row_grid(q.rows, q.cols, v.value, device_sm_count()), 256, 0, st, xp, ldx,
                       ax, q, vp, ldv, av, row_lanes(q.cols, v.value));
        });
    });
    return cudaGetLastError();
}

cudaError_t launch_fp4_dequantize(const Fp4Args &q, bool nv, void *values, int dtype, long ldv, cudaStream_t st) {
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        T *vp = static_cast<T *>(values);
        const int av = row_alignment(vp, ldv);
        by_form<T>(nv, av == 2, [&](auto n, auto v) {
            launch_pdl(fp4_dequantize_kernel<T, decltype(n)::value, decltype(v)::value>, row_grid(q.rows, q.cols, v.value, device_sm_count()), 256, 0, st, q, vp,
                       ldv, av, row_lanes(q.cols, v.value));
        });
    });
    return cudaGetLastError();
}

cudaError_t launch_fp4_quantize_backward(const void *x, int dtype, long ldx, const void *g, long ldg, void *gx, long ldgx, int rows, int cols,
                                         bool nv, float tg, float inv6g, cudaStream_t st) {
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        const T *xp = static_cast<const T *>(x), *gp = static_cast<const T *>(g);
        T *op = static_cast<T *>(gx);
        const int ax = row_alignment(xp, ldx), ag = row_alignment(gp, ldg), ao = row_alignment(op, ldgx);
        by_form<T>(nv, ax == 2 && ag == 2 && ao == 2, [&](auto n, auto v) {
            launch_pdl(fp4_quantize_backward_kernel<T, decltype(n)::value, decltype(v)::value>, row_grid(rows, cols, v.value, device_sm_count()), 256, 0, st, xp,
                       ldx, ax, gp, ldg, ag, op, ldgx, ao, rows, cols, tg, inv6g, row_lanes(cols, v.value));
        });
    });
    return cudaGetLastError();
}

}  // namespace mnmt
