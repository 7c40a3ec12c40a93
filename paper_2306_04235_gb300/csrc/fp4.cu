// fp4.cu -- quantisation to microscaled 4-bit floating point, its inverse and
// its straight-through backward pass (include/mnmt.h, mnmt_fp4_*).
//
// Per block of 32 (MX) or 16 (NV) elements of a row, a = max |x|:
//   MX  e = max(floor(log2 a) - 2, -127), S = 2^e, r = 2^-e;
//   NV  s = E4M3(fl(a fl(1 / fl(6 g)))), S = fl(s g), r = fl(1 / S) (0 where S = 0);
//   q = E2M1(fl(x r)), value fl(q S), gradient |fl(x r)| <= 6 ? g : 0.
// All three are one pass over the data, bound by its bytes.  A warp takes 256
// consecutive elements of a row, eight per lane, so a block is four (MX) or two
// (NV) neighbouring lanes and its maximum two or one shuffles.
#include <type_traits>

#include "fp4.cuh"
#include "internal.h"

namespace mnmt {
namespace {

template <bool NV>
MNMT_DEV uint32_t block_amax(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    if (!NV) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    return m;
}

// chunks in flight per warp
template <typename T>
constexpr int FLIGHT = sizeof(T) == 2 ? 4 : 2;

// codes and scales (q.codes, q.scales) and values, each where its pointer is given
template <typename T, bool NV, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) fp4_quantize_kernel(const T *x, long ldx, bool alx, Fp4Args q, T *values, long ldv, bool alv) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    constexpr int LPB = fp4_block(NV) / 8, U = FLIGHT<T>;  // lanes per block
    const int lane = threadIdx.x & 31;
    const int tiles_k = fp4_tiles_k(q.cols, NV);
    const size_t pitch = fp4_pitch(q.cols);
    for (Walk w(q.cols); w.row < q.rows;) {
        Raw8<T> raw[U];
        long row[U];
        int c0[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            row[u] = w.row, c0[u] = w.chunk * ROW_CHUNK;
            if (row[u] < q.rows) fetch8<T, VEC>(x + row[u] * ldx, c0[u], q.cols, alx, raw[u]);
            w.next();
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (row[u] >= q.rows) break;
            float v[8];
            settle8<T, VEC>(raw[u], alx, buf, v);
            const Fp4Scale s = fp4_scale<NV>(block_amax<NV>(v), q.g, q.inv6g);
            uint32_t codes = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) codes |= fp4_code2(__fmul_rn(v[2 * i], s.r), __fmul_rn(v[2 * i + 1], s.r)) << (8 * i);
            if (!(s.S == s.S)) codes = 0;
            if (values) {
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float2 f = fp4_float2((codes >> (8 * i)) & 0xFFu);
                    v[2 * i] = __fmul_rn(f.x, s.S);
                    v[2 * i + 1] = __fmul_rn(f.y, s.S);
                }
                put8<T, VEC>(values + row[u] * ldv, c0[u], q.cols, alv, buf, v);
            }
            if (q.codes) {
                const int c = c0[u] + 8 * lane;
                if ((size_t)(c >> 1) < pitch) *reinterpret_cast<uint32_t *>(q.codes + row[u] * pitch + (c >> 1)) = codes;
                // the scales of four blocks, a word of a tile
                const int b = c / fp4_block(NV);
                uint32_t word = s.byte << (8 * (b & 3));
                word |= __shfl_xor_sync(0xFFFFFFFFu, word, LPB);
                word |= __shfl_xor_sync(0xFFFFFFFFu, word, 2 * LPB);
                if (lane % (4 * LPB) == 0 && (b >> 2) < tiles_k)
                    *reinterpret_cast<uint32_t *>(q.scales + fp4_scale_at((int)row[u], b, tiles_k)) = word;
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
__global__ void __launch_bounds__(256, ROW_BLOCKS) fp4_dequantize_kernel(Fp4Args q, T *values, long ldv, bool alv) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    const int tiles_k = fp4_tiles_k(q.cols, NV);
    const size_t pitch = fp4_pitch(q.cols);
    for (Walk w(q.cols); w.row < q.rows; w.next()) {
        const int c0 = w.chunk * ROW_CHUNK, c = c0 + 8 * (int)(threadIdx.x & 31);
        float v[8] = {};
        if (c < q.cols) {
            const uint32_t codes = *reinterpret_cast<const uint32_t *>(q.codes + w.row * pitch + (c >> 1));
            const Fp4Scale s = fp4_scale_of<NV>(q.scales[fp4_scale_at((int)w.row, c / fp4_block(NV), tiles_k)], q.g);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 f = fp4_float2((codes >> (8 * i)) & 0xFFu);
                v[2 * i] = __fmul_rn(f.x, s.S);
                v[2 * i + 1] = __fmul_rn(f.y, s.S);
            }
        }
        put8<T, VEC>(values + w.row * ldv, c0, q.cols, alv, buf, v);
    }
}

template <typename T, bool NV, bool VEC>
__global__ void __launch_bounds__(256, ROW_BLOCKS) fp4_quantize_backward_kernel(const T *x, long ldx, bool alx, const T *g, long ldg, bool alg, T *gx,
                                                                                long ldgx, bool algx, int rows, int cols, float tg, float inv6g) {
    pdl_grid_wait();
    MNMT_ROW_BUF(buf, VEC);
    constexpr int U = FLIGHT<T> / 2;
    for (Walk w(cols); w.row < rows;) {
        Raw8<T> rx[U], rg[U];
        long row[U];
        int c0[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            row[u] = w.row, c0[u] = w.chunk * ROW_CHUNK;
            if (row[u] < rows) {
                fetch8<T, VEC>(x + row[u] * ldx, c0[u], cols, alx, rx[u]);
                fetch8<T, VEC>(g + row[u] * ldg, c0[u], cols, alg, rg[u]);
            }
            w.next();
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (row[u] >= rows) break;
            float v[8], d[8];
            settle8<T, VEC>(rx[u], alx, buf, v);
            settle8<T, VEC>(rg[u], alg, buf, d);
            const Fp4Scale s = fp4_scale<NV>(block_amax<NV>(v), tg, inv6g);
#pragma unroll
            for (int i = 0; i < 8; i++) d[i] = fabsf(__fmul_rn(v[i], s.r)) <= 6.0f ? d[i] : 0.0f;
            put8<T, VEC>(gx + row[u] * ldgx, c0[u], cols, algx, buf, d);
        }
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
        const bool ax = row_aligned(xp, ldx), av = !vp || row_aligned(vp, ldv);
        by_form<T>(nv, ax && av, [&](auto n, auto v) {
            launch_pdl(fp4_quantize_kernel<T, decltype(n)::value, decltype(v)::value>, row_grid(q.rows, q.cols, device_sm_count()), 256, 0, st, xp, ldx,
                       ax, q, vp, ldv, av);
        });
    });
    return cudaGetLastError();
}

cudaError_t launch_fp4_dequantize(const Fp4Args &q, bool nv, void *values, int dtype, long ldv, cudaStream_t st) {
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        T *vp = static_cast<T *>(values);
        const bool av = row_aligned(vp, ldv);
        by_form<T>(nv, av, [&](auto n, auto v) {
            launch_pdl(fp4_dequantize_kernel<T, decltype(n)::value, decltype(v)::value>, row_grid(q.rows, q.cols, device_sm_count()), 256, 0, st, q, vp,
                       ldv, av);
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
        const bool ax = row_aligned(xp, ldx), ag = row_aligned(gp, ldg), ao = row_aligned(op, ldgx);
        by_form<T>(nv, ax && ag && ao, [&](auto n, auto v) {
            launch_pdl(fp4_quantize_backward_kernel<T, decltype(n)::value, decltype(v)::value>, row_grid(rows, cols, device_sm_count()), 256, 0, st, xp,
                       ldx, ax, gp, ldg, ag, op, ldgx, ao, rows, cols, tg, inv6g);
        });
    });
    return cudaGetLastError();
}

}  // namespace mnmt
