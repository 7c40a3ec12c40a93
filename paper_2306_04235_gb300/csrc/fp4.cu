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

constexpr int Q_CHUNK = 256;  // elements of a row per warp and step

// The (row, chunk) pairs of a warp: chunk index fastest, advanced without divisions.
struct Walk {
    long row, step_rows;
    int chunk, step_chunks, chunks;
    MNMT_DEV Walk(int cols) {
        chunks = (cols + Q_CHUNK - 1) / Q_CHUNK;
        const long w = ((long)blockIdx.x * blockDim.x + threadIdx.x) >> 5, n = ((long)gridDim.x * blockDim.x) >> 5;
        row = w / chunks, chunk = (int)(w - row * chunks);
        step_rows = n / chunks, step_chunks = (int)(n - step_rows * chunks);
    }
    MNMT_DEV void next() {
        row += step_rows;
        chunk += step_chunks;
        if (chunk >= chunks) chunk -= chunks, row++;
    }
};

template <bool NV>
MNMT_DEV uint32_t block_amax(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    if (!NV) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    return m;
}

template <typename T, bool VEC>
MNMT_DEV void load_row8(const T *row, int c, int cols, float (&v)[8]) {
    if (VEC && c + 8 <= cols) load8<T, true>(row + c, 8, v);
    else load8<T, false>(row + c, cols - c, v);
}
template <typename T, bool VEC>
MNMT_DEV void store_row8(T *row, int c, int cols, const float (&v)[8]) {
    if (VEC && c + 8 <= cols) store8<T, true>(row + c, 8, v);
    else store8<T, false>(row + c, cols - c, v);
}

// codes and scales (q.codes, q.scales) and values, each where its pointer is given
template <typename T, bool NV, bool VEC>
__global__ void __launch_bounds__(256) fp4_quantize_kernel(const T *x, long ldx, Fp4Args q, T *values,
                                                           long ldv) {
    pdl_grid_wait();
    constexpr int LPB = fp4_block(NV) / 8;  // lanes per block
    const int lane = threadIdx.x & 31;
    const int tiles_k = fp4_tiles_k(q.cols, NV);
    const size_t pitch = fp4_pitch(q.cols);
    for (Walk w(q.cols); w.row < q.rows; w.next()) {
        const int c = w.chunk * Q_CHUNK + lane * 8;
        float v[8];
        load_row8<T, VEC>(x + w.row * ldx, c, q.cols, v);
        const Fp4Scale s = fp4_scale<NV>(block_amax<NV>(v), q.g, q.inv6g);
        const bool bad = !(s.S == s.S);
        uint32_t codes = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) codes |= fp4_code2(__fmul_rn(v[2 * i], s.r), __fmul_rn(v[2 * i + 1], s.r)) << (8 * i);
        if (bad) codes = 0;
        if (values) {
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 f = fp4_float2((codes >> (8 * i)) & 0xFFu);
                v[2 * i] = __fmul_rn(f.x, s.S);
                v[2 * i + 1] = __fmul_rn(f.y, s.S);
            }
            store_row8<T, VEC>(values + w.row * ldv, c, q.cols, v);
        }
        if (q.codes) {
            if ((size_t)(c >> 1) < pitch) *reinterpret_cast<uint32_t *>(q.codes + w.row * pitch + (c >> 1)) = codes;
            // the scales of four blocks, a word of a tile
            const int b = c / fp4_block(NV);
            uint32_t word = s.byte << (8 * (b & 3));
            word |= __shfl_xor_sync(0xFFFFFFFFu, word, LPB);
            word |= __shfl_xor_sync(0xFFFFFFFFu, word, 2 * LPB);
            if (lane % (4 * LPB) == 0 && (b >> 2) < tiles_k)
                *reinterpret_cast<uint32_t *>(q.scales + fp4_scale_at((int)w.row, b, tiles_k)) = word;
        }
    }
    if (q.codes) {  // the last tiles' rows beyond the matrix
        const long pad = (long)(-(long)q.rows & 127) * tiles_k;
        for (long i = (long)blockIdx.x * blockDim.x + threadIdx.x; i < pad; i += (long)gridDim.x * blockDim.x)
            *reinterpret_cast<uint32_t *>(q.scales + fp4_scale_at(q.rows + (int)(i / tiles_k), 4 * (int)(i % tiles_k), tiles_k)) = 0;
    }
}

template <typename T, bool NV, bool VEC>
__global__ void __launch_bounds__(256) fp4_dequantize_kernel(Fp4Args q, T *__restrict__ values, long ldv) {
    pdl_grid_wait();
    const int lane = threadIdx.x & 31;
    const int tiles_k = fp4_tiles_k(q.cols, NV);
    const size_t pitch = fp4_pitch(q.cols);
    for (Walk w(q.cols); w.row < q.rows; w.next()) {
        const int c = w.chunk * Q_CHUNK + lane * 8;
        if (c >= q.cols) continue;
        const uint32_t codes = *reinterpret_cast<const uint32_t *>(q.codes + w.row * pitch + (c >> 1));
        const Fp4Scale s = fp4_scale_of<NV>(q.scales[fp4_scale_at((int)w.row, c / fp4_block(NV), tiles_k)], q.g);
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float2 f = fp4_float2((codes >> (8 * i)) & 0xFFu);
            v[2 * i] = __fmul_rn(f.x, s.S);
            v[2 * i + 1] = __fmul_rn(f.y, s.S);
        }
        store_row8<T, VEC>(values + w.row * ldv, c, q.cols, v);
    }
}

template <typename T, bool NV, bool VEC>
__global__ void __launch_bounds__(256) fp4_quantize_backward_kernel(const T *x, long ldx, const T *g, long ldg,
                                                                    T *gx, long ldgx, int rows, int cols, float tg,
                                                                    float inv6g) {
    pdl_grid_wait();
    const int lane = threadIdx.x & 31;
    for (Walk w(cols); w.row < rows; w.next()) {
        const int c = w.chunk * Q_CHUNK + lane * 8;
        float v[8], u[8];
        load_row8<T, VEC>(x + w.row * ldx, c, cols, v);
        load_row8<T, VEC>(g + w.row * ldg, c, cols, u);
        const Fp4Scale s = fp4_scale<NV>(block_amax<NV>(v), tg, inv6g);
#pragma unroll
        for (int i = 0; i < 8; i++) u[i] = fabsf(__fmul_rn(v[i], s.r)) <= 6.0f ? u[i] : 0.0f;
        store_row8<T, VEC>(gx + w.row * ldgx, c, cols, u);
    }
}

int q_grid(long rows, int cols) {
    const long warps = rows * ((cols + Q_CHUNK - 1) / Q_CHUNK), blocks = (warps + 7) / 8;
    const long cap = (long)8 * device_sm_count();
    return (int)(blocks < 1 ? 1 : blocks < cap ? blocks : cap);
}

template <typename T>
bool row_vec(const T *p, long ld) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * sizeof(T) % 16 == 0;
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
        by_form<T>(nv, row_vec(xp, ldx) && (!vp || row_vec(vp, ldv)), [&](auto n, auto v) {
            launch_pdl(fp4_quantize_kernel<T, decltype(n)::value, decltype(v)::value>, q_grid(q.rows, q.cols), 256, 0, st, xp, ldx, q, vp, ldv);
        });
    });
    return cudaGetLastError();
}

cudaError_t launch_fp4_dequantize(const Fp4Args &q, bool nv, void *values, int dtype, long ldv, cudaStream_t st) {
    by_type(dtype, [&](auto t) {
        using T = decltype(t);
        T *vp = static_cast<T *>(values);
        by_form<T>(nv, row_vec(vp, ldv), [&](auto n, auto v) {
            launch_pdl(fp4_dequantize_kernel<T, decltype(n)::value, decltype(v)::value>, q_grid(q.rows, q.cols), 256, 0, st, q, vp, ldv);
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
        by_form<T>(nv, row_vec(xp, ldx) && row_vec(gp, ldg) && row_vec(op, ldgx), [&](auto n, auto v) {
            launch_pdl(fp4_quantize_backward_kernel<T, decltype(n)::value, decltype(v)::value>, q_grid(rows, cols), 256, 0, st, xp, ldx, gp,
                       ldg, op, ldgx, rows, cols, tg, inv6g);
        });
    });
    return cudaGetLastError();
}

}  // namespace mnmt
