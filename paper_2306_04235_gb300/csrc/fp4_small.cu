// fp4_small.cu -- the linear on 4-bit floating-point operands for a few rows (the
// tokens of a decode step), quantisation included, in one launch.
//
// Every block quantises the rows of x for itself (they are few and in L2; block 0
// also stores the packed form) while its first weights are on their way, then its
// warps take rows of W: a lane reads 32 codes (16 bytes) of a row and multiplies
// them as integers, since twice an E2M1 value is one of 0, 1, 2, 3, 4, 6, 8, 12.
// A magnitude is looked up by byte permutation (four codes select four of eight
// bytes); the sign is a second permutation that repeats a byte's sign bit, and
// with t = 0x7F where negative, else 0,  sum x (+-m) = sum x (m ^ t) - sum x t, two
// dot products of four bytes.  A block's sum is exact; blocks are added in fp32.
// Bound by latency: start, the rows of x, one pass of weights (a token through
// 2048 x 512 back to back: 2.8 us, 5.5 as two launches; a program's call costs its host
// more than that).
#include <type_traits>

#include "fp4.cuh"
#include "train.h"

namespace mnmt {
namespace {

constexpr int SM_WARPS = 8;

struct SmallArgs {
    const void *x;  // null: xq holds the packed rows
    int xdtype;
    long ldx;
    Fp4Args xq, w;
    float alpha;
    const float *bias;
    int relu;
    void *y;
    int ydtype;
    long ldy;
    int lanes;  // of a row of W: a power of two
};

// twice the values of four codes (the low half of w), as magnitudes and as 0x7F in the bytes that are negative
MNMT_DEV uint32_t magnitudes(uint32_t w) { return __byte_perm(0x03020100u, 0x0C080604u, w & 0x7777u); }
MNMT_DEV uint32_t negative(uint32_t w) {
    uint32_t r;  // a selector's highest bit repeats the sign of the byte it selects
    asm("prmt.b32 %0, %1, %1, %2;" : "=r"(r) : "r"(0x80808080u), "r"(w & 0x8888u));
    return r & 0x7F7F7F7Fu;
}

// eight elements of x, zeros from n on
template <typename T>
MNMT_DEV void load_x(const T *p, int n, bool al, float *v) {
    float f[8];
    if (al && n >= 8) load8<T, true>(p, 8, f);
    else load8<T, false>(p, n, f);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = f[i];
}

// block b of row m into the doubled codes q2 [block / 4 words], the scale sx (S without the tensor scale) and byte
template <bool NV, typename T>
MNMT_DEV void small_quantize(const SmallArgs &a, int m, int b, uint32_t *q2, float &sx, uint8_t &byte) {
    constexpr int B = fp4_block(NV);
    const T *row = static_cast<const T *>(a.x) + m * a.ldx;
    const bool al = ((reinterpret_cast<uintptr_t>(a.x) | (uintptr_t)a.ldx * sizeof(T)) & 15) == 0;
    float v[B];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < B; i += 8) load_x(row + b * B + i, a.xq.cols - b * B - i, al, v + i);
#pragma unroll
    for (int i = 0; i < B; i++) amax = max(amax, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    const Fp4Scale s = fp4_scale<NV>(amax, a.xq.g, a.xq.inv6g);
    const bool bad = !(s.S == s.S);
    byte = (uint8_t)s.byte;
    sx = NV ? fp4_scale_of<true>(s.byte, 1.0f).S : s.S;
    uint8_t *codes = a.xq.codes + (size_t)m * fp4_pitch(a.xq.cols) + b * (B / 2);
#pragma unroll
    for (int i = 0; i < B; i += 8) {
        uint32_t c = 0;
#pragma unroll
        for (int k = 0; k < 4; k++) c |= fp4_code2(__fmul_rn(v[i + 2 * k], s.r), __fmul_rn(v[i + 2 * k + 1], s.r)) << (8 * k);
        if (bad) c = 0;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t w = c >> (16 * h), mg = magnitudes(w), t = negative(w) * 2 + (negative(w) & 0x01010101u);  // 0xFF where negative
            q2[i / 4 + h] = __vsub4(mg ^ t, t);
        }
        if (blockIdx.x == 0) reinterpret_cast<uint32_t *>(codes)[i / 8] = c;
    }
}

// the same from packed rows
template <bool NV>
MNMT_DEV void small_unpack(const SmallArgs &a, int m, int b, uint32_t *q2, float &sx) {
    constexpr int B = fp4_block(NV);
    const uint32_t *codes = reinterpret_cast<const uint32_t *>(a.xq.codes + (size_t)m * fp4_pitch(a.xq.cols) + b * (B / 2));
    sx = fp4_scale_of<NV>(a.xq.scales[fp4_scale_at(m, b, fp4_tiles_k(a.xq.cols, NV))], 1.0f).S;
#pragma unroll
    for (int i = 0; i < B / 8; i++) {
        const uint32_t c = codes[i];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const uint32_t w = c >> (16 * h), mg = magnitudes(w), t = negative(w) * 2 + (negative(w) & 0x01010101u);
            q2[2 * i + h] = __vsub4(mg ^ t, t);
        }
    }
}

template <bool NV, int MT>
__global__ void __launch_bounds__(SM_WARPS * 32) fp4_small_kernel(SmallArgs a) {
    extern __shared__ uint4 sm_raw[];
    constexpr int B = fp4_block(NV), NS = 32 / B;  // scales of a lane's 32 codes
    const int M = a.xq.rows, K = a.xq.cols, N = a.w.rows, segs = fp4_div_up(K, 32), nb = segs * NS, tiles_k = fp4_tiles_k(K, NV);
    uint32_t *xs = reinterpret_cast<uint32_t *>(sm_raw);            // [M][segs][8] words of doubled codes
    float *sx = reinterpret_cast<float *>(xs + (size_t)M * segs * 8);  // [M][nb]
    uint8_t *sb = reinterpret_cast<uint8_t *>(sx + (size_t)M * nb);    // [M][nb] scale bytes (quantised here)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & (a.lanes - 1);
    const int per = 32 / a.lanes, rows = SM_WARPS * per;  // rows of W per warp, per block

    pdl_grid_wait();
    // the block's first weights, while x is quantised
    const size_t pitch = fp4_pitch(K);
    auto code_at = [&](int n, int s) { return *reinterpret_cast<const uint4 *>(a.w.codes + n * pitch + 16 * s); };
    auto scale_at = [&](int n, int s) {
        const uint8_t *p = a.w.scales + fp4_scale_at(n, s * NS, tiles_k);
        return NV ? (uint32_t)*reinterpret_cast<const uint16_t *>(p) : (uint32_t)*p;
    };
    int n = blockIdx.x * rows + warp * per + lane / a.lanes;
    uint4 w0 = make_uint4(0, 0, 0, 0);
    uint32_t b0 = 0;
    if (n < N && l < segs) w0 = code_at(n, l), b0 = scale_at(n, l);

    for (int i = threadIdx.x; i < M * nb; i += SM_WARPS * 32) {
        const int m = i / nb, b = i - m * nb;
        uint32_t q2[B / 4];
        float s;
        if (!a.x) small_unpack<NV>(a, m, b, q2, s);
        else if (a.xdtype == MNMT_F32) small_quantize<NV, float>(a, m, b, q2, s, sb[i]);
        else if (a.xdtype == MNMT_BF16) small_quantize<NV, __nv_bfloat16>(a, m, b, q2, s, sb[i]);
        else small_quantize<NV, __half>(a, m, b, q2, s, sb[i]);
#pragma unroll
        for (int k = 0; k < B / 16; k++) reinterpret_cast<uint4 *>(xs)[(size_t)i * (B / 16) + k] = make_uint4(q2[4 * k], q2[4 * k + 1], q2[4 * k + 2], q2[4 * k + 3]);
        sx[i] = s * 0.25f;  // both operands are doubled
    }
    __syncthreads();
    if (a.x && blockIdx.x == 0) {  // the scale tiles of the packed form, with their padding
        for (int i = threadIdx.x; i < 128 * tiles_k; i += SM_WARPS * 32) {
            const int m = i & 127, t = i >> 7;
            uint32_t word = 0;
            if (m < M)
                for (int k = 0; k < 4; k++)
                    if (4 * t + k < nb) word |= (uint32_t)sb[m * nb + 4 * t + k] << (8 * k);
            *reinterpret_cast<uint32_t *>(a.xq.scales + fp4_scale_at(m, 4 * t, tiles_k)) = word;
        }
    }

    for (; n - lane / a.lanes < N; n += gridDim.x * rows) {  // alike in all lanes
        float acc[MT];
#pragma unroll
        for (int m = 0; m < MT; m++) acc[m] = 0.0f;
        for (int s = l; s < segs; s += a.lanes) {
            const uint4 w = w0;
            const uint32_t wb = b0;
            if (n < N && s + a.lanes < segs) w0 = code_at(n, s + a.lanes), b0 = scale_at(n, s + a.lanes);
            const uint32_t cw[4] = {w.x, w.y, w.z, w.w};
            uint32_t mg[8], t[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const uint32_t half = cw[i >> 1] >> (16 * (i & 1));
                t[i] = negative(half);
                mg[i] = magnitudes(half) ^ t[i];
            }
            float sw[NS];
#pragma unroll
            for (int k = 0; k < NS; k++) sw[k] = fp4_scale_of<NV>(wb >> (8 * k) & 0xFFu, 1.0f).S;
#pragma unroll
            for (int m = 0; m < MT; m++) {
                if (m >= M) break;
                const uint4 *xp = reinterpret_cast<const uint4 *>(xs) + ((size_t)m * segs + s) * 2;
                const uint4 p0 = xp[0], p1 = xp[1];
                const uint32_t xw[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
#pragma unroll
                for (int k = 0; k < NS; k++) {
                    int d = 0, e = 0;
#pragma unroll
                    for (int i = k * (8 / NS); i < (k + 1) * (8 / NS); i++) {
                        d = __dp4a((int)xw[i], (int)mg[i], d);
                        e = __dp4a((int)xw[i], (int)t[i], e);
                    }
                    // Scaled by one factor after the other: their product may leave fp32 where the
                    // sum is zero.  The smaller first: a whole number of at least 2^-129 is exact, and
                    // infinite only where both scales are so large that the sum is (a NaN stays).
                    // E4M3 scales reach neither end.
                    const float f = sx[m * nb + s * NS + k], g = sw[k];
                    const bool up = !NV && f > g;
                    acc[m] = __fmaf_rn(__fmul_rn((float)(d - e), up ? g : f), up ? f : g, acc[m]);
                }
            }
        }
        const int at = n;
        n += gridDim.x * rows;
        if (n < N && l < segs) w0 = code_at(n, l), b0 = scale_at(n, l);  // the next row's, while this one is summed
        n = at;
#pragma unroll
        for (int m = 0; m < MT; m++) {
            if (m >= M) break;
            float s = acc[m];
            for (int o = a.lanes >> 1; o > 0; o >>= 1) s = __fadd_rn(s, __shfl_xor_sync(0xFFFFFFFFu, s, o));
            if (l == 0 && n < N) {
                float v = NV ? __fmul_rn(s, a.alpha) : s;
                if (a.bias) v = __fadd_rn(v, a.bias[n]);
                if (a.relu && v <= 0.0f) v = 0.0f;  // a NaN stays
                const long i = m * a.ldy + n;
                if (a.ydtype == MNMT_F32) static_cast<float *>(a.y)[i] = v;
                else if (a.ydtype == MNMT_BF16) static_cast<__nv_bfloat16 *>(a.y)[i] = __float2bfloat16_rn(v);
                else static_cast<__half *>(a.y)[i] = __float2half_rn(v);
            }
        }
    }
}

}  // namespace

cudaError_t launch_fp4_small(const Fp4Args &x, const Fp4Args &w, bool nv, const void *xp, int xdtype, long ldx, float alpha, const float *bias, int relu,
                             void *y, int ydtype, long ldy, cudaStream_t st) {
    const int segs = fp4_div_up(x.cols, 32);
    SmallArgs a{xp, xdtype, ldx, x, w, alpha, bias, relu, y, ydtype, ldy, 1};
    while (a.lanes < 32 && a.lanes < segs) a.lanes *= 2;
    const int rows = SM_WARPS * (32 / a.lanes), blocks = fp4_div_up(w.rows, rows), most = 4 * device_sm_count();
    const size_t smem = (size_t)x.rows * segs * (32 + (nv ? 2 : 1) * 5);
    auto go = [&](auto n, auto m) {
        return launch_pdl(fp4_small_kernel<decltype(n)::value, decltype(m)::value>, blocks < most ? blocks : most, SM_WARPS * 32, smem, st, a);
    };
    auto rows_of = [&](auto n) {
        if (x.rows == 1) go(n, std::integral_constant<int, 1>{});
        else if (x.rows <= 4) go(n, std::integral_constant<int, 4>{});
        else go(n, std::integral_constant<int, 8>{});
    };
    nv ? rows_of(std::true_type{}) : rows_of(std::false_type{});
    return cudaGetLastError();
}

}  // namespace mnmt
