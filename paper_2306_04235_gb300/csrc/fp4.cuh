// fp4.cuh -- microscaled 4-bit floating point: E2M1 codes with one scale per
// block of a row (include/mnmt.h), device arithmetic shared by its kernels.
//
// An E2M1 code is sign | 2-bit exponent | 1-bit mantissa: 0, 1/2, 1, 3/2, 2, 3,
// 4, 6.  MX: blocks of 32, scale 2^e in a byte (e + 127).  NV: blocks of 16, an
// E4M3 scale and one fp32 scale of the whole tensor.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"

namespace mnmt {

constexpr int FP4_BLOCK_MX = 32, FP4_BLOCK_NV = 16;

__host__ __device__ constexpr int fp4_block(bool nv) { return nv ? FP4_BLOCK_NV : FP4_BLOCK_MX; }
__host__ __device__ constexpr int fp4_div_up(int a, int b) { return a / b + (a % b != 0); }
// bytes of a row's codes
__host__ __device__ constexpr size_t fp4_pitch(int cols) { return (size_t)fp4_div_up(cols, 32) * 16; }
// scale tiles (128 rows, 4 blocks) along a row
__host__ __device__ constexpr int fp4_tiles_k(int cols, bool nv) { return fp4_div_up(cols, 4 * fp4_block(nv)); }
__host__ __device__ constexpr size_t fp4_scale_bytes(int rows, int cols, bool nv) {
    return (size_t)fp4_div_up(rows, 128) * fp4_tiles_k(cols, nv) * 512;
}
// byte of the scale of (row, block)
__host__ __device__ __forceinline__ size_t fp4_scale_at(int row, int block, int tiles_k) {
    return ((size_t)(row >> 7) * tiles_k + (block >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// the operands of an fp4 matrix as its kernels take them; inv6g = fl(1 / fl(6 g))
struct Fp4Args {
    uint8_t *codes, *scales;
    int rows, cols;
    float g, inv6g;
};

// arguments of the backward pass of a linear (xo, wo: the float originals, for the masks; null: none)
struct Fp4BackwardArgs {
    Fp4Args x, w;
    bool nv;
    const void *g, *xo, *wo;
    long ldg, ldx, ldw;
    int xdtype, wdtype;
    void *workspace, *gx;
    long ldgx, ldgw;
    float *gw, *gb;
    int *status;
};
cudaError_t launch_fp4_linear_backward(const Fp4BackwardArgs &a, cudaStream_t st);

struct Fp4Scale {
    uint32_t byte;
    float S, r;  // the scale, and what elements are multiplied by
};

// scale of a block from the bits of its largest magnitude as fp32 (taken by
// integer comparison, so that a NaN is larger than everything)
template <bool NV>
MNMT_DEV Fp4Scale fp4_scale(uint32_t amax, float g, float inv6g) {
    Fp4Scale s;
    if (amax >= 0x7F800000u) {  // an infinity or a NaN
        s.byte = NV ? 0x7Fu : 0xFFu;
        s.S = __uint_as_float(0x7FFFFFFFu);
        s.r = s.S;
        return s;
    }
    if (NV) {
        // E4M3 nearest, ties to even, held at 448
        uint16_t b;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(0.0f), "f"(__fmul_rn(__uint_as_float(amax), inv6g)));
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(b));
        s.byte = b & 0xFFu;
        s.S = __fmul_rn(__half2float(__ushort_as_half((unsigned short)h)), g);
        s.r = s.S > 0.0f ? __fdiv_rn(1.0f, s.S) : 0.0f;
    } else {
        // floor(log2 amax) - 2 from the exponent field, not below -127
        const uint32_t f = amax >> 23;
        s.byte = f > 2u ? f - 2u : 0u;
        s.S = s.byte ? __uint_as_float(s.byte << 23) : __uint_as_float(0x00400000u);
        s.r = __uint_as_float((254u - s.byte) << 23);
    }
    return s;
}

// scale of a stored byte
template <bool NV>
MNMT_DEV Fp4Scale fp4_scale_of(uint32_t byte, float g) {
    Fp4Scale s;
    s.byte = byte;
    if (NV) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)byte));
        s.S = __fmul_rn(__half2float(__ushort_as_half((unsigned short)h)), g);
        s.r = s.S == 0.0f ? 0.0f : __fdiv_rn(1.0f, s.S);
    } else {
        s.S = byte == 255u ? __uint_as_float(0x7FFFFFFFu) : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
        s.r = byte == 255u ? s.S : byte == 254u ? __uint_as_float(0x00400000u) : __uint_as_float((254u - byte) << 23);
    }
    return s;
}

// codes of two elements, lo in the low half: nearest, ties to even, held at 6
MNMT_DEV uint32_t fp4_code2(float lo, float hi) {
    uint16_t b;
    asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u16.u8 %0, t;\n\t}" : "=h"(b) : "f"(hi), "f"(lo));
    return b;
}

// fp16 values of the two codes of a byte
MNMT_DEV uint32_t fp4_half2(uint32_t byte) {
    uint32_t h;
    asm("{\n\t.reg .b8 t;\n\tcvt.u8.u16 t, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(h) : "h"((uint16_t)byte));
    return h;
}

MNMT_DEV float2 fp4_float2(uint32_t byte) {
    const uint32_t h = fp4_half2(byte);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

// one element of type T as fp32, and back (nearest even)
template <typename T>
MNMT_DEV float to_f32(T v) {
    if constexpr (sizeof(T) == 4) return v;
    else if constexpr (std::is_same_v<T, __half>) return __half2float(v);
    else return __bfloat162float(v);
}
template <typename T>
MNMT_DEV T from_f32(float v) {
    if constexpr (sizeof(T) == 4) return v;
    else if constexpr (std::is_same_v<T, __half>) return __float2half_rn(v);
    else return __float2bfloat16_rn(v);
}

// eight elements at p: 16 bytes at a time where VEC (p 16-byte aligned, all
// eight in range), else one at a time, zeros from element n on
template <typename T, bool VEC>
MNMT_DEV void load8(const T *p, int n, float (&v)[8]) {
    if constexpr (VEC) {
        if constexpr (sizeof(T) == 4) {
            const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4 *>(p);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (std::is_same_v<T, __half>) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                    v[2 * i] = f.x, v[2 * i + 1] = f.y;
                } else {
                    v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < n ? to_f32(p[i]) : 0.0f;
    }
}

template <typename T, bool VEC>
MNMT_DEV void store8(T *p, int n, const float (&v)[8]) {
    if constexpr (VEC) {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (std::is_same_v<T, __half>) {
                    const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t *>(&h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t *>(&h);
                }
            }
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i] = from_f32<T>(v[i]);
    }
}

}  // namespace mnmt
