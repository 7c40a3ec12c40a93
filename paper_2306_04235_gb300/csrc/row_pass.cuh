// row_pass.cuh -- one pass over the rows of a matrix of fp32, bf16 or fp16: how
// the element-wise kernels divide it among warps and move it.
//
// A lane takes E = 16 consecutive elements of a row (one or two 32-byte accesses)
// where every row of every operand starts on 32 bytes (VEC), so that what is done
// per access (addresses, block scales, shuffles) is shared by 16 elements: with
// eight, quantisation was bound by its instructions (16384 x 2048 bf16 33 us, 29
// with 16).  Else E = 8: rows that start anywhere are turned in shared memory,
// which with 16 elements takes the registers of half the warps (dropout backward
// of 5003 x 1001 42 us, 24 with 8).  A warp takes 32 E columns of a row, or of
// narrow rows two or four at a time.
#pragma once

#include <type_traits>

#include "common.cuh"
#include "fp4.cuh"

namespace mnmt {

__host__ __device__ constexpr int row_elements(bool vec) { return vec ? 16 : 8; }
constexpr int ROW_BLOCKS = 4;  // blocks of 256 threads per SM (64 registers a thread)
// how a row's start is aligned, for every row: 2: 32 bytes, 1: 16 bytes, 0: less
template <typename T>
int row_alignment(const T *p, long ld) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * sizeof(T));
    return a % 32 == 0 ? 2 : a % 16 == 0 ? 1 : 0;
}

// lanes of a row: at least those that share a word of scales
inline int row_lanes(int cols, bool vec) { return vec && cols <= 128 ? 8 : cols <= 16 * row_elements(vec) ? 16 : 32; }
inline int row_grid(long rows, int cols, bool vec, int sms) {
    const int lr = row_lanes(cols, vec), per = row_elements(vec) * lr;
    const long steps = (rows + 32 / lr - 1) / (32 / lr) * ((cols + per - 1) / per);
    const long blocks = (steps + 7) / 8, cap = (long)ROW_BLOCKS * sms;
    return (int)(blocks < 1 ? 1 : blocks < cap ? blocks : cap);
}

// A lane's place: row, the columns from c on that it works on, and (unaligned
// rows) its place among the `lanes` lanes of the row, whose columns start at c0.
struct RowAt {
    long row;
    int c, c0;
};
// the steps of a warp: column chunk fastest, advanced without divisions
template <int E>
struct Walk {
    int lanes, sub, l;
    long group, step_groups, groups;
    int chunk, step_chunks, chunks;
    MNMT_DEV Walk(long rows, int cols, int lr) : lanes(lr) {
        const int lane = threadIdx.x & 31;
        l = lane & (lr - 1), sub = lane / lr;
        const int per = E * lr, rp = 32 / lr;
        groups = (rows + rp - 1) / rp;
        chunks = (cols + per - 1) / per;
        const int w = (int)(blockIdx.x * blockDim.x + threadIdx.x) >> 5, n = (int)(gridDim.x * blockDim.x) >> 5;
        group = w / chunks, chunk = w % chunks;
        step_groups = n / chunks, step_chunks = n % chunks;
    }
    MNMT_DEV bool more() const { return group < groups; }  // alike in all lanes
    MNMT_DEV RowAt at() const {
        const int c0 = chunk * E * lanes;
        return RowAt{group * (32 / lanes) + sub, c0 + E * l, c0};
    }
    MNMT_DEV void next() {
        group += step_groups;
        chunk += step_chunks;
        if (chunk >= chunks) chunk -= chunks, group++;
    }
};

// E elements as words
template <typename T, int E>
struct Raw {
    uint32_t w[E * sizeof(T) / 4];
};

MNMT_DEV void ld32(const void *p, uint32_t *w) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
}
MNMT_DEV void st32(void *p, const uint32_t *w) {
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                 "r"(w[6]), "r"(w[7]), "l"(p)
                 : "memory");
}

template <typename T>
MNMT_DEV uint32_t bits_of(T v) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(v);
    else return *reinterpret_cast<const uint16_t *>(&v);
}

// A lane's E elements of `row`, zeros beyond the matrix (ok: the row is in it).
// Aligned rows (al; VEC: all on 32 bytes): its own; else `lanes` lanes load
// `lanes` neighbours at a time, to be turned in shared memory by settle.
template <typename T, bool VEC, int E>
MNMT_DEV void fetch(const T *row, const Walk<E> &w, const RowAt &a, int cols, bool ok, int al, Raw<T, E> &r) {
    constexpr int NW = E * sizeof(T) / 4;
    if (VEC || al) {
        if (ok && a.c + E <= cols) {
            if (NW >= 8 && (VEC || al == 2)) {
#pragma unroll
                for (int i = 0; i < NW / 8; i++) ld32(row + a.c + i * (32 / sizeof(T)), r.w + 8 * i);
            } else {
#pragma unroll
                for (int i = 0; i < NW / 4; i++) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(row + a.c + i * (16 / sizeof(T)));
                    r.w[4 * i] = v.x, r.w[4 * i + 1] = v.y, r.w[4 * i + 2] = v.z, r.w[4 * i + 3] = v.w;
                }
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < NW; i++) r.w[i] = 0;
        if (!ok) return;
#pragma unroll
        for (int k = 0; k < E; k++)
            if (a.c + k < cols) r.w[k * NW / E] |= bits_of(row[a.c + k]) << (sizeof(T) == 2 ? 16 * (k & 1) : 0);
    } else {
#pragma unroll
        for (int i = 0; i < NW; i++) r.w[i] = 0;
#pragma unroll
        for (int j = 0; j < E; j++) {
            const int c = a.c0 + j * w.lanes + w.l;
            if (ok && c < cols) r.w[j * NW / E] |= bits_of(row[c]) << (sizeof(T) == 2 ? 16 * (j & 1) : 0);
        }
    }
}

// element k as fp32
template <typename T, int E>
MNMT_DEV float raw_at(const Raw<T, E> &r, int k) {
    if constexpr (sizeof(T) == 4) {
        return __uint_as_float(r.w[k]);
    } else if constexpr (std::is_same_v<T, __half>) {
        const __half2 h = *reinterpret_cast<const __half2 *>(&r.w[k >> 1]);
        return k & 1 ? __high2float(h) : __low2float(h);
    } else {
        return __uint_as_float(k & 1 ? r.w[k >> 1] & 0xFFFF0000u : r.w[k >> 1] << 16);
    }
}

// buf: 33 E words of the warp, element e of the warp's 32 E at e + e / 32 (no bank
// conflicts: lanes write neighbours and read E apart, or the reverse)
template <typename T, bool VEC, int E>
MNMT_DEV void settle(const Raw<T, E> &r, const Walk<E> &w, int al, float *buf, float (&v)[E]) {
    if (VEC || al) {
#pragma unroll
        for (int k = 0; k < E; k++) v[k] = raw_at(r, k);
    } else {
        const int lane = threadIdx.x & 31, first = w.sub * E * w.lanes + w.l;
        __syncwarp();
#pragma unroll
        for (int j = 0; j < E; j++) {
            const int e = first + j * w.lanes;
            buf[e + (e >> 5)] = raw_at(r, j);
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < E; k++) v[k] = buf[E * lane + (E * lane >> 5) + k];
    }
}

template <typename T, bool VEC, int E>
MNMT_DEV void put(T *row, const Walk<E> &w, const RowAt &a, int cols, bool ok, int al, float *buf, const float (&v)[E]) {
    constexpr int NW = E * sizeof(T) / 4;
    if (VEC || al) {
        if (!ok) return;
        if (a.c + E <= cols) {
            uint32_t u[NW];
#pragma unroll
            for (int i = 0; i < NW; i++) {
                if constexpr (sizeof(T) == 4) {
                    u[i] = __float_as_uint(v[i]);
                } else if constexpr (std::is_same_v<T, __half>) {
                    const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                    u[i] = *reinterpret_cast<const uint32_t *>(&h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                    u[i] = *reinterpret_cast<const uint32_t *>(&h);
                }
            }
            if (NW >= 8 && (VEC || al == 2)) {
#pragma unroll
                for (int i = 0; i < NW / 8; i++) st32(row + a.c + i * (32 / sizeof(T)), u + 8 * i);
            } else {
#pragma unroll
                for (int i = 0; i < NW / 4; i++)
                    *reinterpret_cast<uint4 *>(row + a.c + i * (16 / sizeof(T))) = make_uint4(u[4 * i], u[4 * i + 1], u[4 * i + 2], u[4 * i + 3]);
            }
            return;
        }
#pragma unroll
        for (int k = 0; k < E; k++)
            if (a.c + k < cols) row[a.c + k] = from_f32<T>(v[k]);
    } else {
        const int lane = threadIdx.x & 31, first = w.sub * E * w.lanes + w.l;
        __syncwarp();
#pragma unroll
        for (int k = 0; k < E; k++) buf[E * lane + (E * lane >> 5) + k] = v[k];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < E; j++) {
            const int e = first + j * w.lanes, c = a.c0 + j * w.lanes + w.l;
            if (ok && c < cols) row[c] = from_f32<T>(buf[e + (e >> 5)]);
        }
    }
}

// the warp's buffer for unaligned rows (blocks of 256 threads)
#define MNMT_ROW_BUF(buf, VEC)                     \
    __shared__ float buf##_all[VEC ? 1 : 8 * 264]; \
    float *buf = buf##_all + (VEC ? 0 : (threadIdx.x >> 5) * 264)

}  // namespace mnmt
