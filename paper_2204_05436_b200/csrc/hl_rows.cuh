// Values of a row in 32 bits, whatever they are held in: one at a time, or as many as 16 bytes hold.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hl_common.cuh"

namespace hl {

template <typename T>
__device__ __forceinline__ float as_float(T v) {
    if constexpr (sizeof(T) == 4) return v;
    else if constexpr (std::is_same_v<T, __nv_bfloat16>) return __bfloat162float(v);
    else return __half2float(v);
}
template <typename T>
__device__ __forceinline__ T from_float(float v) {
    if constexpr (sizeof(T) == 4) return v;
    else if constexpr (std::is_same_v<T, __nv_bfloat16>) return __float2bfloat16_rn(v);
    else return __float2half_rn(v);
}

// W values side by side, of a type T: moved as they are where W is 1, in pieces of 16 (or 8) bytes otherwise
template <typename T, int W>
struct Pack {
    static_assert(W == 1 || W * sizeof(T) == 8 || W * sizeof(T) % 16 == 0, "one value, or whole pieces");
    static constexpr int kWords = W * (int)sizeof(T) / 4 > 0 ? W * (int)sizeof(T) / 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (W == 1) {
            if constexpr (sizeof(T) == 4) w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
            else w[0] = __ldg(reinterpret_cast<const unsigned short*>(p));
        } else if constexpr (W * sizeof(T) == 8) {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
            w[0] = v.x, w[1] = v.y;
        } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + i);
                w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ void store(T* p) const {
        if constexpr (W == 1) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
            else *reinterpret_cast<unsigned short*>(p) = (unsigned short)w[0];
        } else if constexpr (W * sizeof(T) == 8) {
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i)
                reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void get(float (&x)[W]) const {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < W; ++i) x[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const unsigned short h = (unsigned short)(w[i / 2] >> (16 * (i & 1)));
                if constexpr (std::is_same_v<T, __nv_bfloat16>) x[i] = __uint_as_float((uint32_t)h << 16);
                else x[i] = __half2float(__ushort_as_half(h));
            }
        }
    }
    __device__ __forceinline__ void set(const float (&x)[W]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = __float_as_uint(x[i]);
        } else if constexpr (W == 1) {
            if constexpr (std::is_same_v<T, __nv_bfloat16>) w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
            else w[0] = __half_as_ushort(__float2half_rn(x[0]));
        } else {
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                if constexpr (std::is_same_v<T, __nv_bfloat16>) {
                    const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&v);
                } else {
                    const __half2 v = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&v);
                }
            }
        }
    }
};

// Eight values side by side of a row that begins anywhere: columns c .. c + 7; what lies outside [0, dim) may be anything.  The 16-byte
// lines that hold some of them are read whole (each has a value of the row, so it lies where the row's memory does), and put in place
// by shifts.
template <typename T>
struct Loose {
    static constexpr int N = 16 / (int)sizeof(T), kLines = 8 / N + 1, kWords = 4 * kLines;
    uint32_t w[kWords];
    int shift;                         // values in the first line that lie before column c
    __device__ __forceinline__ void zero() {
        shift = 0;
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void load(const T* row, int c, int dim) {
        constexpr int kSize = (int)sizeof(T);
        const int in_line = (int)(reinterpret_cast<uintptr_t>(row) & 15), at = c * kSize + in_line;
        const int first = (at & ~15) - in_line, end = min(c + 8, dim) * kSize;         // bytes from the row's begin
        const char* p = reinterpret_cast<const char*>(row) + first;
        shift = (at & 15) / kSize;
#pragma unroll
        for (int i = 0; i < kLines; ++i) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (first + 16 * i < end && first + 16 * i > -16) v = __ldg(reinterpret_cast<const uint4*>(p + 16 * i));
            w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        }
    }
    // the eight, as they are
    __device__ __forceinline__ Pack<T, 8> values() const {
        uint32_t v[kWords];
        const int words = shift * (int)sizeof(T) / 4;            // 0 .. 3
#pragma unroll
        for (int i = 0; i < kWords; ++i) v[i] = words & 2 ? w[i + 2 < kWords ? i + 2 : i] : w[i];
#pragma unroll
        for (int i = 0; i + 1 < kWords; ++i) v[i] = words & 1 ? v[i + 1] : v[i];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(v[i], v[i + 1], 16 * (shift & 1));
        }
        Pack<T, 8> p;
#pragma unroll
        for (int i = 0; i < Pack<T, 8>::kWords; ++i) p.w[i] = v[i];
        return p;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const { values().get(x); }
};

// v[i] for the columns c + i of a row, those outside [0, dim) left out
template <typename T>
__device__ __forceinline__ void store_some(T* row, int c, int dim, const Pack<T, 8>& v) {
    T* p = row + c;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if ((unsigned)(c + i) >= (unsigned)dim) continue;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(p + i) = v.w[i];
        else *reinterpret_cast<unsigned short*>(p + i) = (unsigned short)(v.w[i / 2] >> (16 * (i & 1)));
    }
}
// zeros in a row that begins anywhere, by `threads` threads (at least 8): whole lines, and what lies before and behind them
template <typename T>
__device__ __forceinline__ void zero_row(T* row, int dim, int thread, int threads) {
    constexpr int N = 16 / (int)sizeof(T);
    const int before = min((int)(-(reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (N - 1)), dim);
    const int lines = (dim - before) / N, behind = before + lines * N;
    if (thread < before) row[thread] = from_float<T>(0.f);
    uint4* line = reinterpret_cast<uint4*>(row + before);
    for (int i = thread; i < lines; i += threads) line[i] = make_uint4(0, 0, 0, 0);
    if (behind + thread < dim) row[behind + thread] = from_float<T>(0.f);
}

// ---- arguments: types, and matrices of rows -------------------------------------------------------------------------------
inline int dtype_size(int32_t dtype) { return dtype == HL_F32 ? 4 : dtype == HL_BF16 || dtype == HL_F16 ? 2 : 0; }
inline bool lies_at(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline bool row_matrix_ok(int32_t dtype, int64_t rows, int64_t dim, const void* p, int64_t ld) {
    return dtype_size(dtype) && dim >= 1 && dim <= (int64_t(1) << 24) && ld >= dim && ld < (int64_t(1) << 31) && (p || rows == 0) &&
           lies_at(p, dtype_size(dtype));
}
// whether all rows begin at multiples of `bytes`
inline bool rows_lie_at(int32_t dtype, const void* p, int64_t ld, int64_t bytes) {
    return lies_at(p, bytes) && ld * dtype_size(dtype) % bytes == 0;
}

}  // namespace hl
