// Shared by the kernels of the operators around the step: token log-probabilities (logprobs.hip), 8-bit checkpoints and the gated
// activation (act8.hip), the weight gradient from a checkpoint (act8_wgrad.hip), log-probabilities from the head's input (linear_logprobs.hip),
// gated projections (gated_linear.hip), their products (product_device.h, product.hip), dropout (dropout.hip).
#ifndef ADAGC_OPERATORS_INTERNAL_H
#define ADAGC_OPERATORS_INTERNAL_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "adagc.h"

namespace adagc {

constexpr int64_t kMaxCols = INT32_MAX - 1023;   // columns and leading dimensions: index arithmetic within a row fits 32 bits
constexpr int64_t kMaxLd = kMaxCols;

inline int dtype_size(int32_t dtype) { return dtype == ADAGC_F32 ? 4 : 2; }
inline bool misaligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(to - 1)) != 0; }
inline bool known_dtype(int32_t dtype) { return dtype == ADAGC_F32 || dtype == ADAGC_BF16; }

// Bytes of a checkpoint's row of codes; a row's scales are a 32nd of that.
inline __host__ __device__ int64_t act8_ld(int64_t cols) { return (cols + 31) / 32 * 32; }

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of fp32 or bf16 (uint16_t) values
template <class T>
struct Vector {
    u32x4 w;
};

// 16-byte accesses of arrays whose elements, but nothing more, are aligned: the hardware takes them at any address, and a wave's
// together touch one cache line more.  (Through memcpy the compiler moves the same bytes, but takes them apart one by one.)
typedef u32x4 u32x4_of_f32 __attribute__((aligned(4)));
typedef u32x4 u32x4_of_bf16 __attribute__((aligned(2)));
__device__ __forceinline__ Vector<float> load_whole(const float* p) { return {*reinterpret_cast<const u32x4_of_f32*>(p)}; }
__device__ __forceinline__ Vector<uint16_t> load_whole(const uint16_t* p) { return {*reinterpret_cast<const u32x4_of_bf16*>(p)}; }
__device__ __forceinline__ void store_whole(float* p, const Vector<float>& v) { *reinterpret_cast<u32x4_of_f32*>(p) = v.w; }
__device__ __forceinline__ void store_whole(uint16_t* p, const Vector<uint16_t>& v) { *reinterpret_cast<u32x4_of_bf16*>(p) = v.w; }

// Larger of two, NaN if one is.
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

__device__ __forceinline__ void widen(const Vector<float>& v, float (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v.w[i]);
}
__device__ __forceinline__ void widen(const Vector<uint16_t>& v, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v.w[i] << 16);
        x[2 * i + 1] = __uint_as_float(v.w[i] & 0xFFFF0000u);
    }
}

// Rounded to nearest even where the type is bf16.
template <class T>
__device__ __forceinline__ Vector<T> narrow(const float (&x)[16 / sizeof(T)])
{
    Vector<T> v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            v.w[i] = __float_as_uint(x[i]);
        } else {
            const f32x2_t two = {x[2 * i], x[2 * i + 1]};
            v.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2_t));
        }
    }
    return v;
}

// The 16 bytes at column `col` of a row of n columns, in two steps.  First a load that needs no branch where a row has 16 bytes: the last
// vector of a row that ends inside it is loaded from the row's last 16 bytes; then, where it is used, the values below `col` are
// shifted out and `fill` (a word's bits) takes the places from the row's end on.  (Loading the end one by one costs a wave the memory's
// latency several times, and with short rows every wave has an end.)
template <class T>
__device__ __forceinline__ Vector<T> load_ahead(const T* row, int64_t col, int64_t n, uint32_t fill)
{
    constexpr int N = 16 / sizeof(T);
    if (n >= N) return load_whole(row + (col < n - N ? col : n - N));
    Vector<T> v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            v.w[i] = col + i < n ? __float_as_uint(row[col + i]) : fill;
        } else {
            const uint32_t lo = col + 2 * i < n ? row[col + 2 * i] : fill & 0xFFFFu;
            const uint32_t hi = col + 2 * i + 1 < n ? row[col + 2 * i + 1] : fill >> 16;
            v.w[i] = lo | hi << 16;
        }
    }
    return v;
}
template <class T>
__device__ __forceinline__ void settle(Vector<T>& v, int64_t col, int64_t n, uint32_t fill)
{
    constexpr int N = 16 / sizeof(T);
    if (n < N || col + N <= n) return;
    const int beyond = col < n ? (int)(col + N - n) : N;          // values past the row's end
    const int words = sizeof(T) == 4 ? beyond : beyond / 2;
    if (sizeof(T) == 2 && (beyond & 1)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.w[i] = v.w[i] >> 16 | (i < 3 ? v.w[i + 1] : fill) << 16;
    }
    if (words & 1) v.w = u32x4{v.w[1], v.w[2], v.w[3], fill};
    if (words & 2) v.w = u32x4{v.w[2], v.w[3], fill, fill};
    if (words & 4) v.w = u32x4{fill, fill, fill, fill};
}
template <class T>
__device__ __forceinline__ Vector<T> load_vector(const T* row, int64_t col, int64_t n, uint32_t fill)
{
    Vector<T> v = load_ahead(row, col, n, fill);
    settle(v, col, n, fill);
    return v;
}

// The end of a row is stored in pieces of four, two and one values.
template <class T>
__device__ __forceinline__ void store_vector(T* row, int64_t col, int64_t n, const Vector<T>& v)
{
    constexpr int N = 16 / sizeof(T);
    typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t u32_any __attribute__((aligned(2)));
    if (col + N <= n) {
        store_whole(row + col, v);
    } else if (col < n) {
        T* p = row + col;
        u32x4 w = v.w;
        const int left = (int)(n - col), words = sizeof(T) == 4 ? left : left / 2;
        if (words & 2) {
            *reinterpret_cast<u32x2_any*>(p) = u32x2_any{w[0], w[1]};
            p += 8 / sizeof(T);
            w = u32x4{w[2], w[3], 0, 0};
        }
        if (words & 1) {
            *reinterpret_cast<u32_any*>(p) = w[0];
            p += 4 / sizeof(T);
            w[0] = w[1];
        }
        if constexpr (sizeof(T) == 2) {
            if (left & 1) *p = (uint16_t)w[0];
        }
    }
}

// -inf as `fill`
template <class T>
__device__ __forceinline__ constexpr uint32_t masked()
{
    return sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;
}

}  // namespace adagc
#endif
