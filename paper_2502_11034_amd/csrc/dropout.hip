// Dropout whose mask is never stored, for gfx950:  out = (residual +) keep x / (1 - p),  keep from a counter-based generator: the same
// call on the gradient makes the same mask again.
//
// Random words: block b = (offset + row ceil(cols / 4) + col / 4) mod 2^64 of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random
// numbers: as easy as 1, 2, 3", 2011) with the counter (b's low word, its high word, 0, 0) and the seed as key gives the words of columns
// 4 (col / 4) .. + 3.  A value is kept if its word is at least round(p 2^32).
//
// What bounds it: memory with the vector unit close behind, ten rounds of two 32 x 32 -> 64 bit products for every four values: 16384 x 4096 bf16 60 us,
// with a residual 71 (4.5 and 5.7 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "operators_internal.h"

namespace adagc {
namespace {

struct DropoutArgs {
    const void *    x, *residual;   // residual: or NULL
    void*           out;
    const uint64_t* rng;            // seed, offset
    int64_t         ld_x, ld_residual, ld_out;
    int64_t         cols, blocks;   // of random words in a row
    int64_t         vectors, all;   // of 16 bytes in a row, in all
    uint32_t        least;          // kept words are at least this; keep_none: none is
    int32_t         keep_none;
    float           factor;
};

__device__ __forceinline__ void philox(uint64_t block, uint32_t k0, uint32_t k1, uint32_t (&w)[4])
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = 0, c3 = 0;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0;
    w[1] = c1;
    w[2] = c2;
    w[3] = c3;
}

constexpr int kThreads = 256;

// A lane has 16 bytes of a row: one block of words with fp32, two with bf16.
template <class T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const DropoutArgs a)
{
    constexpr int N = 16 / sizeof(T);
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= a.all) return;
    const uint64_t seed = a.rng[0], offset = a.rng[1];
    const int64_t row = i / a.vectors, v = i - row * a.vectors, col = v * N;
    float x[N], y[N] = {};
    widen(load_vector(static_cast<const T*>(a.x) + row * a.ld_x, col, a.cols, 0), x);
    if (a.residual) widen(load_vector(static_cast<const T*>(a.residual) + row * a.ld_residual, col, a.cols, 0), y);
    const uint64_t block = offset + (uint64_t)(row * a.blocks + v * (N / 4));
#pragma unroll
    for (int b = 0; b < N / 4; ++b) {
        uint32_t w[4];
        philox(block + b, (uint32_t)seed, (uint32_t)(seed >> 32), w);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (w[r] >= a.least && !a.keep_none) y[4 * b + r] = fmaf(x[4 * b + r], a.factor, y[4 * b + r]);
    }
    store_vector(static_cast<T*>(a.out) + row * a.ld_out, col, a.cols, narrow<T>(y));
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int adagc_dropout(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, int32_t dtype, int64_t rows, int64_t cols, double p,
                             const uint64_t* rng, void* out, int64_t ld_out, void* stream)
{
    if (rows < 0 || cols < 1 || !known_dtype(dtype) || !(p >= 0.0 && p <= 1.0)) return ADAGC_ERR_INVALID_ARG;
    if (rows > INT32_MAX || cols > kMaxCols) return ADAGC_ERR_TOO_LARGE;
    if (rows == 0) return ADAGC_OK;
    const int size = dtype_size(dtype);
    if (!x || !out || !rng || ld_x < cols || ld_out < cols || misaligned(x, size) || misaligned(out, size) || misaligned(rng, 8) ||
        (residual && (ld_residual < cols || misaligned(residual, size))))
        return ADAGC_ERR_INVALID_ARG;
    if (ld_x > kMaxLd || ld_out > kMaxLd || (residual && ld_residual > kMaxLd)) return ADAGC_ERR_TOO_LARGE;
    DropoutArgs a{};
    a.x = x;
    a.ld_x = ld_x;
    a.residual = residual;
    a.ld_residual = ld_residual;
    a.out = out;
    a.ld_out = ld_out;
    a.rng = rng;
    a.cols = cols;
    a.blocks = (cols + 3) / 4;
    a.vectors = (cols * size + 15) / 16;
    a.all = rows * a.vectors;
    if (a.all > (int64_t)UINT32_MAX - kThreads) return ADAGC_ERR_TOO_LARGE;
    const double least = std::nearbyint(p * 4294967296.0);
    a.keep_none = least >= 4294967296.0;
    a.least = a.keep_none ? UINT32_MAX : (uint32_t)least;
    a.factor = a.keep_none ? 0.f : (float)(1.0 / (1.0 - p));
    const dim3 grid((uint32_t)((a.all + kThreads - 1) / kThreads));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == ADAGC_F32) dropout_kernel<float><<<grid, dim3(kThreads), 0, s>>>(a);
    else dropout_kernel<uint16_t><<<grid, dim3(kThreads), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}
