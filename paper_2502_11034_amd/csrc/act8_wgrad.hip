// Weight gradient of a linear layer whose input was kept in 8 bits (act8.hip), for gfx950:
//     dW[o][i] = sum_t dY[t][o] X[t][i]  (+ dW[o][i]),   X from a checkpoint, sums in fp32.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "act8_device.h"
#include "operators_internal.h"

namespace adagc {
namespace {

struct WgradArgs {
    const void*    d_out;
    const uint8_t *codes, *scales;
    void*          d_weight;
    int64_t        ld_d, ld_w;
    int64_t        rows;
    int32_t        n_out, n_in, ld;
    uint32_t       tiles_in;
    int32_t        accumulate;
};

constexpr int kThreads = 256, kTile = 64, kDeep = 16;

// One workgroup per 64 x 64 tile, 4 x 4 values a lane.
template <class T, class W>
__global__ __launch_bounds__(kThreads) void wgrad_kernel(const WgradArgs a)
{
    __shared__ float ys[kDeep][kTile], xs[kDeep][kTile];
    const int o0 = (int)(blockIdx.x / a.tiles_in) * kTile, i0 = (int)(blockIdx.x % a.tiles_in) * kTile;
    const int tid = threadIdx.x, to = tid / 16, ti = tid % 16;
    float acc[4][4] = {};
    for (int64_t t0 = 0; t0 < a.rows; t0 += kDeep) {
#pragma unroll
        for (int n = 0; n < kDeep * kTile / kThreads; ++n) {
            const int k = n * (kThreads / kTile) + tid / kTile, c = tid % kTile;
            const int64_t t = t0 + k;
            const bool in = t < a.rows;
            ys[k][c] = in && o0 + c < a.n_out ? to_float(static_cast<const T*>(a.d_out)[t * a.ld_d + o0 + c]) : 0.f;
            float x = 0.f;
            if (in && i0 + c < a.n_in) {
                const int64_t at = t * a.ld + i0 + c;
                x = __builtin_amdgcn_cvt_f32_fp8((int)a.codes[at], 0) * power_of_two((int)a.scales[at / 32] - 127);
            }
            xs[k][c] = x;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDeep; ++k)
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[p][q] = fmaf(ys[k][to + 16 * p], xs[k][ti + 16 * q], acc[p][q]);
        __syncthreads();
    }
    for (int p = 0; p < 4; ++p)
        for (int q = 0; q < 4; ++q) {
            const int o = o0 + to + 16 * p, i = i0 + ti + 16 * q;
            if (o >= a.n_out || i >= a.n_in) continue;
            W* w = static_cast<W*>(a.d_weight) + o * a.ld_w + i;
            const float v = acc[p][q] + (a.accumulate ? to_float(*w) : 0.f);
            if constexpr (sizeof(W) == 4) {
                *w = v;
            } else {
                *w = (uint16_t)__builtin_bit_cast(uint16_t, (__bf16)v);
            }
        }
}

int check(int64_t rows, int64_t n_out, int64_t n_in, int32_t dtype)
{
    if (rows < 0 || n_out < 1 || n_in < 1 || !known_dtype(dtype)) return ADAGC_ERR_INVALID_ARG;
    if (rows > INT32_MAX || n_out > kMaxCols || n_in > kMaxCols) return ADAGC_ERR_TOO_LARGE;
    return ADAGC_OK;
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int64_t adagc_act8_wgrad_workspace_bytes(int64_t rows, int64_t n_out, int64_t n_in, int32_t dtype)
{
    if (const int rc = check(rows, n_out, n_in, dtype)) return rc;
    return 0;
}

extern "C" int adagc_act8_wgrad(const void* d_out, int32_t dtype, int64_t ld_d_out, const void* ckpt, int64_t rows, int64_t n_out,
                                int64_t n_in, void* d_weight, int32_t weight_dtype, int64_t ld_weight, int32_t accumulate,
                                void* workspace, int64_t workspace_bytes, void* stream)
{
    if (const int rc = check(rows, n_out, n_in, dtype)) return rc;
    if (!known_dtype(weight_dtype) || accumulate < 0 || accumulate > 1 || workspace_bytes < 0 || ld_weight < n_in || !d_weight ||
        misaligned(d_weight, dtype_size(weight_dtype)))
        return ADAGC_ERR_INVALID_ARG;
    if (rows > 0 && (!d_out || !ckpt || ld_d_out < n_out || misaligned(d_out, dtype_size(dtype)) || misaligned(ckpt, 16)))
        return ADAGC_ERR_INVALID_ARG;
    if (ld_weight > kMaxLd || (rows > 0 && ld_d_out > kMaxLd)) return ADAGC_ERR_TOO_LARGE;
    const int64_t need = adagc_act8_wgrad_workspace_bytes(rows, n_out, n_in, dtype);
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return ADAGC_ERR_INVALID_ARG;
    WgradArgs a{};
    a.d_out = d_out;
    a.ld = (int32_t)act8_ld(n_in);
    a.codes = static_cast<const uint8_t*>(ckpt);
    a.scales = a.codes + rows * a.ld;
    a.d_weight = d_weight;
    a.ld_d = ld_d_out;
    a.ld_w = ld_weight;
    a.rows = rows;
    a.n_out = (int32_t)n_out;
    a.n_in = (int32_t)n_in;
    a.accumulate = accumulate;
    const int64_t tiles_out = (n_out + kTile - 1) / kTile, tiles_in = (n_in + kTile - 1) / kTile;
    a.tiles_in = (uint32_t)tiles_in;
    if (tiles_out * tiles_in > (1 << 24) - 1) return ADAGC_ERR_TOO_LARGE;
    const dim3 grid((uint32_t)(tiles_out * tiles_in));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == ADAGC_F32 && weight_dtype == ADAGC_F32) wgrad_kernel<float, float><<<grid, dim3(kThreads), 0, s>>>(a);
    else if (dtype == ADAGC_F32) wgrad_kernel<float, uint16_t><<<grid, dim3(kThreads), 0, s>>>(a);
    else if (weight_dtype == ADAGC_F32) wgrad_kernel<uint16_t, float><<<grid, dim3(kThreads), 0, s>>>(a);
    else wgrad_kernel<uint16_t, uint16_t><<<grid, dim3(kThreads), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}
