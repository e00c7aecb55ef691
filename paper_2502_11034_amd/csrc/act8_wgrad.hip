// Weight gradient of a linear layer whose input was kept in 8 bits (act8.hip), for gfx950:
//     dW[o][i] = sum_t dY[t][o] X[t][i]  (+ dW[o][i]),   X from a checkpoint, sums in fp32.
//
// What a code stands for is exact in bf16, so X enters the matrix cores as bf16 without another rounding, and every product is
// exact in fp32.  An fp32 dY is the sum of three bf16 numbers (8 + 8 + 8 significant bits), multiplied one after the other.
//
// Both operands lie with the summed index t as the slow one, and the matrix-core instruction wants 8 consecutive t of one column in a
// lane: the tiles are staged in LDS as they lie (rows of t), the codes turned to bf16 on the way, and read transposed
// (ds_read_b64_tr_b16).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "act8_device.h"
#include "operators_internal.h"

namespace adagc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define ADAGC_LDS __attribute__((address_space(3)))

struct WgradArgs {
    const void*    d_out;
    const uint8_t *codes, *scales;
    void*          d_weight;
    float*         workspace;     // partial sums of the split tiles
    int64_t        ld_d, ld_w;
    int64_t        rows;
    int32_t        n_out, n_in, ld;
    int32_t        tiles_out, tiles_in;
    int32_t        whole;         // tiles computed by one workgroup each; the others by `split`
    int32_t        split;
    int32_t        accumulate;
};

// Compute units: a round of the launch is as many workgroups of the large tile.
constexpr int kUnits = 256;

// Tile number n of the launch.  8 XCDs, each with its own L2, get workgroups in turn: the 32 that one of them has in a round are
// neighbours, in bands of 8 tiles along n_out.
__device__ __forceinline__ void place_of_tile(const WgradArgs& a, int n, int* to, int* ti)
{
    const int round = n / kUnits * kUnits, in_round = min(a.tiles_out * a.tiles_in - round, kUnits);
    int at = n - round;
    if (in_round == kUnits) at = at % 8 * (kUnits / 8) + at / 8;
    at += round;
    const int band = at / (8 * a.tiles_in), in_band = at - band * 8 * a.tiles_in;
    const int high = min(8, a.tiles_out - 8 * band);
    *ti = in_band / high;
    *to = 8 * band + in_band - *ti * high;
}

// A lane's four consecutive values of a row of the result.
template <class W>
__device__ __forceinline__ void store_results(const WgradArgs& a, int64_t o, int64_t i, f32x4 v)
{
    if (o >= a.n_out || i >= a.n_in) return;
    W* w = static_cast<W*>(a.d_weight) + o * a.ld_w + i;
    if (i + 4 <= a.n_in) {
        if constexpr (sizeof(W) == 4) {
            if (a.accumulate) {
                f32x4 old;
                memcpy(&old, w, 16);
                v += old;
            }
            memcpy(w, &v, 16);
        } else {
            uint32_t two[2];
            if (a.accumulate) {
                memcpy(two, w, 8);
                v[0] += __uint_as_float(two[0] << 16);
                v[1] += __uint_as_float(two[0] & 0xFFFF0000u);
                v[2] += __uint_as_float(two[1] << 16);
                v[3] += __uint_as_float(two[1] & 0xFFFF0000u);
            }
            const f32x2_t lo = {v[0], v[1]}, hi = {v[2], v[3]};
            two[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2_t));
            two[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2_t));
            memcpy(w, two, 8);
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (i + r < a.n_in) {
                const float x = v[r] + (a.accumulate ? to_float(w[r]) : 0.f);
                if constexpr (sizeof(W) == 4) w[r] = x;
                else w[r] = __builtin_bit_cast(uint16_t, (__bf16)x);
            }
    }
}

// BM x BN tile of dW (BM along n_out), kWM x kWN waves, kDeep tokens at a time.
template <class T, int BM, int BN, int kWM, int kWN, int kDeep>
struct Tile {
    static constexpr int kThreads = 64 * kWM * kWN;
    static constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    static constexpr int kTM = BM / kWM / 16, kTN = BN / kWN / 16;         // 16 x 16 blocks of a wave
    static constexpr int kY = kDeep * BM, kX = kDeep * BN;                 // elements of a staged operand tile
    static constexpr int kBuffer = (kParts * kY + kX) * 2;                 // bytes
    static constexpr int kLds = 2 * kBuffer;
    static constexpr int kYUnits = kY / 8 / kThreads, kXUnits = kX / 16 / kThreads;     // of a lane: 8 values of dY, 16 codes
    static_assert(kY % (8 * kThreads) == 0 && kX % (16 * kThreads) == 0, "operand tiles are dealt evenly");

    // Byte offset of 16-byte vector v of row r of a staged tile of C columns: its 32-byte units are permuted so that the 8
    // rows a transposed read takes 32 bytes each of (0 .. 3 and 8 .. 11) lie in different banks.
    static __device__ __forceinline__ int swizzle(int r) { return (r & 3) | ((r >> 3) & 1) << 2; }
    template <int C>
    static __device__ __forceinline__ int at(int r, int v) { return r * C * 2 + ((v >> 1) ^ swizzle(r)) * 32 + (v & 1) * 16; }
};

template <class T, class W, int BM, int BN, int kWM, int kWN, int kDeep>
__global__ __launch_bounds__(64 * kWM * kWN, 2) void wgrad_kernel(const WgradArgs a)
{
    typedef Tile<T, BM, BN, kWM, kWN, kDeep> Shape;
    constexpr int kThreads = Shape::kThreads, kTM = Shape::kTM, kTN = Shape::kTN, kParts = Shape::kParts;
    constexpr int kYUnits = Shape::kYUnits, kXUnits = Shape::kXUnits;
    __shared__ __attribute__((aligned(512))) uint8_t lds[Shape::kLds];
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(&lds[0]);      // low half of the flat address = LDS offset
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / kWN, wn = wave % kWN;

    // the tile and the tokens of this workgroup
    const int item = (int)blockIdx.x;
    int tile = item, part = 0;
    if (item >= a.whole) {
        tile = a.whole + (item - a.whole) / a.split;
        part = (item - a.whole) % a.split;
    }
    int to, ti;
    place_of_tile(a, tile, &to, &ti);
    const int64_t o0 = (int64_t)to * BM, i0 = (int64_t)ti * BN;
    const int64_t steps = (a.rows + kDeep - 1) / kDeep;
    const bool alone = item < a.whole;
    const int64_t step0 = alone ? 0 : steps * part / a.split, step1 = alone ? steps : steps * (part + 1) / a.split;

    // staging: a lane's units, in registers between the load and the write to LDS
    struct Staged {
        Vector<T> y[kYUnits][sizeof(T) / 2];
        u32x4     x[kXUnits];
        uint32_t  scale[kXUnits];
    };
    auto load = [&](int64_t step, Staged& s) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < kYUnits; ++n) {
            const int u = n * kThreads + tid, r = u / (BM / 8);
            const int64_t t = step * kDeep + r, o = o0 + u % (BM / 8) * 8;
            const T* row = static_cast<const T*>(a.d_out) + t * a.ld_d;
            const int64_t end = t < a.rows ? a.n_out : 0;
#pragma unroll
            for (int h = 0; h < (int)sizeof(T) / 2; ++h) s.y[n][h] = load_vector(row, o + h * 4, end, 0);
        }
#pragma unroll
        for (int n = 0; n < kXUnits; ++n) {
            const int u = n * kThreads + tid, r = u / (BN / 16);
            const int64_t t = step * kDeep + r, i = i0 + u % (BN / 16) * 16;
            s.x[n] = u32x4{0, 0, 0, 0};
            s.scale[n] = 127;
            if (t < a.rows && i < a.ld) {
                s.x[n] = *reinterpret_cast<const u32x4*>(a.codes + t * a.ld + i);
                s.scale[n] = a.scales[(t * a.ld + i) / 32];
            }
        }
    };
    auto write = [&](const Staged& s, uint8_t* to_lds) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < kYUnits; ++n) {
            const int u = n * kThreads + tid, r = u / (BM / 8), v = u % (BM / 8);
            uint8_t* at = to_lds + Shape::template at<BM>(r, v);
            if constexpr (kParts == 1) {
                *reinterpret_cast<u32x4*>(at) = u32x4{s.y[n][0].w[0], s.y[n][0].w[1], s.y[n][0].w[2], s.y[n][0].w[3]};
            } else {
                // x = hi + mid + lo, each the upper half of what is left: exact.  (An infinity stays one: nothing is left of it.)
                u32x4 p[3];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t two[3] = {0, 0, 0};
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = __uint_as_float(s.y[n][k / 2].w[k % 2 * 2 + e]);
#pragma unroll
                        for (int q = 0; q < 3; ++q) {
                            const uint32_t top = __float_as_uint(x) & 0xFFFF0000u;
                            two[q] |= e ? top : top >> 16;
                            x = x == __uint_as_float(top) ? 0.f : x - __uint_as_float(top);
                        }
                    }
#pragma unroll
                    for (int q = 0; q < 3; ++q) p[q][k] = two[q];
                }
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x4*>(at + q * Shape::kY * 2) = p[q];
            }
        }
        uint8_t* xs = to_lds + kParts * Shape::kY * 2;
#pragma unroll
        for (int n = 0; n < kXUnits; ++n) {
            const int u = n * kThreads + tid, r = u / (BN / 16), v = u % (BN / 16) * 2;
            const float scale = __uint_as_float(s.scale[n] << 23);
            u32x4 w[2];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                w[k / 4][k % 4] = __builtin_bit_cast(uint32_t, k % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(s.x[n][k / 2], scale, true)
                                                                     : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(s.x[n][k / 2], scale, false));
            u32x4* at = reinterpret_cast<u32x4*>(xs + Shape::template at<BN>(r, v));
            at[0] = w[0];
            at[1] = w[1];
        }
    };

    // Fragments.  16 lanes read 4 rows of 16 columns and get a column each; lane l's are rows 8 (l / 16) .. + 7 of column l mod 16.
    const int fr = 8 * (lane >> 4) + ((lane >> 2) & 3);
    const uint32_t fy = fr * BM * 2 + (((wm * kTM) ^ Shape::swizzle(fr)) * 32) + (lane & 3) * 8;
    const uint32_t fx = kParts * Shape::kY * 2 + fr * BN * 2 + (((wn * kTN) ^ Shape::swizzle(fr)) * 32) + (lane & 3) * 8;
    auto fragment = [&](uint32_t from, uint32_t pitch) __attribute__((always_inline)) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ADAGC_LDS s16x4*>(from));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ADAGC_LDS s16x4*>(from + 4 * pitch));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    f32x4 acc[kTM][kTN];
#pragma unroll
    for (int m = 0; m < kTM; ++m)
#pragma unroll
        for (int n = 0; n < kTN; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};

    Staged staged;
    if (step0 < step1) {
        load(step0, staged);
        write(staged, lds);
        if (step0 + 1 < step1) load(step0 + 1, staged);
    }
    __syncthreads();
    int buffer = 0;
    for (int64_t step = step0; step < step1; ++step) {
        const uint32_t from = lds0 + (uint32_t)(buffer * Shape::kBuffer);
        if (step + 1 < step1) write(staged, lds + (buffer ^ 1) * Shape::kBuffer);
        if (step + 2 < step1) load(step + 2, staged);
#pragma unroll
        for (int kk = 0; kk < kDeep / 32; ++kk) {
            bf16x8 x[kTN];
#pragma unroll
            for (int n = 0; n < kTN; ++n) x[n] = fragment(from + (fx ^ (n * 32)) + kk * 32 * BN * 2, BN * 2);
#pragma unroll
            for (int q = 0; q < kParts; ++q)
#pragma unroll
                for (int m = 0; m < kTM; ++m) {
                    const bf16x8 y = fragment(from + (fy ^ (m * 32)) + q * Shape::kY * 2 + kk * 32 * BM * 2, BM * 2);
#pragma unroll
                    for (int n = 0; n < kTN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[n], y, acc[m][n], 0, 0, 0);
                }
        }
        __syncthreads();
        buffer ^= 1;
    }

    // lane l holds rows (l / 16) * 4 .. + 3 (of X's block) of column l mod 16 (of dY's)
    if (alone) {
#pragma unroll
        for (int m = 0; m < kTM; ++m)
#pragma unroll
            for (int n = 0; n < kTN; ++n)
                store_results<W>(a, o0 + (wm * kTM + m) * 16 + (lane & 15), i0 + (wn * kTN + n) * 16 + (lane >> 4) * 4, acc[m][n]);
    } else {
        f32x4* to_ws = reinterpret_cast<f32x4*>(a.workspace) + (size_t)(item - a.whole) * (BM * BN / 4) + tid;
#pragma unroll
        for (int m = 0; m < kTM; ++m)
#pragma unroll
            for (int n = 0; n < kTN; ++n) to_ws[(m * kTN + n) * kThreads] = acc[m][n];
    }
}

// Adds the parts of the split tiles, in order: a workgroup takes one 16 x 16 block of every wave.
template <class T, class W, int BM, int BN, int kWM, int kWN, int kDeep>
__global__ __launch_bounds__(64 * kWM * kWN) void join_kernel(const WgradArgs a)
{
    typedef Tile<T, BM, BN, kWM, kWN, kDeep> Shape;
    constexpr int kTM = Shape::kTM, kTN = Shape::kTN;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / kWN, wn = wave % kWN;
    const int n_tile = (int)blockIdx.x / (kTM * kTN), block = (int)blockIdx.x % (kTM * kTN), m = block / kTN, n = block % kTN;
    int to, ti;
    place_of_tile(a, a.whole + n_tile, &to, &ti);
    const f32x4* from = reinterpret_cast<const f32x4*>(a.workspace) + (size_t)n_tile * a.split * (BM * BN / 4) + (size_t)block * Shape::kThreads + tid;
    f32x4 sum = from[0];
    for (int p = 1; p < a.split; ++p) sum += from[(size_t)p * (BM * BN / 4)];
    store_results<W>(a, (int64_t)to * BM + (wm * kTM + m) * 16 + (lane & 15), (int64_t)ti * BN + (wn * kTN + n) * 16 + (lane >> 4) * 4, sum);
}

int check(int64_t rows, int64_t n_out, int64_t n_in, int32_t dtype)
{
    if (rows < 0 || n_out < 1 || n_in < 1 || !known_dtype(dtype)) return ADAGC_ERR_INVALID_ARG;
    if (rows > INT32_MAX || n_out > kMaxCols || n_in > kMaxCols) return ADAGC_ERR_TOO_LARGE;
    return ADAGC_OK;
}

// How a call is cut: square tiles of dW, and those of the last, partial round of workgroups also along the tokens, so that they
// fill the chip too.
constexpr int kDeep16 = 64, kDeep32 = 32;        // tokens at a time with bf16 and fp32 dY
struct Plan {
    int     side;
    int64_t tiles_out, tiles_in, whole, rest, split;
    int64_t workspace() const { return split > 1 ? rest * split * side * side * 4 : 0; }
};
Plan plan_of(int64_t rows, int64_t n_out, int64_t n_in, int32_t dtype)
{
    Plan p{};
    auto tiles = [&](int64_t side) { return ((n_out + side - 1) / side) * ((n_in + side - 1) / side); };
    p.side = dtype == ADAGC_BF16 && tiles(256) >= kUnits / 2 ? 256 : 128;
    p.tiles_out = (n_out + p.side - 1) / p.side;
    p.tiles_in = (n_in + p.side - 1) / p.side;
    const int64_t all = p.tiles_out * p.tiles_in, round = p.side == 256 ? kUnits : 2 * kUnits;
    const int64_t deep = dtype == ADAGC_BF16 ? kDeep16 : kDeep32, steps = (rows + deep - 1) / deep;
    p.rest = all % round;
    p.split = p.rest ? std::max<int64_t>(1, std::min(round / p.rest, steps / 4)) : 1;
    if (p.split == 1) p.rest = 0;
    p.whole = all - p.rest;
    return p;
}

template <class T, class W, int SIDE, int kWM, int kWN, int kDeep>
int launch(const WgradArgs& a, const Plan& p, hipStream_t s)
{
    typedef Tile<T, SIDE, SIDE, kWM, kWN, kDeep> Shape;
    wgrad_kernel<T, W, SIDE, SIDE, kWM, kWN, kDeep>
        <<<dim3((uint32_t)(p.whole + p.rest * p.split)), dim3(Shape::kThreads), 0, s>>>(a);
    if (p.rest)
        join_kernel<T, W, SIDE, SIDE, kWM, kWN, kDeep>
            <<<dim3((uint32_t)(p.rest * Shape::kTM * Shape::kTN)), dim3(Shape::kThreads), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}
template <class W>
int launch(const WgradArgs& a, const Plan& p, int32_t dtype, hipStream_t s)
{
    if (dtype == ADAGC_F32) return launch<float, W, 128, 2, 2, kDeep32>(a, p, s);
    if (p.side == 256) return launch<uint16_t, W, 256, 2, 4, kDeep16>(a, p, s);
    return launch<uint16_t, W, 128, 2, 2, kDeep16>(a, p, s);
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int64_t adagc_act8_wgrad_workspace_bytes(int64_t rows, int64_t n_out, int64_t n_in, int32_t dtype)
{
    if (const int rc = check(rows, n_out, n_in, dtype)) return rc;
    return plan_of(rows, n_out, n_in, dtype).workspace();
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
    const Plan p = plan_of(rows, n_out, n_in, dtype);
    if (p.whole + p.rest * p.split > (1 << 22)) return ADAGC_ERR_TOO_LARGE;
    const int64_t need = p.workspace();
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return ADAGC_ERR_INVALID_ARG;
    WgradArgs a{};
    a.d_out = d_out;
    a.ld = (int32_t)act8_ld(n_in);
    a.codes = static_cast<const uint8_t*>(ckpt);
    a.scales = a.codes + rows * a.ld;
    a.d_weight = d_weight;
    a.workspace = static_cast<float*>(workspace);
    a.ld_d = ld_d_out;
    a.ld_w = ld_weight;
    a.rows = rows;
    a.n_out = (int32_t)n_out;
    a.n_in = (int32_t)n_in;
    a.tiles_out = (int32_t)p.tiles_out;
    a.tiles_in = (int32_t)p.tiles_in;
    a.whole = (int32_t)p.whole;
    a.split = (int32_t)p.split;
    a.accumulate = accumulate;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return weight_dtype == ADAGC_F32 ? launch<float>(a, p, dtype, s) : launch<uint16_t>(a, p, dtype, s);
}
