// Activations kept in 8 bits between the forward and the backward pass, and the gated activation that keeps its inputs so, for gfx950.
//
// Blocks of 32 values of a row share a power of two: e is the smallest exponent, at least -100, with largest / 2^e <= 448, the
// largest e4m3 number, and a code is the e4m3 number nearest to x / 2^e (ties to even).  Nothing saturates (but what would be rounded
// to 2^128 is held as 1.875 * 2^127), and a value is off by at most 2^-4 of itself down to 2^-6 * 2^e, which is 2^-13 of the block's largest at
// most, and by at most 2^-10 * 2^e below.  The scale being a power of two, what a code stands for has 4 significant bits and is exact in
// bf16 and in fp32.  Infinities and NaN are kept as NaN; the block's scale is that of its finite values.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "act8_device.h"
#include "operators_internal.h"

namespace adagc {
namespace {

constexpr int kThreads = 256;
constexpr int kPerLane = 4;      // 16-byte vectors of a lane and array

struct Matrix {
    void*   p;
    int64_t ld;
};
struct Checkpoint {
    uint8_t *codes, *scales;     // [rows][ld], [rows][ld / 32]
};

struct Args {
    Matrix     x, y, z, w;       // as the kernel has them
    Checkpoint a, b;
    int32_t    cols, ld;         // of the checkpoints
    uint32_t   row_vectors;      // vectors of a row of ld elements: four at least
    uint32_t   reciprocal;       // 2^32 / row_vectors, rounded down
    uint64_t   vectors;
};

struct Place {
    int64_t row;
    int32_t col;
};

template <bool WHOLE, class T>
__device__ __forceinline__ Vector<T> fetch(const T* row, const Args& a, int32_t col)
{
    return WHOLE ? load_whole(row + col) : load_ahead(row, col, a.cols, 0);
}
// What was fetched, with zeros from the row's end on.
template <bool WHOLE, class T>
__device__ __forceinline__ Vector<T> settled(Vector<T> v, const Args& a, int32_t col)
{
    if constexpr (!WHOLE) settle(v, col, a.cols, 0);
    return v;
}
template <bool WHOLE, class T>
__device__ __forceinline__ void put(T* row, const Args& a, int32_t col, const Vector<T>& v)
{
    if constexpr (WHOLE) store_whole(row + col, v);
    else store_vector(row, col, a.cols, v);
}

template <class T>
__device__ __forceinline__ const T* row_of(const Matrix& m, int64_t row) { return static_cast<const T*>(m.p) + row * m.ld; }
template <class T>
__device__ __forceinline__ T* out_row(const Matrix& m, int64_t row) { return static_cast<T*>(m.p) + row * m.ld; }

// Packs a lane's N values; the 32 / N lanes of a block do so together.
template <int N>
__device__ __forceinline__ void pack_vector(const Args& a, const Checkpoint& to, const Place& at, float (&x)[N])
{
    uint32_t largest = 0, lost = 0;                    // lost: a bit for each infinity and NaN
#pragma unroll
    for (int i = 0; i < N; ++i) largest = max(largest, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    if (largest >= 0x7F780000u) {                      // 1.9375 * 2^127, which would be rounded to 2^128, or not finite
        largest = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t b = __float_as_uint(x[i]) & 0x7FFFFFFFu;
            if (b < 0x7F800000u) {
                largest = max(largest, b);
                if (b >= 0x7F780000u) x[i] = copysignf(0x1.Ep127f, x[i]);
            } else {
                lost |= 1u << i;
            }
        }
    }
    // over the block's lanes, by moves between neighbours within the vector unit: lane ^ 1, lane ^ 2, the other four of eight
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, 0xB1, 0xF, 0xF, true));
    largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, 0x4E, 0xF, 0xF, true));
    if constexpr (N == 4) largest = max(largest, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)largest, 0x141, 0xF, 0xF, true));
    const int e = act8_exponent(largest);
    const float inverse = power_of_two(-e);
    uint32_t code[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) code[i] = act8_encode(x[4 * i] * inverse, x[4 * i + 1] * inverse, x[4 * i + 2] * inverse, x[4 * i + 3] * inverse);
    if (lost) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (lost >> i & 1) code[i / 4] = (code[i / 4] & ~(0xFFu << 8 * (i % 4))) | 0x7Fu << 8 * (i % 4);
    }
    uint8_t* codes = to.codes + at.row * a.ld + at.col;      // aligned: ld is a multiple of 32
    if constexpr (N == 8) *reinterpret_cast<uint2*>(codes) = make_uint2(code[0], code[1]);
    else *reinterpret_cast<uint32_t*>(codes) = code[0];
    if (at.col % 32 == 0) to.scales[(at.row * a.ld + at.col) / 32] = (uint8_t)(e + 127);
}

struct Packed {
    uint32_t code[2];
    uint32_t scale;
};
template <int N>
__device__ __forceinline__ Packed load_packed(const Args& a, const Checkpoint& from, const Place& at)
{
    Packed p;
    const uint8_t* codes = from.codes + at.row * a.ld + at.col;
    if constexpr (N == 8) {
        const uint2 c = *reinterpret_cast<const uint2*>(codes);
        p.code[0] = c.x;
        p.code[1] = c.y;
    } else {
        p.code[0] = *reinterpret_cast<const uint32_t*>(codes);
        p.code[1] = 0;
    }
    p.scale = from.scales[(at.row * a.ld + at.col) / 32];
    return p;
}
template <int N>
__device__ __forceinline__ void unpack_vector(const Packed& p, float (&x)[N])
{
    const float scale = power_of_two((int)p.scale - 127);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)p.code[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)p.code[i], true);
        x[4 * i] = lo.x * scale;
        x[4 * i + 1] = lo.y * scale;
        x[4 * i + 2] = hi.x * scale;
        x[4 * i + 3] = hi.y * scale;
    }
}

// t = 1 / (1 + exp(-g)) as p w, w a power of two, and 1 - t.
// FAR, for gates below kFar, where t is exp(g) in all its bits and next to the least normal number or below it (large factors make normal
// results of those too): p is exp(g) 2^116 (0 below -167).  Products are taken with p first and with w last, but for d_gate.  Other gates' results are
// the same either way.
// FINE, for fp32 values: what the exponential's argument g log2 e loses by its rounding is multiplied in after, so that t is off by
// 8 * 2^-24 of itself at most.  Without, that is 2 |g| more, 2^-16 of t at the least: nothing beside the 2^-8 of bf16 results.  The
// five instructions a value cost 2048 x 4096 fp32 5 % forward, from the memory-side cache (19.5 -> 20.4 us), 8192 x 4096 1.5 % (87.9 -> 89.2).
struct Gate {
    float p, w, rest;
};
constexpr float kFar = -87.f;
template <bool FINE, bool FAR>
__device__ __forceinline__ Gate sigmoid(float g)
{
#pragma clang fp contract(off)      // `high` is the product as it was rounded, everywhere
    constexpr float kC = -1.44269504088896340736f, kLow = (float)(-1.44269504088896340736 - (double)kC), kLn2 = 0.69314718055994530942f;
    const float x = FINE ? __builtin_amdgcn_fmed3f(g, -200.f, 200.f) : g;     // an infinite argument has no rest
    const float high = x * kC;
    float e = __builtin_amdgcn_exp2f(high), low = 0.f;
    if constexpr (FINE) {
        low = fmaf(x, kLow, fmaf(x, kC, -high)) * kLn2;
        e = fmaf(e, low, e);
    }
    const float t = __builtin_amdgcn_rcpf(1.f + e);
    Gate gate{t, 1.f, e * t};
    if constexpr (FAR) {
        float p = __builtin_amdgcn_exp2f(116.f - high);
        if constexpr (FINE) p = fmaf(p, -low, p);
        if (g < kFar) gate = Gate{p, 0x1p-116f, 1.f};
    }
    return gate;
}
// f(constant whether FAR) for a lane's gates, of which hardly any is: the wave is asked.
template <int N, class F>
__device__ __forceinline__ void for_gates(const float (&g)[N], F&& f)
{
    float least = g[0];
#pragma unroll
    for (int i = 1; i < N; ++i) least = fminf(least, g[i]);
    if (__builtin_expect(__ballot(least < kFar) != 0, 0)) f(std::true_type{});
    else f(std::false_type{});
}

// finish(place, load(place)) for every vector; a lane's loads come before its first store, of which the compiler could not tell that
// they touch nothing of what is still to be loaded.  Lanes of a block go together: vectors are dealt to lanes in order, and a row has
// whole blocks.
// WHOLE: rows end with a block of 32, so no vector is cut.
template <int N, class Load, class Finish>
__device__ __forceinline__ void each_vector(const Args& a, Load&& load, Finish&& finish)
{
    constexpr uint32_t kItem = kThreads * kPerLane;
    for (uint64_t first = (uint64_t)blockIdx.x * kItem; first < a.vectors; first += (uint64_t)gridDim.x * kItem) {
        // the first vector's row by a division, the same in all lanes; the others' from there, by a product that is one short at most
        const uint64_t row0 = a.vectors >> 32 ? first / a.row_vectors : (uint32_t)first / a.row_vectors;
        const uint32_t col0 = (uint32_t)(first - row0 * a.row_vectors), left = (uint32_t)min(a.vectors - first, (uint64_t)kItem);
        auto place = [&](uint32_t n) __attribute__((always_inline)) {
            const uint32_t from = col0 + n;
            uint32_t rows = __umulhi(from, a.reciprocal), col = from - rows * a.row_vectors;
            if (col >= a.row_vectors) {
                ++rows;
                col -= a.row_vectors;
            }
            return Place{(int64_t)(row0 + rows), (int32_t)(col * N)};
        };
        Place at[kPerLane];
        decltype(load(at[0])) in[kPerLane];
#pragma unroll
        for (int u = 0; u < kPerLane; ++u) {
            const uint32_t n = (uint32_t)(u * kThreads) + threadIdx.x;
            at[u] = place(n < left ? n : 0);
            in[u] = load(at[u]);
        }
#pragma unroll
        for (int u = 0; u < kPerLane; ++u)
            if ((uint32_t)(u * kThreads) + threadIdx.x < left) finish(at[u], in[u]);
    }
}

// Elementwise kernels all: bound by memory on long calls, by a load's and a store's latency on short ones (2 to 3 us).  Lanes take
// neighbouring 16-byte vectors, so that the 4 (bf16) or 8 (fp32) lanes of a block of 32 are neighbours and find its largest value without LDS.
// 16384 x 4096 bf16: packed in 41 us (4.9 TB/s), unpacked in 30 (6.7, from the memory-side cache); fp32 60 (5.6) and 58 (5.8).
template <class T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void pack_kernel(const Args a)
{
    constexpr int N = 16 / sizeof(T);
    each_vector<N>(
        a, [&](const Place& at) { return fetch<WHOLE>(row_of<T>(a.x, at.row), a, at.col); },
        [&](const Place& at, const Vector<T>& in) {
            float x[N];
            widen(settled<WHOLE>(in, a, at.col), x);
            pack_vector(a, a.a, at, x);
        });
}

template <class T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const Args a)
{
    constexpr int N = 16 / sizeof(T);
    each_vector<N>(
        a, [&](const Place& at) { return load_packed<N>(a, a.a, at); },
        [&](const Place& at, const Packed& in) {
            float x[N];
            unpack_vector(in, x);
            put<WHOLE>(out_row<T>(a.x, at.row), a, at.col, narrow<T>(x));
        });
}

// x: gate, y: up, z: out.  Gate and up are read once for the product and both checkpoints: 8192 x 14336 bf16 170 us (5.6 TB/s), without
// checkpoints 126 (5.6); 8192 x 4096 fp32 89 (5.3) and 72 (5.6).
template <class T, bool WHOLE, bool PACK>
__global__ __launch_bounds__(kThreads) void swiglu_kernel(const Args a)
{
    constexpr int N = 16 / sizeof(T);
    struct In {
        Vector<T> gate, up;
    };
    each_vector<N>(
        a,
        [&](const Place& at) {
            return In{fetch<WHOLE>(row_of<T>(a.x, at.row), a, at.col), fetch<WHOLE>(row_of<T>(a.y, at.row), a, at.col)};
        },
        [&](const Place& at, const In& in) {
            float g[N], u[N], h[N];
            widen(settled<WHOLE>(in.gate, a, at.col), g);
            widen(settled<WHOLE>(in.up, a, at.col), u);
            for_gates(g, [&](auto FAR) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const Gate t = sigmoid<sizeof(T) == 4, decltype(FAR)::value>(g[i]);
                    h[i] = g[i] * t.p * u[i] * t.w;
                }
            });
            put<WHOLE>(out_row<T>(a.z, at.row), a, at.col, narrow<T>(h));
            if constexpr (PACK) {
                pack_vector(a, a.a, at, g);
                pack_vector(a, a.b, at, u);
            }
        });
}

// x: d_out, y: d_gate, z: d_up, w: out (or null).  8192 x 14336 bf16 167 us (5.7 TB/s), with `out` 210 (5.6); 8192 x 4096 fp32 83 (5.7).
template <class T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void swiglu_backward_kernel(const Args a)
{
    constexpr int N = 16 / sizeof(T);
    struct In {
        Vector<T> d_out;
        Packed    gate, up;
    };
    each_vector<N>(
        a,
        [&](const Place& at) {
            return In{fetch<WHOLE>(row_of<T>(a.x, at.row), a, at.col), load_packed<N>(a, a.a, at), load_packed<N>(a, a.b, at)};
        },
        [&](const Place& at, const In& in) {
            float g[N], u[N], d[N], dg[N], h[N];
            widen(settled<WHOLE>(in.d_out, a, at.col), d);
            unpack_vector(in.gate, g);
            unpack_vector(in.up, u);
            for_gates(g, [&](auto FAR) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const Gate t = sigmoid<sizeof(T) == 4, decltype(FAR)::value>(g[i]);
                    const float silu = g[i] * t.p;
                    // of a gradient above 1 w is taken first: d u would leave the range, which w brings it back into, and d w does not
                    const bool above = decltype(FAR)::value && __builtin_fabsf(d[i]) > 1.f;
                    dg[i] = d[i] * (above ? t.w : 1.f) * (u[i] * (t.p * fmaf(g[i], t.rest, 1.f))) * (above ? 1.f : t.w);
                    h[i] = silu * u[i] * t.w;
                    d[i] = d[i] * silu * t.w;
                }
            });
            put<WHOLE>(out_row<T>(a.y, at.row), a, at.col, narrow<T>(dg));
            put<WHOLE>(out_row<T>(a.z, at.row), a, at.col, narrow<T>(d));
            if (a.w.p) put<WHOLE>(out_row<T>(a.w, at.row), a, at.col, narrow<T>(h));
        });
}

Checkpoint checkpoint(const void* p, int64_t rows, int64_t cols)
{
    uint8_t* codes = static_cast<uint8_t*>(const_cast<void*>(p));
    return {codes, codes + rows * act8_ld(cols)};
}

Args arguments(int64_t rows, int64_t cols, int32_t dtype)
{
    Args a{};
    a.cols = (int32_t)cols;
    a.ld = (int32_t)act8_ld(cols);
    a.row_vectors = (uint32_t)((int64_t)a.ld * dtype_size(dtype) / 16);
    a.reciprocal = (uint32_t)((1ull << 32) / a.row_vectors);
    a.vectors = (uint64_t)rows * a.row_vectors;
    return a;
}

dim3 grid_of(const Args& a)
{
    const uint64_t per_item = (uint64_t)kThreads * kPerLane;
    return dim3((uint32_t)std::min<uint64_t>((a.vectors + per_item - 1) / per_item, 1u << 23));
}

// Sizes and types; the pointers are looked at where there is a row
int check(int64_t rows, int64_t cols, int32_t dtype)
{
    if (rows < 0 || cols < 1 || !known_dtype(dtype)) return ADAGC_ERR_INVALID_ARG;
    if (rows > INT32_MAX || cols > kMaxCols) return ADAGC_ERR_TOO_LARGE;
    return ADAGC_OK;
}
int check_matrix(const void* p, int64_t ld, int64_t cols, int32_t dtype)
{
    if (!p || ld < cols || misaligned(p, dtype_size(dtype))) return ADAGC_ERR_INVALID_ARG;
    return ld > kMaxLd ? ADAGC_ERR_TOO_LARGE : ADAGC_OK;
}
int check_checkpoint(const void* p) { return !p || misaligned(p, 16) ? ADAGC_ERR_INVALID_ARG : ADAGC_OK; }

// f(T{}, bool constant whether rows end with a block) for the call's type and columns
template <class F>
int dispatch(int32_t dtype, const Args& a, F&& f)
{
    const bool whole = a.cols == a.ld;
    if (dtype == ADAGC_F32) whole ? f(0.0f, std::true_type{}) : f(0.0f, std::false_type{});
    else whole ? f(uint16_t{}, std::true_type{}) : f(uint16_t{}, std::false_type{});
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int64_t adagc_act8_bytes(int64_t rows, int64_t cols)
{
    if (const int rc = check(rows, cols, ADAGC_F32)) return rc;
    return rows * (act8_ld(cols) + act8_ld(cols) / 32);
}

extern "C" int adagc_act8_pack(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, void* ckpt, void* stream)
{
    if (const int rc = check(rows, cols, dtype)) return rc;
    if (rows == 0) return ADAGC_OK;
    if (const int rc = check_matrix(x, ld, cols, dtype)) return rc;
    if (const int rc = check_checkpoint(ckpt)) return rc;
    Args a = arguments(rows, cols, dtype);
    a.x = {const_cast<void*>(x), ld};
    a.a = checkpoint(ckpt, rows, cols);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return dispatch(dtype, a, [&](auto t, auto whole) {
        pack_kernel<decltype(t), decltype(whole)::value><<<grid_of(a), dim3(kThreads), 0, s>>>(a);
    });
}

extern "C" int adagc_act8_unpack(const void* ckpt, int64_t rows, int64_t cols, void* x, int32_t dtype, int64_t ld, void* stream)
{
    if (const int rc = check(rows, cols, dtype)) return rc;
    if (rows == 0) return ADAGC_OK;
    if (const int rc = check_matrix(x, ld, cols, dtype)) return rc;
    if (const int rc = check_checkpoint(ckpt)) return rc;
    Args a = arguments(rows, cols, dtype);
    a.x = {x, ld};
    a.a = checkpoint(ckpt, rows, cols);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return dispatch(dtype, a, [&](auto t, auto whole) {
        unpack_kernel<decltype(t), decltype(whole)::value><<<grid_of(a), dim3(kThreads), 0, s>>>(a);
    });
}

extern "C" int adagc_swiglu(const void* gate, int64_t ld_gate, const void* up, int64_t ld_up, int32_t dtype, int64_t rows, int64_t cols,
                            void* out, int64_t ld_out, void* gate_ckpt, void* up_ckpt, void* stream)
{
    if (const int rc = check(rows, cols, dtype)) return rc;
    if (!gate_ckpt != !up_ckpt) return ADAGC_ERR_INVALID_ARG;
    if (rows == 0) return ADAGC_OK;
    if (const int rc = check_matrix(gate, ld_gate, cols, dtype)) return rc;
    if (const int rc = check_matrix(up, ld_up, cols, dtype)) return rc;
    if (const int rc = check_matrix(out, ld_out, cols, dtype)) return rc;
    if (gate_ckpt && (check_checkpoint(gate_ckpt) || check_checkpoint(up_ckpt) || gate_ckpt == up_ckpt)) return ADAGC_ERR_INVALID_ARG;
    if ((out == gate && ld_out != ld_gate) || (out == up && ld_out != ld_up)) return ADAGC_ERR_INVALID_ARG;
    Args a = arguments(rows, cols, dtype);
    a.x = {const_cast<void*>(gate), ld_gate};
    a.y = {const_cast<void*>(up), ld_up};
    a.z = {out, ld_out};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (gate_ckpt) {
        a.a = checkpoint(gate_ckpt, rows, cols);
        a.b = checkpoint(up_ckpt, rows, cols);
    }
    return dispatch(dtype, a, [&](auto t, auto whole) {
        if (gate_ckpt) swiglu_kernel<decltype(t), decltype(whole)::value, true><<<grid_of(a), dim3(kThreads), 0, s>>>(a);
        else swiglu_kernel<decltype(t), decltype(whole)::value, false><<<grid_of(a), dim3(kThreads), 0, s>>>(a);
    });
}

extern "C" int adagc_swiglu_backward(const void* d_out, int64_t ld_d_out, int32_t dtype, const void* gate_ckpt, const void* up_ckpt,
                                     int64_t rows, int64_t cols, void* d_gate, int64_t ld_d_gate, void* d_up, int64_t ld_d_up, void* out,
                                     int64_t ld_out, void* stream)
{
    if (const int rc = check(rows, cols, dtype)) return rc;
    if (rows == 0) return ADAGC_OK;
    if (const int rc = check_matrix(d_out, ld_d_out, cols, dtype)) return rc;
    if (const int rc = check_matrix(d_gate, ld_d_gate, cols, dtype)) return rc;
    if (const int rc = check_matrix(d_up, ld_d_up, cols, dtype)) return rc;
    if (out)
        if (const int rc = check_matrix(out, ld_out, cols, dtype)) return rc;
    if (check_checkpoint(gate_ckpt) || check_checkpoint(up_ckpt)) return ADAGC_ERR_INVALID_ARG;
    if (d_gate == d_up || out == d_gate || out == d_up || out == d_out) return ADAGC_ERR_INVALID_ARG;
    if ((d_gate == d_out && ld_d_gate != ld_d_out) || (d_up == d_out && ld_d_up != ld_d_out)) return ADAGC_ERR_INVALID_ARG;
    Args a = arguments(rows, cols, dtype);
    a.x = {const_cast<void*>(d_out), ld_d_out};
    a.y = {d_gate, ld_d_gate};
    a.z = {d_up, ld_d_up};
    a.w = {out, ld_out};
    a.a = checkpoint(gate_ckpt, rows, cols);
    a.b = checkpoint(up_ckpt, rows, cols);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return dispatch(dtype, a, [&](auto t, auto whole) {
        swiglu_backward_kernel<decltype(t), decltype(whole)::value><<<grid_of(a), dim3(kThreads), 0, s>>>(a);
    });
}
