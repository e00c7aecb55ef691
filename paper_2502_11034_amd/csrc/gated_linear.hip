// The gated projections of a feed-forward layer, for gfx950:  out = silu(x Wg^T) * (x Wu^T),  silu(g) = g t,  t = 1 / (1 + exp(-g)),
// both products and the activation in one pass, and their gradients
//     d_g = d u t (1 + g (1 - t)),  d_u = d g t,  dx = d_g Wg + d_u Wu,  dWg = d_g^T x,  dWu = d_u^T x.
//
// Blocks of 16 columns of the two weights' rows take turns in a tile, so that a lane holds g and u of the same places.  Backward: d_g and
// d_u go to the workspace (bf16 with bf16 operands: they go into the matrix cores as they are), from g and u that the forward pass kept,
// or from both products made again; from there dx, one product over both, and the two weight gradients, in one launch.
#include "product_device.h"

namespace adagc {
namespace {

using namespace product;

// t and 1 - t: both to full precision, also where one of them is next to 0.  Below -88 t counts as 0.
__device__ __forceinline__ void sigmoid(float g, float* t, float* rest)
{
    const float e = __expf(-g);
    *t = 1.f / (1.f + e);
    *rest = e < 0x1p127f ? e * *t : 1.f;
    if (g != g) *rest = g;
}
__device__ __forceinline__ float silu(float g, float t) { return t == 0.f ? 0.f : g * t; }
// d_g / d and d_u / d
__device__ __forceinline__ void slopes(float g, float u, float* of_gate, float* of_up)
{
    float t, rest;
    sigmoid(g, &t, &rest);
    *of_up = silu(g, t);
    *of_gate = t == 0.f ? 0.f : rest == 0.f ? u * t : u * t * (1.f + g * rest);
}

struct GatedArgs {
    AlongArgs   p;
    void*       out;               // T; backward: or NULL
    void *      gate, *up;         // T, or both NULL; backward: d_g and d_u
    const void* d_out;             // T
    int64_t     ld_out, ld_gate, ld_up, ld_d_out;
};

template <class S, class T, bool BACKWARD>
__global__ __launch_bounds__(S::kThreads, 2) void gated_kernel(const GatedArgs a)
{
    __shared__ __attribute__((aligned(512))) uint8_t lds[S::kLds];
    along_tiles<S, T, true>(a.p, lds, [](int64_t, int64_t) {}, [&](Sums<S>& acc, int64_t m0, int64_t n0, uint8_t*) __attribute__((always_inline)) {
        const int t = thread_anew(), lane = t & 63, wave = t >> 6;
        const int first_row = wave / S::kWN * S::kTM * 16 + lane % 16, first_col = wave % S::kWN * (S::kTN / 2) * 16 + lane / 16 * 4;
        const int64_t row0 = m0 + first_row, col0 = n0 + first_col;
        auto results = [&](int m, int n, f32x4_p& o) __attribute__((always_inline)) {
            const f32x4_p &g = acc[m][n], &u = acc[m][n + 1];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float t, rest;
                sigmoid(g[r], &t, &rest);
                o[r] = silu(g[r], t) * u[r];
            }
        };
        auto gradients = [&](int m, int n, const f32x4_p& d, f32x4_p& o, f32x4_p& dg, f32x4_p& du) __attribute__((always_inline)) {
            const f32x4_p &g = acc[m][n], &u = acc[m][n + 1];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float of_gate, of_up;
                slopes(g[r], u[r], &of_gate, &of_up);
                o[r] = of_up * u[r];
                dg[r] = d[r] * of_gate;
                du[r] = d[r] * of_up;
            }
        };
        if (m0 + S::BM <= a.p.m && n0 + S::BN / 2 <= a.p.n) {
            // a tile inside: one address for each array, no checks
            T* out = static_cast<T*>(a.out) + row0 * a.ld_out + col0;
            T *gate = static_cast<T*>(a.gate) + row0 * a.ld_gate + col0, *up = static_cast<T*>(a.up) + row0 * a.ld_up + col0;
            const T* d_out = static_cast<const T*>(a.d_out) + row0 * a.ld_d_out + col0;
#pragma unroll
            for (int m = 0; m < S::kTM; ++m)
#pragma unroll
                for (int n = 0; n < S::kTN; n += 2) {
                    f32x4_p o;
                    if constexpr (BACKWARD) {
                        f32x4_p dg, du;
                        gradients(m, n, load4(d_out + m * 16 * a.ld_d_out + n * 8), o, dg, du);
                        store4(gate + m * 16 * a.ld_gate + n * 8, dg);
                        store4(up + m * 16 * a.ld_up + n * 8, du);
                    } else {
                        results(m, n, o);
                        if (a.gate) {
                            store4(gate + m * 16 * a.ld_gate + n * 8, acc[m][n]);
                            store4(up + m * 16 * a.ld_up + n * 8, acc[m][n + 1]);
                        }
                    }
                    if (!BACKWARD || a.out) store4(out + m * 16 * a.ld_out + n * 8, o);
                }
            return;
        }
#pragma unroll
        for (int m = 0; m < S::kTM; ++m) {
            const int64_t row = row0 + m * 16;
            if (row >= a.p.m) continue;
#pragma unroll
            for (int n = 0; n < S::kTN; n += 2) {
                const int64_t col = col0 + n * 8;
                if (col >= a.p.n) continue;
                f32x4_p o;
                if constexpr (BACKWARD) {
                    f32x4_p dg, du;
                    gradients(m, n, load4(static_cast<const T*>(a.d_out) + row * a.ld_d_out, col, 0, a.p.n), o, dg, du);
                    store4(static_cast<T*>(a.gate) + row * a.ld_gate, col, 0, a.p.n, dg);
                    store4(static_cast<T*>(a.up) + row * a.ld_up, col, 0, a.p.n, du);
                } else {
                    results(m, n, o);
                    if (a.gate) {
                        store4(static_cast<T*>(a.gate) + row * a.ld_gate, col, 0, a.p.n, acc[m][n]);
                        store4(static_cast<T*>(a.up) + row * a.ld_up, col, 0, a.p.n, acc[m][n + 1]);
                    }
                }
                if (!BACKWARD || a.out) store4(static_cast<T*>(a.out) + row * a.ld_out, col, 0, a.p.n, o);
            }
        }
    });
}

// Few rows: a thread for each result.
template <class T, int TM, bool BACKWARD>
__global__ __launch_bounds__(kThinThreads, 4) void thin_gated_kernel(const GatedArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[kThinLds<TM>];
    constexpr int kColumns = kThinColumns / 2;
    float d = 0.f;
    auto before = [&](int64_t n0) __attribute__((always_inline)) {
        const int64_t row = threadIdx.x / kColumns, col = n0 + threadIdx.x % kColumns;
        if (BACKWARD && row < a.p.m && col < a.p.n) d = to_float(static_cast<const T*>(a.d_out)[row * a.ld_d_out + col]);
    };
    thin_tiles<T, TM, true>(a.p, lds, before, [&](int64_t n0, int64_t row, int at, float g, float u) __attribute__((always_inline)) {
        const int64_t col = n0 + at;
        if (row >= a.p.m || col >= a.p.n) return;
        auto store = [](void* to, int64_t at, float v) __attribute__((always_inline)) {
            if constexpr (sizeof(T) == 4) static_cast<T*>(to)[at] = v;
            else static_cast<T*>(to)[at] = __builtin_bit_cast(uint16_t, (__bf16)v);
        };
        float o;
        if constexpr (BACKWARD) {
            float of_gate, of_up;
            slopes(g, u, &of_gate, &of_up);
            o = of_up * u;
            store(a.gate, row * a.ld_gate + col, d * of_gate);
            store(a.up, row * a.ld_up + col, d * of_up);
        } else {
            float t, rest;
            sigmoid(g, &t, &rest);
            o = silu(g, t) * u;
            if (a.gate) {
                store(a.gate, row * a.ld_gate + col, g);
                store(a.up, row * a.ld_up + col, u);
            }
        }
        if (!BACKWARD || a.out) store(a.out, row * a.ld_out + col, o);
    });
}

struct KeptArgs {
    const void *d_out, *gate, *up;
    void *      d_gate, *d_up, *out;
    int64_t     ld_d_out, ld_gate, ld_up, ld_d, ld_out;
    int64_t     cols, vectors;      // vectors of a row
    int64_t     all;                // of all rows
};

// d_g and d_u from g and u that were kept: 16 bytes of each for a lane.  Bound by memory.
constexpr int kKept = 256;
template <class T>
__global__ __launch_bounds__(kKept) void kept_kernel(const KeptArgs a)
{
    constexpr int N = 16 / sizeof(T);
    const int64_t i = (int64_t)blockIdx.x * kKept + threadIdx.x;
    if (i >= a.all) return;
    const int64_t row = i / a.vectors, col = (i - row * a.vectors) * N;
    float d[N], g[N], u[N], dg[N], du[N], o[N];
    widen(load_vector(static_cast<const T*>(a.d_out) + row * a.ld_d_out, col, a.cols, 0), d);
    widen(load_vector(static_cast<const T*>(a.gate) + row * a.ld_gate, col, a.cols, 0), g);
    widen(load_vector(static_cast<const T*>(a.up) + row * a.ld_up, col, a.cols, 0), u);
#pragma unroll
    for (int r = 0; r < N; ++r) {
        float of_gate, of_up;
        slopes(g[r], u[r], &of_gate, &of_up);
        o[r] = of_up * u[r];
        dg[r] = d[r] * of_gate;
        du[r] = d[r] * of_up;
    }
    store_vector(static_cast<T*>(a.d_gate) + row * a.ld_d, col, a.cols, narrow<T>(dg));
    store_vector(static_cast<T*>(a.d_up) + row * a.ld_d, col, a.cols, narrow<T>(du));
    if (a.out) store_vector(static_cast<T*>(a.out) + row * a.ld_out, col, a.cols, narrow<T>(o));
}

int check(int64_t rows, int64_t dim, int64_t hidden, int32_t dtype)
{
    if (rows < 0 || dim < 1 || hidden < 1 || !known_dtype(dtype)) return ADAGC_ERR_INVALID_ARG;
    if (rows > (1 << 24) - 1 || dim > kMaxCols || hidden > kMaxCols / 2) return ADAGC_ERR_TOO_LARGE;
    const int64_t m = (rows + 127) / 128, k = (dim + 127) / 128, n = (hidden + 63) / 64;
    if (std::max({m * n, m * k, n * k}) >= 1 << 23) return ADAGC_ERR_TOO_LARGE;
    if (rows * ((hidden * dtype_size(dtype) + 15) / 16) > (int64_t)UINT32_MAX - kKept) return ADAGC_ERR_TOO_LARGE;       // lanes
    return ADAGC_OK;
}
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// d_g and d_u, rows x ld each, then partial sums
struct Space {
    int64_t ld, gradients, partial;
    int64_t all() const { return 2 * gradients + partial; }
};
Space space_of(int64_t rows, int64_t dim, int64_t hidden, int32_t dtype)
{
    Space s{};
    s.ld = (hidden + 63) / 64 * 64;
    s.gradients = up16(rows * s.ld * dtype_size(dtype));
    for (const bool aligned : {false, true})
        s.partial = std::max({s.partial, plain_plan((hidden + 7) / 8 * 8, dim, rows, dtype, true, s.ld, dim, 1, 2, aligned).workspace(),
                              plain_plan(rows, dim, hidden, dtype, false, s.ld, dim, 2, 1, aligned).workspace()});
    return s;
}

template <class T, bool BACKWARD>
int projections(GatedArgs a, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    const bool aligned = rows_aligned(a.p.y, a.p.ld_y, dtype) && rows_aligned(a.p.x[0], a.p.ld_x[0], dtype) && rows_aligned(a.p.x[1], a.p.ld_x[1], dtype);
    const AlongPlan p = along_plan(a.p.m, 2 * a.p.n, dtype, aligned, a.p.ld_y, std::max(a.p.ld_x[0], a.p.ld_x[1]));
    a.p.tiles_m = (int32_t)p.tiles_m;
    a.p.tiles_n = (int32_t)p.tiles_n;
    const dim3 grid((uint32_t)(p.tiles_m * p.tiles_n));
    const bool few = thin(a.p, sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16);
    if (few) {
        const dim3 blocks((uint32_t)std::min<int64_t>((a.p.n + kThinColumns / 2 - 1) / (kThinColumns / 2), kThinGrid));
        for_rows(a.p.m, [&](auto TM) { thin_gated_kernel<T, decltype(TM)::value, BACKWARD><<<blocks, dim3(kThinThreads), 0, s>>>(a); });
    } else if constexpr (sizeof(T) == 2) {
        if (p.size == 256) gated_kernel<Large, T, BACKWARD><<<dim3(grid_of<Large>(p.tiles_m * p.tiles_n)), dim3(Large::kThreads), 0, s>>>(a);
        else if (p.direct) gated_kernel<Small, T, BACKWARD><<<grid, dim3(Small::kThreads), 0, s>>>(a);
    }
    if (!few && !p.direct) {
        if constexpr (sizeof(T) == 4) {
            if (p.size == 64) gated_kernel<Smallest, T, BACKWARD><<<grid, dim3(Smallest::kThreads), 0, s>>>(a);
        }
        if (p.size == 128) gated_kernel<Staged<T>, T, BACKWARD><<<grid, dim3(Staged<T>::kThreads), 0, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}

struct Backward {
    GatedArgs   g;                  // the products again
    const void *gate, *up;          // or kept
    int64_t     ld_gate, ld_up;
    void*       d_x;
    int64_t     ld_d_x;
    void *      d_w_gate, *d_w_up;
    int64_t     ld_d_w_gate, ld_d_w_up;
    int32_t     weight_dtype, accumulate;
};

template <class T>
int backward(Backward b, uint8_t* workspace, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    const AlongArgs& p = b.g.p;
    const int64_t rows = p.m, hidden = p.n, dim = p.k;
    const Space space = space_of(rows, dim, hidden, dtype);
    T *d_gate = reinterpret_cast<T*>(workspace), *d_up = reinterpret_cast<T*>(workspace + space.gradients);
    float* partial = reinterpret_cast<float*>(workspace + 2 * space.gradients);
    if (rows > 0 && b.gate) {
        KeptArgs k{};
        k.d_out = b.g.d_out;
        k.ld_d_out = b.g.ld_d_out;
        k.gate = b.gate;
        k.ld_gate = b.ld_gate;
        k.up = b.up;
        k.ld_up = b.ld_up;
        k.d_gate = d_gate;
        k.d_up = d_up;
        k.ld_d = space.ld;
        k.out = b.g.out;
        k.ld_out = b.g.ld_out;
        k.cols = hidden;
        k.vectors = (hidden * (int64_t)sizeof(T) + 15) / 16;
        k.all = rows * k.vectors;
        kept_kernel<T><<<dim3((uint32_t)((k.all + kKept - 1) / kKept)), dim3(kKept), 0, s>>>(k);
        if (hipGetLastError() != hipSuccess) return ADAGC_ERR_HIP;
    } else if (rows > 0) {
        b.g.gate = d_gate;
        b.g.up = d_up;
        b.g.ld_gate = b.g.ld_up = space.ld;
        if (const int rc = projections<T, true>(b.g, s)) return rc;
    }
    if (b.d_w_gate) {
        PlainArgs w{};
        w.y[0] = d_gate;
        w.y[1] = d_up;
        w.ld_y = space.ld;
        w.x[0] = w.x[1] = p.y;
        w.ld_x[0] = w.ld_x[1] = p.ld_y;
        w.out[0] = b.d_w_gate;
        w.out[1] = b.d_w_up;
        w.ld_out[0] = w.ld_add[0] = b.ld_d_w_gate;
        w.ld_out[1] = w.ld_add[1] = b.ld_d_w_up;
        if (b.accumulate) {
            w.add[0] = b.d_w_gate;
            w.add[1] = b.d_w_up;
        }
        w.m = hidden;
        w.m_readable = (hidden + 7) / 8 * 8;
        w.n = dim;
        w.k = rows;
        w.workspace = partial;
        w.factor = 1.f;
        w.pairs = 1;
        w.products = 2;
        w.out_bf16 = w.add_bf16 = b.weight_dtype == ADAGC_BF16;
        if (const int rc = run_plain<T, true>(w, s)) return rc;
    }
    if (b.d_x && rows > 0) {
        PlainArgs x{};
        x.y[0] = d_gate;
        x.y[1] = d_up;
        x.ld_y = space.ld;
        x.x[0] = p.x[0];
        x.x[1] = p.x[1];
        x.ld_x[0] = p.ld_x[0];
        x.ld_x[1] = p.ld_x[1];
        x.out[0] = b.d_x;
        x.ld_out[0] = b.ld_d_x;
        x.m = x.m_readable = rows;
        x.n = dim;
        x.k = hidden;
        x.workspace = partial;
        x.factor = 1.f;
        x.pairs = 2;
        x.products = 1;
        x.out_bf16 = dtype == ADAGC_BF16;
        if (const int rc = run_plain<T, false>(x, s)) return rc;
    }
    return ADAGC_OK;
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int64_t adagc_gated_linear_workspace_bytes(int64_t rows, int64_t dim, int64_t hidden, int32_t dtype)
{
    if (const int rc = check(rows, dim, hidden, dtype)) return rc;
    return 0;
}

extern "C" int adagc_gated_linear(const void* x, int64_t ld_x, const void* w_gate, int64_t ld_w_gate, const void* w_up, int64_t ld_w_up, int32_t dtype,
                                  int64_t rows, int64_t dim, int64_t hidden, void* out, int64_t ld_out, void* gate, int64_t ld_gate, void* up,
                                  int64_t ld_up, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (const int rc = check(rows, dim, hidden, dtype)) return rc;
    const int size = dtype_size(dtype);
    if (workspace_bytes < 0 || (rows > 0 && !gate != !up)) return ADAGC_ERR_INVALID_ARG;
    if (rows == 0) return ADAGC_OK;
    if (!x || !w_gate || !w_up || !out || ld_x < dim || ld_w_gate < dim || ld_w_up < dim || ld_out < hidden || misaligned(x, size) ||
        misaligned(w_gate, size) || misaligned(w_up, size) || misaligned(out, size))
        return ADAGC_ERR_INVALID_ARG;
    if (gate && (ld_gate < hidden || ld_up < hidden || misaligned(gate, size) || misaligned(up, size))) return ADAGC_ERR_INVALID_ARG;
    if (std::max({ld_x, ld_w_gate, ld_w_up, ld_out}) > kMaxLd || (gate && std::max(ld_gate, ld_up) > kMaxLd)) return ADAGC_ERR_TOO_LARGE;
    const int64_t need = adagc_gated_linear_workspace_bytes(rows, dim, hidden, dtype);
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return ADAGC_ERR_INVALID_ARG;
    GatedArgs a{};
    a.p = {x, {w_gate, w_up}, ld_x, {ld_w_gate, ld_w_up}, rows, hidden, dim, 0, 0};
    a.out = out;
    a.ld_out = ld_out;
    a.gate = gate;
    a.up = up;
    a.ld_gate = ld_gate;
    a.ld_up = ld_up;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == ADAGC_F32 ? projections<float, false>(a, s) : projections<uint16_t, false>(a, s);
}

extern "C" int64_t adagc_gated_linear_backward_workspace_bytes(int64_t rows, int64_t dim, int64_t hidden, int32_t dtype)
{
    if (const int rc = check(rows, dim, hidden, dtype)) return rc;
    return space_of(rows, dim, hidden, dtype).all();
}

extern "C" int adagc_gated_linear_backward(const void* d_out, int64_t ld_d_out, const void* x, int64_t ld_x, const void* w_gate, int64_t ld_w_gate,
                                           const void* w_up, int64_t ld_w_up, int32_t dtype, int64_t rows, int64_t dim, int64_t hidden, const void* gate,
                                           int64_t ld_gate, const void* up, int64_t ld_up, void* d_x, int64_t ld_d_x, void* d_w_gate,
                                           int64_t ld_d_w_gate, void* d_w_up, int64_t ld_d_w_up, int32_t weight_dtype, int32_t accumulate, void* out,
                                           int64_t ld_out, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (const int rc = check(rows, dim, hidden, dtype)) return rc;
    const int size = dtype_size(dtype);
    if (workspace_bytes < 0 || !d_w_gate != !d_w_up || (rows > 0 && (!gate != !up || (!d_x && !d_w_gate))) || accumulate < 0 || accumulate > 1) return ADAGC_ERR_INVALID_ARG;
    if (d_w_gate && (!known_dtype(weight_dtype) || ld_d_w_gate < dim || ld_d_w_up < dim || misaligned(d_w_gate, dtype_size(weight_dtype)) ||
                     misaligned(d_w_up, dtype_size(weight_dtype))))
        return ADAGC_ERR_INVALID_ARG;
    if (rows > 0) {
        if (!d_out || !x || !w_gate || !w_up || ld_d_out < hidden || ld_x < dim || ld_w_gate < dim || ld_w_up < dim || misaligned(d_out, size) ||
            misaligned(x, size) || misaligned(w_gate, size) || misaligned(w_up, size) || (d_x && (ld_d_x < dim || misaligned(d_x, size))) ||
            (gate && (ld_gate < hidden || ld_up < hidden || misaligned(gate, size) || misaligned(up, size))) ||
            (out && (ld_out < hidden || misaligned(out, size))))
            return ADAGC_ERR_INVALID_ARG;
        if (std::max({ld_d_out, ld_x, ld_w_gate, ld_w_up}) > kMaxLd || (d_x && ld_d_x > kMaxLd) || (gate && std::max(ld_gate, ld_up) > kMaxLd) ||
            (out && ld_out > kMaxLd))
            return ADAGC_ERR_TOO_LARGE;
    }
    if (d_w_gate && std::max(ld_d_w_gate, ld_d_w_up) > kMaxLd) return ADAGC_ERR_TOO_LARGE;
    const int64_t need = space_of(rows, dim, hidden, dtype).all();
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return ADAGC_ERR_INVALID_ARG;
    Backward b{};
    b.g.p = {x, {w_gate, w_up}, ld_x, {ld_w_gate, ld_w_up}, rows, hidden, dim, 0, 0};
    b.g.out = out;
    b.g.ld_out = ld_out;
    b.g.d_out = d_out;
    b.g.ld_d_out = ld_d_out;
    b.gate = gate;
    b.up = up;
    b.ld_gate = ld_gate;
    b.ld_up = ld_up;
    b.d_x = d_x;
    b.ld_d_x = ld_d_x;
    b.d_w_gate = d_w_gate;
    b.d_w_up = d_w_up;
    b.ld_d_w_gate = ld_d_w_gate;
    b.ld_d_w_up = ld_d_w_up;
    b.weight_dtype = weight_dtype;
    b.accumulate = accumulate;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    return dtype == ADAGC_F32 ? backward<float>(b, ws, s) : backward<uint16_t>(b, ws, s);
}
