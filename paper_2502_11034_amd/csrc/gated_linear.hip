// The gated projections of a feed-forward layer, for gfx950:  out = silu(x Wg^T) * (x Wu^T),  silu(g) = g t,  t = 1 / (1 + exp(-g)),
// both products and the activation in one pass, and their gradients
//     d_g = d u t (1 + g (1 - t)),  d_u = d g t,  dx = d_g Wg + d_u Wu,  dWg = d_g^T x,  dWu = d_u^T x.
//
// Blocks of 16 columns of the two weights' rows take turns in a tile, so that a lane holds g and u of the same places.  Backward: d_g and
// d_u go to the workspace (bf16 with bf16 operands: they go into the matrix cores as they are, and a second part of them would double the time of the
// products), from g and u that the forward pass kept, or from both products made again; from there dx, one product over both, and the two
// weight gradients, in one launch.
//
// What bounds it: the matrix cores.  8192 rows, 14336 from 4096, bf16: forward with g and u kept 1410 - 1620 us (1.19 - 1.37 PFLOP/s), d_g and d_u from
// them 199 (5.9 TB/s), the weights' gradients 1465 - 1660, dx 1350 - 1500.  24 rows: the weights' way to the compute units, 38 us from the memory-side
// cache, 47 from memory (5 TB/s).
#include "product_device.h"

namespace adagc {
namespace {

using namespace product;

// silu(g) = g t and its slope t (1 + g (1 - t)), t = 1 / (1 + exp(-g)): both times 1 / w, w a power of two.  For gates below kFar, where t is exp(g) in all its
// bits and next to the least normal number or below it (large factors make normal results of those too), w is 2^-116 (and t 0 below
// -167); for others it is 1.  Products are taken with silu or slope first and with w last, but for d_g.
// FINE, for fp32 data: what the exponential's argument g log2 e loses by its rounding is multiplied in after, so that t is off by 8 * 2^-24 of
// itself at most.  Without, that is 2 |g| more, 2^-16 of t at the least: nothing beside the 2^-8 of bf16 results.  No branch: 17 fp32 rows, 2 x 12382 from
// 4096 and back, 462 us; with e^-g as it is and a division 457, and every larger case the same either way.
struct Gate {
    float silu, slope, w;
};
constexpr float kFar = -87.f;
template <bool FINE>
__device__ __forceinline__ Gate gate_of(float g)
{
#pragma clang fp contract(off)      // `high` is the product as it was rounded, everywhere
    constexpr float kC = -1.44269504088896340736f, kLow = (float)(-1.44269504088896340736 - (double)kC), kLn2 = 0.69314718055994530942f;
    // beyond 200 either way t is 0 or 1, and no infinity meets a 0; NaN stays
    const float at_least = g < -200.f ? -200.f : g, x = at_least > 200.f ? 200.f : at_least;
    const bool far = x < kFar;
    const float high = x * kC;
    float e = __builtin_amdgcn_exp2f(far ? 116.f - high : high);           // exp(g) 2^116 or exp(-g)
    if constexpr (FINE) {
        const float low = fmaf(x, kLow, fmaf(x, kC, -high)) * kLn2;
        e = fmaf(e, far ? -low : low, e);
    }
    const float t = __builtin_amdgcn_rcpf(1.f + e), p = far ? e : t, rest = far ? 1.f : e * t;
    return {at_least * p, p * fmaf(x, rest, 1.f), far ? 0x1p-116f : 1.f};
}
template <bool FINE>
__device__ __forceinline__ float result_of(float g, float u)
{
    const Gate t = gate_of<FINE>(g);
    return t.silu * u * t.w;
}
template <bool FINE>
__device__ __forceinline__ void gradients_of(float g, float u, float d, float& out, float& d_g, float& d_u)
{
    const Gate t = gate_of<FINE>(g);
    // of a gradient above 1 w is taken first: d u would leave the range, which w brings it back into, and d w does not
    const bool above = __builtin_fabsf(d) > 1.f;
    out = t.silu * u * t.w;
    d_g = d * (above ? t.w : 1.f) * (u * t.slope) * (above ? 1.f : t.w);
    d_u = d * t.silu * t.w;
}

struct GatedArgs {
    AlongArgs   p;
    void*       out;               // O; backward: or NULL
    void *      gate, *up;         // O, or both NULL; backward: d_g and d_u, in kParts of bf16 if there are as many
    const void* d_out;             // O
    int64_t     ld_out, ld_gate, ld_up, ld_d_out;
    int64_t     part, rows;        // d_g and d_u in parts: elements from part to part; rows with those filled with zeros
};

// Four of d_g or d_u in parts.
__device__ __forceinline__ void store_parts(uint16_t* to, int64_t part, const f32x4_p& v)
{
    uint32_t bits[kParts][2];
    split4(v, bits);
#pragma unroll
    for (int p = 0; p < kParts; ++p) *reinterpret_cast<u32x2_of_bf16*>(to + p * part) = u32x2_of_bf16{bits[p][0], bits[p][1]};
}

// T: of the operands; O: of what else is read and written.  PARTS: of d_g and d_u, 1 or kParts, the latter with zeros in rows past the last one
// and columns past the last one.
template <class S, class T, class O, bool BACKWARD, int PARTS, Sum SUM>
__global__ __launch_bounds__(S::kThreads, 2) void gated_kernel(const GatedArgs a)
{
    __shared__ __attribute__((aligned(512))) uint8_t lds[S::kLds];
    constexpr bool kFine = sizeof(O) == 4;
    along_tiles<S, T, true, SUM>(a.p, lds, [](int64_t, int64_t) {}, [&](Sums<S>& acc, int64_t m0, int64_t n0, uint8_t*) __attribute__((always_inline)) {
        const int t = thread_anew(), lane = t & 63, wave = t >> 6;
        const int first_row = wave / S::kWN * S::kTM * 16 + lane % 16, first_col = wave % S::kWN * (S::kTN / 2) * 16 + lane / 16 * 4;
        const int64_t row0 = m0 + first_row, col0 = n0 + first_col;
        auto results = [&](int m, int n, f32x4_p& o) __attribute__((always_inline)) {
            const f32x4_p &g = acc[m][n], &u = acc[m][n + 1];
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = result_of<kFine>(g[r], u[r]);
        };
        auto gradients = [&](int m, int n, const f32x4_p& d, f32x4_p& o, f32x4_p& dg, f32x4_p& du) __attribute__((always_inline)) {
            const f32x4_p &g = acc[m][n], &u = acc[m][n + 1];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float out, d_g, d_u;
                gradients_of<kFine>(g[r], u[r], d[r], out, d_g, d_u);
                o[r] = out;
                dg[r] = d_g;
                du[r] = d_u;
            }
        };
        if constexpr (PARTS > 1) {
            uint16_t *gate = static_cast<uint16_t*>(a.gate) + row0 * a.ld_gate + col0, *up = static_cast<uint16_t*>(a.up) + row0 * a.ld_up + col0;
#pragma unroll
            for (int m = 0; m < S::kTM; ++m) {
                const int64_t row = row0 + m * 16;
                if (row >= a.rows) continue;
#pragma unroll
                for (int n = 0; n < S::kTN; n += 2) {
                    const int64_t col = col0 + n * 8;
                    if (col >= a.ld_gate) continue;
                    const f32x4_p none = {0.f, 0.f, 0.f, 0.f};
                    f32x4_p o, dg, du;
                    gradients(m, n, row < a.p.m ? load4(static_cast<const O*>(a.d_out) + row * a.ld_d_out, col, 0, a.p.n) : none, o, dg, du);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (row >= a.p.m || col + r >= a.p.n) dg[r] = du[r] = 0.f;
                    store_parts(gate + m * 16 * a.ld_gate + n * 8, a.part, dg);
                    store_parts(up + m * 16 * a.ld_up + n * 8, a.part, du);
                    if (a.out && row < a.p.m) store4(static_cast<O*>(a.out) + row * a.ld_out, col, 0, a.p.n, o);
                }
            }
            return;
        }
        if (m0 + S::BM <= a.p.m && n0 + S::BN / 2 <= a.p.n) {
            // a tile inside: one address for each array, no checks
            O* out = static_cast<O*>(a.out) + row0 * a.ld_out + col0;
            O *gate = static_cast<O*>(a.gate) + row0 * a.ld_gate + col0, *up = static_cast<O*>(a.up) + row0 * a.ld_up + col0;
            const O* d_out = static_cast<const O*>(a.d_out) + row0 * a.ld_d_out + col0;
            // blocks of the same array at a time: two where a wave has two, stored together
            constexpr int kOf = S::kTN % 4 == 0 ? 2 : 1;
            auto store = [](O* to, const f32x4_p (&v)[kOf]) __attribute__((always_inline)) {
                if constexpr (kOf == 2) store_blocks(to, v[0], v[1]);
                else store4(to, v[0]);
            };
#pragma unroll
            for (int m = 0; m < S::kTM; ++m)
#pragma unroll
                for (int n = 0; n < S::kTN; n += 2 * kOf) {
                    f32x4_p o[kOf], first[kOf], second[kOf];
#pragma unroll
                    for (int i = 0; i < kOf; ++i) {
                        if constexpr (BACKWARD) {
                            gradients(m, n + 2 * i, load4(d_out + m * 16 * a.ld_d_out + (n + 2 * i) * 8), o[i], first[i], second[i]);
                        } else {
                            results(m, n + 2 * i, o[i]);
                            first[i] = acc[m][n + 2 * i];
                            second[i] = acc[m][n + 2 * i + 1];
                        }
                    }
                    if (BACKWARD || a.gate) {
                        store(gate + m * 16 * a.ld_gate + n * 8, first);
                        store(up + m * 16 * a.ld_up + n * 8, second);
                    }
                    if (!BACKWARD || a.out) store(out + m * 16 * a.ld_out + n * 8, o);
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
                    gradients(m, n, load4(static_cast<const O*>(a.d_out) + row * a.ld_d_out, col, 0, a.p.n), o, dg, du);
                    store4(static_cast<O*>(a.gate) + row * a.ld_gate, col, 0, a.p.n, dg);
                    store4(static_cast<O*>(a.up) + row * a.ld_up, col, 0, a.p.n, du);
                } else {
                    results(m, n, o);
                    if (a.gate) {
                        store4(static_cast<O*>(a.gate) + row * a.ld_gate, col, 0, a.p.n, acc[m][n]);
                        store4(static_cast<O*>(a.up) + row * a.ld_up, col, 0, a.p.n, acc[m][n + 1]);
                    }
                }
                if (!BACKWARD || a.out) store4(static_cast<O*>(a.out) + row * a.ld_out, col, 0, a.p.n, o);
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
        constexpr bool kFine = sizeof(T) == 4;
        if constexpr (BACKWARD) {
            float d_g, d_u;
            gradients_of<kFine>(g, u, d, o, d_g, d_u);
            store(a.gate, row * a.ld_gate + col, d_g);
            store(a.up, row * a.ld_up + col, d_u);
        } else {
            o = result_of<kFine>(g, u);
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
    int64_t     rows, cols, vectors;       // vectors of a row
    int64_t     all;                // of all rows
    int64_t     part;               // d_g and d_u in parts: elements from part to part
};

// d_g and d_u from g and u that were kept: 16 bytes of each for a lane.  Bound by memory.
constexpr int kKept = 256;
template <class T, int PARTS>
__global__ __launch_bounds__(kKept) void kept_kernel(const KeptArgs a)
{
    constexpr int N = 16 / sizeof(T);
    const int64_t i = (int64_t)blockIdx.x * kKept + threadIdx.x;
    if (i >= a.all) return;
    const int64_t row = i / a.vectors, col = (i - row * a.vectors) * N;
    float d[N], g[N], u[N], dg[N], du[N], o[N];
    const int64_t cols = PARTS > 1 && row >= a.rows ? 0 : a.cols;          // (0 times what is there past the end is 0)
    widen(load_vector(static_cast<const T*>(a.d_out) + row * a.ld_d_out, col, cols, 0), d);
    widen(load_vector(static_cast<const T*>(a.gate) + row * a.ld_gate, col, cols, 0), g);
    widen(load_vector(static_cast<const T*>(a.up) + row * a.ld_up, col, cols, 0), u);
#pragma unroll
    for (int r = 0; r < N; ++r) gradients_of<sizeof(T) == 4>(g[r], u[r], d[r], o[r], dg[r], du[r]);
    if constexpr (PARTS > 1) {
        store_parts(static_cast<uint16_t*>(a.d_gate) + row * a.ld_d + col, a.part, f32x4_p{dg[0], dg[1], dg[2], dg[3]});
        store_parts(static_cast<uint16_t*>(a.d_up) + row * a.ld_d + col, a.part, f32x4_p{du[0], du[1], du[2], du[3]});
    } else {
        store_vector(static_cast<T*>(a.d_gate) + row * a.ld_d, col, cols, narrow<T>(dg));
        store_vector(static_cast<T*>(a.d_up) + row * a.ld_d, col, cols, narrow<T>(du));
    }
    if (a.out) store_vector(static_cast<T*>(a.out) + row * a.ld_out, col, cols, narrow<T>(o));
}

int check(int64_t rows, int64_t dim, int64_t hidden, int32_t dtype)
{
    if (rows < 0 || dim < 1 || hidden < 1 || !known_dtype(dtype)) return ADAGC_ERR_INVALID_ARG;
    if (rows > (1 << 24) - 1 || dim > kMaxCols || hidden > kMaxCols / 2) return ADAGC_ERR_TOO_LARGE;
    const int64_t m = (rows + 63) / 64, k = (dim + 63) / 64, n = (hidden + 31) / 32;
    // lanes of a launch are within 32 bits
    if (m * n >= 1 << 23 || std::max(n * k, m * k) >= 1 << 22 || m * 64 * (n * 32 / 4) > (int64_t)UINT32_MAX - kKept) return ADAGC_ERR_TOO_LARGE;
    // x and both weights are laid out in one launch
    const Layout l = layout_of(rows, hidden, dim, dtype, true);
    if (l.anew && (l.part(rows) + 2 * l.part(hidden)) / 8 > (int64_t)UINT32_MAX - 3 * kLay) return ADAGC_ERR_TOO_LARGE;
    return ADAGC_OK;
}
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// What a call needs, in bytes: operands laid out anew; backward: d_g and d_u, rows x ld each, and partial sums of a product.
struct Work {
    Layout  layout;
    int64_t x, weight;                             // weight: of each
    int64_t along;                                 // partial sums of the projections
    int64_t ld, rows, gradients, partial;          // partial: of them and of the products
    int64_t forward() const { return x + 2 * weight + along; }
    int64_t backward() const { return 2 * gradients + partial + x + 2 * weight; }
};
Work work_of(int64_t rows, int64_t dim, int64_t hidden, int32_t dtype, bool backward)
{
    Work w{};
    w.layout = layout_of(rows, hidden, dim, dtype, backward);
    w.ld = (hidden + 63) / 64 * 64;
    // d_g and d_u in parts are for the rings alone, which their rows are too far apart for
    if (backward && w.layout.parts > 1 && w.ld >= kFarAlong) w.layout = Layout{false, 1, 1, w.layout.ld};
    if (w.layout.anew) {
        w.x = w.layout.bytes(rows);
        w.weight = w.layout.bytes(hidden);
    }
    const bool parts = w.layout.parts > 1;
    w.rows = parts ? Layout::rows_of(rows) : rows;
    w.gradients = up16(w.rows * w.ld * (parts ? 2 * kParts : dtype_size(dtype)));
    const int32_t type = w.layout.anew ? ADAGC_BF16 : dtype;
    const int64_t columns = w.layout.anew ? (dim + 7) / 8 * 8 : dim;
    const int64_t k = w.layout.anew ? w.layout.ld : dim;
    for (const bool aligned : {false, true})
        if (!always_thin(rows, dtype)) w.along = std::max(w.along, along_plan(rows, 2 * hidden, k, w.layout.segments, type, aligned, k, k).workspace());
    w.partial = w.along;
    for (const bool aligned : {false, true})
        w.partial = std::max({w.partial, plain_plan((hidden + 7) / 8 * 8, columns, w.rows, type, true, w.ld, columns, w.layout.segments, 2, aligned).workspace(),
                              plain_plan(rows, columns, parts ? w.ld : hidden, type, false, w.ld, columns, 2 * w.layout.segments, 1, aligned).workspace()});
    return w;
}

int launched() { return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP; }

// Lays x and both weights out anew, if the call does that.
template <class T>
int lay_operands(const Work& w, AlongArgs* p, uint8_t* space, hipStream_t s)
{
    p->segments = w.layout.segments;
    if (!w.layout.anew || p->m == 0) return ADAGC_OK;
    const LaySource sources[3] = {{p->x[0], p->ld_x[0], p->n, space + w.x}, {p->x[1], p->ld_x[1], p->n, space + w.x + w.weight}, {p->y, p->ld_y, p->m, space}};
    if (const int rc = lay<T>(sources, 3, p->k, w.layout, s)) return rc;
    p->y = space;
    p->x[0] = space + w.x;
    p->x[1] = space + w.x + w.weight;
    p->ld_y = p->ld_x[0] = p->ld_x[1] = p->k = w.layout.ld;
    p->part_y = w.layout.part(p->m);
    p->part_x = w.layout.part(p->n);
    return ADAGC_OK;
}

// T: of the operands, as they are or laid out anew; O: of the call's data
template <class T, class O, bool BACKWARD>
int projections(GatedArgs a, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    if constexpr (sizeof(T) == sizeof(O)) {
        if (thin(a.p, dtype)) {
            const dim3 blocks((uint32_t)std::min<int64_t>((a.p.n + kThinColumns / 2 - 1) / (kThinColumns / 2), kThinGrid));
            for_rows(a.p.m, [&](auto TM) { thin_gated_kernel<T, decltype(TM)::value, BACKWARD><<<blocks, dim3(kThinThreads), 0, s>>>(a); });
            return launched();
        }
    }
    const bool aligned = rows_aligned(a.p.y, a.p.ld_y, dtype) && rows_aligned(a.p.x[0], a.p.ld_x[0], dtype) && rows_aligned(a.p.x[1], a.p.ld_x[1], dtype);
    const AlongPlan p = along_plan(a.p.m, 2 * a.p.n, a.p.k, a.p.segments, dtype, aligned, a.p.ld_y, std::max(a.p.ld_x[0], a.p.ld_x[1]));
    a.p.tiles_m = (int32_t)p.tiles_m;
    a.p.tiles_n = (int32_t)p.tiles_n;
    a.p.split = (int32_t)p.split;
    const dim3 grid((uint32_t)(p.tiles_m * p.tiles_n));
    if constexpr (sizeof(T) == 2) {
        constexpr int kOf = BACKWARD && sizeof(O) == 4 ? kParts : 1;       // (fp32 data is laid out in parts)
        if (p.size == 256) {
            if constexpr (sizeof(O) == 2)
                gated_kernel<Large, T, O, BACKWARD, 1, Sum::kWhole><<<dim3(grid_of<Large>(p.tiles_m * p.tiles_n)), dim3(Large::kThreads), 0, s>>>(a);
        } else if (p.direct && p.split > 1) {
            launch_parts<Small, T, true>(a.p, s);
            gated_kernel<Small, T, O, BACKWARD, kOf, Sum::kJoined><<<grid, dim3(Small::kThreads), 0, s>>>(a);
        } else if (p.direct) {
            gated_kernel<Small, T, O, BACKWARD, kOf, Sum::kWhole><<<dim3(grid_of<Small>(p.tiles_m * p.tiles_n)), dim3(Small::kThreads), 0, s>>>(a);
        }
    }
    if constexpr (sizeof(T) == sizeof(O)) {
        if (!p.direct)
            staged_tile<T>(p, [&](auto tile) {
                using S = decltype(tile);
                if (p.split > 1) {
                    launch_parts<S, T, true>(a.p, s);
                    gated_kernel<S, T, O, BACKWARD, 1, Sum::kJoined><<<grid, dim3(S::kThreads), 0, s>>>(a);
                } else {
                    gated_kernel<S, T, O, BACKWARD, 1, Sum::kWhole><<<grid, dim3(S::kThreads), 0, s>>>(a);
                }
            });
    }
    return launched();
}

template <class T>
int forward(const Work& w, GatedArgs a, uint8_t* workspace, hipStream_t s)
{
    if (const int rc = lay_operands<T>(w, &a.p, workspace, s)) return rc;
    a.p.partial = reinterpret_cast<float*>(workspace + w.x + 2 * w.weight);
    return w.layout.anew ? projections<uint16_t, T, false>(a, s) : projections<T, T, false>(a, s);
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
int backward(const Work& w, Backward b, uint8_t* workspace, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    const int64_t rows = b.g.p.m, hidden = b.g.p.n, dim = b.g.p.k;
    const bool anew = w.layout.anew, parts = w.layout.parts > 1;
    uint8_t *d_gate = workspace, *d_up = workspace + w.gradients;
    const int64_t part = w.rows * w.ld;
    if (const int rc = lay_operands<T>(w, &b.g.p, workspace + 2 * w.gradients + w.partial, s)) return rc;
    const AlongArgs& p = b.g.p;
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
        k.ld_d = w.ld;
        k.part = part;
        k.out = b.g.out;
        k.ld_out = b.g.ld_out;
        k.rows = rows;
        k.cols = hidden;
        k.vectors = ((parts ? w.ld : hidden) * (int64_t)sizeof(T) + 15) / 16;
        k.all = w.rows * k.vectors;
        const dim3 grid((uint32_t)((k.all + kKept - 1) / kKept));
        if constexpr (sizeof(T) == 4) {
            if (parts) kept_kernel<T, kParts><<<grid, dim3(kKept), 0, s>>>(k);
        }
        if (!parts) kept_kernel<T, 1><<<grid, dim3(kKept), 0, s>>>(k);
        if (const int rc = launched()) return rc;
    } else if (rows > 0) {
        b.g.gate = d_gate;
        b.g.up = d_up;
        b.g.ld_gate = b.g.ld_up = w.ld;
        b.g.part = part;
        b.g.rows = w.rows;
        b.g.p.partial = reinterpret_cast<float*>(workspace + 2 * w.gradients);
        if (const int rc = anew ? projections<uint16_t, T, true>(b.g, s) : projections<T, T, true>(b.g, s)) return rc;
    }
    PlainArgs both{};
    both.y[0] = d_gate;
    both.y[1] = d_up;
    both.ld_y = w.ld;
    both.part_y = part;
    both.segments = w.layout.segments;
    both.n = dim;
    both.n_readable = anew ? (dim + 7) / 8 * 8 : dim;
    both.workspace = reinterpret_cast<float*>(workspace + 2 * w.gradients);
    both.factor = 1.f;
    if (b.d_w_gate) {
        PlainArgs a = both;
        a.x[0] = a.x[1] = p.y;
        a.ld_x[0] = a.ld_x[1] = p.ld_y;
        a.part_x = p.part_y;
        a.out[0] = b.d_w_gate;
        a.out[1] = b.d_w_up;
        a.ld_out[0] = a.ld_add[0] = b.ld_d_w_gate;
        a.ld_out[1] = a.ld_add[1] = b.ld_d_w_up;
        if (b.accumulate) {
            a.add[0] = b.d_w_gate;
            a.add[1] = b.d_w_up;
        }
        a.m = hidden;
        a.m_readable = (hidden + 7) / 8 * 8;
        a.k = w.rows;
        a.pairs = 1;
        a.products = 2;
        a.out_bf16 = a.add_bf16 = b.weight_dtype == ADAGC_BF16;
        if (const int rc = anew ? run_plain<uint16_t, true>(a, s) : run_plain<T, true>(a, s)) return rc;
    }
    if (b.d_x && rows > 0) {
        PlainArgs a = both;
        a.x[0] = p.x[0];
        a.x[1] = p.x[1];
        a.ld_x[0] = p.ld_x[0];
        a.ld_x[1] = p.ld_x[1];
        a.part_x = p.part_x;
        a.out[0] = b.d_x;
        a.ld_out[0] = b.ld_d_x;
        a.m = a.m_readable = rows;
        a.k = parts ? w.ld : hidden;
        a.pairs = 2;
        a.products = 1;
        a.out_bf16 = dtype == ADAGC_BF16;
        if (const int rc = anew ? run_plain<uint16_t, false>(a, s) : run_plain<T, false>(a, s)) return rc;
    }
    return ADAGC_OK;
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int64_t adagc_gated_linear_workspace_bytes(int64_t rows, int64_t dim, int64_t hidden, int32_t dtype)
{
    if (const int rc = check(rows, dim, hidden, dtype)) return rc;
    return work_of(rows, dim, hidden, dtype, false).forward();
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
    const Work w = work_of(rows, dim, hidden, dtype, false);
    const int64_t need = w.forward();
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return ADAGC_ERR_INVALID_ARG;
    GatedArgs a{};
    a.p = {x, {w_gate, w_up}, ld_x, {ld_w_gate, ld_w_up}, rows, hidden, dim, 0, 0, 1, 0, 0, nullptr, 1};
    a.out = out;
    a.ld_out = ld_out;
    a.gate = gate;
    a.up = up;
    a.ld_gate = ld_gate;
    a.ld_up = ld_up;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    return dtype == ADAGC_F32 ? forward<float>(w, a, ws, s) : forward<uint16_t>(w, a, ws, s);
}

extern "C" int64_t adagc_gated_linear_backward_workspace_bytes(int64_t rows, int64_t dim, int64_t hidden, int32_t dtype)
{
    if (const int rc = check(rows, dim, hidden, dtype)) return rc;
    return work_of(rows, dim, hidden, dtype, true).backward();
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
    const Work w = work_of(rows, dim, hidden, dtype, true);
    const int64_t need = w.backward();
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return ADAGC_ERR_INVALID_ARG;
    Backward b{};
    b.g.p = {x, {w_gate, w_up}, ld_x, {ld_w_gate, ld_w_up}, rows, hidden, dim, 0, 0, 1, 0, 0, nullptr, 1};
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
    return dtype == ADAGC_F32 ? backward<float>(w, b, ws, s) : backward<uint16_t>(w, b, ws, s);
}
