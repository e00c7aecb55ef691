// Log-probabilities of given tokens straight from the head's input x and weights W, and their gradients, without the logits, for gfx950:
//     z = x W^T,  M = max_j z_j,  L = ln sum_j exp(s (z_j - M)),  log p(t) = s (z_t - M) - L;
//     dz_j = d (1[j = t] - p_j),  dx = s dz W,  dW = s dz^T x.
//
// Forward: the product's tiles stay in registers; of every row a tile leaves its maximum and its sum of exponentials relative to that,
// and the target's logit, and a second kernel joins a row's tiles in order.  Backward: the logits of a piece of the vocabulary again, their
// gradients (bf16 with bf16 operands: they go into the matrix cores as they are) to the workspace, and from there the two products; dx is
// summed over the pieces in fp32.
#include "product_device.h"

namespace adagc {
namespace {

using namespace product;

constexpr float kLog2e = 1.44269504088896340736f;

struct StatsArgs {
    AlongArgs      p;
    const int64_t* targets;        // or NULL
    float          scale;
    float2*        parts;          // [rows][tiles_n]: maximum, sum
    float*         target_logit;   // [rows]
};

// sum of exp(scale (m_i - m) ) s_i for the joint maximum m; a part of -inf has sum 0
__device__ __forceinline__ float rescaled(float mi, float si, float m, float c) { return mi == -__builtin_inff() ? 0.f : si * __builtin_amdgcn_exp2f((mi - m) * c); }

template <class S, class T>
__global__ __launch_bounds__(S::kThreads, 2) void stats_kernel(const StatsArgs a)
{
    __shared__ __attribute__((aligned(512))) uint8_t lds[S::kLds];
    const float c = a.scale * kLog2e;
    int target[S::kTM];            // its column from the lane's first one, if in the wave's columns
    auto before = [&](int64_t m0, int64_t n0) __attribute__((always_inline)) {
        const LanePlace<S> at;
#pragma unroll
        for (int m = 0; m < S::kTM; ++m) {
            const int64_t row = m0 + at.row + m * 16;
            target[m] = -1;
            if (a.targets && row < a.p.m) {
                const int64_t t = a.targets[row];
                if (t >= n0 + at.col && t < min(n0 + at.col + S::kTN * 16, a.p.n)) target[m] = (int)(t - n0 - at.col);
            }
        }
        settle_now(target);
    };
    along_tiles<S, T, false>(a.p, lds, before, [&](Sums<S>& acc, int64_t m0, int64_t n0, uint8_t* scratch) __attribute__((always_inline)) {
        const LanePlace<S> at;
        const int tid = thread_anew(), lane = tid & 63, wave = tid >> 6;
        if (n0 + S::BN > a.p.n) {
            each_piece<S>(acc, [&](int m, int n, int, int col, const f32x4_p&) __attribute__((always_inline)) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (n0 + col + r >= a.p.n) acc[m][n][r] = -__builtin_inff();
            });
        }
        float2* shared = reinterpret_cast<float2*>(scratch);       // [BM][kWN]
#pragma unroll
        for (int m = 0; m < S::kTM; ++m) {
            float most = -__builtin_inff();
#pragma unroll
            for (int n = 0; n < S::kTN; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) most = maximum(most, acc[m][n][r]);
            most = maximum(most, __shfl_xor(most, 16));
            most = maximum(most, __shfl_xor(most, 32));
            // relative to from, most c as an fp32 number: an exponent is rounded once, and the sum then put right for what that number is off by
            const float from = most == -__builtin_inff() ? 0.f : most * c;
            float sum = 0.f;
            if (__builtin_fabsf(from) < 0x1p20f) {         // (then it is off by less than 2^-4)
#pragma unroll
                for (int n = 0; n < S::kTN; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[m][n][r], c, -from));
                if (from != 0.f) sum *= __builtin_amdgcn_exp2f(-__builtin_fmaf(most, c, -from));
            } else {
#pragma unroll
                for (int n = 0; n < S::kTN; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f((acc[m][n][r] - most) * c);
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            const int row = at.row + m * 16;
            if (lane < 16) shared[row * S::kWN + wave % S::kWN] = float2{most, sum};
            if (target[m] >= 0) {
#pragma unroll
                for (int n = 0; n < S::kTN; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (target[m] == n * 16 + r) a.target_logit[m0 + row] = acc[m][n][r];
            }
        }
        meet_keeping_loads();
        if (tid < S::BM && m0 + tid < a.p.m) {
            float2 part[S::kWN];
            float most = -__builtin_inff(), sum = 0.f;
#pragma unroll
            for (int w = 0; w < S::kWN; ++w) {
                part[w] = shared[tid * S::kWN + w];
                most = maximum(most, part[w].x);
            }
#pragma unroll
            for (int w = 0; w < S::kWN; ++w) sum += rescaled(part[w].x, part[w].y, most, c);
            a.parts[(m0 + tid) * a.p.tiles_n + n0 / S::BN] = float2{most, sum};
        }
    });
}

// Few rows: a thread for each value.
template <class T, int TM>
__global__ __launch_bounds__(kThinThreads, 4) void thin_stats_kernel(const StatsArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[kThinLds<TM>];
    const int own_row = threadIdx.x / kThinColumns;
    const int64_t target = a.targets && own_row < a.p.m ? a.targets[own_row] : -1;
    const float c = a.scale * kLog2e;
    thin_tiles<T, TM, false>(a.p, lds, [](int64_t) {}, [&](int64_t n0, int row, int at, float z, float) __attribute__((always_inline)) {
        if (row >= a.p.m) return;                          // (whole halves of waves)
        const int64_t col = n0 + at;
        if (col >= a.p.n) z = -__builtin_inff();
        float most = z;
#pragma unroll
        for (int d = 1; d < kThinColumns; d *= 2) most = maximum(most, __shfl_xor(most, d));
        float sum = __builtin_amdgcn_exp2f((z - (most == -__builtin_inff() ? 0.f : most)) * c);
#pragma unroll
        for (int d = 1; d < kThinColumns; d *= 2) sum += __shfl_xor(sum, d);
        if (at == 0) a.parts[row * (int64_t)a.p.tiles_n + n0 / kThinColumns] = float2{most, sum};
        if (target == col && col < a.p.n) a.target_logit[row] = z;
    });
}

struct JoinArgs {
    const float2*  parts;
    const float*   target_logit;
    const int64_t* targets;
    float          scale;
    int64_t        vocab;
    int32_t        tiles;
    float*         logprob;        // or NULL
    float2*        stats;          // or NULL
};

// A row's tiles: a workgroup for each row.
constexpr int kJoin = 256;
__global__ __launch_bounds__(kJoin) void join_kernel(const JoinArgs a)
{
    __shared__ float most_of[kJoin / 64], sum_of[kJoin / 64];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const float2* parts = a.parts + row * a.tiles;
    const float c = a.scale * kLog2e;
    float most = -__builtin_inff(), sum = 0.f;
    for (int i = tid; i < a.tiles; i += kJoin) most = maximum(most, parts[i].x);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = maximum(most, __shfl_xor(most, d));
    if (tid % 64 == 0) most_of[tid / 64] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoin / 64; ++w) most = maximum(most, most_of[w]);
    for (int i = tid; i < a.tiles; i += kJoin) sum += rescaled(parts[i].x, parts[i].y, most, c);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (tid % 64 == 0) sum_of[tid / 64] = sum;
    __syncthreads();
    if (tid) return;
    sum = 0.f;
    for (int w = 0; w < kJoin / 64; ++w) sum += sum_of[w];
    const float log_sum = most == -__builtin_inff() ? 0.f : logf(sum);
    if (a.stats) a.stats[row] = float2{most, log_sum};
    if (a.logprob) {
        const int64_t t = a.targets[row];
        float logp = 0.f;
        if (t >= 0 && t < a.vocab) {
            const float z = a.target_logit[row];
            // halves, whose difference does not leave fp32's range
            logp = most == -__builtin_inff() ? most : (0.5f * z - 0.5f * most) * a.scale * 2.f - log_sum;
        }
        a.logprob[row] = logp;
    }
}

struct GradArgs {
    AlongArgs      p;              // n: of the piece
    const int64_t* targets;
    const float*   stats;
    const float*   d_logprob;
    float          scale;
    int64_t        first;          // of the vocabulary
    int64_t        vocab;
    void*          d_logits;       // T[rows][ld]
    int64_t        ld;
};

template <class S, class T>
__global__ __launch_bounds__(S::kThreads, 2) void grad_kernel(const GradArgs a)
{
    __shared__ __attribute__((aligned(512))) uint8_t lds[S::kLds];
    const float c = a.scale * kLog2e;
    // of a row: the target's column from the lane's first one (or none of them), M, L in powers of two, d (0: all of the row's gradients are 0)
    int target[S::kTM];
    float most[S::kTM], log2_sum[S::kTM], d[S::kTM];
    auto before = [&](int64_t m0, int64_t n0) __attribute__((always_inline)) {
        const LanePlace<S> at;
#pragma unroll
        for (int m = 0; m < S::kTM; ++m) {
            const int64_t row = min(m0 + at.row + m * 16, a.p.m - 1), t = a.targets[row];
            most[m] = a.stats[2 * row];
            log2_sum[m] = a.stats[2 * row + 1] * kLog2e;
            d[m] = a.d_logprob[row];
            const int64_t from = t - a.first - n0 - at.col;
            target[m] = from >= 0 && from < S::kTN * 16 ? (int)from : -1;
            if (t < 0 || t >= a.vocab || most[m] == -__builtin_inff()) d[m] = 0.f;
        }
        settle_now(target);
        settle_now(most);
        settle_now(log2_sum);
        settle_now(d);
    };
    along_tiles<S, T, false>(a.p, lds, before, [&](Sums<S>& acc, int64_t m0, int64_t n0, uint8_t*) __attribute__((always_inline)) {
        const LanePlace<S> at;
#pragma unroll
        for (int m = 0; m < S::kTM; ++m) {
            const int64_t row = m0 + at.row + m * 16;
            if (row >= a.p.m) continue;
            T* to = static_cast<T*>(a.d_logits) + row * a.ld + n0 + at.col;
#pragma unroll
            for (int n = 0; n < S::kTN; ++n) {
                f32x4_p v;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __builtin_amdgcn_exp2f((acc[m][n][r] - most[m]) * c - log2_sum[m]);
                    v[r] = d[m] == 0.f ? 0.f : ((target[m] == n * 16 + r ? 1.f : 0.f) - p) * d[m];
                }
                store4(to + n * 16, v);            // (columns past the piece's end are within ld, and not read)
            }
        }
    });
}

template <class T, int TM>
__global__ __launch_bounds__(kThinThreads, 4) void thin_grad_kernel(const GradArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[kThinLds<TM>];
    const int64_t own_row = min((int64_t)threadIdx.x / kThinColumns, a.p.m - 1), target = a.targets[own_row];
    const float most = a.stats[2 * own_row], log2_sum = a.stats[2 * own_row + 1] * kLog2e, c = a.scale * kLog2e;
    const float d = target < 0 || target >= a.vocab || most == -__builtin_inff() ? 0.f : a.d_logprob[own_row];
    thin_tiles<T, TM, false>(a.p, lds, [](int64_t) {}, [&](int64_t n0, int row, int at, float z, float) __attribute__((always_inline)) {
        if (row >= a.p.m) return;
        const int64_t col = n0 + at;                       // (columns past the piece's end are within ld, and not read)
        const float p = __builtin_amdgcn_exp2f((z - most) * c - log2_sum);
        const float v = d == 0.f ? 0.f : ((target - a.first == col ? 1.f : 0.f) - p) * d;
        T* to = static_cast<T*>(a.d_logits) + row * a.ld + col;
        if constexpr (sizeof(T) == 4) *to = v;
        else *to = __builtin_bit_cast(uint16_t, (__bf16)v);
    });
}

int check(int64_t rows, int64_t vocab, int64_t dim, int32_t dtype)
{
    if (rows < 0 || vocab < 1 || dim < 1 || !known_dtype(dtype)) return ADAGC_ERR_INVALID_ARG;
    if (rows > (1 << 24) - 1 || vocab > kMaxCols || dim > kMaxCols) return ADAGC_ERR_TOO_LARGE;
    return ADAGC_OK;
}
bool scale_in_range(float scale) { return scale >= 0x1p-100f && scale <= 0x1p100f; }
int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// at most: of the smallest tile that a call of this size may take
int64_t parts_of_row(int64_t rows, int64_t vocab)
{
    const int64_t tile = rows <= kThinRows ? kThinColumns : ((rows + 127) / 128) * ((vocab + 127) / 128) < 4 * kUnits ? 64 : 128;
    return (vocab + tile - 1) / tile;
}
int64_t forward_workspace(int64_t rows, int64_t vocab)
{
    return up16(rows * parts_of_row(rows, vocab) * 8) + rows * 4;
}

// Pieces of the vocabulary: 2^26 gradients of logits a piece, which the memory-side cache holds as bf16, and 2048 columns at least.
struct Pieces {
    int64_t size, number, ld;
    int64_t d_logits, sums, partial;       // bytes
    int64_t all() const { return d_logits + sums + partial; }
};
Pieces pieces_of(int64_t rows, int64_t vocab, int64_t dim, int32_t dtype)
{
    Pieces p{};
    const int64_t most = std::max<int64_t>(2048, ((int64_t)1 << 26) / std::max<int64_t>(rows, 1) / 256 * 256);
    p.number = (vocab + most - 1) / most;
    p.size = p.number == 1 ? vocab : ((vocab + p.number - 1) / p.number + 255) / 256 * 256;
    p.number = (vocab + p.size - 1) / p.size;
    p.ld = (p.size + 255) / 256 * 256;
    p.d_logits = up16(rows * p.ld * dtype_size(dtype));
    p.sums = p.number > 1 && dtype == ADAGC_BF16 ? up16(rows * dim * 4) : 0;
    for (const int64_t n : {p.size, vocab - (p.number - 1) * p.size})
        for (const bool aligned : {false, true}) {
            const int64_t readable = (n + 7) / 8 * 8;
            p.partial = std::max({p.partial, plain_plan(readable, dim, rows, dtype, true, p.ld, dim, 1, 1, aligned).workspace(),
                                  plain_plan(rows, dim, n, dtype, false, p.ld, dim, 1, 1, aligned).workspace()});
        }
    return p;
}
bool launchable(int64_t rows, int64_t vocab, int64_t dim)
{
    const int64_t tiles = ((rows + 127) / 128) * ((vocab + 127) / 128), weight = ((vocab + 127) / 128) * ((dim + 127) / 128),
                  input = ((rows + 127) / 128) * ((dim + 127) / 128);
    return std::max({tiles, weight, input}) < 1 << 23;
}

AlongArgs along_args(const void* x, int64_t ld_x, const void* weight, int64_t ld_weight, int64_t rows, int64_t vocab, int64_t dim)
{
    AlongArgs p{};
    p.y = x;
    p.ld_y = ld_x;
    p.x[0] = p.x[1] = weight;
    p.ld_x[0] = p.ld_x[1] = ld_weight;
    p.m = rows;
    p.n = vocab;
    p.k = dim;
    return p;
}
AlongPlan plan_of(AlongArgs* p, int32_t dtype)
{
    const AlongPlan plan = along_plan(p->m, p->n, dtype, rows_aligned(p->y, p->ld_y, dtype) && rows_aligned(p->x[0], p->ld_x[0], dtype), p->ld_y, p->ld_x[0]);
    p->tiles_m = (int32_t)plan.tiles_m;
    p->tiles_n = (int32_t)plan.tiles_n;
    return plan;
}

template <class T>
int forward(StatsArgs a, const JoinArgs& join, hipStream_t s)
{
    const AlongPlan p = plan_of(&a.p, sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16);
    const dim3 grid((uint32_t)(p.tiles_m * p.tiles_n));
    const bool few = thin(a.p, sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16);
    if (few) {
        a.p.tiles_n = (int32_t)((a.p.n + kThinColumns - 1) / kThinColumns);
        for_rows(a.p.m, [&](auto TM) { thin_stats_kernel<T, decltype(TM)::value><<<dim3(std::min(a.p.tiles_n, kThinGrid)), dim3(kThinThreads), 0, s>>>(a); });
    } else if constexpr (sizeof(T) == 2) {
        if (p.size == 256) stats_kernel<Large, T><<<dim3(grid_of<Large>(p.tiles_m * p.tiles_n)), dim3(Large::kThreads), 0, s>>>(a);
        else if (p.direct) stats_kernel<Small, T><<<grid, dim3(Small::kThreads), 0, s>>>(a);
    }
    if (!few && !p.direct) {
        if constexpr (sizeof(T) == 4) {
            if (p.size == 64) stats_kernel<Smallest, T><<<grid, dim3(Smallest::kThreads), 0, s>>>(a);
        }
        if (p.size == 128) stats_kernel<Staged<T>, T><<<grid, dim3(Staged<T>::kThreads), 0, s>>>(a);
    }
    JoinArgs j = join;
    j.tiles = a.p.tiles_n;
    join_kernel<<<dim3((uint32_t)a.p.m), dim3(kJoin), 0, s>>>(j);
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}

template <class T>
int gradient(GradArgs a, hipStream_t s)
{
    const AlongPlan p = plan_of(&a.p, sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16);
    const dim3 grid((uint32_t)(p.tiles_m * p.tiles_n));
    const bool few = thin(a.p, sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16);
    if (few) {
        const dim3 blocks((uint32_t)std::min<int64_t>((a.p.n + kThinColumns - 1) / kThinColumns, kThinGrid));
        for_rows(a.p.m, [&](auto TM) { thin_grad_kernel<T, decltype(TM)::value><<<blocks, dim3(kThinThreads), 0, s>>>(a); });
    } else if constexpr (sizeof(T) == 2) {
        if (p.size == 256) grad_kernel<Large, T><<<dim3(grid_of<Large>(p.tiles_m * p.tiles_n)), dim3(Large::kThreads), 0, s>>>(a);
        else if (p.direct) grad_kernel<Small, T><<<grid, dim3(Small::kThreads), 0, s>>>(a);
    }
    if (!few && !p.direct) {
        if constexpr (sizeof(T) == 4) {
            if (p.size == 64) grad_kernel<Smallest, T><<<grid, dim3(Smallest::kThreads), 0, s>>>(a);
        }
        if (p.size == 128) grad_kernel<Staged<T>, T><<<grid, dim3(Staged<T>::kThreads), 0, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}

struct Outputs {
    void*   d_x;
    int64_t ld_d_x;
    void*   d_weight;
    int32_t weight_dtype;
    int64_t ld_d_weight;
    int32_t accumulate;
};

template <class T>
int backward(const GradArgs& all, const Outputs& o, uint8_t* workspace, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    const int64_t rows = all.p.m, vocab = all.vocab, dim = all.p.k;
    const Pieces pieces = pieces_of(rows, vocab, dim, dtype);
    float* sums = reinterpret_cast<float*>(workspace + pieces.d_logits);
    float* partial = reinterpret_cast<float*>(workspace + pieces.d_logits + pieces.sums);
    const int w_size = dtype_size(o.weight_dtype);
    for (int64_t i = 0; i < pieces.number; ++i) {
        const int64_t first = i * pieces.size, n = std::min(pieces.size, vocab - first);
        const T* weight = static_cast<const T*>(all.p.x[0]) + first * all.p.ld_x[0];
        if (rows > 0) {
            GradArgs a = all;
            a.p.x[0] = a.p.x[1] = weight;
            a.p.n = n;
            a.first = first;
            a.d_logits = workspace;
            a.ld = pieces.ld;
            if (const int rc = gradient<T>(a, s)) return rc;
        }
        if (o.d_weight) {
            PlainArgs w{};
            w.y[0] = workspace;
            w.ld_y = pieces.ld;
            w.x[0] = all.p.y;
            w.ld_x[0] = all.p.ld_y;
            w.out[0] = static_cast<uint8_t*>(o.d_weight) + first * o.ld_d_weight * w_size;
            w.ld_out[0] = o.ld_d_weight;
            w.add[0] = o.accumulate ? w.out[0] : nullptr;
            w.ld_add[0] = o.ld_d_weight;
            w.m = n;
            w.m_readable = (n + 7) / 8 * 8;
            w.n = dim;
            w.k = rows;
            w.workspace = partial;
            w.factor = all.scale;
            w.pairs = w.products = 1;
            w.out_bf16 = w.add_bf16 = o.weight_dtype == ADAGC_BF16;
            if (const int rc = run_plain<T, true>(w, s)) return rc;
        }
        if (o.d_x && rows > 0) {
            const bool last = i == pieces.number - 1;
            PlainArgs x{};
            x.y[0] = workspace;
            x.ld_y = pieces.ld;
            x.x[0] = weight;
            x.ld_x[0] = all.p.ld_x[0];
            const bool direct = last || dtype == ADAGC_F32;
            x.out[0] = direct ? o.d_x : sums;
            x.ld_out[0] = direct ? o.ld_d_x : dim;
            x.out_bf16 = direct && dtype == ADAGC_BF16;
            x.add[0] = i == 0 ? nullptr : dtype == ADAGC_F32 ? o.d_x : sums;
            x.ld_add[0] = dtype == ADAGC_F32 ? o.ld_d_x : dim;
            x.m = x.m_readable = rows;
            x.n = dim;
            x.k = n;
            x.workspace = partial;
            x.factor = all.scale;
            x.pairs = x.products = 1;
            if (const int rc = run_plain<T, false>(x, s)) return rc;
        }
    }
    return ADAGC_OK;
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int64_t adagc_linear_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int64_t dim, int32_t dtype)
{
    if (const int rc = check(rows, vocab, dim, dtype)) return rc;
    return launchable(rows, vocab, 1) ? forward_workspace(rows, vocab) : (int64_t)ADAGC_ERR_TOO_LARGE;
}

extern "C" int adagc_linear_logprobs(const void* x, int64_t ld_x, const void* weight, int64_t ld_weight, int32_t dtype, int64_t rows, int64_t vocab,
                                     int64_t dim, const int64_t* targets, float scale, float* logprob, float* stats, void* workspace,
                                     int64_t workspace_bytes, void* stream)
{
    if (const int rc = check(rows, vocab, dim, dtype)) return rc;
    const int size = dtype_size(dtype);
    if (!scale_in_range(scale) || workspace_bytes < 0 || (rows > 0 && !logprob && !stats)) return ADAGC_ERR_INVALID_ARG;
    if (rows == 0) return ADAGC_OK;
    if (!x || !weight || ld_x < dim || ld_weight < dim || misaligned(x, size) || misaligned(weight, size) || (logprob && !targets) ||
        misaligned(targets, 8) || misaligned(logprob, 4) || misaligned(stats, 4))
        return ADAGC_ERR_INVALID_ARG;
    if (ld_x > kMaxLd || ld_weight > kMaxLd || !launchable(rows, vocab, 1)) return ADAGC_ERR_TOO_LARGE;
    if (!workspace || workspace_bytes < forward_workspace(rows, vocab) || misaligned(workspace, 16)) return ADAGC_ERR_INVALID_ARG;
    StatsArgs a{};
    a.p = along_args(x, ld_x, weight, ld_weight, rows, vocab, dim);
    a.targets = logprob ? targets : nullptr;
    a.scale = scale;
    a.parts = static_cast<float2*>(workspace);
    a.target_logit = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + up16(rows * parts_of_row(rows, vocab) * 8));
    JoinArgs j{};
    j.parts = a.parts;
    j.target_logit = a.target_logit;
    j.targets = targets;
    j.scale = scale;
    j.vocab = vocab;
    j.logprob = logprob;
    j.stats = reinterpret_cast<float2*>(stats);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == ADAGC_F32 ? forward<float>(a, j, s) : forward<uint16_t>(a, j, s);
}

extern "C" int64_t adagc_linear_logprobs_backward_workspace_bytes(int64_t rows, int64_t vocab, int64_t dim, int32_t dtype)
{
    if (const int rc = check(rows, vocab, dim, dtype)) return rc;
    return launchable(rows, vocab, dim) ? pieces_of(rows, vocab, dim, dtype).all() : (int64_t)ADAGC_ERR_TOO_LARGE;
}

extern "C" int adagc_linear_logprobs_backward(const void* x, int64_t ld_x, const void* weight, int64_t ld_weight, int32_t dtype, int64_t rows,
                                              int64_t vocab, int64_t dim, const int64_t* targets, float scale, const float* stats,
                                              const float* d_logprob, void* d_x, int64_t ld_d_x, void* d_weight, int32_t weight_dtype,
                                              int64_t ld_d_weight, int32_t accumulate, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (const int rc = check(rows, vocab, dim, dtype)) return rc;
    const int size = dtype_size(dtype);
    if (!scale_in_range(scale) || workspace_bytes < 0 || (rows > 0 && !d_x && !d_weight) || accumulate < 0 || accumulate > 1) return ADAGC_ERR_INVALID_ARG;
    if (d_weight && (!known_dtype(weight_dtype) || ld_d_weight < dim || misaligned(d_weight, dtype_size(weight_dtype)))) return ADAGC_ERR_INVALID_ARG;
    if (rows > 0 && (!x || !weight || ld_x < dim || ld_weight < dim || misaligned(x, size) || misaligned(weight, size) || !targets || !stats ||
                     !d_logprob || misaligned(targets, 8) || misaligned(stats, 4) || misaligned(d_logprob, 4) ||
                     (d_x && (ld_d_x < dim || misaligned(d_x, size)))))
        return ADAGC_ERR_INVALID_ARG;
    if ((d_weight && ld_d_weight > kMaxLd) || (rows > 0 && (ld_x > kMaxLd || ld_weight > kMaxLd || (d_x && ld_d_x > kMaxLd))) || !launchable(rows, vocab, dim))
        return ADAGC_ERR_TOO_LARGE;
    const int64_t need = pieces_of(rows, vocab, dim, dtype).all();
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return ADAGC_ERR_INVALID_ARG;
    GradArgs a{};
    a.p = along_args(x, ld_x, weight, ld_weight, rows, vocab, dim);
    a.targets = targets;
    a.stats = stats;
    a.d_logprob = d_logprob;
    a.scale = scale;
    a.vocab = vocab;
    const Outputs o = {d_x, ld_d_x, d_weight, weight_dtype, ld_d_weight, accumulate};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    return dtype == ADAGC_F32 ? backward<float>(a, o, ws, s) : backward<uint16_t>(a, o, ws, s);
}
