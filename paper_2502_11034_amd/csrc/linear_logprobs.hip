// Log-probabilities of given tokens straight from the head's input x and weights W, and their gradients, without the logits, for gfx950:
//     z = x W^T,  M = max_j z_j,  L = ln sum_j exp(s (z_j - M)),  log p(t) = s (z_t - M) - L;
//     dz_j = d (1[j = t] - p_j),  dx = s dz W,  dW = s dz^T x.
//
// Forward: the product's tiles stay in registers; of every row a tile leaves its maximum and its sum of exponentials relative to that,
// and the target's logit, and a second kernel joins a row's tiles in order.  Backward: the logits of a piece of the vocabulary again, their
// gradients (bf16 with bf16 operands: they go into the matrix cores as they are, and a second part of them would double the time of both products)
// to the workspace, and from there the two products; dx is summed over the pieces in fp32.
//
// What bounds it: the matrix cores, and of short sums what a tile takes beside them, 3 - 4 us of a 256-tile's exponentials among it.  4096 rows,
// 128256 from 4096, bf16: forward 3050 - 3240 us and 10 for joining; a piece of 16384 columns 399 - 429 for its gradients, 404 - 432 for the weight's,
// 382 - 406 for x's.  1024 rows, 50257 from 768, forward: 77 + 11 + 5.  One row, 128256 from 4096: 179 + 5, memory (5.9 TB/s).
#include "product_device.h"

namespace adagc {
namespace {

using namespace product;

constexpr float kLog2e = 1.44269504088896340736f;

struct StatsArgs {
    AlongArgs      p;              // n: of a piece of the vocabulary
    const int64_t* targets;        // or NULL
    float          scale;
    float2*        parts;          // [rows][pitch]: maximum, sum of each tile
    int64_t        pitch;
    int64_t        first;          // of the vocabulary
    float*         target_logit;   // [rows]
};

// sum of exp(scale (m_i - m) ) s_i for the joint maximum m; a part of -inf has sum 0
__device__ __forceinline__ float rescaled(float mi, float si, float m, float c) { return mi == -__builtin_inff() ? 0.f : si * __builtin_amdgcn_exp2f((mi - m) * c); }

template <class S, class T, Sum SUM>
__global__ __launch_bounds__(S::kThreads, 2) void stats_kernel(const StatsArgs a)
{
    __shared__ __attribute__((aligned(512))) uint8_t lds[S::kLds];
    const float c = a.scale * kLog2e;
    along_tiles<S, T, false, SUM>(a.p, lds, [](int64_t, int64_t) {}, [&](Sums<S>& acc, int64_t m0, int64_t n0, uint8_t* scratch) __attribute__((always_inline)) {
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
        }
        // the targets last: their loads come after the next tile's in the order that loads are waited for in
        if (a.targets) {
            int target[S::kTM];            // the column from the lane's first one, if in the wave's columns
#pragma unroll
            for (int m = 0; m < S::kTM; ++m) {
                const int64_t t = a.targets[min(m0 + at.row + m * 16, a.p.m - 1)] - a.first;
                target[m] = t >= n0 + at.col && t < min(n0 + at.col + S::kTN * 16, a.p.n) && m0 + at.row + m * 16 < a.p.m ? (int)(t - n0 - at.col) : -1;
            }
#pragma unroll
            for (int m = 0; m < S::kTM; ++m)
                if (target[m] >= 0) {
#pragma unroll
                    for (int n = 0; n < S::kTN; ++n)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (target[m] == n * 16 + r) a.target_logit[m0 + at.row + m * 16] = acc[m][n][r];
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
            a.parts[(m0 + tid) * a.pitch + n0 / S::BN] = float2{most, sum};
        }
    });
}

// Few rows: a thread for each value; a workgroup leaves one part of each row, of all its columns.
template <class T, int TM>
__global__ __launch_bounds__(kThinThreads, 4) void thin_stats_kernel(const StatsArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[kThinLds<TM>];
    const int own_row = threadIdx.x / kThinColumns;
    const int64_t target = a.targets && own_row < a.p.m ? a.targets[own_row] : -1;
    const float c = a.scale * kLog2e;
    float most_yet = -__builtin_inff(), sum_yet = 0.f;
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
        const float both = maximum(most_yet, most);
        sum_yet = rescaled(most_yet, sum_yet, both, c) + rescaled(most, sum, both, c);
        most_yet = both;
        if (target == col && col < a.p.n) a.target_logit[row] = z;
    });
    if (own_row < a.p.m && threadIdx.x % kThinColumns == 0) a.parts[own_row * a.pitch + blockIdx.x] = float2{most_yet, sum_yet};
}

struct JoinArgs {
    const float2*  parts;
    const float*   target_logit;
    const int64_t* targets;
    float          scale;
    int64_t        vocab;
    int64_t        pitch, tiles;
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
    const float2* parts = a.parts + row * a.pitch;
    const float c = a.scale * kLog2e;
    float most = -__builtin_inff(), sum = 0.f;
    for (int64_t i = tid; i < a.tiles; i += kJoin) most = maximum(most, parts[i].x);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = maximum(most, __shfl_xor(most, d));
    if (tid % 64 == 0) most_of[tid / 64] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoin / 64; ++w) most = maximum(most, most_of[w]);
    for (int64_t i = tid; i < a.tiles; i += kJoin) sum += rescaled(parts[i].x, parts[i].y, most, c);
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
    void*          d_logits;       // T[rows][ld], or kParts of them in bf16
    int64_t        ld;
    int64_t        part, rows;     // in parts: elements from part to part; rows with those filled with zeros
};

// PARTS: 1, or kParts, with zeros in rows past the last one and columns past the piece's end.
template <class S, class T, int PARTS, Sum SUM>
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
    along_tiles<S, T, false, SUM>(a.p, lds, before, [&](Sums<S>& acc, int64_t m0, int64_t n0, uint8_t*) __attribute__((always_inline)) {
        const LanePlace<S> at;
#pragma unroll
        for (int m = 0; m < S::kTM; ++m) {
            const int64_t row = m0 + at.row + m * 16;
            if (row >= (PARTS == 1 ? a.p.m : a.rows)) continue;
            T* to = static_cast<T*>(a.d_logits) + row * a.ld + n0 + at.col;
            auto gradients = [&](int n) __attribute__((always_inline)) {
                f32x4_p v;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float p = __builtin_amdgcn_exp2f((acc[m][n][r] - most[m]) * c - log2_sum[m]);
                    v[r] = d[m] == 0.f ? 0.f : ((target[m] == n * 16 + r ? 1.f : 0.f) - p) * d[m];
                }
                return v;
            };
            if constexpr (PARTS == 1) {
                // (columns past the piece's end are within ld, and not read)
#pragma unroll
                for (int n = 0; n < S::kTN; n += 2) store_blocks(to + n * 16, gradients(n), gradients(n + 1));
            } else {
#pragma unroll
                for (int n = 0; n < S::kTN; ++n) {
                    if (n0 + at.col + n * 16 >= a.ld) continue;
                    f32x4_p v = gradients(n);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (row >= a.p.m || n0 + at.col + n * 16 + r >= a.p.n) v[r] = 0.f;
                    uint32_t bits[kParts][2];
                    split4(v, bits);
#pragma unroll
                    for (int p = 0; p < kParts; ++p) *reinterpret_cast<u32x2_of_bf16*>(to + p * a.part + n * 16) = u32x2_of_bf16{bits[p][0], bits[p][1]};
                }
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

// What a call needs, in bytes, and how it goes through the vocabulary.
//
// The backward pass and operands that are laid out anew go in pieces: 2^26 gradients of logits, which the memory-side cache holds as bf16 (as three
// parts half as many), and as many weights, laid out, at most, or 2048 columns where that is more; up to twice that where fewer would not fill a round
// of the weight's gradient (piece_of).
struct Work {
    Layout  layout;
    int64_t size, number;                          // of a piece, of pieces
    int64_t pitch, parts, targets;                 // forward: tiles of a row at most; their parts, the targets' logits
    int64_t ld, d_logits, sums, partial;           // backward: the gradients of a piece's logits; sums of dx in fp32; partial: sums of a product
    int64_t x, weight;                             // operands laid out
    int64_t forward() const { return parts + targets + x + weight + partial; }
    int64_t backward() const { return d_logits + sums + partial + x + weight; }
};
// Columns of a piece, so many at most: the weight's gradient takes 256-tiles in whole rounds of the compute units where that many fill some, or one
// round where twice as many do.
int64_t piece_of(int64_t vocab, int64_t dim, int64_t most)
{
    if (vocab <= most) return vocab;
    const int64_t wide = (dim + 255) / 256;
    int64_t rounds = most / 256 * wide / kUnits;
    if (rounds == 0) rounds = 2 * most / 256 * wide / kUnits;
    return rounds ? std::min(vocab, rounds * kUnits / wide * 256) : most;
}
// Columns of W whose tiles fill whole rounds; 0: those after them are no smaller tiles.  They are, if those are a round at most: 1024 x 50257 from
// 768, 788 tiles, 95 us, and 78 and 12 with the last five columns of tiles small.
int64_t columns_of_whole_rounds(const AlongPlan& p, int64_t m, int64_t n)
{
    if (p.size < 256) return 0;
    const int64_t columns = p.tiles_m * p.tiles_n / kUnits * kUnits / p.tiles_m * 256;
    return columns < n && (m + 127) / 128 * ((n - columns + 127) / 128) <= kUnits ? columns : 0;
}
// Columns of a piece's gradients that the weight's product may read, n or more.  Parts are multiplied by the small tile's ring alone, which wants a whole
// tile of them: those past a shorter piece's end are 0, to the end of the tile that made them (ld is two tiles at least).
int64_t readable_of(const Layout& l, int64_t n)
{
    const int64_t up = (n + 7) / 8 * 8;
    return l.parts > 1 ? std::max<int64_t>(up, Small::BM) : up;
}
Work work_of(int64_t rows, int64_t vocab, int64_t dim, int32_t dtype, bool backward)
{
    Work w{};
    w.layout = layout_of(rows, vocab, dim, dtype, backward);
    const int64_t cap = (int64_t)1 << (w.layout.parts > 1 ? 25 : 26);
    int64_t most = std::max<int64_t>(2048, cap / std::max<int64_t>(rows, 1) / 256 * 256);
    if (w.layout.anew) most = std::max<int64_t>(2048, std::min(backward ? most : INT64_MAX, cap / w.layout.ld / 256 * 256));
    w.size = backward || w.layout.anew ? piece_of(vocab, dim, most) : vocab;
    w.number = (vocab + w.size - 1) / w.size;
    const int64_t tile = rows <= kThinRows ? kThinColumns : dtype == ADAGC_F32 && !w.layout.anew ? 64 : 128;
    w.pitch = (vocab + tile - 1) / tile + w.number;
    w.parts = up16(rows * w.pitch * 8);
    w.targets = up16(rows * 4);
    w.ld = (w.size + 255) / 256 * 256;
    const int dz_size = w.layout.parts > 1 ? 2 * kParts : dtype_size(dtype);
    w.d_logits = up16((w.layout.parts > 1 ? Layout::rows_of(rows) : rows) * w.ld * dz_size);
    w.sums = w.number > 1 && dtype == ADAGC_BF16 ? up16(rows * dim * 4) : 0;
    if (w.layout.anew) {
        w.x = w.layout.bytes(rows);
        w.weight = w.layout.bytes(w.size);
    }
    const int32_t type = w.layout.anew ? ADAGC_BF16 : dtype;
    const int64_t k_along = w.layout.anew ? w.layout.ld : dim;
    for (const int64_t n : {w.size, vocab - (w.number - 1) * w.size})
        for (const bool aligned : {false, true}) {
            if (always_thin(rows, dtype)) continue;
            const AlongPlan p = along_plan(rows, n, k_along, w.layout.segments, type, aligned, k_along, k_along);
            w.partial = std::max(w.partial, p.workspace());
            if (const int64_t columns = columns_of_whole_rounds(p, rows, n))
                w.partial = std::max(w.partial, along_plan(rows, n - columns, k_along, w.layout.segments, type, aligned, k_along, k_along).workspace());
        }
    if (!backward) return w;
    const int64_t columns = w.layout.anew ? (dim + 7) / 8 * 8 : dim;
    for (const int64_t n : {w.size, vocab - (w.number - 1) * w.size})
        for (const bool aligned : {false, true}) {
            const int64_t readable = readable_of(w.layout, n), k = w.layout.parts > 1 ? Layout::rows_of(rows) : rows;
            w.partial = std::max({w.partial, plain_plan(readable, columns, k, type, true, w.ld, columns, w.layout.segments, 1, aligned).workspace(),
                                  plain_plan(rows, columns, w.layout.parts > 1 ? Layout::rows_of(n) : n, type, false, w.ld, columns, w.layout.segments, 1, aligned).workspace()});
        }
    return w;
}
bool launchable(int64_t rows, int64_t vocab, int64_t dim)
{
    const int64_t tiles = ((rows + 63) / 64) * ((vocab + 63) / 64), weight = ((vocab + 63) / 64) * ((dim + 63) / 64), input = ((rows + 63) / 64) * ((dim + 63) / 64);
    return std::max(tiles, weight) < 1 << 23 && input < 1 << 22;       // lanes of a launch are within 32 bits
}

// A piece's operands, laid out by the time its kernels run.
struct Operands {
    const void *x, *weight;
    int64_t     ld_x, ld_weight;
};
// The piece of the weights from `first` on, and with the first one x too.
template <class T>
int lay_piece(const Work& w, int64_t rows, int64_t first, int64_t n, int64_t dim, Operands* all, Operands* piece, uint8_t* space, hipStream_t s)
{
    const void* weight = static_cast<const T*>(all->weight) + first * all->ld_weight;
    *piece = *all;
    piece->weight = weight;
    if (!w.layout.anew) return ADAGC_OK;
    const LaySource sources[2] = {{weight, all->ld_weight, n, space + w.x}, {all->x, all->ld_x, rows, space}};
    if (const int rc = lay<T>(sources, first == 0 ? 2 : 1, dim, w.layout, s)) return rc;
    all->x = piece->x = space;
    all->ld_x = piece->ld_x = w.layout.ld;
    piece->weight = space + w.x;
    piece->ld_weight = w.layout.ld;
    return ADAGC_OK;
}
AlongArgs along_args(const Operands& o, const Work& w, int64_t rows, int64_t n, int64_t dim)
{
    AlongArgs p{};
    p.y = o.x;
    p.ld_y = o.ld_x;
    p.x[0] = p.x[1] = o.weight;
    p.ld_x[0] = p.ld_x[1] = o.ld_weight;
    p.m = rows;
    p.n = n;
    p.k = w.layout.anew ? w.layout.ld : dim;
    p.part_y = w.layout.part(rows);
    p.part_x = w.layout.part(n);
    p.segments = w.layout.segments;
    return p;
}
AlongPlan plan_of(AlongArgs* p, int32_t dtype)
{
    const AlongPlan plan = along_plan(p->m, p->n, p->k, p->segments, dtype, rows_aligned(p->y, p->ld_y, dtype) && rows_aligned(p->x[0], p->ld_x[0], dtype), p->ld_y, p->ld_x[0]);
    p->tiles_m = (int32_t)plan.tiles_m;
    p->tiles_n = (int32_t)plan.tiles_n;
    p->split = (int32_t)plan.split;
    return plan;
}
int launched() { return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP; }

// One piece; *tiles: the parts of a row that it adds.
template <class T>
int stats_of(StatsArgs a, int64_t* tiles, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    if (thin(a.p, dtype)) {
        *tiles = std::min<int64_t>((a.p.n + kThinColumns - 1) / kThinColumns, kThinGrid);
        for_rows(a.p.m, [&](auto TM) { thin_stats_kernel<T, decltype(TM)::value><<<dim3((uint32_t)*tiles), dim3(kThinThreads), 0, s>>>(a); });
        return launched();
    }
    const AlongPlan p = plan_of(&a.p, dtype);
    *tiles = p.tiles_n;
    const dim3 grid((uint32_t)(p.tiles_m * p.tiles_n));
    if constexpr (sizeof(T) == 2) {
        if (const int64_t columns = columns_of_whole_rounds(p, a.p.m, a.p.n)) {
            StatsArgs last = a;
            last.p.x[0] = last.p.x[1] = static_cast<const T*>(a.p.x[0]) + columns * a.p.ld_x[0];
            last.p.n -= columns;
            last.first += columns;
            last.parts += columns / 256;
            a.p.n = columns;
            int64_t more = 0;
            if (const int rc = stats_of<T>(a, tiles, s)) return rc;
            const int rc = stats_of<T>(last, &more, s);
            *tiles += more;
            return rc;
        }
        const dim3 small(grid_of<Small>(p.tiles_m * p.tiles_n));
        if (p.size == 256) {
            stats_kernel<Large, T, Sum::kWhole><<<dim3(grid_of<Large>(p.tiles_m * p.tiles_n)), dim3(Large::kThreads), 0, s>>>(a);
        } else if (p.direct && p.split > 1) {
            launch_parts<Small, T, false>(a.p, s);
            stats_kernel<Small, T, Sum::kJoined><<<grid, dim3(Small::kThreads), 0, s>>>(a);
        } else if (p.direct) {
            stats_kernel<Small, T, Sum::kWhole><<<small, dim3(Small::kThreads), 0, s>>>(a);
        }
    }
    if (!p.direct)
        staged_tile<T>(p, [&](auto tile) {
            using S = decltype(tile);
            if (p.split > 1) {
                launch_parts<S, T, false>(a.p, s);
                stats_kernel<S, T, Sum::kJoined><<<grid, dim3(S::kThreads), 0, s>>>(a);
            } else {
                stats_kernel<S, T, Sum::kWhole><<<grid, dim3(S::kThreads), 0, s>>>(a);
            }
        });
    return launched();
}

template <class T>
int forward(const Work& w, Operands o, int64_t rows, int64_t vocab, int64_t dim, StatsArgs a, JoinArgs join, uint8_t* workspace, hipStream_t s)
{
    uint8_t* laid = workspace + w.parts + w.targets;
    float* partial = reinterpret_cast<float*>(laid + w.x + w.weight);
    for (int64_t first = 0; first < vocab; first += w.size) {
        const int64_t n = std::min(w.size, vocab - first);
        Operands piece;
        if (const int rc = lay_piece<T>(w, rows, first, n, dim, &o, &piece, laid, s)) return rc;
        StatsArgs b = a;
        b.p = along_args(piece, w, rows, n, dim);
        b.p.partial = partial;
        b.first = first;
        b.parts += join.tiles;
        int64_t tiles = 0;
        if (const int rc = w.layout.anew ? stats_of<uint16_t>(b, &tiles, s) : stats_of<T>(b, &tiles, s)) return rc;
        join.tiles += tiles;
    }
    join_kernel<<<dim3((uint32_t)rows), dim3(kJoin), 0, s>>>(join);
    return launched();
}

template <class T>
int gradient(GradArgs a, int parts, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    if (parts == 1 && thin(a.p, dtype)) {
        const dim3 blocks((uint32_t)std::min<int64_t>((a.p.n + kThinColumns - 1) / kThinColumns, kThinGrid));
        for_rows(a.p.m, [&](auto TM) { thin_grad_kernel<T, decltype(TM)::value><<<blocks, dim3(kThinThreads), 0, s>>>(a); });
        return launched();
    }
    const AlongPlan p = plan_of(&a.p, dtype);
    const dim3 grid((uint32_t)(p.tiles_m * p.tiles_n));
    if constexpr (sizeof(T) == 2) {
        const dim3 large(grid_of<Large>(p.tiles_m * p.tiles_n)), small(grid_of<Small>(p.tiles_m * p.tiles_n));
        auto small_ones = [&](auto PARTS) {
            constexpr int kOf = decltype(PARTS)::value;
            if (p.split > 1) {
                launch_parts<Small, T, false>(a.p, s);
                grad_kernel<Small, T, kOf, Sum::kJoined><<<grid, dim3(Small::kThreads), 0, s>>>(a);
            } else {
                grad_kernel<Small, T, kOf, Sum::kWhole><<<small, dim3(Small::kThreads), 0, s>>>(a);
            }
        };
        if (p.size == 256) grad_kernel<Large, T, 1, Sum::kWhole><<<large, dim3(Large::kThreads), 0, s>>>(a);
        else if (p.direct && parts > 1) small_ones(std::integral_constant<int, kParts>{});
        else if (p.direct) small_ones(std::integral_constant<int, 1>{});
    }
    if (!p.direct)
        staged_tile<T>(p, [&](auto tile) {
            using S = decltype(tile);
            if (p.split > 1) {
                launch_parts<S, T, false>(a.p, s);
                grad_kernel<S, T, 1, Sum::kJoined><<<grid, dim3(S::kThreads), 0, s>>>(a);
            } else {
                grad_kernel<S, T, 1, Sum::kWhole><<<grid, dim3(S::kThreads), 0, s>>>(a);
            }
        });
    return launched();
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
int backward(const Work& w, Operands o, int64_t rows, int64_t vocab, int64_t dim, const GradArgs& all, const Outputs& out, uint8_t* workspace, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    float* sums = reinterpret_cast<float*>(workspace + w.d_logits);
    float* partial = reinterpret_cast<float*>(workspace + w.d_logits + w.sums);
    uint8_t* laid = workspace + w.d_logits + w.sums + w.partial;
    const bool anew = w.layout.anew, parts = w.layout.parts > 1;
    const int w_size = dtype_size(out.weight_dtype);
    const int64_t rows_dz = parts ? Layout::rows_of(rows) : rows, columns = anew ? (dim + 7) / 8 * 8 : dim;
    auto product_across = [&](const PlainArgs& a) { return anew ? run_plain<uint16_t, true>(a, s) : run_plain<T, true>(a, s); };
    auto product_along = [&](const PlainArgs& a) { return anew ? run_plain<uint16_t, false>(a, s) : run_plain<T, false>(a, s); };
    for (int64_t first = 0; first < vocab; first += w.size) {
        const int64_t n = std::min(w.size, vocab - first);
        Operands piece = o;
        PlainArgs both{};
        both.y[0] = workspace;
        both.ld_y = w.ld;
        both.part_y = rows_dz * w.ld;
        both.segments = w.layout.segments;
        both.n = dim;
        both.n_readable = columns;
        both.workspace = partial;
        both.factor = all.scale;
        both.pairs = both.products = 1;
        if (rows > 0) {
            if (const int rc = lay_piece<T>(w, rows, first, n, dim, &o, &piece, laid, s)) return rc;
            GradArgs a = all;
            a.p = along_args(piece, w, rows, n, dim);
            a.p.partial = partial;
            a.first = first;
            a.d_logits = workspace;
            a.ld = w.ld;
            a.part = both.part_y;
            a.rows = rows_dz;
            if (const int rc = anew ? gradient<uint16_t>(a, w.layout.parts, s) : gradient<T>(a, 1, s)) return rc;
        }
        if (out.d_weight) {
            PlainArgs a = both;
            a.x[0] = piece.x;
            a.ld_x[0] = piece.ld_x;
            a.part_x = w.layout.part(rows);
            a.out[0] = static_cast<uint8_t*>(out.d_weight) + first * out.ld_d_weight * w_size;
            a.ld_out[0] = out.ld_d_weight;
            a.add[0] = out.accumulate ? a.out[0] : nullptr;
            a.ld_add[0] = out.ld_d_weight;
            a.m = n;
            a.m_readable = readable_of(w.layout, n);
            a.k = rows_dz;
            a.out_bf16 = a.add_bf16 = out.weight_dtype == ADAGC_BF16;
            if (const int rc = product_across(a)) return rc;
        }
        if (out.d_x && rows > 0) {
            PlainArgs a = both;
            a.x[0] = piece.weight;
            a.ld_x[0] = piece.ld_weight;
            a.part_x = w.layout.part(n);
            const bool direct = first + n == vocab || dtype == ADAGC_F32;
            a.out[0] = direct ? out.d_x : sums;
            a.ld_out[0] = direct ? out.ld_d_x : dim;
            a.out_bf16 = direct && dtype == ADAGC_BF16;
            a.add[0] = first == 0 ? nullptr : dtype == ADAGC_F32 ? out.d_x : sums;
            a.ld_add[0] = dtype == ADAGC_F32 ? out.ld_d_x : dim;
            a.m = a.m_readable = rows;
            a.k = parts ? Layout::rows_of(n) : n;
            if (const int rc = product_along(a)) return rc;
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
    return launchable(rows, vocab, dim) ? work_of(rows, vocab, dim, dtype, false).forward() : (int64_t)ADAGC_ERR_TOO_LARGE;
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
    if (ld_x > kMaxLd || ld_weight > kMaxLd || !launchable(rows, vocab, dim)) return ADAGC_ERR_TOO_LARGE;
    const Work w = work_of(rows, vocab, dim, dtype, false);
    if (!workspace || workspace_bytes < w.forward() || misaligned(workspace, 16)) return ADAGC_ERR_INVALID_ARG;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    StatsArgs a{};
    a.targets = logprob ? targets : nullptr;
    a.scale = scale;
    a.parts = reinterpret_cast<float2*>(ws);
    a.pitch = w.pitch;
    a.target_logit = reinterpret_cast<float*>(ws + w.parts);
    JoinArgs j{};
    j.parts = a.parts;
    j.pitch = w.pitch;
    j.target_logit = a.target_logit;
    j.targets = targets;
    j.scale = scale;
    j.vocab = vocab;
    j.logprob = logprob;
    j.stats = reinterpret_cast<float2*>(stats);
    const Operands o = {x, weight, ld_x, ld_weight};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == ADAGC_F32 ? forward<float>(w, o, rows, vocab, dim, a, j, ws, s) : forward<uint16_t>(w, o, rows, vocab, dim, a, j, ws, s);
}

extern "C" int64_t adagc_linear_logprobs_backward_workspace_bytes(int64_t rows, int64_t vocab, int64_t dim, int32_t dtype)
{
    if (const int rc = check(rows, vocab, dim, dtype)) return rc;
    return launchable(rows, vocab, dim) ? work_of(rows, vocab, dim, dtype, true).backward() : (int64_t)ADAGC_ERR_TOO_LARGE;
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
    const Work w = work_of(rows, vocab, dim, dtype, true);
    const int64_t need = w.backward();
    if (need > 0 && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return ADAGC_ERR_INVALID_ARG;
    GradArgs a{};
    a.targets = targets;
    a.stats = stats;
    a.d_logprob = d_logprob;
    a.scale = scale;
    a.vocab = vocab;
    const Operands o = {x, weight, ld_x, ld_weight};
    const Outputs out = {d_x, ld_d_x, d_weight, weight_dtype, ld_d_weight, accumulate};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    return dtype == ADAGC_F32 ? backward<float>(w, o, rows, vocab, dim, a, out, ws, s) : backward<uint16_t>(w, o, rows, vocab, dim, a, out, ws, s);
}
