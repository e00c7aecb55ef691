// Log-probabilities of target tokens, with entropy, the most likely alternatives and the gradient of the logits, for gfx950.
//
// With M = max_j z_j and L = ln sum_j exp(s (z_j - M)) of a row of logits z and a scale s (the inverse temperature),
//   logp_j = s (z_j - M) - L,   p_j = exp(logp_j),   entropy H = -sum_j p_j logp_j = L - s sum_j p_j (z_j - M),
//   d z_j = s ( d_logprob (1[j = target] - p_j) - d_entropy p_j (logp_j + H) ).
// M and L are kept apart: s M + L in one fp32 number would lose L's digits where logits are large (a row of the type's lowest
// value, which masks are often made of, is uniform here).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "adagc.h"
#include "operators_internal.h"

namespace adagc {
namespace {

constexpr float kLowest = -3.402823466e38f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int64_t kMaxRows = (1 << 24) - 1;      // a launch has at most 2^32 - 1 lanes
// Scales with which s (z - M) log2 e neither overflows next to M nor needs the differences of z that do.
constexpr float kLeastScale = 0x1p-100f, kMostScale = 0x1p100f;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Partial result of a part of a row: sums relative to the part's largest value.
struct RowPart {
    float most;      // max z; -inf: nothing but masked values
    float sum;       // sum exp(s (z - most))
    float weighted;  // sum (z - most) exp(s (z - most))
    float pad;
};

struct ForwardArgs {
    const void*    logits;
    const int64_t* targets;
    int64_t        ld;
    int64_t        rows;
    int32_t        vocab;
    int32_t        parts;         // of a row
    int32_t        part_vectors;  // 16-byte vectors of a part
    int32_t        top_k;
    float          scale;
    float*         logprob;
    float*         entropy;
    float*         stats;
    float*         top_logprob;
    int32_t*       top_index;
    RowPart*       part;          // [rows][parts]
    uint64_t*      part_keys;     // [rows][parts][top_k]
};

// exp(x) of a difference already times log2 e
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A running sum of exponentials relative to `ref`, which trails the largest value by kSlack at most: moving it along with
// every new maximum would cost an exponential and a few products each time, and any reference within a few powers of e is as exact.
constexpr float kSlack = 4.0f;   // in units of s z
template <bool ENTROPY>
struct Running {
    float ref = kLowest, most = -INFINITY, sum = 0.f, weighted = 0.f;

    __device__ __forceinline__ void move_to(float m, float c)
    {
        if (sum != 0.f) {                        // also with NaN
            const float f = exp2_fast((ref - m) * c);
            // a distance that exp takes to 0 may be infinite in fp32
            if (ENTROPY) weighted = f == 0.f ? 0.f : (weighted + (ref - m) * sum) * f;
            sum *= f;
        }
        ref = m;
    }
    template <int N>
    __device__ __forceinline__ void add(const float (&z)[N], float vmax, float c, float slack)
    {
        most = maximum(most, vmax);
        if (vmax > ref + slack) move_to(vmax, c);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = z[i] - ref;
            const float e = exp2_fast(d * c);    // NaN stays NaN; -inf gives 0
            sum += e;
            if (ENTROPY) weighted += fmaxf(d, kLowest) * e;
        }
    }
    // both relative to the larger of the two maxima
    __device__ __forceinline__ void join(float m2, float s2, float w2, float c)
    {
        const float m = maximum(most, m2);
        const float to = m == -INFINITY ? kLowest : m;
        Running other;
        other.ref = m2;
        other.sum = s2;
        other.weighted = w2;
        move_to(to, c);
        other.move_to(to, c);
        most = m;
        sum += other.sum;
        weighted += other.weighted;
    }
};

// The top_k largest values that a wave has seen, as keys in its lanes, largest first: the value's bits in an order-keeping form, then
// the index's complement, so that keys are unique and equal values go to the lower index.  0: none.
//
// Candidates, values above the bar, wait in LDS and are sorted into the list many at a time: one alone costs the latencies of some
// thirty dependent instructions (about 600 clocks, seven microseconds for the 30 of a row's wave with top_k = 8), while the ranks
// of n of them are n independent comparisons.  Called by whole waves.
struct TopList {
    uint64_t  mine = 0;                          // this lane's
    int       count = 0, waiting = 0;            // in the list, in LDS
    // Values of -inf do not come in: a row with too few others has its list filled up at the end (write_row), which spares masked parts of rows
    // the sorting of equal values.
    float     bar = -INFINITY;                   // a later vector has to have a larger value: just below the least that counts, or the full list's last
    float     below = -INFINITY;                 // values that come in are larger: just below the least that counts, or just below the full list's last
    uint64_t* lds;                               // 64 of the wave's own
    int       k;

    __device__ __forceinline__ TopList(uint64_t* lds_, int k_) : lds(lds_), k(k_) {}

    static __device__ __forceinline__ uint64_t key(float z, uint32_t index)
    {
        uint32_t b = __float_as_uint(z + 0.0f);  // -0 is 0
        if (z != z) b = 0x7FFFFFFFu;
        b = (b & 0x80000000u) ? ~b : b | 0x80000000u;
        return (uint64_t)b << 32 | (0xFFFFFFFFu - index);
    }
    static __device__ __forceinline__ float value(uint64_t key)
    {
        const uint32_t b = (uint32_t)(key >> 32);
        return __uint_as_float((b & 0x80000000u) ? b & 0x7FFFFFFFu : ~b);
    }
    // The largest value below that with the upper half `bits` of a key; 0 and -0 count as one value.
    static __device__ __forceinline__ float just_below(uint32_t bits) { return value((uint64_t)(bits - (bits == 0x80000000u ? 2 : 1)) << 32); }
    static __device__ __forceinline__ uint32_t index(uint64_t key) { return 0xFFFFFFFFu - (uint32_t)key; }
    static __device__ __forceinline__ uint64_t of_lane(uint64_t x, int lane)
    {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
    }
    // LDS accesses of a wave are carried out in order; the compiler is told that other lanes' are meant
    static __device__ __forceinline__ void in_order()
    {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }

    // Sorts the keys in the first n lanes' `fresh` (0: none) into the list.
    __device__ __forceinline__ void merge(uint64_t fresh, int n)
    {
        const int lane = threadIdx.x & 63;
        int rank = lane, fresh_rank = 0;
        for (int j = 0; j < n; ++j) {
            const uint64_t other = of_lane(fresh, j);
            rank += other > mine;
            fresh_rank += other > fresh;
        }
        for (int j = 0; j < count; ++j) fresh_rank += of_lane(mine, j) > fresh;
        in_order();
        if (lane < count && rank < k) lds[rank] = mine;
        const bool there = lane < n && fresh != 0;
        if (there && fresh_rank < k) lds[fresh_rank] = fresh;
        in_order();
        count = min(k, count + __builtin_popcountll(__ballot(there)));
        mine = lane < count ? lds[lane] : 0;
        in_order();
        if (count == k) {
            const uint64_t last = of_lane(mine, k - 1);
            bar = value(last);
            below = just_below((uint32_t)(last >> 32));
        }
    }
    __device__ __forceinline__ void flush()
    {
        const int lane = threadIdx.x & 63, n = waiting;
        waiting = 0;
        if (n) {
            in_order();
            merge(lane < n ? lds[lane] : 0, n);
        }
    }
    // A value of each lane, or none.  Of ones that equal a full list's last only those of lower indices wait.
    __device__ __forceinline__ void offer(float z, uint32_t index, bool there)
    {
        uint64_t mask = __ballot(there && !(z <= below));
        if (!mask) return;
        const uint64_t own = key(z, index);
        if (count == k) mask = __ballot(there && own > of_lane(mine, k - 1));
        if (waiting + __builtin_popcountll(mask) > 64) {
            flush();
            mask = __ballot(there && (count == k ? own > of_lane(mine, k - 1) : !(z <= below)));
        }
        const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
        if (mask >> (threadIdx.x & 63) & 1) lds[waiting + before] = own;
        waiting += __builtin_popcountll(mask);
    }

    // The bar for a list that gets none of what lies below the k-th largest of 64 J values (J of each lane, 0 < k <= 64 J): just below
    // that, found bit by bit, its upper half being enough; -inf if it is -inf or NaN.
    template <int J>
    static __device__ __forceinline__ float bar_of(const float (&values)[J], int k)
    {
        uint32_t bits[J], at = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) bits[j] = (uint32_t)(key(values[j], 0) >> 32);
        for (uint32_t bit = 0x80000000u; bit != 0x8000u; bit >>= 1) {
            int above = 0;
#pragma unroll
            for (int j = 0; j < J; ++j) above += __builtin_popcountll(__ballot(bits[j] >= (at | bit)));
            if (above >= k) at |= bit;
        }
        const float kth = value((uint64_t)at << 32);
        return kth > -INFINITY ? just_below(at) : -INFINITY;
    }
};

template <int N>
__device__ __forceinline__ float largest_of(const float (&x)[N])
{
    float m = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = maximum(m, x[i]);
    return m;
}

// op over the wave's lanes, in all of them; op(x, y) = op(y, x).
template <class Op>
__device__ __forceinline__ float all_lanes(float x, Op&& op)
{
    auto moved = [](float v, auto CTRL) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(CTRL)::value, 0xF, 0xF, true)); };
    x = op(x, moved(x, std::integral_constant<int, 0xB1>{}));      // lane ^ 1
    x = op(x, moved(x, std::integral_constant<int, 0x4E>{}));      // lane ^ 2
    x = op(x, moved(x, std::integral_constant<int, 0x141>{}));     // the other four of eight
    x = op(x, moved(x, std::integral_constant<int, 0x140>{}));     // the other eight of sixteen
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = op(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return op(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
}

// Every lane's sums become the wave's, relative to its largest value.
template <bool ENTROPY>
__device__ __forceinline__ void reduce_lanes(Running<ENTROPY>& r, float c)
{
    r.most = all_lanes(r.most, [](float x, float y) { return maximum(x, y); });
    r.move_to(r.most == -INFINITY ? kLowest : r.most, c);
    r.sum = all_lanes(r.sum, [](float x, float y) { return x + y; });
    if (ENTROPY) r.weighted = all_lanes(r.weighted, [](float x, float y) { return x + y; });
}

// Results of a row from its sums, by one wave.
template <bool ENTROPY, bool TOP, class T>
__device__ __forceinline__ void write_row(const ForwardArgs& a, int64_t row, const Running<ENTROPY>& r, const TopList& top)
{
    const int lane = threadIdx.x & 63;
    const bool none = r.most == -INFINITY && r.sum == 0.f;
    // scale (z - M), also where the difference is beyond fp32's range and the product is not
    auto relative = [&](float z) __attribute__((always_inline)) {
        const float d = z - r.most;
        return d == -INFINITY && z != -INFINITY ? 2.f * a.scale * (0.5f * z - 0.5f * r.most) : a.scale * d;
    };
    // relative to ref, which is the maximum here
    const float log_sum = none ? 0.f : logf(r.sum);
    if (lane == 0) {
        if (a.logprob) {
            const int64_t t = a.targets[row];
            float v = 0.f;
            if (t >= 0 && t < a.vocab) {
                const float z = to_float(static_cast<const T*>(a.logits)[row * a.ld + t]);
                v = none ? -INFINITY : relative(z) - log_sum;
            }
            a.logprob[row] = v;
        }
        if (ENTROPY && a.entropy) a.entropy[row] = none ? 0.f : log_sum - a.scale * (r.weighted / r.sum);
        if (a.stats) {
            a.stats[2 * row] = r.most;
            a.stats[2 * row + 1] = log_sum;
        }
    }
    if constexpr (TOP) {
        auto put = [&](int place, float z, int32_t index) __attribute__((always_inline)) {
            a.top_logprob[row * a.top_k + place] = none ? -INFINITY : relative(z) - log_sum;
            a.top_index[row * a.top_k + place] = index;
        };
        const bool there = lane < a.top_k && top.mine != 0;
        if (there) put(lane, TopList::value(top.mine), (int32_t)TopList::index(top.mine));
        // all others are -inf: the first of them in order
        const T* z = static_cast<const T*>(a.logits) + row * a.ld;
        int have = __builtin_popcountll(__ballot(there));
        for (int64_t j0 = 0; have < a.top_k && j0 < a.vocab; j0 += 64) {
            const int64_t j = j0 + lane;
            const bool is = j < a.vocab && to_float(z[j]) == -INFINITY;
            const uint64_t mask = __ballot(is);
            const int place = have + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
            if (is && place < a.top_k) put(place, -INFINITY, (int32_t)j);
            have += __builtin_popcountll(mask);
        }
    }
}

constexpr int kAhead = 4;        // 16-byte vectors of a lane in a group

// One workgroup per part of a row, one pass: each lane keeps a running sum of exponentials (and of z - M times them), lanes and waves are
// joined at the end.  A row is one part unless there are too few rows to fill the chip.  Bound by memory on long calls, with the vector
// unit busy two thirds of the time (the exponential is a quarter of its instructions' time and a row's largest value another eighth): 4096 x
// 128256 bf16 208 us (5.1 TB/s), 1024 x 50257 with top 8 29 us (3.5 TB/s from the memory-side cache; 22 without the list, 25 with top 1, 36 with
// top 20, 72 with top 64).  One row of 128256 with top 5 in 31 parts 7 us: the 518 vectors of a part go round three times, each time waiting for
// their loads, the last time for 6 lanes; then the lists are joined.
template <class T, bool ENTROPY, bool TOP, bool SPLIT>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(const ForwardArgs a)
{
    constexpr int N = 16 / sizeof(T);
    const int64_t row = SPLIT ? blockIdx.x / (uint32_t)a.parts : blockIdx.x;
    const int part = SPLIT ? (int)(blockIdx.x - (uint32_t)row * (uint32_t)a.parts) : 0;
    const T* z = static_cast<const T*>(a.logits) + row * a.ld;
    const int all = (a.vocab + N - 1) / N;
    const int first = SPLIT ? part * a.part_vectors : 0;
    const int last = SPLIT ? min(first + a.part_vectors, all) : all;
    const int last_whole = min(last, a.vocab / N);         // all but one at most
    const float c = a.scale * kLog2e, slack = kSlack / a.scale;
    const int tid = (int)threadIdx.x;
    const int wave = tid >> 6, lane = tid & 63;
    __shared__ RowPart wave_part[kWaves];
    __shared__ uint64_t wave_keys[TOP ? kWaves * 64 : 1];    // what waits for each wave's list
    Running<ENTROPY> r;
    TopList top(wave_keys + (TOP ? wave * 64 : 0), a.top_k);
    // returns the lane's largest value
    auto add = [&](const Vector<T>& v) __attribute__((always_inline)) {
        float x[N];
        widen(v, x);
        const float vmax = largest_of(x);
        r.add(x, vmax, c, slack);
        return vmax;
    };
    auto offer = [&](const Vector<T>& v, float vmax, int vector, int count) __attribute__((always_inline)) {
        // these values have higher indices than all in the list, so one of them has to be larger
        if (!__ballot(!(vmax <= top.bar))) return;
        float x[N];
        widen(v, x);
#pragma unroll
        for (int i = 0; i < N; ++i) top.offer(x[i], (uint32_t)(vector * N + i), i < count);
    };
    // The bar of the workgroup's lists from its first values, the largest of each lane: the k-th largest of those is no larger than
    // the row's k-th.  Then all lists together get about top_k values of the first group, and as many of each later one.
    __shared__ float lane_most[kThreads + 1];
    auto begin = [&](float m) __attribute__((always_inline)) {
        lane_most[tid] = m;
        __syncthreads();
        if (wave == 0) {
            float values[kWaves];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) values[w] = lane_most[w * 64 + lane];
            const float bar = TopList::bar_of(values, a.top_k);
            if (lane == 0) lane_most[kThreads] = bar;
        }
        __syncthreads();
        top.bar = top.below = lane_most[kThreads];
    };
    // Whole waves go round together.  A group's loads are on their way while the group before is worked on (the last group loads
    // itself again: a loop without conditions).
    constexpr int kGroup = kAhead * kThreads;
    int v0 = first;
    if (v0 + kGroup <= last_whole) {
        Vector<T> v[kAhead], next[kAhead];
        auto load = [&](int from, Vector<T> (&to)[kAhead]) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) to[u] = load_whole(z + (size_t)(from + u * kThreads) * N + (uint32_t)(tid * N));
        };
        load(v0, v);
        if constexpr (TOP) {
            float m = -INFINITY;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                float x[N];
                widen(v[u], x);
                m = maximum(m, largest_of(x));
            }
            begin(m);
        }
        for (; v0 + kGroup <= last_whole; v0 += kGroup) {
            load(v0 + 2 * kGroup <= last_whole ? v0 + kGroup : v0, next);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const float vmax = add(v[u]);
                if constexpr (TOP) offer(v[u], vmax, v0 + u * kThreads + tid, N);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) v[u] = next[u];
        }
    }
    for (; v0 < last; v0 += kThreads) {
        const int i = v0 + tid, count = i < last ? min(N, a.vocab - i * N) : 0;
        // lanes past the part's end hold masked values
        const Vector<T> v = load_vector(z, i < last ? (int64_t)i * N : (int64_t)a.vocab, a.vocab, masked<T>());
        if constexpr (TOP) {
            if (v0 == first) {
                float x[N];
                widen(v, x);
                begin(largest_of(x));
            }
        }
        const float vmax = add(v);
        if constexpr (TOP) offer(v, vmax, i, count);
    }

    reduce_lanes(r, c);
    if (lane == 0) wave_part[wave] = {r.most, r.sum, r.weighted, 0.f};
    if constexpr (TOP) {
        // What the waves' lists hold and what waits for them, side by side; a key's place in the workgroup's list is the number of
        // larger ones, counted by all lanes: n^2 / 256 independent comparisons a lane for n keys, where merging list by list takes
        // dependent steps of one wave (1024 x 50257 with top 8 32.6 -> 31.4 us, one row of 128256 with top 5 13.3 -> 12.8, top 64 the same).
        constexpr int kMost = kWaves * (ADAGC_MAX_TOP + 64);
        constexpr int kAtOnce = 8, kBeyond = kAtOnce * 16;     // groups are 16 at most
        __shared__ uint64_t all_keys[kMost + kBeyond], sorted[ADAGC_MAX_TOP];
        __shared__ uint32_t rank[kMost];
        __shared__ int held[kWaves];
        if (lane == 0) held[wave] = top.count + top.waiting;
        if (tid < ADAGC_MAX_TOP) sorted[tid] = 0;
        for (int i = tid; i < kMost; i += kThreads) rank[i] = 0;
        for (int i = tid; i < kMost + kBeyond; i += kThreads) all_keys[i] = 0;
        __syncthreads();
        int before = 0, n = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            before += w < wave ? held[w] : 0;
            n += held[w];
        }
        if (lane < top.count) all_keys[before + lane] = top.mine;
        if (lane < top.waiting) all_keys[before + top.count + lane] = top.lds[lane];
        __syncthreads();
        int width = 16;                                    // lanes with a key each; the others take part of their comparisons
        while (width < n && width < kThreads) width *= 2;
        const int groups = kThreads / width, group = tid / width;
        for (int i = tid % width; i < n; i += width) {
            const uint64_t key = all_keys[i];
            uint32_t larger = 0;
            for (int j = group; j < n; j += kAtOnce * groups) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) larger += all_keys[j + u * groups] > key;       // 0 from n on
            }
            atomicAdd(&rank[i], larger);
        }
        __syncthreads();
        for (int i = tid; i < n; i += kThreads)
            if (rank[i] < (uint32_t)a.top_k) sorted[rank[i]] = all_keys[i];
        __syncthreads();
        top.mine = lane < a.top_k ? sorted[lane] : 0;
    } else {
        __syncthreads();
    }
    if (wave != 0) return;
    for (int w = 1; w < kWaves; ++w) r.join(wave_part[w].most, wave_part[w].sum, wave_part[w].weighted, c);
    if constexpr (SPLIT) {
        if (lane == 0) a.part[row * a.parts + part] = {r.most, r.sum, r.weighted, 0.f};
        if (TOP && lane < a.top_k) a.part_keys[(row * a.parts + part) * a.top_k + lane] = top.mine;
    } else {
        write_row<ENTROPY, TOP, T>(a, row, r, top);
    }
}

// One wave per row joins the row's parts, at most 64, one in each lane.  3.6 us for a row of 31 parts with top 5: a chain of latencies.
template <class T, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(64) void join_parts_kernel(const ForwardArgs a)
{
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    const float c = a.scale * kLog2e;
    __shared__ uint64_t waiting[64];
    Running<ENTROPY> r;
    TopList top(waiting, a.top_k);
    const bool has = lane < a.parts;
    if (has) {
        const RowPart x = a.part[row * a.parts + lane];
        r.join(x.most, x.sum, x.weighted, c);
    }
    reduce_lanes(r, c);
    if constexpr (TOP) {
        const uint64_t* keys = a.part_keys + row * a.parts * a.top_k;
        const uint64_t first = has ? keys[lane * a.top_k] : 0;
        const float largest[1] = {first ? TopList::value(first) : -INFINITY};
        top.bar = top.below = TopList::bar_of(largest, a.top_k);
        for (int j = 0; j < a.parts * a.top_k; j += 64) {
            const uint64_t key = j + lane < a.parts * a.top_k ? keys[j + lane] : 0;
            top.offer(TopList::value(key), TopList::index(key), key != 0);
        }
        top.flush();
    }
    write_row<ENTROPY, TOP, T>(a, row, r, top);
}

struct BackwardArgs {
    const void*    logits;
    void*          d_logits;
    const int64_t* targets;
    const float*   stats;
    const float*   entropy;
    const float*   d_logprob;
    const float*   d_entropy;
    int64_t        ld, ld_d;
    int32_t        vocab;
    float          scale;
    uint32_t       row_blocks;    // workgroup items per row
    uint64_t       items;
};

// Gradient of the logits, elementwise: a lane has four vectors loaded before its first store.  Bound by memory: 4096 x 128256 bf16 read and
// written in 356 us (5.9 TB/s), the vector unit busy for half of that.
constexpr float kMaskedLogp = -1e4f;
constexpr int kBackwardVectors = 4;  // per lane and item

template <class T>
__global__ __launch_bounds__(kThreads) void logprobs_backward_kernel(const BackwardArgs a)
{
    constexpr int N = 16 / sizeof(T);
    for (uint64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
        // last rows first: the forward pass has left them in the memory-side cache
        const uint64_t back = a.items - 1 - item;
        const int64_t row = (int64_t)(back / a.row_blocks);
        const uint32_t block = (uint32_t)(back - (uint64_t)row * a.row_blocks);
        const T* z = static_cast<const T*>(a.logits) + row * a.ld;
        T* d_z = static_cast<T*>(a.d_logits) + row * a.ld_d;
        const float stat = a.stats[2 * row];
        // nothing but masked values: every p is 0
        const float most = stat == -INFINITY ? 0.f : stat, log_sum = stat == -INFINITY ? INFINITY : a.stats[2 * row + 1];
        const int64_t t = a.targets ? a.targets[row] : -1;
        const int target = t >= 0 && t < a.vocab && stat != -INFINITY ? (int)t : -1;
        // a row of nothing but masked values asks for no gradient, which may be no number (of a ratio of its probabilities, for one)
        float d_lp = target >= 0 ? a.d_logprob[row] : 0.f;
        float d_h = a.d_entropy && stat != -INFINITY ? a.d_entropy[row] : 0.f;
        const float h = a.d_entropy ? a.entropy[row] : 0.f;
        // Gradients with which scale (d_lp + d_h (logp + h)) might be no number where p takes it back to one, or to 0: the larger is moved
        // to 2^99 or above and the scale next to 1 first, results by `after` powers of two last.
        const float size = fmaxf(fabsf(d_lp), fabsf(d_h));
        const bool huge = size > 0x1p100f || size > 0x1p100f / a.scale;
        float scale = a.scale;
        int after = 0;
        if (huge) {
            const int of_size = __builtin_amdgcn_frexp_expf(size), of_scale = __builtin_amdgcn_frexp_expf(scale);
            d_lp = __builtin_ldexpf(d_lp, 100 - of_size);
            d_h = __builtin_ldexpf(d_h, 100 - of_size);
            scale = __builtin_ldexpf(scale, -of_scale);
            after = of_size + of_scale - 100;
        }
        const float k0 = -scale * (d_lp + d_h * h), k1 = -scale * d_h;
        auto one = [&](const Vector<T>& v, uint32_t col) __attribute__((always_inline)) {
            float x[N];
            widen(v, x);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float logp = a.scale * (x[i] - most) - log_sum;
                // p as the square of the root, which is no subnormal number (the instruction would make those 0, and factors may raise them);
                // 0 from far above kMaskedLogp on
                const float root = exp2_fast(logp * (0.5f * kLog2e));
                x[i] = root * (root * fmaf(k1, fmaxf(logp, kMaskedLogp), k0));
            }
            if ((uint32_t)target - col < (uint32_t)N) {
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] += (uint32_t)target == col + i ? scale * d_lp : 0.f;
            }
            if (huge) {
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = __builtin_ldexpf(x[i], after);
            }
            return narrow<T>(x);
        };
        const int col0 = (int)block * kBackwardVectors * kThreads * N, col = col0 + (int)threadIdx.x * N;
        Vector<T> v[kBackwardVectors];
        if (kBackwardVectors * kThreads * N <= a.vocab - col0) {
#pragma unroll
            for (int u = 0; u < kBackwardVectors; ++u) v[u] = load_whole(z + col + u * kThreads * N);
#pragma unroll
            for (int u = 0; u < kBackwardVectors; ++u) store_whole(d_z + col + u * kThreads * N, one(v[u], (uint32_t)col + u * kThreads * N));
        } else {
#pragma unroll
            for (int u = 0; u < kBackwardVectors; ++u) v[u] = load_ahead(z, (int64_t)col + u * kThreads * N, a.vocab, masked<T>());
#pragma unroll
            for (int u = 0; u < kBackwardVectors; ++u) {
                settle(v[u], (int64_t)col + u * kThreads * N, a.vocab, masked<T>());
                store_vector(d_z, (int64_t)col + u * kThreads * N, a.vocab, one(v[u], (uint32_t)col + u * kThreads * N));
            }
        }
    }
}

// Parts of a row: one, unless there are too few rows to fill the chip.
int parts_of(int64_t rows, int64_t vocab)
{
    const int64_t wanted = 1024 / std::max<int64_t>(rows, 1), most = vocab / 4096;
    return (int)std::max<int64_t>(1, std::min<int64_t>({wanted, most, 64}));
}

template <class T, bool ENTROPY, bool TOP>
void launch_forward(const ForwardArgs& a, hipStream_t stream)
{
    if (a.parts == 1) {
        logprobs_kernel<T, ENTROPY, TOP, false><<<dim3((uint32_t)a.rows), dim3(kThreads), 0, stream>>>(a);
    } else {
        logprobs_kernel<T, ENTROPY, TOP, true><<<dim3((uint32_t)(a.rows * a.parts)), dim3(kThreads), 0, stream>>>(a);
        join_parts_kernel<T, ENTROPY, TOP><<<dim3((uint32_t)a.rows), dim3(64), 0, stream>>>(a);
    }
}

template <class T>
void launch_forward(const ForwardArgs& a, hipStream_t stream)
{
    if (a.entropy && a.top_k) launch_forward<T, true, true>(a, stream);
    else if (a.entropy) launch_forward<T, true, false>(a, stream);
    else if (a.top_k) launch_forward<T, false, true>(a, stream);
    else launch_forward<T, false, false>(a, stream);
}

int check_rows(int64_t rows, int64_t vocab, int32_t dtype, float scale)
{
    if (rows < 0 || vocab < 1 || !known_dtype(dtype) || !(scale >= kLeastScale) || !(scale <= kMostScale)) return ADAGC_ERR_INVALID_ARG;
    if (rows > kMaxRows || vocab > kMaxCols) return ADAGC_ERR_TOO_LARGE;
    return ADAGC_OK;
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int64_t adagc_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int32_t top_k)
{
    if (rows < 0 || vocab < 1 || top_k < 0 || top_k > ADAGC_MAX_TOP || top_k > vocab) return ADAGC_ERR_INVALID_ARG;
    if (rows > kMaxRows || vocab > kMaxCols) return ADAGC_ERR_TOO_LARGE;
    const int64_t parts = parts_of(rows, vocab);
    return parts == 1 ? 0 : rows * parts * (int64_t)(sizeof(RowPart) + 8 * top_k);
}

extern "C" int adagc_token_logprobs(const void* logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t ld, const int64_t* targets,
                                    float scale, int32_t top_k, float* logprob, float* entropy, float* stats, float* top_logprob,
                                    int32_t* top_index, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (const int rc = check_rows(rows, vocab, dtype, scale)) return rc;
    if (top_k < 0 || top_k > ADAGC_MAX_TOP || top_k > vocab || ld < vocab || workspace_bytes < 0) return ADAGC_ERR_INVALID_ARG;
    if (ld > kMaxLd) return ADAGC_ERR_TOO_LARGE;
    if (rows == 0) return ADAGC_OK;
    if (!logits || (logprob && !targets) || (top_k > 0) != (top_logprob != nullptr) || (top_k > 0) != (top_index != nullptr) ||
        (!logprob && !entropy && !stats && top_k == 0))
        return ADAGC_ERR_INVALID_ARG;
    const int64_t need = adagc_token_logprobs_workspace_bytes(rows, vocab, top_k);
    if (need > 0 && (!workspace || workspace_bytes < need)) return ADAGC_ERR_INVALID_ARG;
    if (misaligned(logits, dtype_size(dtype)) || misaligned(targets, 8) || misaligned(logprob, 4) || misaligned(entropy, 4) ||
        misaligned(stats, 4) || misaligned(top_logprob, 4) || misaligned(top_index, 4) || (need > 0 && misaligned(workspace, 16)))
        return ADAGC_ERR_INVALID_ARG;
    ForwardArgs a{};
    a.logits = logits;
    a.targets = targets;
    a.ld = ld;
    a.rows = rows;
    a.vocab = (int32_t)vocab;
    a.parts = parts_of(rows, vocab);
    const int64_t n = 16 / dtype_size(dtype), vectors = (vocab + n - 1) / n;
    a.part_vectors = (int32_t)((vectors + a.parts - 1) / a.parts);
    a.top_k = top_k;
    a.scale = scale;
    a.logprob = logprob;
    a.entropy = entropy;
    a.stats = stats;
    a.top_logprob = top_logprob;
    a.top_index = top_index;
    a.part = static_cast<RowPart*>(workspace);
    a.part_keys = reinterpret_cast<uint64_t*>(a.part + rows * a.parts);
    if (dtype == ADAGC_F32) launch_forward<float>(a, static_cast<hipStream_t>(stream));
    else launch_forward<uint16_t>(a, static_cast<hipStream_t>(stream));
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}

extern "C" int adagc_token_logprobs_backward(const void* logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t ld,
                                             const int64_t* targets, float scale, const float* stats, const float* entropy,
                                             const float* d_logprob, const float* d_entropy, void* d_logits, int64_t ld_d, void* stream)
{
    if (const int rc = check_rows(rows, vocab, dtype, scale)) return rc;
    if (ld < vocab || ld_d < vocab) return ADAGC_ERR_INVALID_ARG;
    if (ld > kMaxLd || ld_d > kMaxLd) return ADAGC_ERR_TOO_LARGE;
    if (rows == 0) return ADAGC_OK;
    if (!logits || !stats || !d_logits || (d_logprob && !targets) || (d_entropy && !entropy) || (d_logits == logits && ld_d != ld))
        return ADAGC_ERR_INVALID_ARG;
    if (misaligned(logits, dtype_size(dtype)) || misaligned(d_logits, dtype_size(dtype)) || misaligned(targets, 8) || misaligned(stats, 4) ||
        misaligned(entropy, 4) || misaligned(d_logprob, 4) || misaligned(d_entropy, 4))
        return ADAGC_ERR_INVALID_ARG;
    BackwardArgs a{};
    a.logits = logits;
    a.d_logits = d_logits;
    a.targets = d_logprob ? targets : nullptr;
    a.stats = stats;
    a.entropy = entropy;
    a.d_logprob = d_logprob;
    a.d_entropy = d_entropy;
    a.ld = ld;
    a.ld_d = ld_d;
    a.vocab = (int32_t)vocab;
    a.scale = scale;
    const int64_t per_block = (int64_t)kThreads * kBackwardVectors * (16 / dtype_size(dtype));
    a.row_blocks = (uint32_t)((vocab + per_block - 1) / per_block);
    a.items = (uint64_t)rows * a.row_blocks;
    const uint32_t grid = (uint32_t)std::min<uint64_t>(a.items, 1u << 23);
    if (dtype == ADAGC_F32) logprobs_backward_kernel<float><<<dim3(grid), dim3(kThreads), 0, static_cast<hipStream_t>(stream)>>>(a);
    else logprobs_backward_kernel<uint16_t><<<dim3(grid), dim3(kThreads), 0, static_cast<hipStream_t>(stream)>>>(a);
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}
