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
#include <type_traits>
#include <utility>

#include "act8_device.h"
#include "operators_internal.h"

namespace adagc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
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
    int32_t        weight_bf16;
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

// A lane's four consecutive values of row o of the result, from column i on; rows below o_least and columns below i_least belong to
// another tile.
template <class W>
__device__ __forceinline__ void store_typed(const WgradArgs& a, int64_t o, int64_t i, int64_t i_least, f32x4 v)
{
    W* w = static_cast<W*>(a.d_weight) + o * a.ld_w + i;
    if (i >= i_least && i + 4 <= a.n_in) {
        if constexpr (sizeof(W) == 4) {
            if (a.accumulate) {
                float old[4];
                widen(load_whole(w), old);
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] += old[r];
            }
            store_whole(w, {__builtin_bit_cast(u32x4, v)});
        } else {
            typedef uint32_t u32x2_of_bf16 __attribute__((ext_vector_type(2), aligned(2)));
            u32x2_of_bf16 two;
            if (a.accumulate) {
                two = *reinterpret_cast<const u32x2_of_bf16*>(w);
                v[0] += __uint_as_float(two[0] << 16);
                v[1] += __uint_as_float(two[0] & 0xFFFF0000u);
                v[2] += __uint_as_float(two[1] << 16);
                v[3] += __uint_as_float(two[1] & 0xFFFF0000u);
            }
            const f32x2_t lo = {v[0], v[1]}, hi = {v[2], v[3]};
            two[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2_t));
            two[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2_t));
            *reinterpret_cast<u32x2_of_bf16*>(w) = two;
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (i + r >= i_least && i + r < a.n_in) {
                const float x = v[r] + (a.accumulate ? to_float(w[r]) : 0.f);
                if constexpr (sizeof(W) == 4) w[r] = x;
                else w[r] = __builtin_bit_cast(uint16_t, (__bf16)x);
            }
    }
}
__device__ __forceinline__ void store_results(const WgradArgs& a, int64_t o, int64_t o_least, int64_t i, int64_t i_least, f32x4 v)
{
    if (o < o_least || o >= a.n_out || i >= a.n_in) return;
    if (a.weight_bf16) store_typed<uint16_t>(a, o, i, i_least, v);
    else store_typed<float>(a, o, i, i_least, v);
}

// f(integral_constant 0), ..., f(integral_constant N-1)
template <class F, int... I>
__device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f)
{
    static_for_impl(f, std::make_integer_sequence<int, N>{});
}

// Tokens of a step, and the places of LDS that steps go round in.
constexpr int kDeep = 32, kPlaces = 3;

// BM x BN tile of dW (BM along n_out), kWM x kWN waves, matrix-core instructions of kBlock x kBlock results.
//
// kBlock: with 32 the matrix cores read half the operand registers for the same products, in half the instructions: fp32 2048 tokens
// 1024 x 2816 52.7 -> 49.5 us.  On the 256 x 256 tile, where the chip's power limit sets the clock, 16 is ahead: 8192 tokens
// 14336 x 4096 816 against 853 us, and back to back 906 - 924 against 949 (on zeros, which take less power, 758 against 737).
template <class T, int BM_, int BN_, int kWM_, int kWN_, int kBlock_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, kWM = kWM_, kWN = kWN_, kBlock = kBlock_;
    static constexpr int kThreads = 64 * kWM * kWN;
    static constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    static constexpr int kTM = BM / kWM / kBlock, kTN = BN / kWN / kBlock; // blocks of a wave
    static constexpr int kHalves = kBlock / 16;                            // instructions of a step and block: one takes 512 / kBlock tokens
    static constexpr int kPieces = kBlock * kBlock / 256;                  // of four results in a lane's part of a block
    static constexpr int kY = kDeep * BM, kX = kDeep * BN;                 // elements of a staged operand tile
    static constexpr int kPlace = (kParts * kY + kX) * 2;                  // bytes
    static constexpr int kYUnits = kY / 8 / kThreads, kXUnits = kX / 16 / kThreads;     // of a lane: 8 values of dY, 16 codes
    static_assert(kY % (8 * kThreads) == 0 && kX % (16 * kThreads) == 0, "operand tiles are dealt evenly");

    // Byte offset of 16-byte vector v of row r of a staged tile of C columns: its 32-byte units are permuted so that the eight that half
    // a wave's transposed read takes (one of the rows 0 .. 3 and 8 .. 11 each, or two of 0 .. 3) lie in different banks.
    static __device__ __forceinline__ int swizzle(int r) { return kBlock == 16 ? (r & 3) | ((r >> 3) & 1) << 2 : (r & 3) << 1; }
    template <int C>
    static __device__ __forceinline__ int at(int r, int v) { return r * C * 2 + ((v >> 1) ^ swizzle(r)) * 32 + (v & 1) * 16; }
};

// s_waitcnt for "at most n LDS accesses of this wave still outstanding", nothing else waited for
#define ADAGC_WAIT_LDS(n) __builtin_amdgcn_s_waitcnt(0xF | (3 << 14) | (7 << 4) | ((n) << 8))
// nothing is moved across this point by the compiler's instruction scheduler
#define ADAGC_SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)

// EDGE: dW is smaller than a tile in one direction, or rows of an operand are too far apart for 32-bit offsets.  Otherwise the last tile of a
// direction begins a tile before the end, so that every tile is whole, and stores only what no other tile does.
//
// Main loop.  A step's operands are staged in a place of LDS; while step k is multiplied from registers, step k + 1 is read to
// registers from its place (each fragment as soon as its multiplications are issued, or to a second set), step k + 2 goes from
// the registers it was loaded to into its place, and those take step k + 4.  One barrier a step: what it orders is the writes of k + 2
// before their reads in the next step; the reads of a place are done a step before it is written again.  Loads past the last step take
// the last one again: a loop without conditions lets the compiler count what is outstanding.
//
// What bounds large calls is power, and what the two waves of a SIMD wait for each other: 8192 tokens 14336 x 4096 bf16 816 us (1.18 PFLOP/s;
// 923 back to back, where a library product of bf16 matrices lying like these takes 1049), the matrix cores busy 53 % of the time at
// some 1.9 GHz, LDS 40 %; with zeros for values 738.  Reads beyond the L2s are 4.5 times the operands, 1.5 TB/s.  Small calls are a chain of
// latencies: 123 tokens 768 x 768 8 us.
template <class S, class T, bool EDGE>
__global__ __launch_bounds__(S::kThreads, S::kThreads == 256 && S::kParts == 3 ? 1 : 2) void wgrad_kernel(const WgradArgs a)
{
    constexpr int BM = S::BM, BN = S::BN, kThreads = S::kThreads, kTM = S::kTM, kTN = S::kTN, kParts = S::kParts;
    constexpr int kHalves = S::kHalves, kYUnits = S::kYUnits, kXUnits = S::kXUnits, kH = (int)sizeof(T) / 2;
    __shared__ __attribute__((aligned(512))) uint8_t lds[kPlaces * S::kPlace];
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(&lds[0]);      // low half of the flat address = LDS offset
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / S::kWN, wn = wave % S::kWN;

    // the tile and the tokens of this workgroup
    const int item = (int)blockIdx.x;
    int tile = item, part = 0;
    const bool alone = item < a.whole;
    if (!alone) {
        tile = a.whole + (item - a.whole) / a.split;
        part = (item - a.whole) % a.split;
    }
    int to, ti;
    place_of_tile(a, tile, &to, &ti);
    const int64_t o_least = (int64_t)to * BM, i_least = (int64_t)ti * BN;
    const int64_t o0 = EDGE ? o_least : min(o_least, (int64_t)a.n_out - BM), i0 = EDGE ? i_least : min(i_least, (int64_t)a.ld - BN);
    const int64_t full = a.rows / kDeep;
    const int64_t step0 = alone ? 0 : full * part / a.split, step1 = alone ? full : full * (part + 1) / a.split;
    const bool last = alone || part == a.split - 1;

    // Staging: a lane's units, in registers between the load and the write to LDS.  A lane's units are whole rows apart.
    struct Staged {
        Vector<T> y[kYUnits][kH];
        u32x4     x[kXUnits];
        uint32_t  scale[kXUnits];
    };
    const int yr = tid / (BM / 8), yv = tid % (BM / 8), xr = tid / (BN / 16), xv = tid % (BN / 16) * 2;
    constexpr int kYRows = kThreads / (BM / 8), kXRows = kThreads / (BN / 16);
    const uint32_t lane_y = (uint32_t)(yr * (uint32_t)a.ld_d + (uint32_t)yv * 8) * sizeof(T);
    const uint32_t lane_x = (uint32_t)xr * (uint32_t)a.ld + (uint32_t)xv * 8;
    const uint32_t lane_scale = (uint32_t)xr * (uint32_t)(a.ld / 32) + (uint32_t)xv / 4;
    // inside the matrices nothing is checked, and a lane's address is a wave-wide base and 32 bits
    auto load_y = [&](int64_t step, int n, Staged& s) __attribute__((always_inline)) {
        const uint8_t* row = static_cast<const uint8_t*>(a.d_out) + ((step * kDeep + n * kYRows) * a.ld_d + o0) * sizeof(T);
#pragma unroll
        for (int h = 0; h < kH; ++h) s.y[n][h] = load_whole(reinterpret_cast<const T*>(row + lane_y) + h * 4);
    };
    auto load_x = [&](int64_t step, int n, Staged& s) __attribute__((always_inline)) {
        const int64_t at = (step * kDeep + n * kXRows) * a.ld + i0;
        s.x[n] = *reinterpret_cast<const u32x4*>(a.codes + at + lane_x);
        s.scale[n] = (a.scales + at / 32)[lane_scale];
    };
    auto load = [&](int64_t step, Staged& s) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < kYUnits; ++n) load_y(step, n, s);
#pragma unroll
        for (int n = 0; n < kXUnits; ++n) load_x(step, n, s);
    };
    auto load_checked = [&](int64_t step, Staged& s) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < kYUnits; ++n) {
            const int64_t t = step * kDeep + yr + n * kYRows;
            const T* row = static_cast<const T*>(a.d_out) + t * a.ld_d;
#pragma unroll
            for (int h = 0; h < kH; ++h) s.y[n][h] = load_vector(row, o0 + yv * 8 + h * 4, t < a.rows ? a.n_out : 0, 0);
        }
#pragma unroll
        for (int n = 0; n < kXUnits; ++n) {
            const int64_t t = step * kDeep + xr + n * kXRows, i = i0 + xv * 8;
            s.x[n] = u32x4{0, 0, 0, 0};
            s.scale[n] = 127;
            if (t < a.rows && i < a.ld) {
                s.x[n] = *reinterpret_cast<const u32x4*>(a.codes + t * a.ld + i);
                s.scale[n] = a.scales[(t * a.ld + i) / 32];
            }
        }
    };
    const uint32_t write_y_at = (uint32_t)S::template at<BM>(yr, yv), write_x_at = (uint32_t)(kParts * S::kY * 2 + S::template at<BN>(xr, xv));
    static_assert(kYRows % 16 == 0 && kXRows % 16 == 0, "a lane's units are at the same place of the swizzle");
    auto write_y = [&](const Staged& s, int n, uint32_t place) __attribute__((always_inline)) {
        const uint32_t at = place + write_y_at + (uint32_t)(n * kYRows * BM * 2);
        if constexpr (kParts == 1) {
            *reinterpret_cast<ADAGC_LDS u32x4*>(at) = s.y[n][0].w;
        } else {
            // x = hi + mid + lo, each the upper half of what is left: exact.  (Of an infinity nothing is left.)
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
            for (int q = 0; q < 3; ++q) *reinterpret_cast<ADAGC_LDS u32x4*>(at + q * S::kY * 2) = p[q];
        }
    };
    auto write_x = [&](const Staged& s, int n, uint32_t place) __attribute__((always_inline)) {
        const float scale = __uint_as_float(s.scale[n] << 23);
        u32x4 w[2];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            w[k / 4][k % 4] = __builtin_bit_cast(uint32_t, k % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(s.x[n][k / 2], scale, true)
                                                                 : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(s.x[n][k / 2], scale, false));
        const uint32_t at = place + write_x_at + (uint32_t)(n * kXRows * BN * 2);
        *reinterpret_cast<ADAGC_LDS u32x4*>(at) = w[0];
        *reinterpret_cast<ADAGC_LDS u32x4*>(at + 16) = w[1];
    };
    auto write = [&](const Staged& s, uint32_t place) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < kYUnits; ++n) write_y(s, n, place);
#pragma unroll
        for (int n = 0; n < kXUnits; ++n) write_x(s, n, place);
    };

    // Fragments.  16 lanes read 4 rows of 16 columns and get a column each; lane l's are rows 8 (l / kBlock) .. + 7 of column l mod kBlock.
    constexpr int kBlock = S::kBlock, kUnits32 = kBlock / 16;       // 32-byte units of a block's row
    const int fr = 8 * (lane / kBlock) + ((lane >> 2) & 3), fu = (lane >> 4) % kUnits32;
    const uint32_t fy = fr * BM * 2 + (((wm * kTM * kUnits32 + fu) ^ S::swizzle(fr)) * 32) + (lane & 3) * 8;
    const uint32_t fx = kParts * S::kY * 2 + fr * BN * 2 + (((wn * kTN * kUnits32 + fu) ^ S::swizzle(fr)) * 32) + (lane & 3) * 8;
    auto read4 = [](uint32_t at) __attribute__((always_inline)) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ADAGC_LDS s16x4*>(at)); };
    auto fragment = [&](uint32_t at, uint32_t pitch) __attribute__((always_inline)) {
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(read4(at), read4(at + 4 * pitch), 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // fragment g of dY: block g mod kTM, half, part; fragment f of X: block f mod kTN, half
    auto read_y = [&](int g, uint32_t place) __attribute__((always_inline)) {
        return fragment(place + (fy ^ (uint32_t)(g % kTM * kBlock * 2)) + (uint32_t)(g / kTM % kHalves * 16 * BM * 2 + g / kTM / kHalves * S::kY * 2), BM * 2);
    };
    auto read_x = [&](int f, uint32_t place) __attribute__((always_inline)) {
        return fragment(place + (fx ^ (uint32_t)(f % kTN * kBlock * 2)) + (uint32_t)(f / kTN * 16 * BN * 2), BN * 2);
    };

    typedef std::conditional_t<kBlock == 16, f32x4, f32x16> Results;
    Results acc[kTM][kTN];
#pragma unroll
    for (int m = 0; m < kTM; ++m)
#pragma unroll
        for (int n = 0; n < kTN; ++n)
#pragma unroll
            for (int r = 0; r < 4 * S::kPieces; ++r) acc[m][n][r] = 0.f;
    constexpr int kG = kParts * kHalves * kTM, kF = kHalves * kTN;         // fragments of dY, of X
    constexpr int kSets = kHalves == 1 ? 2 : 1;      // of X's: with one half they are all in use to the step's end
    bf16x8 y[kG], x[kSets][kF];

    // acc[m][n] += x y^T
    auto multiply = [](const bf16x8& x, const bf16x8& y, Results& sum) __attribute__((always_inline)) {
        if constexpr (kBlock == 16) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, sum, 0, 0, 0);
        else sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, sum, 0, 0, 0);
    };

    // a step from the place at `place`, whose staged units are loaded
    auto plain_step = [&](const Staged& s, uint32_t place, auto&& meanwhile) __attribute__((always_inline)) {
        write(s, place);
        meanwhile();
        __syncthreads();
#pragma unroll
        for (int f = 0; f < kF; ++f) x[0][f] = read_x(f, place);
#pragma unroll
        for (int g = 0; g < kG; ++g) {
            y[0] = read_y(g, place);
#pragma unroll
            for (int n = 0; n < kTN; ++n) multiply(x[0][g / kTM % kHalves * kTN + n], y[0], acc[g % kTM][n]);
        }
    };
    // Tokens after the last full step come first, so that their loads and the main loop's first are on their way together.
    const bool rest = last && a.rows % kDeep;
    constexpr uint32_t kRestPlace = (kPlaces - 1) * S::kPlace;

    if constexpr (EDGE) {
        // two steps' loads are on their way; a step's writes and the reads of the step before take different places
        const int64_t end = step1 + rest;
        Staged staged[2];
        if (step0 < end) load_checked(step0, staged[0]);
        if (step0 + 1 < end) load_checked(step0 + 1, staged[1]);
        for (int64_t step = step0; step < end; step += 2)
            static_for<2>([&](auto P) __attribute__((always_inline)) {
                constexpr int p = decltype(P)::value;
                if (step + p >= end) return;
                plain_step(staged[p], lds0 + p * S::kPlace, [&] {
                    if (step + p + 2 < end) load_checked(step + p + 2, staged[p]);
                });
            });
    } else if (step0 == step1) {
        if (rest) {
            Staged s;
            load_checked(full, s);
            plain_step(s, lds0 + kRestPlace, [] {});
        }
    } else {
        Staged staged[2];
        auto clamp = [&](int64_t step) { return min(step, step1 - 1); };
        if (rest) {
            Staged s;
            load_checked(full, s);
            load(step0, staged[0]);
            load(clamp(step0 + 1), staged[1]);
            plain_step(s, lds0 + kRestPlace, [] {});
        } else {
            load(step0, staged[0]);
            load(clamp(step0 + 1), staged[1]);
        }
        write(staged[0], lds0);
        load(clamp(step0 + 2), staged[0]);
        write(staged[1], lds0 + S::kPlace);
        load(clamp(step0 + 3), staged[1]);
        __syncthreads();
#pragma unroll
        for (int f = 0; f < kF; ++f) x[0][f] = read_x(f, lds0);
#pragma unroll
        for (int g = 0; g < kG; ++g) y[g] = read_y(g, lds0);
        uint32_t next = lds0 + S::kPlace;          // the place of step k + 1
        auto after = [&](uint32_t place) { return place == lds0 + (kPlaces - 1) * S::kPlace ? lds0 : place + S::kPlace; };
        auto one_step = [&](auto PARITY, int64_t step) __attribute__((always_inline)) {
            constexpr int p = decltype(PARITY)::value;
            constexpr int kSlots = kG * kTN;
            constexpr int kWrites = kYUnits + kXUnits;
            const uint32_t to_place = after(next);
            const int64_t ahead = clamp(step + 4);
            static_for<kSlots>([&](auto SLOT) __attribute__((always_inline)) {
                constexpr int slot = decltype(SLOT)::value, g = slot / kTN, n = slot % kTN;
                multiply(x[p % kSets][g / kTM % kHalves * kTN + n], y[g], acc[g % kTM][n]);
                ADAGC_SCHED_FENCE();
                // into the other set, or where a fragment's last multiplication is issued (a half step before its next)
                if constexpr (kSets == 2) {
                    if constexpr (slot % 2 == 0 && slot / 2 < kF) x[p ^ 1][slot / 2] = read_x(slot / 2, next);
                } else if constexpr (g >= kG - kTM * kHalves && g % kTM == kTM - 1) {
                    x[0][g / kTM % kHalves * kTN + n] = read_x(g / kTM % kHalves * kTN + n, next);
                }
                if constexpr (n == kTN - 1) y[g] = read_y(g, next);
                static_for<kWrites>([&](auto N) __attribute__((always_inline)) {
                    constexpr int w = decltype(N)::value;
                    if constexpr (kSlots / 4 + w * (kSlots / 4) / kWrites + 1 == slot) {
                        if constexpr (w < kYUnits) write_y(staged[p], w, to_place);
                        else write_x(staged[p], w - kYUnits, to_place);
                    }
                    if constexpr (kSlots / 2 + 2 + w * (kSlots / 4) / kWrites == slot) {
                        if constexpr (w < kYUnits) load_y(ahead, w, staged[p]);
                        else load_x(ahead, w - kYUnits, staged[p]);
                    }
                });
                ADAGC_SCHED_FENCE();
            });
            // the writes, in the first half of the step, are done; the fragments read since may still be on their way
            constexpr int kSince = 2 * (kG / 2 - 1);
            ADAGC_WAIT_LDS(kSince < 15 ? kSince : 15);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            ADAGC_SCHED_FENCE();
            next = to_place;
        };
        int64_t step = step0;
        for (; step + 1 < step1; step += 2) {
            one_step(std::integral_constant<int, 0>{}, step);
            one_step(std::integral_constant<int, 1>{}, step + 1);
        }
        if (step < step1) one_step(std::integral_constant<int, 0>{}, step);
    }
    // lane l holds rows 8 q + 4 (l / kBlock) .. + 3 (of X's block), q = 0 .. kPieces - 1, of column l mod kBlock (of dY's)
    auto each_piece = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
        for (int m = 0; m < kTM; ++m)
#pragma unroll
            for (int n = 0; n < kTN; ++n)
#pragma unroll
                for (int q = 0; q < S::kPieces; ++q)
                    f(m, n, q, f32x4{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]});
    };
    if (alone) {
        each_piece([&](int m, int n, int q, f32x4 v) __attribute__((always_inline)) {
            store_results(a, o0 + (wm * kTM + m) * kBlock + lane % kBlock, o_least, i0 + (wn * kTN + n) * kBlock + q * 8 + lane / kBlock * 4, i_least, v);
        });
    } else {
        f32x4* to_ws = reinterpret_cast<f32x4*>(a.workspace) + (size_t)(item - a.whole) * (BM * BN / 4) + tid;
        each_piece([&](int m, int n, int q, f32x4 v) __attribute__((always_inline)) { to_ws[((m * kTN + n) * S::kPieces + q) * kThreads] = v; });
    }
}

// Adds the parts of the split tiles, in order: a workgroup takes one piece of four results of every lane.  Bound by memory and latency: 128
// tiles of 256 x 256 in two parts 17 us.
template <class S, bool EDGE>
__global__ __launch_bounds__(S::kThreads) void join_kernel(const WgradArgs a)
{
    constexpr int kTN = S::kTN, kPieces = S::kTM * kTN * S::kPieces, BM = S::BM, BN = S::BN, kBlock = S::kBlock;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / S::kWN, wn = wave % S::kWN;
    const int n_tile = (int)blockIdx.x / kPieces, piece = (int)blockIdx.x % kPieces, q = piece % S::kPieces;
    const int m = piece / S::kPieces / kTN, n = piece / S::kPieces % kTN;
    int to, ti;
    place_of_tile(a, a.whole + n_tile, &to, &ti);
    const int64_t o_least = (int64_t)to * BM, i_least = (int64_t)ti * BN;
    const int64_t o0 = EDGE ? o_least : min(o_least, (int64_t)a.n_out - BM), i0 = EDGE ? i_least : min(i_least, (int64_t)a.ld - BN);
    const f32x4* from = reinterpret_cast<const f32x4*>(a.workspace) + (size_t)n_tile * a.split * (BM * BN / 4) + (size_t)piece * S::kThreads + tid;
    f32x4 sum = from[0];
    int p = 1;
    constexpr int kTogether = 4;                       // loads on their way
    for (; p + kTogether <= a.split; p += kTogether) {
        f32x4 v[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) v[u] = from[(size_t)(p + u) * (BM * BN / 4)];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) sum += v[u];
    }
    for (; p < a.split; ++p) sum += from[(size_t)p * (BM * BN / 4)];
    store_results(a, o0 + (wm * S::kTM + m) * kBlock + lane % kBlock, o_least, i0 + (wn * kTN + n) * kBlock + q * 8 + lane / kBlock * 4, i_least, sum);
}

int check(int64_t rows, int64_t n_out, int64_t n_in, int32_t dtype)
{
    if (rows < 0 || n_out < 1 || n_in < 1 || !known_dtype(dtype)) return ADAGC_ERR_INVALID_ARG;
    if (rows > INT32_MAX || n_out > kMaxCols || n_in > kMaxCols) return ADAGC_ERR_TOO_LARGE;
    return ADAGC_OK;
}

// How a call is cut: tiles of dW, and those of the last, partial round of workgroups also along the tokens, so that they
// fill the chip too.
struct Plan {
    int     bm, bn;
    int64_t tiles_out, tiles_in, whole, rest, split;
    int64_t workspace() const { return split > 1 ? rest * split * bm * bn * 4 : 0; }
    bool    launchable() const { return (whole + rest * split) * (bm + bn > 256 ? 512 : 256) <= UINT32_MAX; }      // lanes
};
Plan plan_of(int64_t rows, int64_t n_out, int64_t n_in, int32_t dtype)
{
    Plan p{};
    auto tiles = [&](int64_t bm, int64_t bn) { return ((n_out + bm - 1) / bm) * ((n_in + bn - 1) / bn); };
    const bool large = dtype == ADAGC_BF16 && n_out >= 256 && act8_ld(n_in) >= 256 && tiles(256, 256) >= kUnits / 2;
    const bool wide = dtype == ADAGC_F32 && n_out >= 128 && act8_ld(n_in) >= 256;
    p.bm = large ? 256 : 128;
    p.bn = large || wide ? 256 : 128;
    p.tiles_out = (n_out + p.bm - 1) / p.bm;
    p.tiles_in = (n_in + p.bn - 1) / p.bn;
    const int64_t all = p.tiles_out * p.tiles_in, steps = rows / kDeep;
    // the smaller tile's workgroups with bf16 dY share a compute unit in pairs; the others fill its LDS
    const int64_t round = dtype == ADAGC_BF16 && !large ? 2 * kUnits : kUnits;
    p.rest = all % round;
    // A part has four steps at least, and eight where there are few: what another workgroup saves has to pay for the partial sums and the second
    // kernel (us with eight everywhere, with four everywhere: 660 tokens 74 x 125 15.2, 10.0; 1000 tokens 300 x 900 fp32 22.4, 19.2;
    // 256 tokens 768 x 768 8.3, 10.2; 300 tokens 2000 x 2000 12.0, 26.7).
    // In the checked loop of matrices smaller than a tile a step takes twice as long: parts of two steps (215 tokens 2947 x 84 fp32 17.7 -> 13.8).
    const bool checked = n_out < p.bm || act8_ld(n_in) < p.bn;
    const int64_t most = steps >= 16 ? steps / 4 : checked ? steps / 2 : steps / 8;
    p.split = p.rest ? std::max<int64_t>(1, std::min(round / p.rest, most)) : 1;
    if (p.split == 1) p.rest = 0;
    p.whole = all - p.rest;
    return p;
}

template <class S, class T, bool EDGE>
int launch(const WgradArgs& a, const Plan& p, hipStream_t s)
{
    wgrad_kernel<S, T, EDGE><<<dim3((uint32_t)(p.whole + p.rest * p.split)), dim3(S::kThreads), 0, s>>>(a);
    if (p.rest) join_kernel<S, EDGE><<<dim3((uint32_t)(p.rest * S::kTM * S::kTN * S::kPieces)), dim3(S::kThreads), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}
template <class T>
int launch(const WgradArgs& a, const Plan& p, hipStream_t s)
{
    // 32 rows are not within 32 bits, or less than a tile
    const bool edge = a.ld_d >= (int64_t)1 << 24 || a.ld >= 1 << 26 || a.n_out < p.bm || a.ld < p.bn;
    if constexpr (sizeof(T) == 2) {
        if (p.bm == 256) return edge ? launch<Tile<T, 256, 256, 2, 4, 16>, T, true>(a, p, s) : launch<Tile<T, 256, 256, 2, 4, 16>, T, false>(a, p, s);
    } else {
        if (p.bn == 256) return edge ? launch<Tile<T, 128, 256, 2, 4, 32>, T, true>(a, p, s) : launch<Tile<T, 128, 256, 2, 4, 32>, T, false>(a, p, s);
    }
    return edge ? launch<Tile<T, 128, 128, 2, 2, 32>, T, true>(a, p, s) : launch<Tile<T, 128, 128, 2, 2, 32>, T, false>(a, p, s);
}

}  // namespace
}  // namespace adagc

using namespace adagc;

extern "C" int64_t adagc_act8_wgrad_workspace_bytes(int64_t rows, int64_t n_out, int64_t n_in, int32_t dtype)
{
    if (const int rc = check(rows, n_out, n_in, dtype)) return rc;
    const Plan p = plan_of(rows, n_out, n_in, dtype);
    return p.launchable() ? p.workspace() : (int64_t)ADAGC_ERR_TOO_LARGE;
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
    if (!p.launchable()) return ADAGC_ERR_TOO_LARGE;
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
    a.weight_bf16 = weight_dtype == ADAGC_BF16;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return dtype == ADAGC_F32 ? launch<float>(a, p, s) : launch<uint16_t>(a, p, s);
}
