// The tile loop of the matrix products behind the operators that make their intermediate results again instead of keeping them
// (linear_logprobs.hip, gated_linear.hip), and a product with a plain result.
//
// A block tile's sums  acc[row][col] += sum_k Y[row][k] X[col][k]  on the matrix cores, fp32 accumulation.  Each operand lies in memory
// either with k consecutive ("along": rows of k) or with k as the slow index ("across": k rows of consecutive rows or columns of the
// result).  bf16 products are exact in fp32; fp32 operands go through the matrix cores' fp32 instruction, or, for more rows, are three bf16
// numbers each (kSegments below).
//
// What bounds it, bf16: of large products the power limit (a step of 32 k on a 256-tile 0.72 - 0.75 us at some 1.8 GHz, 0.55 if the matrix cores never
// waited) and what a tile takes beside its steps, 8 - 10 us of which the next tile's first loads hide a part.  4096 x 128256 from 4096, both along:
// 3050 - 3240 us, 1330 - 1410 TFLOP/s (a library product of this shape 1452); 16384 x 4096 from 4096, both across: 404 - 432 us, 1270 - 1360 (1007);
// 4096 x 4096 from 16384, one across: 382 - 406 us, 1350 - 1440 (1166).  Of the small tile what it loads from the L2s, some 8.4 TB/s.
#ifndef ADAGC_PRODUCT_DEVICE_H
#define ADAGC_PRODUCT_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>
#include <utility>

#include "operators_internal.h"

namespace adagc {

typedef __bf16 bf16x8_p __attribute__((ext_vector_type(8)));
typedef float f32x4_p __attribute__((ext_vector_type(4)));
typedef short s16x4_p __attribute__((ext_vector_type(4)));

namespace product {

#define ADAGC_P_LDS __attribute__((address_space(3)))
// s_waitcnt for "at most n vector-memory operations of this wave still outstanding", nothing else waited for
#define ADAGC_P_WAIT_VMEM(n) __builtin_amdgcn_s_waitcnt(((n) & 0xF) | (((n) >> 4) << 14) | (7 << 4) | (0xF << 8))
// s_waitcnt for "at most n LDS accesses of this wave still outstanding", nothing else waited for
#define ADAGC_P_WAIT_LDS(n) __builtin_amdgcn_s_waitcnt(0xF | (3 << 14) | (7 << 4) | ((n) << 8))
// nothing is moved across this point by the compiler's instruction scheduler
#define ADAGC_P_FENCE() __builtin_amdgcn_sched_barrier(0)

// f(integral_constant 0), ..., f(integral_constant N-1)
template <class F, int... I>
__device__ __forceinline__ void each_impl(F&& f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F&& f)
{
    each_impl(f, std::make_integer_sequence<int, N>{});
}

// Compute units: a round of a launch is as many workgroups of the large tile.
constexpr int kUnits = 256;
constexpr int kPlaces = 3;                 // of LDS, that steps staged through registers go round in
constexpr int kStepBytes = 64;             // of k, a step

// BM x BN tile (BM rows of Y), kWM x kWN waves of kTM x kTN blocks of 16 x 16.  A step is 64 bytes of k: 32 bf16 or 16 fp32 numbers, so that
// an operand's tile has the same bytes and a lane's fragment the same 16 with both types.  RING: operands go from global memory straight into LDS,
// into a ring of so many places, which wants rows at multiples of 16 bytes; 0: through registers, rows at any element.
template <class T, int BM_, int BN_, int kWM_, int kWN_, int RING_>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, kWM = kWM_, kWN = kWN_;
    static constexpr int kThreads = 64 * kWM * kWN;
    static constexpr int kTM = BM / kWM / 16, kTN = BN / kWN / 16;
    static constexpr int kDeep = kStepBytes / (int)sizeof(T);
    static constexpr int kY = BM * kStepBytes, kX = BN * kStepBytes, kPlace = kY + kX;      // bytes
    static constexpr int kYUnits = kY / 16 / kThreads, kXUnits = kX / 16 / kThreads;       // of 16 bytes, a lane's
    static constexpr bool kDirect = RING_ > 0;
    static constexpr bool kEven = RING_ % 2 == 0;
    static constexpr int kRing = RING_, kAhead = RING_ / 2;                                // places of the ring; pairs of steps that loads are ahead
    static constexpr int kYLoads = 2 * kYUnits, kXLoads = 2 * kXUnits;                     // straight into LDS, of two steps, a lane's
    static constexpr int kLds = (RING_ ? RING_ : kPlaces) * kPlace;
    static_assert(!RING_ || (BM_ == BN_ && RING_ >= 5), "a place of the ring takes either operand, X and Y in turn");
    static_assert(kY % (16 * kThreads) == 0 && kX % (16 * kThreads) == 0, "operand tiles are dealt evenly");
};

// 16 bytes per lane from global memory straight into LDS: lane i's, at base + off_i bytes (base: the same in all lanes), land at
// lds_at + 16 i (the same in all lanes).  The instruction takes the LDS address from M0 and wants a wait state after M0 is written; M0 is put
// back afterwards.  Inline assembly rather than the compiler's builtin so that the compiler does not track these loads: it would turn every wait
// for an LDS read into a wait for all of them.  The waits for these loads are explicit (ADAGC_P_WAIT_VMEM) wherever their data is needed.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t lds_at)
{
    uint32_t saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved_m0)
                 : "s"(lds_at), "v"(off), "s"(base)
                 : "memory");
}

// The thread's number, where what follows from it is made anew instead of being kept through a main loop, which leaves no registers for that.
__device__ __forceinline__ int thread_anew()
{
    int t = (int)threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// Values that were loaded are waited for here, not where they are used: by then younger loads may be on their way, which the wait would take in.
template <class V, int N>
__device__ __forceinline__ void settle_now(V (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// A value that is the same in all lanes, in scalar registers.
__device__ __forceinline__ int64_t scalar(int64_t v)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
template <class T>
__device__ __forceinline__ const T* scalar(const T* p)
{
    return reinterpret_cast<const T*>(scalar((int64_t)reinterpret_cast<uintptr_t>(p)));
}

// Number n of a launch of tiles_m x tiles_n: 8 XCDs, each with its own L2, get workgroups in turn; the 32 that one of them has in a round are
// neighbours, in bands of 8 tiles along m.
__device__ __forceinline__ void place_of_tile(int n, int tiles_m, int tiles_n, int* tm, int* tn)
{
    const int all = tiles_m * tiles_n, round = n / kUnits * kUnits, in_round = min(all - round, kUnits);
    int at = n - round;
    if (in_round == kUnits) at = at % 8 * (kUnits / 8) + at / 8;
    at += round;
    const int band = at / (8 * tiles_n), in_band = at - band * 8 * tiles_n;
    const int high = min(8, tiles_m - 8 * band);
    *tn = __builtin_amdgcn_readfirstlane(in_band / high);          // the same in all lanes: kept in scalar registers
    *tm = __builtin_amdgcn_readfirstlane(8 * band + in_band - *tn * high);
}

// fp32 operands in three bf16 parts, hi + mid + lo, each the nearest to what the ones before it leave (8 + 8 + 8 significant bits, exact but
// next to the type's ends): of the nine products of parts the six that count, smallest first; the others are some 2^-26 of the whole.  The
// matrix cores' bf16 rate is 16 times the fp32 one.  Segments: products that are summed, one of operands as they are, or these.
constexpr int kSegments = 6, kParts = 3;

// How one operand's tile (B rows or columns of the result) is loaded, staged in LDS and read: kUnits units of 16 bytes a step for a lane.
//
// Along: LDS rows of a step's 64 bytes (DIRECT: of two steps' 128), one for a row of the result.  The 16-byte vector v of row r is at position
// v ^ f((r / 4) mod 4), f = 0, 3, 2, 1 (DIRECT: v ^ ((r / 2) mod 8)): the 16 lanes that read at a time (vector v of rows 0 .. 3 and 12 .. 15
// with v ^ 1 of rows 4 .. 11) so meet different banks.  (With f = 0, 1, 2, 3, which separates 16 rows of one vector, half of the LDS
// cycles were conflicts.)
// Across, bf16: LDS rows of B numbers, one for each k; 16 lanes read 4 rows of 16 columns and get a column each (ds_read_b64_tr_b16); the
// 32-byte units of a row are permuted so that the eight that half a wave takes (rows 0 .. 3 and 8 .. 11) lie in different banks.
// Across, fp32: the same with 64-byte units, read number by number.
template <class T, int B, int kThreads, int kUnits, int kBlocks, bool ACROSS, bool DIRECT>
struct Side {
    static constexpr int kE = 16 / (int)sizeof(T);                 // numbers in a vector
    static constexpr int kDeep = kStepBytes / (int)sizeof(T);
    static constexpr int kVectors = ACROSS ? B / kE : 4;            // of a row and a step
    static constexpr int kPitch = ACROSS ? B * (int)sizeof(T) : DIRECT ? 2 * kStepBytes : kStepBytes;      // bytes of a row in LDS
    static constexpr bool kHalf = sizeof(T) == 2;
    static_assert(!DIRECT || kHalf);

    const T* row[ACROSS ? 1 : kUnits];     // along: a unit's address at k = 0, less its vector
    uint32_t lane_at;                      // across: bytes from the step's address, unit 0
    int64_t  ld;
    uint32_t write_at, read_at;

    static __device__ __forceinline__ int row_of(int tid, int u) { return (tid + u * kThreads) / kVectors; }
    static __device__ __forceinline__ int vector_of(int tid, int u) { return (tid + u * kThreads) % kVectors; }
    static __device__ __forceinline__ uint32_t place(int r, int v)
    {
        if constexpr (!ACROSS && DIRECT) return (uint32_t)(r * kPitch + (v ^ ((r >> 1) & 7)) * 16);
        else if constexpr (!ACROSS) return (uint32_t)(r * kPitch + (v ^ ((r >> 2) & 3) ^ ((r >> 1) & 2)) * 16);
        else if constexpr (kHalf) return (uint32_t)(r * kPitch + ((v >> 1) ^ ((r & 3) | ((r >> 3) & 1) << 2)) * 32 + (v & 1) * 16);
        else return (uint32_t)(r * kPitch + ((v >> 2) ^ ((r >> 2) & 3)) * 64 + (v & 3) * 16);
    }
    // lds0: the first byte of the tile's place, wave_block: the wave's first block
    __device__ __forceinline__ void set_places(int tid, uint32_t lds0, int wave_block)
    {
        write_at = lds0 + place(row_of(tid, 0), vector_of(tid, 0));
        const int l = tid & 63;
        if constexpr (!ACROSS) {
            read_at = lds0 + place(l & 15, l >> 4) + (uint32_t)(wave_block * 16 * kPitch);
        } else if constexpr (kHalf) {
            const int r = 8 * (l >> 4) + ((l >> 2) & 3);
            read_at = lds0 + (uint32_t)(r * kPitch + (wave_block ^ ((r & 3) | ((r >> 3) & 1) << 2)) * 32 + (l & 3) * 8);
        } else {
            const int r = 4 * (l >> 4);
            read_at = lds0 + (uint32_t)(r * kPitch + (wave_block ^ ((r >> 2) & 3)) * 64 + (l & 15) * 4);
        }
    }

    // ---- through registers
    // along: row_at(r): the address of row r of the tile (rows beyond the matrix: any of its rows)
    template <class F>
    __device__ __forceinline__ void set_rows(int tid, F&& row_at)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) row[u] = row_at(row_of(tid, u)) + vector_of(tid, u) * kE;
    }
    // across: k rows from `at` on, B whole columns of them inside the matrix, kDeep * ld_ numbers within 32 bits of bytes
    __device__ __forceinline__ void set_columns(int tid, const T* at, int64_t ld_)
    {
        row[0] = at;
        ld = ld_;
        lane_at = (uint32_t)(row_of(tid, 0) * (uint32_t)ld_ + (uint32_t)vector_of(tid, 0) * kE) * (uint32_t)sizeof(T);
    }
    __device__ __forceinline__ u32x4 load(int64_t step, int u) const
    {
        if constexpr (!ACROSS) {
            return load_whole(row[u] + step * kDeep).w;
        } else {
            const uint8_t* at = reinterpret_cast<const uint8_t*>(row[0] + (step * kDeep + u * (kThreads / kVectors)) * ld);
            return load_whole(reinterpret_cast<const T*>(at + lane_at)).w;
        }
    }
    // the same where k or (across) the columns may end inside: zeros there
    __device__ __forceinline__ u32x4 load_checked(int tid, int64_t step, int u, int64_t k, int64_t columns) const
    {
        if constexpr (!ACROSS) {
            const int v = vector_of(tid, u);
            return load_vector(row[u] - v * kE, step * kDeep + v * kE, k, 0).w;
        } else {
            const int64_t t = step * kDeep + row_of(tid, u);
            return load_vector(row[0] + t * ld, vector_of(tid, u) * kE, t < k ? columns : 0, 0).w;
        }
    }
    __device__ __forceinline__ void write(int u, uint32_t place, const u32x4& w) const
    {
        // a unit's rows are kRows below the last one's: at the same place of the permutation but for fp32 across, where 8 rows flip a bit of it
        constexpr int kRows = kThreads / kVectors;
        static_assert(kRows % 16 == 0 || (ACROSS && !kHalf && kRows == 8 && kUnits <= 2), "the permutation of a unit's rows");
        const uint32_t at = kRows % 16 && u ? write_at ^ 128u : write_at;
        *reinterpret_cast<ADAGC_P_LDS u32x4*>(at + place + (uint32_t)(u * kRows * kPitch)) = w;
    }

    // ---- straight into LDS, two steps at a time: a lane's kLoads vectors, kAlong of a row
    static constexpr int kLoads = 2 * kUnits, kAlong = ACROSS ? kVectors : 8;
    uint32_t off[ACROSS ? 1 : kLoads];     // bytes from the first step's address, which is the same in all lanes
    const T* base;
    // the next pair of steps to load, and the first one
    const T* at;
    int      first;
    int64_t  part;

    // Position i of row r gets vector unplaced(r, i), so that vector v is where place(r, v) says (its own inverse).
    static __device__ __forceinline__ int unplaced(int r, int i) { return (int)(place(r, i) % (uint32_t)kPitch) / 16; }
    // along: rows of one matrix within 32 bits of bytes from `at`; number_of(r): the number of row r of the tile, from `at` (a row inside the matrix)
    template <class F>
    __device__ __forceinline__ void set_rows_direct(int tid, const T* at, int64_t ld_, F&& number_of)
    {
        base = scalar(at);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int i = tid + u * kThreads, r = i / kAlong;
            off[u] = ((uint32_t)number_of(r) * (uint32_t)ld_ + (uint32_t)unplaced(r, i % kAlong) * kE) * (uint32_t)sizeof(T);
        }
    }
    __device__ __forceinline__ void set_columns_direct(int tid, const T* at, int64_t ld_)
    {
        base = scalar(at);
        ld = scalar(ld_);
        const int r = tid / kAlong;
        off[0] = ((uint32_t)r * (uint32_t)ld_ + (uint32_t)unplaced(r, tid % kAlong) * kE) * (uint32_t)sizeof(T);
    }
    // first_: of the pairs of steps; part_: operands in parts: elements from part to part
    __device__ __forceinline__ void set_first(int first_, int64_t part_)
    {
        first = first_;
        part = part_;
        at = part_at(0, 0);
    }
    __device__ __forceinline__ void load_direct(int u, uint32_t lds_at) const
    {
        constexpr int kRows = kThreads / kAlong;       // of a load, across: the permutation repeats after 16
        static_assert(!ACROSS || kRows % 16 == 0);
        if constexpr (ACROSS) load_to_lds(at + (int64_t)(u * kRows) * ld, off[0], lds_at + (uint32_t)(u * kThreads * 16));
        else load_to_lds(at, off[u], lds_at + (uint32_t)(u * kThreads * 16));
    }
    __device__ __forceinline__ void advance() { at += ACROSS ? 2 * kDeep * ld : (int64_t)(2 * kDeep); }

    // the same for part p of operands in parts, pair of steps d from the first one on
    __device__ __forceinline__ const T* part_at(int p, int d) const
    {
        return base + p * part + (int64_t)(first + d) * (2 * kDeep) * (ACROSS ? ld : 1);
    }
    __device__ __forceinline__ void load_part(const T* from, int u, uint32_t lds_at) const
    {
        if constexpr (ACROSS) load_to_lds(from + (int64_t)(u * (kThreads / kAlong)) * ld, off[0], lds_at + (uint32_t)(u * kThreads * 16));
        else load_to_lds(from, off[u], lds_at + (uint32_t)(u * kThreads * 16));
    }

    // second: of two steps in a place
    __device__ __forceinline__ u32x4 read(int block, uint32_t place, bool second = false) const
    {
        if constexpr (!ACROSS) {
            const uint32_t at = DIRECT && second ? read_at ^ 64u : read_at;
            return *reinterpret_cast<const ADAGC_P_LDS u32x4*>(at + place + (uint32_t)(block * 16 * kPitch));
        } else if constexpr (kHalf) {
            static_assert((kBlocks & (kBlocks - 1)) == 0, "blocks are exclusive-ored into an address");
            const uint32_t at = (read_at ^ (uint32_t)(block * 32)) + place + (second ? kDeep * kPitch : 0);
            const s16x4_p a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ADAGC_P_LDS s16x4_p*>(at));
            const s16x4_p b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ADAGC_P_LDS s16x4_p*>(at + 4 * kPitch));
            return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const uint32_t at = (read_at ^ (uint32_t)(block * 64)) + place;
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const ADAGC_P_LDS uint32_t*>(at + (uint32_t)(j * kPitch));
            return w;
        }
    }
};

// sum += x y^T of one block: lane l gets columns 4 (l / 16) .. + 3 of row l mod 16.
template <class T>
__device__ __forceinline__ void multiply(const u32x4& x, const u32x4& y, f32x4_p& sum)
{
    if constexpr (sizeof(T) == 2) {
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_p, x), __builtin_bit_cast(bf16x8_p, y), sum, 0, 0, 0);
    } else {
        // four k of every four: both operands give the same ones
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[j]), __uint_as_float(y[j]), sum, 0, 0, 0);
    }
}

template <class S>
using Sums = f32x4_p[S::kTM][S::kTN];

template <class S>
__device__ __forceinline__ void clear(Sums<S>& acc)
{
#pragma unroll
    for (int m = 0; m < S::kTM; ++m)
#pragma unroll
        for (int n = 0; n < S::kTN; ++n) acc[m][n] = f32x4_p{0.f, 0.f, 0.f, 0.f};
}

// Steps step0 .. step1 - 1 of k, and with `rest` the numbers after the last whole step (number `full`).  CHECKED: every load looks where the
// operands end.
//
// Main loop.  A step's operands are staged in a place of LDS; while step i is multiplied from registers, step i + 1 is read to registers
// from its place (each fragment of Y as soon as its multiplications are issued, those of X to a second set), step i + 2 goes from the
// registers it was loaded to into its place, and those take step i + 4.  One barrier a step: what it orders is the writes of i + 2
// before their reads in the next step; the reads of a place are done a step before it is written again.  Loads past the last step take
// the last one again: a loop without conditions lets the compiler count what is outstanding.  All waves leave with LDS free to use.
template <class S, class T, bool CHECKED, class SideY, class SideX>
__device__ __forceinline__ void accumulate(Sums<S>& acc, const SideY& sy, const SideX& sx, int64_t step0, int64_t step1, bool rest, int64_t full,
                                           int64_t k, int64_t columns_y, int64_t columns_x)
{
    constexpr int kTM = S::kTM, kTN = S::kTN, kYU = S::kYUnits, kXU = S::kXUnits;
    const int tid = threadIdx.x;
    struct Staged {
        u32x4 y[kYU], x[kXU];
    };
    auto load = [&](int64_t step, Staged& s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kYU; ++u) s.y[u] = sy.load(step, u);
#pragma unroll
        for (int u = 0; u < kXU; ++u) s.x[u] = sx.load(step, u);
    };
    auto load_checked = [&](int64_t step, Staged& s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kYU; ++u) s.y[u] = sy.load_checked(tid, step, u, k, columns_y);
#pragma unroll
        for (int u = 0; u < kXU; ++u) s.x[u] = sx.load_checked(tid, step, u, k, columns_x);
    };
    auto write = [&](const Staged& s, uint32_t place) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kYU; ++u) sy.write(u, place, s.y[u]);
#pragma unroll
        for (int u = 0; u < kXU; ++u) sx.write(u, place, s.x[u]);
    };
    u32x4 y[kTM], x[2][kTN];
    auto plain_step = [&](const Staged& s, uint32_t place, auto&& meanwhile) __attribute__((always_inline)) {
        write(s, place);
        meanwhile();
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kTN; ++n) x[0][n] = sx.read(n, place);
#pragma unroll
        for (int m = 0; m < kTM; ++m) {
            y[0] = sy.read(m, place);
#pragma unroll
            for (int n = 0; n < kTN; ++n) multiply<T>(x[0][n], y[0], acc[m][n]);
        }
    };
    constexpr uint32_t kRestPlace = (kPlaces - 1) * S::kPlace;

    if constexpr (CHECKED) {
        // two steps' loads are on their way; a step's writes and the reads of the step before take different places
        const int64_t end = step1 + rest;
        Staged staged[2];
        if (step0 < end) load_checked(step0, staged[0]);
        if (step0 + 1 < end) load_checked(step0 + 1, staged[1]);
        for (int64_t step = step0; step < end; step += 2)
            each<2>([&](auto P) __attribute__((always_inline)) {
                constexpr int p = decltype(P)::value;
                if (step + p >= end) return;
                plain_step(staged[p], p * S::kPlace, [&] {
                    if (step + p + 2 < end) load_checked(step + p + 2, staged[p]);
                });
            });
    } else if (step0 == step1) {
        if (rest) {
            Staged s;
            load_checked(full, s);
            plain_step(s, kRestPlace, [] {});
        }
    } else {
        // what is left over comes first (with the main loop's first loads on their way at the same time registers would be short)
        Staged staged[2];
        auto clamp = [&](int64_t step) { return min(step, step1 - 1); };
        if (rest) {
            load_checked(full, staged[0]);
            plain_step(staged[0], kRestPlace, [] {});
            ADAGC_P_FENCE();
        }
        load(step0, staged[0]);
        load(clamp(step0 + 1), staged[1]);
        write(staged[0], 0);
        load(clamp(step0 + 2), staged[0]);
        write(staged[1], S::kPlace);
        load(clamp(step0 + 3), staged[1]);
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kTN; ++n) x[0][n] = sx.read(n, 0);
#pragma unroll
        for (int m = 0; m < kTM; ++m) y[m] = sy.read(m, 0);
        uint32_t next = S::kPlace;                 // the place of step i + 1
        auto after = [](uint32_t place) { return place == (kPlaces - 1) * S::kPlace ? 0u : place + S::kPlace; };
        auto one_step = [&](auto PARITY, int64_t step) __attribute__((always_inline)) {
            constexpr int p = decltype(PARITY)::value;
            constexpr int kSlots = kTM * kTN, kMoves = kYU + kXU;
            const uint32_t to_place = after(next);
            const int64_t ahead = clamp(step + 4);
            each<kSlots>([&](auto SLOT) __attribute__((always_inline)) {
                constexpr int slot = decltype(SLOT)::value, m = slot / kTN, n = slot % kTN;
                multiply<T>(x[p][n], y[m], acc[m][n]);
                ADAGC_P_FENCE();
                if constexpr (slot % 2 == 0 && slot / 2 < kTN) x[p ^ 1][slot / 2] = sx.read(slot / 2, next);
                if constexpr (n == kTN - 1) y[m] = sy.read(m, next);
                each<kMoves>([&](auto N) __attribute__((always_inline)) {
                    constexpr int w = decltype(N)::value;
                    constexpr int kLate = kSlots >= 16 ? 1 : 0;
                    if constexpr (kSlots / 4 + w * (kSlots / 4) / kMoves + kLate == slot) {
                        if constexpr (w < kYU) sy.write(w, to_place, staged[p].y[w]);
                        else sx.write(w - kYU, to_place, staged[p].x[w - kYU]);
                    }
                    if constexpr (kSlots / 2 + w * (kSlots / 4) / kMoves + 1 + kLate == slot) {
                        if constexpr (w < kYU) staged[p].y[w] = sy.load(ahead, w);
                        else staged[p].x[w - kYU] = sx.load(ahead, w - kYU);
                    }
                });
                ADAGC_P_FENCE();
            });
            // the writes, in the first half of the step, are done; the fragments read since (one access each at least) may still be on their way
            ADAGC_P_WAIT_LDS(kTM / 2 - 1);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            ADAGC_P_FENCE();
            next = to_place;
        };
        int64_t step = step0;
        for (; step + 1 < step1; step += 2) {
            one_step(std::integral_constant<int, 0>{}, step);
            one_step(std::integral_constant<int, 1>{}, step + 1);
        }
        if (step < step1) one_step(std::integral_constant<int, 0>{}, step);
    }
    __syncthreads();
}

// What is left over after `first` steps, a step at a time: for the tiles whose whole pairs of steps go straight into LDS.
template <class S, class T, class SideY, class SideX>
__device__ __forceinline__ void accumulate_rest(Sums<S>& acc, const SideY& sy, const SideX& sx, int64_t first, int64_t k, int64_t columns_y, int64_t columns_x)
{
    const int tid = thread_anew();
    constexpr uint32_t kXPlace = S::kXLoads * S::kThreads * 16;            // the next place of the ring
    for (int64_t step = first; step * S::kDeep < k; ++step) {
        u32x4 w[S::kYUnits + S::kXUnits];
#pragma unroll
        for (int u = 0; u < S::kYUnits; ++u) w[u] = sy.load_checked(tid, step, u, k, columns_y);
#pragma unroll
        for (int u = 0; u < S::kXUnits; ++u) w[S::kYUnits + u] = sx.load_checked(tid, step, u, k, columns_x);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < S::kYUnits; ++u) sy.write(u, 0, w[u]);
#pragma unroll
        for (int u = 0; u < S::kXUnits; ++u) sx.write(u, kXPlace, w[S::kYUnits + u]);
        __syncthreads();
        u32x4 x[S::kTN];
#pragma unroll
        for (int n = 0; n < S::kTN; ++n) x[n] = sx.read(n, kXPlace);
#pragma unroll
        for (int m = 0; m < S::kTM; ++m) {
            const u32x4 y = sy.read(m, 0);
#pragma unroll
            for (int n = 0; n < S::kTN; ++n) multiply<T>(x[n], y, acc[m][n]);
        }
    }
    __syncthreads();
}

// Pairs of steps with operands that go straight into LDS, into a ring of places.  A place holds one operand's tile of two
// steps, so that a row along k is loaded 128 bytes at a time: with the 64 of one step the L2s had twice the requests.
//
// While a step is multiplied from registers, the next one is read to registers.  In the first step of pair d the X of pair d + kAhead is
// loaded into the place of the Y of pair d - 1, in the second its Y into the place of the X of pair d.  What a place held before has been read by then: the
// Y were waited for by the multiplications before the last barrier, and the X, which are read first, by a wait for all but the later LDS
// reads.  With five places a load has one and a half or two and a half steps to arrive.
//
// An even number of places, for tiles with registers to spare: fragments of Y too are read to a second set, early in the step, and waited for before
// the waves meet, which they do once a pair.  In the second step of pair d the X of pair d + kAhead is loaded into the place of its own X, in the
// first step of pair d + 1 the Y into that of its Y.
//
// A workgroup with a ring has its compute unit for itself: it stays, and starts the next tile's first loads before it deals with the
// results of the last one, for which the last place of the ring is free meanwhile.
template <class S, class SideY, class SideX>
__device__ __forceinline__ void start_direct(SideY& sy, SideX& sx, uint32_t lds0, int total)
{
    const uint32_t lds_wave = lds0 + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 1024u;
#pragma unroll
    for (int d = 0; d < S::kAhead; ++d)
        if (d < total) {
#pragma unroll
            for (int u = 0; u < S::kXLoads; ++u) sx.load_direct(u, lds_wave + 2 * d * S::kPlace);
            sx.advance();
            if (S::kEven && d == S::kAhead - 1) continue;
#pragma unroll
            for (int u = 0; u < S::kYLoads; ++u) sy.load_direct(u, lds_wave + (2 * d + 1) * S::kPlace);
            sy.advance();
        }
}

// total: pairs of steps
template <class S, class T, class SideY, class SideX>
__device__ __forceinline__ void accumulate_direct(Sums<S>& acc, SideY& sy, SideX& sx, uint32_t lds0, int total)
{
    constexpr int kTM = S::kTM, kTN = S::kTN, kLoads = S::kYLoads, kSize = S::kPlace, kEnd = S::kRing * kSize, kAhead = S::kAhead;      // kSize: one operand, two steps
    static_assert(S::kYLoads == S::kXLoads && kLoads * S::kThreads * 16 == kSize);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const uint32_t lds_wave = lds0 + (uint32_t)wave * 1024u;
    if (total <= 0) return;
    auto meet = []() __attribute__((always_inline)) {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        ADAGC_P_FENCE();
    };
    auto later = [](uint32_t place, int n) { return place + (uint32_t)(n * kSize) >= (uint32_t)kEnd ? place + (uint32_t)(n * kSize) - kEnd : place + (uint32_t)(n * kSize); };
    // all but the loads of so many pairs, fewer than kAhead, are there
    auto wait_but = [](int pairs) __attribute__((always_inline)) {
        if (kAhead > 4 && pairs >= 4) ADAGC_P_WAIT_VMEM(8 * kLoads);
        else if (kAhead > 3 && pairs >= 3) ADAGC_P_WAIT_VMEM(6 * kLoads);
        else if (kAhead > 2 && pairs >= 2) ADAGC_P_WAIT_VMEM(4 * kLoads);
        else if (pairs >= 1) ADAGC_P_WAIT_VMEM(2 * kLoads);
        else ADAGC_P_WAIT_VMEM(0);
    };
    static_assert(kAhead <= 5);
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> odd{};
    uint32_t here = 0;                             // the place of X of pair d; its Y's is the next one
    int d = 0;
    if constexpr (S::kEven) {
        u32x4 y[2][kTM], x[2][kTN];
        // (results stored since the loads were started are waited for too: they are younger)
        wait_but(min(total, kAhead - 1) - 1);
        meet();
#pragma unroll
        for (int n = 0; n < kTN; ++n) x[0][n] = sx.read(n, 0);
#pragma unroll
        for (int m = 0; m < kTM; ++m) y[0][m] = sy.read(m, kSize);
        // LOAD: there is something left to load
        auto one_step = [&](auto SECOND, auto LOAD, int d) __attribute__((always_inline)) {
            constexpr int second = decltype(SECOND)::value;
            constexpr int kSlots = kTM * kTN, kReads = kTM + kTN;
            // of the step that is read: the second one of pair d, the first one of pair d + 1
            const uint32_t from_x = second ? later(here, 2) : here, from_y = later(here, second ? 3 : 1);
            const uint32_t to = second ? here : later(here, 2 * kAhead - 1);
            each<kSlots>([&](auto SLOT) __attribute__((always_inline)) {
                constexpr int slot = decltype(SLOT)::value, m = slot / kTN, n = slot % kTN;
                multiply<T>(x[second][n], y[second][m], acc[m][n]);
                ADAGC_P_FENCE();
                each<kReads>([&](auto R) __attribute__((always_inline)) {
                    constexpr int r = decltype(R)::value;
                    if constexpr (r * (kSlots / 2) / kReads == slot) {
                        if constexpr (r < kTN) x[second ^ 1][r] = sx.read(r, from_x, !second);
                        else y[second ^ 1][r - kTN] = sy.read(r - kTN, from_y, !second);
                    }
                });
                if constexpr (decltype(LOAD)::value) {
                    each<kLoads>([&](auto N) __attribute__((always_inline)) {
                        constexpr int u = decltype(N)::value;
                        if constexpr (kSlots / 2 + u * (kSlots / 2) / kLoads == slot) {
                            if constexpr (second) sx.load_direct(u, lds_wave + to);
                            else sy.load_direct(u, lds_wave + to);
                            if constexpr (u == kLoads - 1) {
                                if constexpr (second) sx.advance();
                                else sy.advance();
                            }
                        }
                    });
                }
                ADAGC_P_FENCE();
            });
            if constexpr (!second) {
                // pair d + 1 has to be there, and pair d read
                if constexpr (decltype(LOAD)::value) ADAGC_P_WAIT_VMEM(2 * (kAhead - 2) * kLoads);
                else wait_but(total - 2 - d);
                ADAGC_P_WAIT_LDS(0);
                meet();
            }
        };
        for (; d + kAhead < total; ++d) {
            one_step(even, std::true_type{}, d);
            one_step(odd, std::true_type{}, d);
            here = later(here, 2);
        }
        if (d + kAhead == total) {                 // the last Y
            one_step(even, std::true_type{}, d);
            one_step(odd, std::false_type{}, d);
            here = later(here, 2);
            ++d;
        }
        for (; d < total; ++d) {
            one_step(even, std::false_type{}, d);
            one_step(odd, std::false_type{}, d);
            here = later(here, 2);
        }
        __syncthreads();
        return;
    }
    u32x4 y[kTM], x[2][kTN];
    wait_but(min(total, kAhead) - 1);
    meet();
#pragma unroll
    for (int n = 0; n < kTN; ++n) x[0][n] = sx.read(n, 0);
#pragma unroll
    for (int m = 0; m < kTM; ++m) y[m] = sy.read(m, kSize);
    auto one_step = [&](auto SECOND, auto MORE, int d) __attribute__((always_inline)) {
        constexpr int second = decltype(SECOND)::value;
        constexpr bool more = decltype(MORE)::value;       // pair d + kAhead exists
        constexpr int kSlots = kTM * kTN;
        // of the step that is read: the second one of pair d, the first one of pair d + 1
        const uint32_t from_x = second ? later(here, 2) : here, from_y = later(here, second ? 3 : 1);
        const uint32_t to = second ? here : later(here, 2 * kAhead);
        each<kSlots>([&](auto SLOT) __attribute__((always_inline)) {
            constexpr int slot = decltype(SLOT)::value, m = slot / kTN, n = slot % kTN;
            multiply<T>(x[second][n], y[m], acc[m][n]);
            ADAGC_P_FENCE();
            if constexpr (slot % 2 == 0 && slot / 2 < kTN) x[second ^ 1][slot / 2] = sx.read(slot / 2, from_x, !second);
            if constexpr (n == kTN - 1) y[m] = sy.read(m, from_y, !second);
            if constexpr (more) {
                each<kLoads>([&](auto N) __attribute__((always_inline)) {
                    constexpr int u = decltype(N)::value;
                    if constexpr (1 + u * kSlots / kLoads == slot) {
                        if constexpr (second) sy.load_direct(u, lds_wave + to);
                        else sx.load_direct(u, lds_wave + to);
                        if constexpr (u == kLoads - 1) {
                            if constexpr (second) sy.advance();
                            else sx.advance();
                        }
                    }
                });
            }
            ADAGC_P_FENCE();
        });
        if constexpr (!second) {
            // pair d + 1 has to be there, and X of pair d read: kTM - 1 fragments of Y, one access each at least, are read after it
            if constexpr (more) ADAGC_P_WAIT_VMEM((2 * kAhead - 3) * kLoads);
            else wait_but(total - 2 - d);
            ADAGC_P_WAIT_LDS(kTM - 1);
        }
        meet();
    };
    for (; d + kAhead < total; ++d) {
        one_step(even, std::true_type{}, d);
        one_step(odd, std::true_type{}, d);
        here = later(here, 2);
    }
    // the fragments of the step after the last one are read from some place of the ring and not used
    for (; d < total; ++d) {
        one_step(even, std::false_type{}, d);
        one_step(odd, std::false_type{}, d);
        here = later(here, 2);
    }
    __syncthreads();
}

// Operands in three parts, with a ring of ten places: of a pair of steps' six tiles, loaded once, all six products of the first step, then all of the
// second, in an order in which each takes over an operand of the one before, in registers: 18 fragments read for six products instead of 36.
// (The products one after the other over all of k, 192 tiles of 765 numbers, were bound by the loads, 55 us; a pair's products two steps each, by
// the reads from LDS, 39, and 40 with both operands across k; now 38 and 35.)
// The large tile's ring does not hold six tiles: with twelve loaded for six products, 597 rows, 2 x 11373 from 4096 and back took 3440 us, now 2810;
// 300 x 128256 from 1024 906, now 756; 512 x 32000 from 1024 205, now 213.
//
// Tile u of pair c, in the order y lo, x hi, y mid, x mid, y hi, x lo, is in place 6 c + u (mod 10), and gives it to the tile ten later.  Step k of six
// multiplies (y lo, x hi), (y mid, x hi), (y mid, x mid), (y hi, x mid), (y hi, x lo), (y hi, x hi); what the next one needs is read meanwhile.  Waves
// meet three times in a pair's twelve steps: after step 5, when y lo and x hi have been read for the last time, their places are loaded, with y hi and x lo of
// the next pair; after step 9 the other four, with the first four tiles of the pair after it; the first time after step 1, when this pair's y hi and x lo
// have to be there, six steps after their loads.  What is loaded past the last pair is the last pair again: every wait counts the same loads.
struct PartsOrder {
    static constexpr int part[6] = {2, 0, 1, 1, 0, 2};                     // of a tile
    static constexpr bool is_y[6] = {true, false, true, false, true, false};
};
template <class S, int TILE, class SideY, class SideX>
__device__ __forceinline__ void load_tile(const SideY& sy, const SideX& sx, int d, uint32_t lds_at)
{
    if constexpr (PartsOrder::is_y[TILE]) {
        const auto* from = sy.part_at(PartsOrder::part[TILE], d);
#pragma unroll
        for (int u = 0; u < S::kYLoads; ++u) sy.load_part(from, u, lds_at);
    } else {
        const auto* from = sx.part_at(PartsOrder::part[TILE], d);
#pragma unroll
        for (int u = 0; u < S::kXLoads; ++u) sx.load_part(from, u, lds_at);
    }
}
// (the last place of the ring is left free)
template <class S, class SideY, class SideX>
__device__ __forceinline__ void start_parts(const SideY& sy, const SideX& sx, uint32_t lds0, int pairs)
{
    if (pairs <= 0) return;
    const uint32_t lds_wave = lds0 + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 1024u;
    each<9>([&](auto I) __attribute__((always_inline)) {
        constexpr int i = decltype(I)::value;
        load_tile<S, i % 6>(sy, sx, min(i / 6, pairs - 1), lds_wave + i * S::kPlace);
    });
}
template <class S, class T, class SideY, class SideX>
__device__ __forceinline__ void accumulate_parts(Sums<S>& acc, const SideY& sy, const SideX& sx, uint32_t lds0, int pairs)
{
    static_assert(S::kRing == 10 && S::kYLoads == S::kXLoads);
    constexpr int kTM = S::kTM, kTN = S::kTN, kLoads = S::kYLoads;
    if (pairs <= 0) return;
    const uint32_t lds_wave = lds0 + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 1024u;
    auto meet = []() __attribute__((always_inline)) {
        ADAGC_P_WAIT_LDS(0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        ADAGC_P_FENCE();
    };
    int base = 0;                                  // the place of the pair's first tile
    auto place = [&](int u) __attribute__((always_inline)) { return (uint32_t)((base + u >= 10 ? base + u - 10 : base + u) * S::kPlace); };
    u32x4 y[2][kTM], x_hi[2][kTN], x[2][kTN];      // x: mid, lo
    ADAGC_P_WAIT_VMEM(5 * kLoads);                 // four of nine tiles
    meet();
    load_tile<S, 3>(sy, sx, min(1, pairs - 1), lds_wave + 9 * S::kPlace);
#pragma unroll
    for (int n = 0; n < kTN; ++n) x_hi[0][n] = sx.read(n, S::kPlace);
#pragma unroll
    for (int m = 0; m < kTM; ++m) y[0][m] = sy.read(m, 0);
    for (int d = 0; d < pairs; ++d) {
        each<12>([&](auto STEP) __attribute__((always_inline)) {
            constexpr int step = decltype(STEP)::value, second = step / 6, k = step % 6, kSlots = kTM * kTN;
            constexpr int of_y = (k == 0 ? 0 : k < 3 ? 1 : 0) ^ second;                         // the set of y that is multiplied; the other one is read to
            constexpr bool reads_y = k % 2 == 0 ? k < 4 : k == 5, reads_x = k % 2 == 1;
            constexpr int next_second = k == 5 ? second ^ 1 : second;
            const uint32_t from_y = place(k == 0 ? 2 : k == 2 ? 4 : second ? 6 : 0), from_x = place(k == 1 ? 3 : k == 3 ? 5 : second ? 7 : 1);
            each<kSlots>([&](auto SLOT) __attribute__((always_inline)) {
                constexpr int slot = decltype(SLOT)::value, m = slot / kTN, n = slot % kTN;
                multiply<T>(k == 2 || k == 3 ? x[0][n] : k == 4 ? x[1][n] : x_hi[second][n], y[of_y][m], acc[m][n]);
                ADAGC_P_FENCE();
                constexpr int kReads = (reads_x ? kTN : 0) + (reads_y ? kTM : 0);
                each<kReads>([&](auto R) __attribute__((always_inline)) {
                    constexpr int r = decltype(R)::value;
                    if constexpr (r * (kSlots / 2) / kReads == slot) {
                        if constexpr (reads_x && r < kTN) {
                            if constexpr (k == 5) x_hi[second ^ 1][r] = sx.read(r, from_x, next_second);
                            else x[k / 2][r] = sx.read(r, from_x, next_second);
                        } else {
                            constexpr int block = reads_x ? r - kTN : r;
                            y[of_y ^ 1][block] = sy.read(block, from_y, next_second);
                        }
                    }
                });
                if constexpr (slot == kSlots / 2) {
                    if constexpr (step == 6) load_tile<S, 4>(sy, sx, min(d + 1, pairs - 1), lds_wave + place(0));
                    if constexpr (step == 7) load_tile<S, 5>(sy, sx, min(d + 1, pairs - 1), lds_wave + place(1));
                    if constexpr (step == 10) load_tile<S, 0>(sy, sx, min(d + 2, pairs - 1), lds_wave + place(2));
                    if constexpr (step == 11) load_tile<S, 2>(sy, sx, min(d + 2, pairs - 1), lds_wave + place(4));
                }
                if constexpr (slot == kSlots - 1) {
                    if constexpr (step == 10) load_tile<S, 1>(sy, sx, min(d + 2, pairs - 1), lds_wave + place(3));
                    if constexpr (step == 11) load_tile<S, 3>(sy, sx, min(d + 2, pairs - 1), lds_wave + place(5));
                }
                ADAGC_P_FENCE();
            });
            if constexpr (step == 1) ADAGC_P_WAIT_VMEM(4 * kLoads);        // y hi and x lo of this pair
            if constexpr (step == 9) ADAGC_P_WAIT_VMEM(2 * kLoads);        // the first four tiles of the next one
            if constexpr (step == 1 || step == 5 || step == 9) meet();
        });
        base = base + 6 >= 10 ? base - 4 : base + 6;
    }
    ADAGC_P_WAIT_VMEM(0);
    __syncthreads();
}

// The one or the other: `pairs` of steps, from the sides' first one on.
template <class S, class SideY, class SideX>
__device__ __forceinline__ void start_products(SideY& sy, SideX& sx, uint32_t lds0, int pairs, int segments)
{
    if constexpr (S::kRing == 10) {
        if (segments == kSegments) return start_parts<S>(sy, sx, lds0, pairs);
    }
    start_direct<S>(sy, sx, lds0, pairs);
}
template <class S, class T, class SideY, class SideX>
__device__ __forceinline__ void accumulate_products(Sums<S>& acc, SideY& sy, SideX& sx, uint32_t lds0, int pairs, int segments)
{
    if constexpr (S::kRing == 10) {
        if (segments == kSegments) return accumulate_parts<S, T>(acc, sy, sx, lds0, pairs);
    }
    accumulate_direct<S, T>(acc, sy, sx, lds0, pairs);
}

// The lane's first row and column of a tile.
template <class S>
struct LanePlace {
    int row, col;
    __device__ __forceinline__ LanePlace()
    {
        const int t = thread_anew(), lane = t & 63, wave = t >> 6;
        row = wave / S::kWN * S::kTM * 16 + lane % 16;
        col = wave % S::kWN * S::kTN * 16 + lane / 16 * 4;
    }
};

// f(m, n, row, column, sums of 4 consecutive columns): rows and columns within the tile
template <class S, class F>
__device__ __forceinline__ void each_piece(const Sums<S>& acc, F&& f)
{
    const int t = thread_anew(), lane = t & 63, wave = t >> 6, wm = wave / S::kWN, wn = wave % S::kWN;
#pragma unroll
    for (int m = 0; m < S::kTM; ++m)
#pragma unroll
        for (int n = 0; n < S::kTN; ++n)
            f(m, n, (wm * S::kTM + m) * 16 + lane % 16, (wn * S::kTN + n) * 16 + lane / 16 * 4, acc[m][n]);
}

// Four consecutive results.
typedef uint32_t u32x2_of_bf16 __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void store4(float* p, const f32x4_p& v) { store_whole(p, {__builtin_bit_cast(u32x4, v)}); }
__device__ __forceinline__ void store4(uint16_t* p, const f32x4_p& v)
{
    const f32x2_t lo = {v[0], v[1]}, hi = {v[2], v[3]};
    *reinterpret_cast<u32x2_of_bf16*>(p) =
        u32x2_of_bf16{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2_t)), __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2_t))};
}
__device__ __forceinline__ f32x4_p load4(const float* p) { return __builtin_bit_cast(f32x4_p, load_whole(p).w); }
__device__ __forceinline__ f32x4_p load4(const uint16_t* p)
{
    const u32x2_of_bf16 two = *reinterpret_cast<const u32x2_of_bf16*>(p);
    return f32x4_p{__uint_as_float(two[0] << 16), __uint_as_float(two[0] & 0xFFFF0000u), __uint_as_float(two[1] << 16), __uint_as_float(two[1] & 0xFFFF0000u)};
}

// Two blocks' four consecutive results each, of blocks next to each other, `to`: of the lane's first column of the first.  bf16: lanes 16 apart exchange
// halves, so that a lane stores eight consecutive ones.
__device__ __forceinline__ void store_blocks(float* to, const f32x4_p& a, const f32x4_p& b)
{
    store4(to, a);
    store4(to + 16, b);
}
__device__ __forceinline__ void store_blocks(uint16_t* to, const f32x4_p& a, const f32x4_p& b)
{
    uint32_t w[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x2_t two = {a[2 * h], a[2 * h + 1]}, other = {b[2 * h], b[2 * h + 1]};
        const auto swapped = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2_t)),
                                                              __builtin_bit_cast(uint32_t, __builtin_convertvector(other, bf16x2_t)), false, false);
        w[0][h] = swapped[0];
        w[1][h] = swapped[1];
    }
    store_whole(to + (threadIdx.x / 16 % 2 ? 12 : 0), {u32x4{w[0][0], w[0][1], w[1][0], w[1][1]}});
}

// Four consecutive results from column `col` of a row that ends at `end` on; those before `least` are left as they are.
template <class T>
__device__ __forceinline__ void store4(T* row, int64_t col, int64_t least, int64_t end, const f32x4_p& v)
{
    if (col >= least && col + 4 <= end) {
        store4(row + col, v);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (col + r >= least && col + r < end) {
                if constexpr (sizeof(T) == 4) row[col + r] = v[r];
                else row[col + r] = __builtin_bit_cast(uint16_t, (__bf16)v[r]);
            }
    }
}
// The four there; 0 outside.
template <class T>
__device__ __forceinline__ f32x4_p load4(const T* row, int64_t col, int64_t least, int64_t end)
{
    f32x4_p v = {0.f, 0.f, 0.f, 0.f};
    if (col >= least && col + 4 <= end) {
        v = load4(row + col);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (col + r >= least && col + r < end) v[r] = to_float(row[col + r]);
    }
    return v;
}

using Large = Tile<uint16_t, 256, 256, 2, 4, 5>;
using Small = Tile<uint16_t, 128, 128, 2, 4, 10>;
template <class T> using Staged = Tile<T, sizeof(T) == 4 ? 64 : 128, sizeof(T) == 4 ? 64 : 128, 2, 2, 0>;
// Up to 32 fp32 rows, whose matrix instructions take the time: 128256 from 29 rows of 4096 698 us in 64-tiles, 451; the gradient of 17 rows of 4096 from
// 2 x 12382 155, 124.
using Slim = Tile<float, 32, 64, 1, 2, 0>;

// Rows of an operand start at multiples of 16 bytes.
inline bool rows_aligned(const void* p, int64_t ld, int32_t dtype) { return !misaligned(p, 16) && ld * dtype_size(dtype) % 16 == 0; }


// Elements from row to row from which on 256 rows along k are not within 32 bits of bytes: no operand of the rings.
constexpr int64_t kFarAlong = (int64_t)1 << 23;

// Tiles for a product of rows along k; n: of both matrices where there are two.
struct AlongPlan {
    int     size, rows;           // columns: 256, 128 or 64; rows: as many, or 32
    bool    direct;
    int64_t tiles_m, tiles_n, split;       // split: workgroups that share a tile's k
    int64_t workspace() const { return split > 1 ? tiles_m * tiles_n * split * rows * size * 4 : 0; }
};
// fp32 as it is: the matrix cores' rate is a sixteenth, which staging and a small tile keep up with.
template <class F>
inline int tile_size(bool direct, int32_t dtype, F&& tiles)
{
    return direct && tiles(256) >= kUnits / 2 ? 256 : dtype == ADAGC_F32 ? 64 : 128;
}
inline AlongPlan along_plan(int64_t m, int64_t n, int64_t k, int segments, int32_t dtype, bool aligned, int64_t ld_y, int64_t ld_x)
{
    AlongPlan p{};
    auto tiles = [&](int64_t size) { return ((m + size - 1) / size) * ((n + size - 1) / size); };
    p.direct = aligned && dtype == ADAGC_BF16 && ld_y < kFarAlong && ld_x < kFarAlong;
    p.size = tile_size(p.direct, dtype, tiles);
    if (p.size == 256 && segments > 1) p.size = 128;        // parts stay in the small tile's ring; see accumulate_parts
    p.rows = p.size == 64 && m <= Slim::BM ? Slim::BM : p.size;
    p.tiles_m = (m + p.rows - 1) / p.rows;
    p.tiles_n = (n + p.size - 1) / p.size;
    // Tiles that leave half of the chip without work or more, along a long k: parts of 16 steps at least, whose sums a second launch joins.  56 rows of
    // 4096 to 2 x 1719, fp32: 54 tiles 100 us, in nine parts 31; 128 rows of 768 to 2 x 768, three bf16 parts, 12 tiles 37, in nine 28.  Below 64 steps, 12 - 24 us, the second
    // launch costs what it saves.  Workgroups of 32 rows are small: six on a compute unit, 12382 x 2 from 17 rows of 4096 162 us in 387 whole tiles, 92 and
    // 5 in three parts each.
    const int64_t round = p.direct ? kUnits : p.rows == 32 ? 6 * kUnits : 2 * kUnits, all = p.tiles_m * p.tiles_n, steps = k / (kStepBytes / dtype_size(dtype)) * segments;
    // (Large tiles are half as many as compute units at least, and whole.)
    p.split = p.size < 256 && steps >= 64 ? std::max<int64_t>(1, std::min(round / all, steps / 16)) : 1;
    return p;
}

// ---------------------------------------------------------------------------------------- both operands along k

// Four values in parts: bits of bf16 pairs.  What is not finite is in the first part alone; what rounds beyond bf16's range keeps its largest number.
__device__ __forceinline__ void split4(const f32x4_p& v, uint32_t (&bits)[kParts][2])
{
    float left[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
    for (int p = 0; p < kParts; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x2_t two = {left[2 * i], left[2 * i + 1]};
            uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector(two, bf16x2_t));
            if (p == 0) {
                if ((w & 0x7FFFu) == 0x7F80u && __builtin_isfinite(left[2 * i])) w -= 1;
                if ((w & 0x7FFF0000u) == 0x7F800000u && __builtin_isfinite(left[2 * i + 1])) w -= 0x10000u;
            }
            bits[p][i] = w;
            const float lo = left[2 * i] - __uint_as_float(w << 16), hi = left[2 * i + 1] - __uint_as_float(w & 0xFFFF0000u);
            left[2 * i] = __builtin_isfinite(left[2 * i]) ? lo : 0.f;
            left[2 * i + 1] = __builtin_isfinite(left[2 * i + 1]) ? hi : 0.f;
        }
}

// Rows of Y, and of X or, as the gated projections take them, of two matrices in turn: blocks of 16 columns of the result belong to x[0] and
// x[1] alternately, so that a lane has both results of a place next to each other.
struct AlongArgs {
    const void* y;
    const void* x[2];
    int64_t     ld_y, ld_x[2];
    int64_t     m, n, k;          // n: rows of one X
    int64_t     part_y, part_x;   // operands in parts: elements from part to part
    int32_t     segments;         // products that are summed: 1, or kSegments of operands in three parts
    int32_t     tiles_m, tiles_n;
    float*      partial;          // sums of the parts of split tiles
    int32_t     split;
};

// Whole tiles; one part of a tile's k, whose sums go to `partial`; a tile's parts, added in order.
enum class Sum { kWhole, kPart, kJoined };

// The workgroup's tiles.  before(m0, n0): loads for finish, which come before the next tile's in the order that loads are waited for in;
// finish(acc, m0, n0, scratch): the sums of the tile whose first row is m0 and whose first row of X (or of each) is n0, and an LDS place
// free to use.
template <class S, class T, bool PAIR, Sum SUM, class Before, class Finish>
__device__ __forceinline__ void along_tiles(const AlongArgs& a, uint8_t* lds, Before&& before, Finish&& finish)
{
    constexpr int kColumns = PAIR ? S::BN / 2 : S::BN;
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(lds);      // low half of the flat address = LDS offset
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const T* y = static_cast<const T*>(a.y);
    Side<T, S::BM, S::kThreads, S::kYUnits, S::kTM, false, S::kDirect> sy;
    Side<T, S::BN, S::kThreads, S::kXUnits, S::kTN, false, S::kDirect> sx;
    sy.set_places(tid, lds0, wave / S::kWN * S::kTM);
    sx.set_places(tid, S::kDirect ? lds0 : lds0 + S::kY, wave % S::kWN * S::kTN);
    int64_t m0, n0;
    Sums<S> acc;
    auto row_of_x = [&](int r) __attribute__((always_inline)) { return min(n0 + (PAIR ? (r >> 5) * 16 + (r & 15) : r), a.n - 1); };
    auto aim_staged = [&]() __attribute__((always_inline)) {
        const int tid = thread_anew();
        sy.set_rows(tid, [&](int r) { return y + min(m0 + r, a.m - 1) * a.ld_y; });
        sx.set_rows(tid, [&](int r) {
            const bool second = PAIR && (r >> 4 & 1);
            return static_cast<const T*>(second ? a.x[1] : a.x[0]) + row_of_x(r) * (second ? a.ld_x[1] : a.ld_x[0]);
        });
    };
    auto to_tile = [&](int n) __attribute__((always_inline)) {
        int tm, tn;
        place_of_tile(n, a.tiles_m, a.tiles_n, &tm, &tn);
        m0 = (int64_t)tm * S::BM;
        n0 = (int64_t)tn * kColumns;
    };
    auto aim = [&](int first) __attribute__((always_inline)) {
        // a load of a wave is 8 rows, and a lane's are a multiple of 32 apart: with two matrices, all of one
        static_assert(!S::kDirect || S::kThreads / 8 % 32 == 0);
        const int tid = thread_anew();
        const bool second = PAIR && (wave >> 1 & 1);
        const int64_t ld_x = second ? a.ld_x[1] : a.ld_x[0];
        sy.set_rows_direct(tid, y + m0 * a.ld_y, a.ld_y, [&](int r) { return min(m0 + r, a.m - 1) - m0; });
        sy.set_first(first, a.part_y);
        sx.set_rows_direct(tid, static_cast<const T*>(second ? a.x[1] : a.x[0]) + n0 * ld_x, ld_x, [&](int r) { return row_of_x(r) - n0; });
        sx.set_first(first, a.part_x);
    };
    if constexpr (SUM == Sum::kJoined) {
        to_tile((int)blockIdx.x);
        before(m0, n0);
        const f32x4_p* from = reinterpret_cast<const f32x4_p*>(a.partial) + (size_t)blockIdx.x * a.split * (S::BM * S::BN / 4) + tid;
        clear<S>(acc);
        for (int p = 0; p < a.split; ++p)
#pragma unroll
            for (int m = 0; m < S::kTM; ++m)
#pragma unroll
                for (int n = 0; n < S::kTN; ++n) acc[m][n] += from[((size_t)p * S::kTM * S::kTN + m * S::kTN + n) * S::kThreads];
        finish(acc, m0, n0, lds);
    } else if constexpr (SUM == Sum::kPart) {
        // an XCD has neighbours: tiles of the same part
        const int items = (int)gridDim.x, xcd = (int)blockIdx.x % 8, at = xcd * (items / 8) + min(xcd, items % 8) + (int)blockIdx.x / 8;
        const int tiles = a.tiles_m * a.tiles_n, part = __builtin_amdgcn_readfirstlane(at / tiles), tile = __builtin_amdgcn_readfirstlane(at % tiles);
        constexpr int kTogether = (S::kDirect ? 2 : 1) * S::kDeep;
        const int full = (int)(a.k / kTogether), first = __builtin_amdgcn_readfirstlane((int)((int64_t)full * part / a.split));
        const int number = __builtin_amdgcn_readfirstlane((int)((int64_t)full * (part + 1) / a.split)) - first;
        const bool rest = a.k % kTogether && part == a.split - 1;
        to_tile(tile);
        clear<S>(acc);
        if constexpr (S::kDirect) {
            if (rest) {
                aim_staged();
                accumulate_rest<S, T>(acc, sy, sx, 2 * (int64_t)full, a.k, 0, 0);
            }
            aim(first);
            start_products<S>(sy, sx, lds0, number, a.segments);
            accumulate_products<S, T>(acc, sy, sx, lds0, number, a.segments);
        } else {
            aim_staged();
            accumulate<S, T, false>(acc, sy, sx, first, first + number, rest, full, a.k, 0, 0);
        }
        f32x4_p* to = reinterpret_cast<f32x4_p*>(a.partial) + ((size_t)tile * a.split + part) * (S::BM * S::BN / 4) + thread_anew();
        each_piece<S>(acc, [&](int m, int n, int, int, const f32x4_p& v) __attribute__((always_inline)) { to[(m * S::kTN + n) * S::kThreads] = v; });
    } else if constexpr (!S::kDirect) {
        to_tile((int)blockIdx.x);
        aim_staged();
        clear<S>(acc);
        const int64_t full = a.k / S::kDeep;
        accumulate<S, T, false>(acc, sy, sx, 0, full, a.k % S::kDeep, full, a.k, 0, 0);
        before(m0, n0);
        finish(acc, m0, n0, lds);
    } else {
        const int pairs = (int)(a.k / (2 * S::kDeep)), tiles = a.tiles_m * a.tiles_n;
        const bool rest = a.k % (2 * S::kDeep);        // (not with several segments)
        int n = (int)blockIdx.x;
        to_tile(n);
        if (!rest) {
            aim(0);
            start_products<S>(sy, sx, lds0, pairs, a.segments);
        }
        while (true) {
            clear<S>(acc);
            if (rest) {
                aim_staged();
                accumulate_rest<S, T>(acc, sy, sx, 2 * pairs, a.k, 0, 0);
                aim(0);
                start_products<S>(sy, sx, lds0, pairs, a.segments);
            }
            accumulate_products<S, T>(acc, sy, sx, lds0, pairs, a.segments);
            const int64_t m_now = m0, n_now = n0;
            before(m_now, n_now);
            n += (int)gridDim.x;
            if (n < tiles) {
                to_tile(n);
                if (!rest) {
                    aim(0);
                    start_products<S>(sy, sx, lds0, pairs, a.segments);
                }
            }
            finish(acc, m_now, n_now, lds + (S::kRing - 1) * S::kPlace);
            if (n >= tiles) break;
        }
    }
}

// Workgroups of a launch of so many tiles (or parts of them).
template <class S>
inline uint32_t grid_of(int64_t tiles)
{
    return (uint32_t)(S::kDirect ? std::min<int64_t>(tiles, kUnits) : tiles);
}

template <class S, class T, bool PAIR>
__global__ __launch_bounds__(S::kThreads, 2) void part_kernel(const AlongArgs a)
{
    __shared__ __attribute__((aligned(512))) uint8_t lds[S::kLds];
    along_tiles<S, T, PAIR, Sum::kPart>(a, lds, [](int64_t, int64_t) {}, [](Sums<S>&, int64_t, int64_t, uint8_t*) {});
}
// The parts of split tiles; Sum::kJoined is to follow.
template <class S, class T, bool PAIR>
void launch_parts(const AlongArgs& a, hipStream_t s)
{
    part_kernel<S, T, PAIR><<<dim3((uint32_t)(a.tiles_m * a.tiles_n * a.split)), dim3(S::kThreads), 0, s>>>(a);
}

// Waves meet, their LDS accesses done; loads into LDS may be on their way (which __syncthreads would not leave).
__device__ __forceinline__ void meet_keeping_loads()
{
    ADAGC_P_WAIT_LDS(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    ADAGC_P_FENCE();
}

// ---- few rows
//
// Up to 16 rows of Y: memory bounds it, the rows of X that go past once.  A workgroup of 8 waves has 32 rows of X at a time (of two matrices 16
// each) and all of Y; its waves share k out and their sums meet in LDS, in their order.  Operands go from memory to registers as the matrix
// cores want them, a batch on its way while one is multiplied, the next rows' first one while the sums meet.
//
// A load takes 128 bytes each of 8 rows, whole lines of the cache (of the instruction's natural 16 rows 64 bytes each, lines came from
// memory twice where they had left the L2 between the halves: one row, 128256 x 4096 bf16 215 - 255 us, with loads past the caches 296; now 178,
// 5.9 TB/s).  So an operand of 16 rows is 8 rows with the first 64 bytes and the same 8 with the second; of the 16 x 16 results the quadrants that belong together
// are added, the others not used.
constexpr int kThinRows = 16, kThinColumns = 32, kThinWaves = 8, kThinThreads = 64 * kThinWaves, kThinBlocks = kThinColumns / 8;
template <int TM>
constexpr int kThinLds = kThinWaves * TM * kThinBlocks * 64 * 16;
constexpr int kThinGrid = 2 * kUnits;      // workgroups that fill the chip

// The workgroup's rows of X; k is a vector at least.  before(n0): loads for finish; finish(n0, row, col, sum, sum_of_second): of row `row` of Y with row n0 + col of X (of
// each), a thread for each: all threads call it, those with row 8 TM or more, or beyond the matrices, with nothing.
template <class T, int TM, bool PAIR, class Before, class Finish>
__device__ __forceinline__ void thin_tiles(const AlongArgs& a, uint8_t* lds, Before&& before, Finish&& finish)
{
    constexpr int kE = 16 / (int)sizeof(T), kDeep = 2 * kStepBytes / (int)sizeof(T), kU = 1, kB = kThinBlocks;
    constexpr int kColumns = PAIR ? kThinColumns / 2 : kThinColumns;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane_k = (lane / 8 % 2 * 4 + lane / 16) * kE, k = (int)a.k;
    const int full = k / kDeep, steps = (k + kDeep - 1) / kDeep;           // the last one may be cut
    const int first = __builtin_amdgcn_readfirstlane((int)((int64_t)steps * wave / kThinWaves));
    const int own = __builtin_amdgcn_readfirstlane((int)((int64_t)steps * (wave + 1) / kThinWaves)) - first;
    const T *y[TM], *x[kB];
#pragma unroll
    for (int m = 0; m < TM; ++m) y[m] = static_cast<const T*>(a.y) + min((int64_t)(m * 8 + lane % 8), a.m - 1) * a.ld_y;
    auto aim = [&](int64_t n0) __attribute__((always_inline)) {
        const int l = thread_anew();
#pragma unroll
        for (int n = 0; n < kB; ++n) {
            const bool second = PAIR && (n & 1);
            const int64_t row = min(n0 + (PAIR ? n / 2 : n) * 8 + l % 8, a.n - 1);
            x[n] = static_cast<const T*>(second ? a.x[1] : a.x[0]) + row * (second ? a.ld_x[1] : a.ld_x[0]);
        }
    };
    struct Batch {
        u32x4 y[kU][TM], x[kU][kB];
    };
    // a batch's steps that do not exist are the last one again, and not multiplied
    auto load = [&](int i, Batch& b) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const int at = min((first + min(i + u, own - 1)) * kDeep + lane_k, k - kE);       // (k's last vector is put right in use)
#pragma unroll
            for (int n = 0; n < kB; ++n) b.x[u][n] = load_whole(x[n] + at).w;
#pragma unroll
            for (int m = 0; m < TM; ++m) b.y[u][m] = load_whole(y[m] + at).w;
        }
    };
    f32x4_p acc[TM][kB];
    auto use = [&](int i, Batch& b) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kU; ++u)
            if (i + u < own) {
                if (first + i + u == full) {
                    const int l = thread_anew() & 63, col = full * kDeep + (l / 8 % 2 * 4 + l / 16) * kE;
                    auto cut = [&](u32x4& w) __attribute__((always_inline)) {
                        Vector<T> v{w};
                        settle(v, col, k, 0);
                        w = v.w;
                    };
#pragma unroll
                    for (int m = 0; m < TM; ++m) cut(b.y[u][m]);
#pragma unroll
                    for (int n = 0; n < kB; ++n) cut(b.x[u][n]);
                }
#pragma unroll
                for (int m = 0; m < TM; ++m)
#pragma unroll
                    for (int n = 0; n < kB; ++n) multiply<T>(b.x[u][n], b.y[u][m], acc[m][n]);
            }
    };
    const int64_t step = (int64_t)gridDim.x * kColumns;
    int64_t n0 = (int64_t)blockIdx.x * kColumns;
    Batch b[2];
    aim(n0);
    if (own > 0) load(0, b[0]);
    while (true) {
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int n = 0; n < kB; ++n) acc[m][n] = f32x4_p{0.f, 0.f, 0.f, 0.f};
        before(n0);
        const int64_t next = n0 + step;
        if (own > 0) {
            int i = 0;
            for (; i + 2 * kU < own; i += 2 * kU) {
                load(i + kU, b[1]);
                use(i, b[0]);
                load(i + 2 * kU, b[0]);
                use(i + kU, b[1]);
            }
            if (i + kU < own) load(i + kU, b[1]);
            use(i, b[0]);
            if (next < a.n) {
                aim(next);
                load(0, b[0]);
            }
            if (i + kU < own) use(i + kU, b[1]);
        } else if (next < a.n) {
            aim(next);
        }
        // value r of lane l: row (l mod 16) mod 8 of Y, row (4 (l / 16) + r) mod 8 of X; valid where both are in the same half
        float* parts = reinterpret_cast<float*>(lds);
        const int own_part = thread_anew() & 63;
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int n = 0; n < kB; ++n) reinterpret_cast<f32x4_p*>(parts)[((wave * TM + m) * kB + n) * 64 + own_part] = acc[m][n];
        meet_keeping_loads();
        const int t = thread_anew(), row = t / kColumns, col = t % kColumns;
        float sum[2] = {0.f, 0.f};
        if (row < 8 * TM) {
#pragma unroll
            for (int p = 0; p < (PAIR ? 2 : 1); ++p) {
                const int block = PAIR ? col / 8 * 2 + p : col / 8;
                const float* from = parts + ((row / 8 * kB + block) * 64 + col % 8 / 4 * 16 + row % 8) * 4 + col % 4;
#pragma unroll
                for (int w = 0; w < kThinWaves; ++w) sum[p] += from[w * TM * kB * 256] + from[w * TM * kB * 256 + 40 * 4];
            }
        }
        if (next < a.n) meet_keeping_loads();
        finish(n0, row, col, sum[0], sum[1]);
        if (next >= a.n) break;
        n0 = next;
    }
}

// whatever the matrices (those with less than a vector along k have no parts either)
inline bool always_thin(int64_t rows, int32_t dtype) { return rows <= (dtype == ADAGC_F32 ? 8 : kThinRows); }
// fp32, more than 8 rows: 128256 x 4096 from 10 rows 545 us, 32 x 64-tiles 433 - 488; 32000 x 1024 from 12 rows 44 and 52
inline bool thin(const AlongArgs& a, int32_t dtype)
{
    return a.k >= 16 / dtype_size(dtype) && (always_thin(a.m, dtype) || (a.m <= kThinRows && a.n * a.k < (int64_t)1 << 28));
}

// f(integral_constant blocks of 8 rows) for up to kThinRows rows
template <class F>
inline void for_rows(int64_t rows, F&& f)
{
    if (rows <= 8) f(std::integral_constant<int, 1>{});
    else f(std::integral_constant<int, 2>{});
}

// ---------------------------------------------------------------------------------------- a product with a plain result

// out = (add +) factor times the sum over up to two pairs of operands, or two products side by side.
struct PlainArgs {
    const void* y[2];
    const void* x[2];
    int64_t     ld_y, ld_x[2];
    void*       out[2];
    int64_t     ld_out[2];
    const void* add[2];           // NULL: nothing
    int64_t     ld_add[2];
    int64_t     m, n, k;
    int64_t     m_readable;       // Y across k: columns of it that may be read, m or more
    int64_t     n_readable;       // columns of X that may be read, n or more
    int64_t     part_y, part_x;   // operands in parts: elements from part to part
    int32_t     segments;         // products that are summed for a pair: 1, or kSegments of operands in three parts
    float*      workspace;        // partial sums of the split tiles
    float       factor;
    int32_t     pairs;            // 1, or 2: both pairs' products are summed
    int32_t     products;         // 1, or 2: out[0], out[1] of the two pairs
    int32_t     out_bf16, add_bf16;
    int32_t     tiles_m, tiles_n; // of one product
    int32_t     whole;            // tiles computed by one workgroup each; the others by `split`
    int32_t     split;
};

__device__ __forceinline__ void store_plain(const PlainArgs& a, int product, int64_t row, int64_t row_least, int64_t col, int64_t col_least, f32x4_p v)
{
    if (row < row_least || row >= a.m || col >= a.n) return;
    v *= a.factor;
    const void* add = product ? a.add[1] : a.add[0];
    void* out = product ? a.out[1] : a.out[0];
    if (add) {
        const int64_t at = row * (product ? a.ld_add[1] : a.ld_add[0]);
        v += a.add_bf16 ? load4(static_cast<const uint16_t*>(add) + at, col, col_least, a.n) : load4(static_cast<const float*>(add) + at, col, col_least, a.n);
    }
    const int64_t at = row * (product ? a.ld_out[1] : a.ld_out[0]);
    if (a.out_bf16) store4(static_cast<uint16_t*>(out) + at, col, col_least, a.n, v);
    else store4(static_cast<float*>(out) + at, col, col_least, a.n, v);
}

// The first row or column that a tile computes and the first that it stores: the last tile across columns begins a tile before the end, so that
// every tile is whole.
template <bool SHIFT>
__device__ __forceinline__ int64_t first_of_tile(int tile, int size, int64_t n)
{
    const int64_t first = (int64_t)tile * size;
    return SHIFT ? min(first, n - size) : first;
}

// Y along k or across it, X across it (the products of a backward pass).  CHECKED: a side across k is smaller than a tile, or its rows are too
// far apart for 32-bit offsets.
template <class S, class T, bool ACROSS_Y, bool CHECKED>
__global__ __launch_bounds__(S::kThreads, 2) void plain_kernel(const PlainArgs a)
{
    static_assert(!(CHECKED && S::kDirect));
    __shared__ __attribute__((aligned(512))) uint8_t lds[S::kLds];
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(&lds[0]);      // low half of the flat address = LDS offset
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Side<T, S::BM, S::kThreads, S::kYUnits, S::kTM, ACROSS_Y, S::kDirect> sy;
    Side<T, S::BN, S::kThreads, S::kXUnits, S::kTN, true, S::kDirect> sx;
    sy.set_places(tid, lds0, wave / S::kWN * S::kTM);
    sx.set_places(tid, S::kDirect ? lds0 : lds0 + S::kY, wave % S::kWN * S::kTN);

    constexpr int kTogether = (S::kDirect ? 2 : 1) * S::kDeep;     // of k: a step, or a pair of them
    const int full = (int)(a.k / kTogether), items = a.whole + (a.tiles_m * a.tiles_n * a.products - a.whole) * a.split;
    const bool uneven = a.k % kTogether;
    const int64_t m_readable = ACROSS_Y ? a.m_readable : a.m;
    struct Place {
        int     item, product, slot;           // slot: of a split tile's part in the workspace
        int64_t m0, n0, m_least, n_least;
    };
    int step0, step1;
    bool rest;
    auto place_of = [&](int item) __attribute__((always_inline)) {
        int tile = item, slot = 0;
        step0 = 0;
        step1 = full;
        rest = uneven;
        if (item >= a.whole) {
            // an XCD has neighbours here too: tiles of the same part of k
            const int split_items = items - a.whole, tiles = split_items / a.split, i = item - a.whole, xcd = i % 8;
            const int at = xcd * (split_items / 8) + min(xcd, split_items % 8) + i / 8;
            const int part = __builtin_amdgcn_readfirstlane(at / tiles);
            tile = __builtin_amdgcn_readfirstlane(a.whole + at % tiles);
            slot = (tile - a.whole) * a.split + part;
            step0 = __builtin_amdgcn_readfirstlane((int)((int64_t)full * part / a.split));
            step1 = __builtin_amdgcn_readfirstlane((int)((int64_t)full * (part + 1) / a.split));
            rest = uneven && part == a.split - 1;
        }
        const int per_product = a.tiles_m * a.tiles_n;
        Place p;
        p.item = item;
        p.slot = slot;
        p.product = a.products > 1 && tile >= per_product;
        int tm, tn;
        place_of_tile(tile - p.product * per_product, a.tiles_m, a.tiles_n, &tm, &tn);
        p.m0 = scalar(first_of_tile<ACROSS_Y && !CHECKED>(tm, S::BM, m_readable));
        p.n0 = scalar(first_of_tile<!CHECKED>(tn, S::BN, a.n_readable));
        p.m_least = (int64_t)tm * S::BM;
        p.n_least = (int64_t)tn * S::BN;
        return p;
    };
    // (an index would put the arguments into memory)
    auto y_of = [&](bool second) __attribute__((always_inline)) { return static_cast<const T*>(second ? a.y[1] : a.y[0]); };
    auto x_of = [&](bool second) __attribute__((always_inline)) { return static_cast<const T*>(second ? a.x[1] : a.x[0]); };
    auto aim_staged = [&](const Place& p, bool second) __attribute__((always_inline)) {
        const int tid = thread_anew();
        const T* y = y_of(second);
        if constexpr (ACROSS_Y) sy.set_columns(tid, y + p.m0, a.ld_y);
        else sy.set_rows(tid, [&](int r) { return y + min(p.m0 + r, a.m - 1) * a.ld_y; });
        sx.set_columns(tid, x_of(second) + p.n0, second ? a.ld_x[1] : a.ld_x[0]);
    };
    // (what is left over after whole pairs of steps comes with a single segment only)
    auto aim = [&](const Place& p, bool second) __attribute__((always_inline)) {
        const int tid = thread_anew();
        const T* y = y_of(second);
        if constexpr (ACROSS_Y) sy.set_columns_direct(tid, y + p.m0, a.ld_y);
        else sy.set_rows_direct(tid, y + p.m0 * a.ld_y, a.ld_y, [&](int r) { return min(p.m0 + r, a.m - 1) - p.m0; });
        sx.set_columns_direct(tid, x_of(second) + p.n0, second ? a.ld_x[1] : a.ld_x[0]);
        sy.set_first(step0, a.part_y);
        sx.set_first(step0, a.part_x);
    };
    Sums<S> acc;
    auto finish_inside = [&](const Place& p, auto* out, const auto* add) __attribute__((always_inline)) {
        const LanePlace<S> at;
        const int64_t ld = p.product ? a.ld_out[1] : a.ld_out[0], ld_add = p.product ? a.ld_add[1] : a.ld_add[0];
        auto* to = out + ((p.m0 + at.row) * ld + p.n0 + at.col);
        if (add) {
            const auto* from = add + ((p.m0 + at.row) * ld_add + p.n0 + at.col);
#pragma unroll
            for (int m = 0; m < S::kTM; ++m) {
                f32x4_p old[S::kTN];
#pragma unroll
                for (int n = 0; n < S::kTN; ++n) old[n] = load4(from + m * 16 * ld_add + n * 16);
#pragma unroll
                for (int n = 0; n < S::kTN; n += 2)
                    store_blocks(to + m * 16 * ld + n * 16, acc[m][n] * a.factor + old[n], acc[m][n + 1] * a.factor + old[n + 1]);
            }
        } else {
#pragma unroll
            for (int m = 0; m < S::kTM; ++m)
#pragma unroll
                for (int n = 0; n < S::kTN; n += 2) store_blocks(to + m * 16 * ld + n * 16, acc[m][n] * a.factor, acc[m][n + 1] * a.factor);
        }
    };
    auto finish = [&](const Place& p) __attribute__((always_inline)) {
        // (a tile at the matrix's end looks where it ends; within it an address and a check for every four results showed: 5 of 459 us of a weight
        // gradient of 16128 x 4096 from 4096 tokens.  bf16 results with nothing added, d_x but the fp32 sums of its pieces, have add_bf16 = 0 and take the
        // way of the ends too.)
        const bool inside = p.m0 == p.m_least && p.m0 + S::BM <= a.m && p.n0 == p.n_least && p.n0 + S::BN <= a.n && a.out_bf16 == a.add_bf16;
        if (p.item < a.whole && inside) {
            void* out = p.product ? a.out[1] : a.out[0];
            const void* add = p.product ? a.add[1] : a.add[0];
            if (a.out_bf16) finish_inside(p, static_cast<uint16_t*>(out), static_cast<const uint16_t*>(add));
            else finish_inside(p, static_cast<float*>(out), static_cast<const float*>(add));
        } else if (p.item < a.whole) {
            each_piece<S>(acc, [&](int, int, int r, int c, const f32x4_p& v) __attribute__((always_inline)) {
                store_plain(a, p.product, p.m0 + r, p.m_least, p.n0 + c, p.n_least, v);
            });
        } else {
            f32x4_p* to = reinterpret_cast<f32x4_p*>(a.workspace) + (size_t)p.slot * (S::BM * S::BN / 4) + thread_anew();
            each_piece<S>(acc, [&](int m, int n, int, int, const f32x4_p& v) __attribute__((always_inline)) { to[(m * S::kTN + n) * S::kThreads] = v; });
        }
    };

    clear<S>(acc);
    Place now = place_of((int)blockIdx.x);
    int pair = now.product;
    if constexpr (!S::kDirect) {
        for (; pair < now.product + a.pairs; ++pair) {
            aim_staged(now, pair);
            accumulate<S, T, CHECKED>(acc, sy, sx, step0, step1, rest, full, a.k, m_readable - now.m0, a.n_readable - now.n0);
        }
        finish(now);
    } else {
        if (!uneven) {
            aim(now, pair);
            start_products<S>(sy, sx, lds0, step1 - step0, a.segments);
        }
        while (true) {
            if (uneven) {
                if (rest) {
                    aim_staged(now, pair);
                    accumulate_rest<S, T>(acc, sy, sx, 2 * (int64_t)full, a.k, m_readable - now.m0, a.n_readable - now.n0);
                }
                aim(now, pair);
                start_products<S>(sy, sx, lds0, step1 - step0, a.segments);
            }
            accumulate_products<S, T>(acc, sy, sx, lds0, step1 - step0, a.segments);
            const bool last = pair + 1 == now.product + a.pairs;
            const int item = now.item + (int)gridDim.x;
            const Place done = now;
            if (!last) {
                ++pair;
            } else if (item < items) {
                now = place_of(item);
                pair = now.product;
            }
            if ((!last || item < items) && !uneven) {
                aim(now, pair);
                start_products<S>(sy, sx, lds0, step1 - step0, a.segments);
            }
            if (!last) continue;
            finish(done);
            if (item >= items) break;
            clear<S>(acc);
        }
    }
}

// Adds the parts of the split tiles, in order: a workgroup takes one block of every wave.
template <class S, bool ACROSS_Y, bool CHECKED>
__global__ __launch_bounds__(S::kThreads) void plain_join_kernel(const PlainArgs a)
{
    constexpr int kBlocks = S::kTM * S::kTN;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / S::kWN, wn = wave % S::kWN;
    const int n_tile = (int)blockIdx.x / kBlocks, block = (int)blockIdx.x % kBlocks, m = block / S::kTN, n = block % S::kTN;
    const int tile = a.whole + n_tile, per_product = a.tiles_m * a.tiles_n, product = tile / per_product;
    int tm, tn;
    place_of_tile(tile - product * per_product, a.tiles_m, a.tiles_n, &tm, &tn);
    const int64_t m0 = first_of_tile<ACROSS_Y && !CHECKED>(tm, S::BM, ACROSS_Y ? a.m_readable : a.m), n0 = first_of_tile<!CHECKED>(tn, S::BN, a.n_readable);
    const f32x4_p* from = reinterpret_cast<const f32x4_p*>(a.workspace) + (size_t)n_tile * a.split * (S::BM * S::BN / 4) + (size_t)block * S::kThreads + tid;
    f32x4_p sum = from[0];
    int p = 1;
    constexpr int kTogether = 4;                       // loads on their way
    for (; p + kTogether <= a.split; p += kTogether) {
        f32x4_p v[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) v[u] = from[(size_t)(p + u) * (S::BM * S::BN / 4)];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) sum += v[u];
    }
    for (; p < a.split; ++p) sum += from[(size_t)p * (S::BM * S::BN / 4)];
    store_plain(a, product, m0 + (wm * S::kTM + m) * 16 + lane % 16, (int64_t)tm * S::BM, n0 + (wn * S::kTN + n) * 16 + lane / 16 * 4, (int64_t)tn * S::BN, sum);
}

// How a product is cut: tiles, and those of the last, partial round of workgroups also along k, so that they fill the chip too.
struct PlainPlan {
    int     size, rows;           // columns: 256, 128 or 64; rows: as many, or 32
    bool    checked, direct;
    int64_t tiles_m, tiles_n, whole, rest, split;
    int64_t workspace() const { return split > 1 ? rest * split * rows * size * 4 : 0; }
};
// m (with Y across k) and n: of the readable columns; pairs: of operands that are summed, times segments; products: side by side; aligned: the rows of both
// operands are.  A workspace is sized for both.
inline PlainPlan plain_plan(int64_t m, int64_t n, int64_t k, int32_t dtype, bool across_y, int64_t ld_y, int64_t ld_x, int pairs, int products, bool aligned)
{
    PlainPlan p{};
    auto tiles = [&](int64_t size) { return products * ((m + size - 1) / size) * ((n + size - 1) / size); };
    // 32 rows across k are not within 32 bits
    const bool far = ld_x >= (int64_t)1 << 24 || (across_y && ld_y >= (int64_t)1 << 24);
    p.direct = aligned && !far && dtype == ADAGC_BF16 && (across_y || ld_y < kFarAlong) && n >= 128 && n % 8 == 0 &&
               (!across_y || (m >= 128 && m % 8 == 0));
    const int64_t steps = k / (kStepBytes / dtype_size(dtype)) / (p.direct ? 2 : 1) * (p.direct ? 2 : 1);
    p.size = tile_size(p.direct, dtype, tiles);
    // Few large tiles, if along k there are 64 steps for each compute unit, by which the partial sums are paid for: 4096 x 768 from 16384, 48 tiles in
    // five parts 110 - 128 us and 14 - 18 for joining, 192 small tiles 175.
    if (p.direct && p.size < 256 && steps * pairs * tiles(256) >= 64 * kUnits) p.size = 256;
    if (p.size == 256 && (m < 256 || n < 256 || pairs >= kSegments)) p.size = 128;
    p.checked = far || n < p.size || (across_y && m < p.size);
    p.rows = p.size == 64 && !across_y && m <= Slim::BM ? Slim::BM : p.size;
    p.tiles_m = (m + p.rows - 1) / p.rows;
    p.tiles_n = (n + p.size - 1) / p.size;
    const int64_t all = products * p.tiles_m * p.tiles_n;
    // a ring fills a compute unit's LDS; the others' workgroups share a unit in pairs, small ones six at a time
    const int64_t round = p.direct ? kUnits : p.rows == 32 ? 6 * kUnits : 2 * kUnits;
    p.rest = all % round;
    // a part has eight steps at least (of each pair)
    p.split = p.rest ? std::max<int64_t>(1, std::min(round / p.rest, steps * pairs / 8)) : 1;
    p.split = std::min(p.split, std::max<int64_t>(1, steps / 2));
    if (p.split == 1) p.rest = 0;
    p.whole = all - p.rest;
    return p;
}

template <class S, class T, bool ACROSS_Y, bool CHECKED>
int launch_plain(const PlainArgs& a, const PlainPlan& p, hipStream_t s)
{
    plain_kernel<S, T, ACROSS_Y, CHECKED><<<dim3(grid_of<S>(p.whole + p.rest * p.split)), dim3(S::kThreads), 0, s>>>(a);
    if (p.rest) plain_join_kernel<S, ACROSS_Y, CHECKED><<<dim3((uint32_t)(p.rest * S::kTM * S::kTN)), dim3(S::kThreads), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}
// Fills in how the product is cut and launches it.
template <class T, bool ACROSS_Y>
int run_plain(PlainArgs a, hipStream_t s)
{
    constexpr int32_t dtype = sizeof(T) == 4 ? ADAGC_F32 : ADAGC_BF16;
    const int both = std::max(a.pairs, a.products);
    const int64_t m = ACROSS_Y ? a.m_readable : a.m;
    bool aligned = true;
    int64_t ld_x = 0;
    for (int i = 0; i < both; ++i) {
        aligned = aligned && rows_aligned(a.y[i], a.ld_y, dtype) && rows_aligned(a.x[i], a.ld_x[i], dtype);      // (parts are multiples of 16 bytes apart)
        ld_x = std::max(ld_x, a.ld_x[i]);
    }
    const PlainPlan p = plain_plan(m, a.n_readable, a.k, dtype, ACROSS_Y, a.ld_y, ld_x, a.pairs * a.segments, a.products, aligned);
    if (a.segments > 1 && !p.direct) return ADAGC_ERR_TOO_LARGE;           // the staged tiles take operands as they are, and would multiply the first parts alone
    a.tiles_m = (int32_t)p.tiles_m;
    a.tiles_n = (int32_t)p.tiles_n;
    a.whole = (int32_t)p.whole;
    a.split = (int32_t)p.split;
    if constexpr (sizeof(T) == 2) {
        if (p.size == 256) return launch_plain<Large, T, ACROSS_Y, false>(a, p, s);
        if (p.direct) return launch_plain<Small, T, ACROSS_Y, false>(a, p, s);
    }
    if constexpr (sizeof(T) == 4 && !ACROSS_Y) {
        if (p.rows == Slim::BM) return p.checked ? launch_plain<Slim, T, false, true>(a, p, s) : launch_plain<Slim, T, false, false>(a, p, s);
    }
    return p.checked ? launch_plain<Staged<T>, T, ACROSS_Y, true>(a, p, s) : launch_plain<Staged<T>, T, ACROSS_Y, false>(a, p, s);
}

// ---------------------------------------------------------------------------------------- operands laid out anew
//
// fp32 operands in three parts, and bf16 ones whose rows have no whole number of 16-byte vectors (k no multiple of 8), are copied to the workspace first,
// rows and columns filled up to multiples of 64 with zeros, and multiplied by the bf16 tiles that load straight into LDS.  The workspace's size knows no
// addresses: bf16 rows of whole vectors that start elsewhere than at multiples of 16 bytes are taken as they are, through registers (1024 x 50257 from
// 768 forward 93 us, from rows 769 apart 166; 4096 x 14336 from 4096 364 and 760).  Laying out has to be paid for: bf16 rows are laid out from 128 rows on
// (1024 x 50257 from 767 113 us); fp32 ones too, those of a single product (a forward pass) from 193, of 2^29 multiplications at least.  fp32, us as they are and in
// parts: 192 and 256 rows, 32000 from 1024, forward 117 and 150, 153 and 146; 128 rows, all of a training pass 343 and 340; 256 rows, 2 x 1719 from 4096,
// all of it 335 and 262; 2 x 2138 from 1024, forward 44 and 40; 2 x 768 from 768, all of it 74 and 101.
struct Layout {
    bool    anew;
    int     parts, segments;
    int64_t ld;                   // of rows of k numbers
    int64_t bytes(int64_t rows) const { return parts * rows_of(rows) * ld * 2; }
    int64_t part(int64_t rows) const { return rows_of(rows) * ld; }                // elements
    static int64_t rows_of(int64_t rows) { return (rows + 63) / 64 * 64; }
};
inline Layout layout_of(int64_t rows, int64_t wide, int64_t k, int32_t dtype, bool backward)
{
    Layout l{};
    const bool fp32 = dtype == ADAGC_F32;
    l.anew = wide >= 128 && k >= 128 && k < (int64_t)1 << 22 &&
             (fp32 ? rows >= (backward ? 128 : 193) && (double)rows * (double)wide * (double)k >= 0x1p29 : rows >= 128 && k % 8);
    l.parts = l.anew && fp32 ? kParts : 1;
    l.segments = l.parts == 1 ? 1 : kSegments;
    l.ld = (k + 63) / 64 * 64;
    return l;
}

// Up to three matrices in a launch.
struct LayArgs {
    const void* from[3];
    uint16_t*   to[3];
    int64_t     ld_from[3], rows[3], part[3];
    uint32_t    end[3];           // workgroups of the matrix and those before it
    int64_t     ld_to, cols;
};
constexpr int kLay = 256;
// 8 numbers of a row for a lane.  Bound by memory.
template <class T>
__global__ __launch_bounds__(kLay) void lay_kernel(const LayArgs a)
{
    const uint32_t block = blockIdx.x;
    const bool first = block < a.end[0], second = block < a.end[1];        // (an index would put the arguments into memory)
    const int64_t rows = first ? a.rows[0] : second ? a.rows[1] : a.rows[2], part = first ? a.part[0] : second ? a.part[1] : a.part[2];
    const int64_t ld_from = first ? a.ld_from[0] : second ? a.ld_from[1] : a.ld_from[2];
    const void* source = first ? a.from[0] : second ? a.from[1] : a.from[2];
    uint16_t* target = first ? a.to[0] : second ? a.to[1] : a.to[2];
    const int64_t i = (int64_t)(block - (first ? 0 : second ? a.end[0] : a.end[1])) * kLay + threadIdx.x, vectors = a.ld_to / 8;
    if (i >= part / 8) return;
    const int64_t row = i / vectors, col = (i - row * vectors) * 8;
    const T* from = static_cast<const T*>(source) + row * ld_from;
    u32x4* to = reinterpret_cast<u32x4*>(target + row * a.ld_to + col);
    const int64_t n = row < rows ? a.cols : 0;
    if constexpr (sizeof(T) == 2) {
        *to = load_vector(from, col, n, 0).w;
    } else {
        uint32_t bits[2][kParts][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) split4(__builtin_bit_cast(f32x4_p, load_vector(from, col + 4 * h, n, 0).w), bits[h]);
#pragma unroll
        for (int p = 0; p < kParts; ++p) to[p * (part / 8)] = u32x4{bits[0][p][0], bits[0][p][1], bits[1][p][0], bits[1][p][1]};
    }
}
struct LaySource {
    const void* from;
    int64_t     ld, rows;
    void*       to;
};
// `number` matrices of cols columns
template <class T>
int lay(const LaySource* sources, int number, int64_t cols, const Layout& l, hipStream_t s)
{
    LayArgs a{};
    uint32_t blocks = 0;
    for (int i = 0; i < 3; ++i) {
        if (i < number) {
            a.from[i] = sources[i].from;
            a.to[i] = static_cast<uint16_t*>(sources[i].to);
            a.ld_from[i] = sources[i].ld;
            a.rows[i] = sources[i].rows;
            a.part[i] = l.part(sources[i].rows);
            blocks += (uint32_t)((a.part[i] / 8 + kLay - 1) / kLay);
        }
        a.end[i] = blocks;
    }
    a.ld_to = l.ld;
    a.cols = cols;
    if (blocks == 0) return ADAGC_OK;
    lay_kernel<T><<<dim3(blocks), dim3(kLay), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? ADAGC_OK : ADAGC_ERR_HIP;
}

// f(the tile of operands staged through registers)
template <class T, class F>
inline void staged_tile(const AlongPlan& p, F&& f)
{
    if constexpr (sizeof(T) == 4) {
        if (p.rows == Slim::BM) return f(Slim{});
    }
    f(Staged<T>{});
}

// instantiated in product.hip
extern template int run_plain<float, false>(PlainArgs, hipStream_t);
extern template int run_plain<float, true>(PlainArgs, hipStream_t);
extern template int run_plain<uint16_t, false>(PlainArgs, hipStream_t);
extern template int run_plain<uint16_t, true>(PlainArgs, hipStream_t);
extern template int lay<float>(const LaySource*, int, int64_t, const Layout&, hipStream_t);
extern template int lay<uint16_t>(const LaySource*, int, int64_t, const Layout&, hipStream_t);
extern template void launch_parts<Small, uint16_t, false>(const AlongArgs&, hipStream_t);
extern template void launch_parts<Small, uint16_t, true>(const AlongArgs&, hipStream_t);
extern template void launch_parts<Staged<uint16_t>, uint16_t, false>(const AlongArgs&, hipStream_t);
extern template void launch_parts<Staged<uint16_t>, uint16_t, true>(const AlongArgs&, hipStream_t);
extern template void launch_parts<Slim, float, false>(const AlongArgs&, hipStream_t);
extern template void launch_parts<Slim, float, true>(const AlongArgs&, hipStream_t);
extern template void launch_parts<Staged<float>, float, false>(const AlongArgs&, hipStream_t);
extern template void launch_parts<Staged<float>, float, true>(const AlongArgs&, hipStream_t);

}  // namespace product
}  // namespace adagc
#endif
