// The products of the gated block on the matrix cores, one kernel template for all five (see GatedOp).
//
// A workgroup makes a tile of BM x BN results.  Steps of 64 along the summed index go from memory straight to shared memory, one to three steps ahead
// of the matrix instructions, 16 bytes a lane; where rows begin anywhere all but the largest tiles take them through registers (Loose).
//   adjacent operand   tile [rows][64]: 128 bytes a row, eight pieces of 16; piece c of row r lies in place c ^ (r & 7), so that the 16 rows
//                      that an instruction's lanes read at the same piece lie in different banks
//   strided operand    tile [64][columns]; read with the transposing read of shared memory: of 16 lanes each gives the address of four
//                      neighbouring columns (four lanes to a row, four rows), and gets four rows of one column.  Piece c of row k lies in
//                      place c ^ (2 (k & 3) + 8 (k >> 3 & 1)): the rows that are read together lie in different banks
// The instruction (v_mfma_f32_16x16x32: a = A[lane % 16][8 (lane / 16) + i], b = B[8 (lane / 16) + i][lane % 16], c[v] = C[4 (lane / 16) + v][lane % 16])
// forms the transpose of the result, so that a lane ends with four neighbouring columns of a row.
// Sums are in fp32.  Where few tiles leave compute units idle several workgroups share a tile's sum: each writes its part, the last one to
// arrive adds the parts in the order of their index (the result does not depend on who was last) and goes on.
//
// What bounds it (bf16, microseconds of the kernels alone).
//   8,192 rows, p = out = 4,096, hidden 8,192: kOpUp 945, kOpMul 443, kOpDown 521, the gradients 2,116: 1.16, 1.24, 1.05 and 1.30 PFLOP/s, where a library's plain
//   products of these sizes reach 1.05 to 1.35.  Matrix units busy half to two thirds of the time (57, 61, 49 and 62 %) at 1.85 GHz (2.1 without load): they and the
//   way from L2 through shared memory to registers, 256 KB of reads and writes a step, share what shared memory delivers.
//   One row of the same block: kOpUp 33.2 (134 MB at 4.0 TB/s), kOpMul 16.0: memory, and 2.8 us of an empty launch.
//   100 rows, p = 200, hidden 600, out 130: kOpDown 5.6, the gradients 9.7: an empty launch, one trip to memory that nothing precedes (2 us) and the
//   trips of shared sums (0.8 us each); both loose, which adds 0.5 and 1.0 and saves copies of 3.3.
#pragma once

#include "gated_internal.h"
#include "lds_load.h"

#include <hip/hip_runtime.h>

#include <type_traits>

namespace bmgd {
namespace {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) short4v lds_short4;
typedef __attribute__((address_space(3))) short8v lds_short8;

template <typename T> struct Half;
template <> struct Half<__bf16> {
    static __device__ __forceinline__ float4v mma(short8v a, short8v b, float4v c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Half<_Float16> {
    static __device__ __forceinline__ float4v mma(short8v a, short8v b, float4v c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

// act(g) and its derivative.  silu g s, s = 1 / (1 + e^-g): derivative s + g s (1 - s); gelu g F(g), F the normal distribution's: F + g f;
// relu: 0 at 0.  s and F keep their relative accuracy far out on the left, where they are small: an exponential of -|g|, taken 2^32 times too
// large, since the hardware's knows no numbers below 2^-126, and a tail of F of its own.  The hardware's exponential and reciprocal are
// good to 2^-22 here (for |g| < 20; the exponent's own rounding adds 2^-24 |g|).
__device__ __forceinline__ float logistic(float g)
{
    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(fabsf(g), -1.4426950408889634f, 32.f)) * 0x1p-32f;
    return (g < 0.f ? e : 1.f) * __builtin_amdgcn_rcpf(1.f + e);
}
// The normal distribution's F(g), and e^(-g^2 / 2) in `bell`.  1 - F(|g|) = e^(-g^2 / 2) P(1 / (1 + 0.35 |g|)): P is the polynomial of degree 7 that is nearest to
// erfcx(|g| / sqrt 2) / 2 in relative error for |g| up to 13.5 (fitted here; with these coefficients 3.6e-7); with the rounding of the exponent 1.5e-6 for |g| < 5.
__device__ __forceinline__ float normal_cdf(float g, float& bell)
{
    bell = __builtin_amdgcn_exp2f(g * g * -0.72134752044448170f);
    const float s = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(g), 0.35f, 1.f));
    float p = 0.048942551f;
    p = __builtin_fmaf(p, s, -0.202119678f);
    p = __builtin_fmaf(p, s, 0.240641415f);
    p = __builtin_fmaf(p, s, -0.0170239024f);
    p = __builtin_fmaf(p, s, 0.155961677f);
    p = __builtin_fmaf(p, s, 0.133355066f);
    p = __builtin_fmaf(p, s, 0.140270352f);
    p = __builtin_fmaf(p, s, -2.73154237e-5f);
    const float tail = bell * p;
    return g < 0.f ? tail : 1.f - tail;
}

template <int ACT> __device__ __forceinline__ float act_value(float g)
{
    if constexpr (ACT == kActSilu) return g * logistic(g);
    else if constexpr (ACT == kActGelu) {
        float bell;
        return g * normal_cdf(g, bell);
    }
    else return g <= 0.f ? 0.f : g;
}

template <int ACT> __device__ __forceinline__ float act_both(float g, float& slope)
{
    if constexpr (ACT == kActSilu) {
        const float s = logistic(g);
        const float a = g * s;
        slope = __builtin_fmaf(a, 1.f - s, s);
        return a;
    } else if constexpr (ACT == kActGelu) {
        float bell;
        const float cdf = normal_cdf(g, bell);
        slope = __builtin_fmaf(g * 0.39894228040143268f, bell, cdf);
        return g * cdf;
    } else {
        slope = g <= 0.f ? 0.f : 1.f;
        return g <= 0.f ? 0.f : g;
    }
}

// f(constant) with the activation that `act` names
template <typename F> __device__ __forceinline__ void with_act(int act, F f)
{
    if (act == kActSilu) f(std::integral_constant<int, kActSilu>());
    else if (act == kActGelu) f(std::integral_constant<int, kActGelu>());
    else f(std::integral_constant<int, kActRelu>());
}

template <typename T> __device__ __forceinline__ short bits_of(float x)
{
    const T t = (T)x;
    return __builtin_bit_cast(short, t);
}
template <typename T> __device__ __forceinline__ float value_of(short b) { return (float)__builtin_bit_cast(T, b); }

// Rounded elements as they are, whatever is done with them next: a product and its rounding can be one instruction with one rounding, and for another use of the same element
// two with two, which at ties differ by a last place.
__device__ __forceinline__ short8v settled(short8v v)
{
    uint4v w = __builtin_bit_cast(uint4v, v);
    asm("" : "+v"(w));
    return __builtin_bit_cast(short8v, w);
}
__device__ __forceinline__ bool is_number(float x) { return fabsf(x) < __builtin_inff(); }
// What is left of x beside the value it was rounded to; nothing where that is no number.
template <typename T> __device__ __forceinline__ short rest_of(float x, short b)
{
    const float v = value_of<T>(b);
    return bits_of<T>(is_number(v) ? x - v : 0.f);
}
// Result (m, n) of kOpWeight in a call of few rows, from what its operands were rounded to: where an infinity is among the products, which a rest may turn into a NaN.
template <typename T> __device__ __forceinline__ float without_rest(const GatedProduct& q, int64_t m, int64_t n)
{
    float sum = 0.f;
#pragma unroll 1
    for (int64_t k = 0; k < q.K; k += 2) {
        const int64_t at_a = (k >> q.twice_a) * q.a.ld + m, at_b = (k >> q.twice_b) * q.b.ld + n;
        float a = 0.f, b = 0.f;
        if (m < q.M) a = value_of<T>(((const short*)q.a.p)[at_a]);
        if (n < (q.half ? 2 * q.half : q.N)) b = value_of<T>(((const short*)q.b.p)[at_b]);
        const float ab = a * b;
        sum += std::is_same<T, _Float16>::value ? ldexpf(ab, q.scale[(q.twice_b ? at_a : at_b) >> 3]) : ab;
    }
    return sum;
}

// Eight neighbouring elements at any even address: one instruction all the same.
typedef short short8u __attribute__((ext_vector_type(8), aligned(2)));
__device__ __forceinline__ short* element(const GatedMat& m, int64_t r, int64_t c) { return (short*)m.p + r * m.ld + c; }
__device__ __forceinline__ void store8(const GatedMat& m, int64_t r, int64_t c, short8v v) { *(short8u*)element(m, r, c) = v; }
__device__ __forceinline__ short8v load8(const GatedMat& m, int64_t r, int64_t c) { return *(const short8u*)element(m, r, c); }

// The first `n` of eight elements, zeros behind them (bits, whatever they mean: NaN goes too); a vector without its first `n` (1 to 7).
__device__ __forceinline__ short8v first_of(short8v v, int n)
{
    uint4v w = __builtin_bit_cast(uint4v, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = n >= 2 * j + 2 ? w[j] : n == 2 * j + 1 ? w[j] & 0xffffu : 0u;
    return __builtin_bit_cast(short8v, w);
}
__device__ __forceinline__ short8v without_first(short8v v, int n)
{
    uint4v w = __builtin_bit_cast(uint4v, v);
    if (n & 4) w = uint4v{w[2], w[3], 0u, 0u};
    if (n & 2) w = uint4v{w[1], w[2], w[3], 0u};
    if (n & 1) w = uint4v{__builtin_amdgcn_alignbit(w[1], w[0], 16), __builtin_amdgcn_alignbit(w[2], w[1], 16), __builtin_amdgcn_alignbit(w[3], w[2], 16), w[3] >> 16};
    return __builtin_bit_cast(short8v, w);
}
// Columns c to c + 7 of row r as far as there are `cols`: the last piece of a row goes out element by element, all at once.
__device__ __forceinline__ void store_some(const GatedMat& m, int64_t r, int64_t c, int64_t cols, short8v v)
{
    if (c + 8 <= cols) store8(m, r, c, v);
    else {
        short* const to = element(m, r, c);
        const int n = (int)(cols - c);
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < n) to[k] = v[k];
    }
}

constexpr int kStep = kGatedStep;

// Wait until at most N of this wavefront's loads to shared memory are on their way and its reads of shared memory are done, then for the others.
template <int N> __device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// One operand's way to shared memory: R rows (adjacent) or columns (strided) of the tile, by `THREADS` threads.
template <bool ADJ, int R, int THREADS> struct Mover {
    static constexpr int kPieces = R * 8 / THREADS;           // 16-byte pieces a thread moves per step
    static_assert(R * 8 % THREADS == 0, "");
    static constexpr int kRow = ADJ ? 8 : R / 8;              // pieces in a row of the tile
    const unsigned short* src[kPieces];
    int at;                                                   // adjacent: the piece's place along the sum; strided: the first piece's row

    static __device__ __forceinline__ int turn(int k)         // strided: how row k's pieces are turned
    {
        return 2 * (k & 3) + (R >= 128 ? 8 * ((k >> 3) & 1) : 0);
    }
    // Adjacent: element (row, k) at base + row * ld + k; pick(row of the tile) is where its row begins.
    // Strided: element (k, column) at base + k * ld + column; pick(piece of a row of the tile) is where its eight columns begin.
    // (twice: 1 where the operand has each row twice, which is so in sums of one step only)
    template <typename Pick>
    __device__ __forceinline__ void start(int64_t ld, int64_t k0, int tid, Pick pick, int twice = 0)
    {
        if constexpr (ADJ) {
            const int s = tid & 7;
            at = 8 * (s ^ ((tid >> 3) & 7));                  // (rows of one thread's pieces are multiples of 8 apart)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) src[i] = pick(i * (THREADS / 8) + (tid >> 3)) + k0 + at;
        } else {
            at = tid / kRow;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int k = i * (THREADS / kRow) + tid / kRow;
                const int c = (tid % kRow) ^ turn(k);
                src[i] = pick(c) + ((k0 + k) >> twice) * ld;
            }
        }
    }
    // Requests the next step; `left` elements of the sum are left (what is behind them is taken as zero).
    __device__ __forceinline__ void request(unsigned lds, int64_t ld, int64_t left, const unsigned short* zeros)
    {
        if (left >= kStep) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) load_to_lds(src[i], lds + i * THREADS * 16);
        } else {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int k = ADJ ? at : at + i * (THREADS / kRow);
                load_to_lds(k < left ? src[i] : zeros, lds + i * THREADS * 16);
            }
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) src[i] += ADJ ? (int64_t)kStep : kStep * ld;
    }
};

// The same way by registers, for rows at any address and of any length of 8 or more: pieces that end behind the last element of a row are its last eight,
// shifted when they go to shared memory.
template <bool ADJ, int R, int THREADS> struct Loose {
    using Whole = Mover<ADJ, R, THREADS>;
    static constexpr int kPieces = Whole::kPieces, kRow = Whole::kRow, kShifts = ADJ ? 1 : kPieces;
    const unsigned short* src[kPieces];
    int at, shift[kShifts];

    // Adjacent: pick(row of the tile) is where its row begins.  Strided: pick(piece of a row of the tile, its first column) is where column 0 of its matrix begins; the
    // matrix has `cols` columns.
    template <typename Pick>
    __device__ __forceinline__ void start(int64_t ld, int64_t k0, int64_t cols, int tid, Pick pick, int twice = 0)
    {
        if constexpr (ADJ) {
            const int s = tid & 7;
            at = 8 * (s ^ ((tid >> 3) & 7));
#pragma unroll
            for (int i = 0; i < kPieces; ++i) src[i] = pick(i * (THREADS / 8) + (tid >> 3)) + k0 + at;
        } else {
            at = tid / kRow;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int k = i * (THREADS / kRow) + tid / kRow;
                int64_t col;
                const unsigned short* const base = pick((tid % kRow) ^ Whole::turn(k), col);
                src[i] = base + min(col, cols - 8) + ((k0 + k) >> twice) * ld;
                shift[i] = col < cols ? (int)max(col + 8 - cols, (int64_t)0) : 0;         // (results of columns that are not there go nowhere)
            }
        }
    }
    __device__ __forceinline__ void request(short8v* v, int64_t ld, int64_t left, const unsigned short* zeros)
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const unsigned short* from = src[i];
            if constexpr (ADJ) {
                const int64_t n = left - at;
                if (n < 8) from = n > 0 ? from - (8 - n) : zeros;
            } else if (at + i * (THREADS / kRow) >= left) from = zeros;
            v[i] = *(const short8u*)from;
            src[i] += ADJ ? (int64_t)kStep : kStep * ld;
        }
    }
    __device__ __forceinline__ void put(unsigned lds, const short8v* v, int64_t left, int tid) const
    {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int n = ADJ ? (int)max(min(at + 8 - left, (int64_t)8), (int64_t)0) & 7 : shift[i < kShifts ? i : 0];     // (8: nothing but zeros)
            *(lds_short8*)(size_t)(lds + (i * THREADS + tid) * 16) = n ? without_first(v[i], n) : v[i];
        }
    }
};

// Operands of an instruction from the tile: fragment f covers rows (columns) first + 16 f .. + 15, summed index 32 h + 8 (lane / 16) + i.
template <bool ADJ, int R> struct Reader {
    int lane_off;                                             // adjacent: bytes of this lane's place for h = 0 ...
    int other;                                                // ... and for h = 1; strided: the lane's turn
    int first;
    __device__ __forceinline__ void start(int first_, int lane)
    {
        first = first_;
        const int i = lane & 15, q = lane >> 4;
        if constexpr (ADJ) {
            lane_off = (first + i) * 128 + ((q ^ (i & 7)) << 4);
            other = (first + i) * 128 + (((4 + q) ^ (i & 7)) << 4);
        } else {
            lane_off = (8 * q + (i >> 2)) * (2 * R) + ((i & 1) << 3) + (((i & 3) >> 1) << 4);
            other = 2 * (i >> 2) + (R >= 128 ? 8 * (q & 1) : 0);
        }
    }
    __device__ __forceinline__ short8v read(unsigned tile, int f, int h) const
    {
        if constexpr (ADJ) {
            return *(lds_short8*)(size_t)(tile + (h ? other : lane_off) + f * 16 * 128);
        } else {
            const unsigned at = tile + lane_off + ((((first >> 3) + 2 * f) ^ other) << 4) + h * 32 * 2 * R;
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(size_t)at);
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(size_t)(at + 4 * 2 * R));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// Tile, wavefronts along its rows and columns, steps in shared memory (all but one of them on their way).  A unit holds one workgroup of the large kind, two of the
// medium, three of the small, two of those for 16 rows, one of those for 32, whose steps take a little more than half of its shared memory.  Measured beside these: small tiles with four steps (two workgroups to a unit, 3 to 25 %
// slower), medium ones on four wavefronts (5 to 10 % slower) or with four steps (faster by as much on fewer tiles than units, slower by 20 % on more), tiles
// for few rows with five to eight steps (the same), 256 x 128 with three steps (of 90 products from 500 to 8,192 rows 4 to 10 % faster in three, the same in six, slower in the others).
template <int TILE> struct Shape;
template <> struct Shape<kTileLarge> { static constexpr int BM = 256, BN = 256, WM = 2, WN = 4, STAGES = 2; };
template <> struct Shape<kTileMedium> { static constexpr int BM = 128, BN = 128, WM = 2, WN = 4, STAGES = 2; };
template <> struct Shape<kTileDeep> { static constexpr int BM = 128, BN = 128, WM = 2, WN = 4, STAGES = 3; };
template <> struct Shape<kTileSmall> { static constexpr int BM = 64, BN = 64, WM = 2, WN = 2, STAGES = 3; };
template <> struct Shape<kTile32> { static constexpr int BM = 32, BN = 128, WM = 1, WN = 2, STAGES = 4; };
template <> struct Shape<kTile16> { static constexpr int BM = 16, BN = 128, WM = 1, WN = 2, STAGES = 4; };

template <int TILE> constexpr int tile_threads() { return 64 * Shape<TILE>::WM * Shape<TILE>::WN; }
// Wavefronts that share a SIMD's registers: two workgroups of the medium kind to a unit need 128 a lane (one register more, and 1,910 rows of hidden 2,688 in kOpDown
// take 88 us for 57), three of the small kind 168.
template <int TILE> constexpr int tile_waves() { return TILE == kTileMedium ? 4 : TILE == kTileSmall ? 3 : 2; }
// The results leave through shared memory, in turns; kOpDown's have G and U beside them.
template <GatedOp OP, int TILE> constexpr int tile_turns() { return TILE == kTileLarge ? (OP == kOpDown ? 4 : 2) : (TILE == kTileMedium || TILE == kTileDeep) && OP == kOpDown ? 2 : 1; }
template <int TILE> constexpr int tile_pitch() { return Shape<TILE>::BN + 4; }             // floats from one row to the next
template <GatedOp OP, int TILE> constexpr unsigned tile_lds()
{
    using S = Shape<TILE>;
    constexpr unsigned stages = (unsigned)S::STAGES * (S::BM + S::BN) * 128u, rows = S::BM / tile_turns<OP, TILE>();
    constexpr unsigned out = rows * (tile_pitch<TILE>() * 4u + (OP == kOpDown ? S::BN * 4u : 0u));
    return stages > out ? stages : out;
}

// Parts of a sum on their way between workgroups of different dies: written through to where all dies see them, and read from there.
// (No inline assembly for the stores: only the compiler knows how long a matrix instruction's result must not be read.)
__device__ __forceinline__ void store_shared(float4v* to, float4v v)
{
    typedef unsigned long long word2 __attribute__((ext_vector_type(2)));
    const word2 w = __builtin_bit_cast(word2, v);
    unsigned long long* at = reinterpret_cast<unsigned long long*>(to);
    __hip_atomic_store(at, w[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(at + 1, w[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename P> __device__ __forceinline__ P* uniform(P* p)           // a wavefront's common address, for scalar registers
{
    const uint64_t a = (uint64_t)p;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)a), hi = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));
    return (P*)((uint64_t)hi << 32 | lo);
}

// Four pieces of each of four parts, which begin at the addresses p: 16 bytes a lane at far[k] behind them.  (The wait stands in the same block as the loads: the
// compiler does not know that they are on their way.)
__device__ __forceinline__ void load_shared(const float4v* const* p, const unsigned* far, float4v* v)
{
    asm volatile("global_load_dwordx4 %0, %16, %20 sc1\n\t"
                 "global_load_dwordx4 %1, %17, %20 sc1\n\t"
                 "global_load_dwordx4 %2, %18, %20 sc1\n\t"
                 "global_load_dwordx4 %3, %19, %20 sc1\n\t"
                 "global_load_dwordx4 %4, %16, %21 sc1\n\t"
                 "global_load_dwordx4 %5, %17, %21 sc1\n\t"
                 "global_load_dwordx4 %6, %18, %21 sc1\n\t"
                 "global_load_dwordx4 %7, %19, %21 sc1\n\t"
                 "global_load_dwordx4 %8, %16, %22 sc1\n\t"
                 "global_load_dwordx4 %9, %17, %22 sc1\n\t"
                 "global_load_dwordx4 %10, %18, %22 sc1\n\t"
                 "global_load_dwordx4 %11, %19, %22 sc1\n\t"
                 "global_load_dwordx4 %12, %16, %23 sc1\n\t"
                 "global_load_dwordx4 %13, %17, %23 sc1\n\t"
                 "global_load_dwordx4 %14, %18, %23 sc1\n\t"
                 "global_load_dwordx4 %15, %19, %23 sc1\n\t"
                 "s_waitcnt vmcnt(0)"
                 : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7]), "=&v"(v[8]), "=&v"(v[9]),
                   "=&v"(v[10]), "=&v"(v[11]), "=&v"(v[12]), "=&v"(v[13]), "=&v"(v[14]), "=&v"(v[15])
                 : "v"(far[0]), "v"(far[1]), "v"(far[2]), "v"(far[3]), "s"(p[0]), "s"(p[1]), "s"(p[2]), "s"(p[3]) : "memory");
}

// H, dG and dU in f16: the operands of the next product, whose range the sums that make them need not keep to (G = U = 300 make 90,000).  Eight neighbouring elements of a row whose
// largest would be rounded to infinity are held as multiples of 2^e, as small as it takes to bring that one below 2^15, and e goes into a byte of its own.  They have the
// relative accuracy of f16, and absolutely that of 2^-39 of the eight's largest.  Infinities and NaN stay what they are.  Where nothing is that large this costs a few
// instructions for eight elements; bytes are written once it has happened to this block.
constexpr float kLargestHalf = 65520.f;                        // and beyond: rounded to infinity
__device__ __forceinline__ bool has_no_number(short8v v)       // of f16: infinities and NaN
{
    const uint4v w = (__builtin_bit_cast(uint4v, v) & 0x7c007c00u) + 0x04000400u;
    return ((w[0] | w[1] | w[2] | w[3]) & 0x80008000u) != 0u;
}
// value(k): element k of the eight.  pair: rows 2 r and 2 r + 1 are theirs (see GatedProduct).
template <typename T, typename F> __device__ __forceinline__ void store_scaled(const GatedProduct& q, bool pair, const GatedMat& to, int64_t r, int64_t c, unsigned char* scale, F value)
{
    float top = 0.f;
#pragma unroll 1
    for (int k = 0; k < 8; ++k) {
        const float size = fabsf(value(k));
        if (size < __builtin_inff()) top = fmaxf(top, size);
    }
    const int64_t row = pair ? 2 * r : r;
    int e = 0;
    if (top >= kLargestHalf) {
        e = (int)(__float_as_uint(top) >> 23) - 127 - 14;
        q.scaled[0] = 1u;
        q.scaled[1 + q.turn] = 1u;
#pragma unroll 1
        for (int k = 0; k < 8; ++k) {
            const float v = ldexpf(value(k), -e);
            unsigned b = (unsigned short)bits_of<T>(v);
            asm("" : "+v"(b));
            *element(to, row, c + k) = (short)b;
            if (pair) *element(to, row + 1, c + k) = rest_of<T>(v, (short)b);
        }
    }
    scale[(row * to.ld + c) >> 3] = (unsigned char)e;          // (0: the eight stand there as they were rounded)
    if (pair) scale[((row + 1) * to.ld + c) >> 3] = (unsigned char)e;
}

// And their part in the next product: its sum took such elements for what they are held as, so (2^e - 1) times their products are added to the results of this turn, in
// shared memory.  `found`: for every 16 rows (columns) of the tile a bit for each 32 of the summed index that have an e, 16,384 at a time.  What is not finite is in the sum
// already.  This is slow, since operands come element by element, and rare (4,096 rows, p = out = 2,048, hidden 4,096: three columns of H out of range 0.41 ms forward for
// 0.20 and 2.0 backward for 0.45, all of them 7.9 and 27; the widest training step that has none takes as long as before).
constexpr int kFoundWords = 16;
__device__ __forceinline__ short finite_or_zero(short b) { return (b & 0x7c00) == 0x7c00 ? (short)0 : b; }

template <typename T, GatedOp OP, int TILE>
__device__ __forceinline__ void add_scaled(const GatedProduct& q, float* res, int turn, int64_t m0, int64_t n0, int tid, unsigned* found)
{
    using S = Shape<TILE>;
    constexpr int threads = tile_threads<TILE>(), BM = S::BM, BN = S::BN, waves = threads / 64, chunk = 32 * 32 * kFoundWords;
    constexpr int turns = tile_turns<OP, TILE>(), pitch = tile_pitch<TILE>(), wm = BM / S::WM, wt = wm / turns;
    const int lane = tid & 63, wave = tid >> 6, i = lane & 15, o = lane >> 4;
    const bool left = OP != kOpWeight || q.half == 0;          // which operand has exponents
    const int64_t ld = left ? q.a.ld : q.b.ld, len = OP == kOpInput ? 2 * q.half : q.K, cols = OP == kOpWeight && q.half ? 2 * q.half : q.N;
    const short *const pa = (const short*)q.a.p, *const pb = (const short*)q.b.p, *const pb2 = (const short*)q.b2.p;
    for (int64_t k0 = 0; k0 < len; k0 += chunk) {
        const int64_t here = min(len - k0, (int64_t)chunk);
        __syncthreads();
        for (int w = tid; w < 16 * kFoundWords; w += threads) found[w] = 0u;
        __syncthreads();
        auto eight = [&](int64_t r, int64_t c) { return *(const unsigned long long*)(q.scale + ((r * ld + c) >> 3)); };        // of columns c to c + 63
        auto mark = [&](int strip, int64_t block) { atomicOr(found + strip * kFoundWords + (block >> 5), 1u << (block & 31)); };
        if constexpr (OP != kOpWeight) {
            const int64_t words = (here + 63) / 64, rows = min((int64_t)BM, q.M - m0);
            for (int64_t id = tid; id < rows * words; id += threads) {
                const unsigned long long v = eight(m0 + id / words, k0 + id % words * 64);
                if ((unsigned)v) mark((int)(id / words) / 16, id % words * 2);
                if ((unsigned)(v >> 32)) mark((int)(id / words) / 16, id % words * 2 + 1);
            }
        } else {
            const int64_t first = left ? m0 : n0;
            const int words = (left ? BM : BN) / 64;
            for (int64_t id = tid; id < here * words; id += threads) {
                const int64_t c = first + id % words * 64;
                const unsigned long long v = c < ld ? eight(k0 + id / words, c) : 0u;
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if ((unsigned short)(v >> (16 * t))) mark((int)(id % words) * 4 + t, id / words / 32);
            }
        }
        __syncthreads();
        for (int piece = wave; piece < BM / turns / 16 * (BN / 16); piece += waves) {
            const int lr = piece / (BN / 16) * 16, lc = piece % (BN / 16) * 16;
            const int64_t r = m0 + (lr / wt) * wm + turn * wt + lr % wt + i, c = n0 + lc + i;
            if (r - i >= q.M || c - i >= cols) continue;
            const int strip = (int)(left ? r - i - m0 : (int64_t)lc) / 16;
            float4v* const to = reinterpret_cast<float4v*>(res + (lr + i) * pitch + lc + 4 * o);
            float4v sum = *to;
            for (int w = 0; w < kFoundWords; ++w)
                for (unsigned bits = __builtin_amdgcn_readfirstlane(found[strip * kFoundWords + w]); bits; bits &= bits - 1) {
                    const int64_t k = k0 + 32 * (32 * w + __builtin_ctz(bits)) + 8 * o;
                    short8v a, b;
                    int e[8], most = 0;
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        const bool second = OP == kOpInput && k >= q.half;
                        const int64_t kb = k + t - (second ? q.half : 0);
                        const bool in_a = r < q.M && (OP != kOpWeight || k + t < q.K), in_b = c < cols && kb < q.K;
                        a[t] = in_a ? finite_or_zero(OP == kOpWeight ? pa[((k + t) >> q.twice_a) * q.a.ld + r] : pa[r * q.a.ld + k + t]) : (short)0;
                        b[t] = in_b ? finite_or_zero(OP == kOpInput ? (second ? pb2 : pb)[c * q.b.ld + kb] : pb[(OP == kOpWeight ? kb >> q.twice_b : kb) * q.b.ld + c]) : (short)0;
                        const int64_t at = OP != kOpWeight ? r * ld + k + t : (k + t) * ld + (left ? r : c);
                        e[t] = (left ? in_a : in_b) ? (int)q.scale[at >> 3] : 0;
                        most = max(most, e[t]);
                    }
                    // the largest e of the wavefront's elements, those that have it; the next one
                    for (;;) {
                        int top = most;
#pragma unroll
                        for (int d = 1; d < 64; d *= 2) top = max(top, __shfl_xor(top, d));
                        if (top == 0) break;
                        short8v only;
                        most = 0;
#pragma unroll
                        for (int t = 0; t < 8; ++t) {
                            only[t] = e[t] == top ? (left ? a[t] : b[t]) : (short)0;
                            e[t] = e[t] == top ? 0 : e[t];
                            most = max(most, e[t]);
                        }
                        const float4v part = Half<T>::mma(left ? b : only, left ? only : a, float4v{0.f, 0.f, 0.f, 0.f});
                        sum += part * (ldexpf(1.f, top) - 1.f);
                    }
                }
            *to = sum;
        }
    }
    __syncthreads();
}

// Workgroup `id` of a product's tiles_m * tiles_n * splits.  LOOSE: operands at any address, widths as they are.
template <typename T, GatedOp OP, int TILE, bool LOOSE>
__device__ __forceinline__ void tile_body(const GatedProduct& q, int id)
{
    using S = Shape<TILE>;
    constexpr int threads = tile_threads<TILE>(), BM = S::BM, BN = S::BN;
    constexpr int wm = BM / S::WM, wn = BN / S::WN, fm = wm / 16, fn = wn / 16;    // of a wavefront
    constexpr bool a_adj = OP != kOpWeight, b_adj = OP == kOpDown || OP == kOpInput;
    constexpr unsigned a_bytes = BM * 128, b_bytes = BN * 128;
    constexpr int stages = S::STAGES;
    extern __shared__ __align__(1024) unsigned short stage[];
    __shared__ unsigned arrived;
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned short*)stage;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // f16: whether bytes of exponents are written in any case (the products that make H and D), whether there are any (those that read them).  The word comes to
    // shared memory behind the first operands: in a register it would be waited for, and with it whatever is on its way; in front of them they would wait for it.
    constexpr bool scales = std::is_same<T, _Float16>::value, makes = OP == kOpUp || OP == kOpDown;
    unsigned* found = nullptr;
    if constexpr (scales) {
        __shared__ unsigned words[16 * kFoundWords];            // (the word fills the first 64)
        static_assert(BM <= 256 && BN <= 256 && 16 * kFoundWords >= 64, "");
        found = words;
        if (!makes && blockIdx.x == 0 && tid == 0) q.scaled[2 - q.turn] = 0u;
    }
    auto ask_word = [&]() {
        if constexpr (scales)
            if (wave == 0) load_word_to_lds((const int*)(q.scaled + (makes ? 0 : 1 + q.turn)), (unsigned)(size_t)(__attribute__((address_space(3))) unsigned*)found);
    };
    const int split = id % q.splits;
    const int tile = id / q.splits;
    constexpr int kGroup = 8;                                  // tile rows that are walked through together
    const int group = tile / (kGroup * q.tiles_n), in_group = tile % (kGroup * q.tiles_n);
    const int rows_here = min(kGroup, q.tiles_m - group * kGroup);
    const int tm = group * kGroup + in_group % rows_here, tn = in_group / rows_here;
    const int64_t m0 = (int64_t)tm * BM;
    const int64_t n0 = (int64_t)tn * (OP == kOpUp ? BN / 2 : BN);

    // the share of the sum: steps [s0, s1); kOpInput: the steps of the first half, then those of the second
    const int64_t len = OP == kOpInput ? 2 * q.half : q.K;
    const int steps = (int)((len + kStep - 1) / kStep);
    const int s0 = split * q.per_split, s1 = min(steps, s0 + q.per_split);
    const unsigned short* zeros = (const unsigned short*)q.zeros;

    const unsigned short* pa = (const unsigned short*)q.a.p;
    const unsigned short* pb = (const unsigned short*)q.b.p;
    const unsigned short* pb2 = (const unsigned short*)q.b2.p;
    // where row (adjacent) or the eight columns from `at` on (strided) of the left tile begin; what is behind the last ones is read from these
    auto left_at = [&](int at) {
        if constexpr (a_adj) { const int64_t r = m0 + at; return pa + (r < q.M ? r : q.M - 1) * q.a.ld; }
        else { const int64_t c = m0 + at; return pa + (c < q.a_cols ? c : q.a_cols - 8); }
    };
    const int half_steps = OP == kOpInput ? (int)(q.half / kStep) : 0, twice_a = OP == kOpWeight ? q.twice_a : 0;
    Mover<b_adj, BN, threads> mb;
    auto start_b = [&](int step) {
        const bool second = OP == kOpInput && step >= half_steps;
        mb.start(q.b.ld, (int64_t)(second ? step - half_steps : step) * kStep, tid, [&](int c) {
            if constexpr (b_adj) { const int64_t r = n0 + c; return (second ? pb2 : pb) + (r < q.N ? r : q.N - 1) * q.b.ld; }
            else if constexpr (OP == kOpUp) {                  // a wavefront's columns: wn / 2 of Wg, then the same of Wu
                const int w = c / (wn / 8), in = c % (wn / 8);
                const int64_t col = n0 + w * (wn / 2) + (in % (wn / 16)) * 8;
                return (in >= wn / 16 ? pb2 : pb) + (col < q.b_cols ? col : q.b_cols - 8);
            } else { const int64_t col = n0 + 8 * c; return pb + (col < q.b_cols ? col : q.b_cols - 8); }
        }, OP == kOpWeight ? q.twice_b : 0);
    };
    if constexpr (!LOOSE) start_b(s0);
    const unsigned lds_a = lds0 + (unsigned)__builtin_amdgcn_readfirstlane(wave * 1024), lds_b = lds_a + stages * a_bytes;
    // elements of the sum that are left from `step` on; the left operand of kOpMul and kOpInput has zeros behind its columns
    auto left_a = [&](int step) { return OP == kOpMul || OP == kOpInput ? (int64_t)kStep : q.K - (int64_t)step * kStep; };
    auto request_b = [&](int step, int buf) {
        if (OP == kOpInput && step == half_steps && step > s0) start_b(step);
        mb.request(lds_b + buf * b_bytes, q.b.ld, q.K - (int64_t)(OP == kOpInput && step >= half_steps ? step - half_steps : step) * kStep, zeros);
    };

    Reader<b_adj, BN> rb;
    const int wrow = (wave / S::WN) * wm, wcol = (wave % S::WN) * wn;
    rb.start(wcol, lane);

    float4v acc[fm][fn];
#pragma unroll
    for (int i = 0; i < fm; ++i)
#pragma unroll
        for (int j = 0; j < fn; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};

    if constexpr (TILE == kTileLarge) {
        // One workgroup to a unit, so the matrix units wait for whatever its wavefronts wait for.  What took the time was the way from L2 to shared memory:
        // 64 KB a step, 2,760 cycles if nothing else is done and requests never pause, against 2,048 of the matrix units; asked for in one go at the head
        // of a step and waited for at its end it took 3,600.  So the requests are spread over the step, and each has a whole step to come back.
        // The left tile is two sub-tiles, of the first and of the second 64 rows of both rows of wavefronts, and a step's matrix instructions go through
        // the first, then through the second.  The right operands of a step are all in registers before its first half is done: with the first half, the place of
        // the right tile and of the first sub-tile are free for the step after the next.
        //   first half    requests the second sub-tile of the next step;    ends when this step's second sub-tile has come
        //   second half   requests the right tile and the first sub-tile of the step after the next;    ends when those of the next step have come
        // Operands are read two fragments ahead, across the meetings too.
        static_assert(S::WM == 2 && wm == 128 && fn == 4 && stages == 2, "");
        using Sub = Mover<a_adj, 128, threads>;
        constexpr unsigned sub_bytes = 128 * 128;
        constexpr int sub_loads = Sub::kPieces, late = sub_loads, early = sub_loads + Mover<b_adj, BN, threads>::kPieces;
        Sub sub[2];
#pragma unroll
        for (int x = 0; x < 2; ++x)
            sub[x].start(q.a.ld, (int64_t)s0 * kStep, tid, [&](int r) { const int at = a_adj ? r : 8 * r; return left_at(at + (at & 64) + 64 * x); }, twice_a);
        Reader<a_adj, 128> ra;
        ra.start((wave / S::WN) * 64, lane);
        auto request_sub = [&](int step, int x) { sub[x].request(lds_a + ((step - s0) & 1) * a_bytes + x * sub_bytes, q.a.ld, left_a(step), zeros); };
        // fragment e of a step: rows 16 (e / 2) .. + 15 of the wavefront's, half e % 2 of the sum
        auto read_a = [&](unsigned t, int e) { return ra.read(t + (e >= 8 ? sub_bytes : 0u), (e >> 1) & 3, e & 1); };
        short8v af[4], bf[2][fn];
        ask_word();
        if (s0 < s1) {
            request_b(s0, 0);
            request_sub(s0, 0);
            request_sub(s0, 1);
            if (s0 + 1 < s1) {
                request_b(s0 + 1, 1);
                request_sub(s0 + 1, 0);
                wait_and_meet<late + early>();
            } else {
                wait_and_meet<0>();
            }
#pragma unroll
            for (int j = 0; j < fn; ++j) {
                bf[0][j] = rb.read(lds0 + stages * a_bytes, j, 0);
                bf[1][j] = rb.read(lds0 + stages * a_bytes, j, 1);
            }
            af[0] = read_a(lds0, 0);
            af[1] = read_a(lds0, 1);
        }
        for (int s = s0; s < s1; ++s) {
            const int buf = (s - s0) & 1;
            const unsigned ta = lds0 + buf * a_bytes, na = lds0 + (buf ^ 1) * a_bytes, nb = lds0 + stages * a_bytes + (buf ^ 1) * b_bytes;
            const bool next = s + 1 < s1, after = s + 2 < s1;
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                if (e == 2 && next) request_sub(s + 1, 1);
                if (e == 6) {
                    if (next) wait_and_meet<late + early>();
                    else wait_and_meet<0>();
                }
                if (e == 8 && after) request_sub(s + 2, 0);
                if (e == 10 && after) request_b(s + 2, buf);
                if (e == 14) {
                    if (after) wait_and_meet<late + early>();
                    else wait_and_meet<0>();
                }
                if (e < 14) {
                    af[(e + 2) & 3] = read_a(ta, e + 2);
                    af[(e + 3) & 3] = read_a(ta, e + 3);
                } else if (next) {
                    af[0] = read_a(na, 0);
                    af[1] = read_a(na, 1);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int j = 0; j < fn; ++j) acc[e >> 1][j] = Half<T>::mma(bf[h][j], af[(e + h) & 3], acc[e >> 1][j]);
                    if (e == 14 && next) {
#pragma unroll
                        for (int j = 0; j < fn; ++j) bf[h][j] = rb.read(nb, j, h);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    } else if constexpr (TILE == kTileDeep && !LOOSE) {
        // As many tiles as units or fewer: one workgroup to a unit, three steps in shared memory, operands read two fragments ahead, across steps too (a
        // step's last two rows of fragments are multiplied when all its operands have been read and the next step has come).
        // Against the medium kind at up to 256 tiles up to 30 % less time, 8 % in the middle (500 rows, p = 2,048, hidden 4,096, kOpUp: 27.7 us for 35.3),
        // beyond 10 to 50 % more.
        Mover<a_adj, BM, threads> ma;
        ma.start(q.a.ld, (int64_t)s0 * kStep, tid, [&](int r) { return left_at(a_adj ? r : 8 * r); }, twice_a);
        Reader<a_adj, BM> ra;
        ra.start(wrow, lane);
        auto request = [&](int step, int buf) {
            ma.request(lds_a + buf * a_bytes, q.a.ld, left_a(step), zeros);
            request_b(step, buf);
        };
        constexpr int loads = Mover<a_adj, BM, threads>::kPieces + Mover<b_adj, BN, threads>::kPieces, groups = 2 * fm;
        static_assert(groups % 4 == 0 && fn <= fm && stages >= 3, "");
        short8v af[4], bf[2][fn];
        unsigned ta = lds0, tb = lds0 + stages * a_bytes;
        int buf = 0;
#pragma unroll
        for (int i = 0; i < stages - 1; ++i)
            if (s0 + i < s1) request(s0 + i, i);
        ask_word();
        if (s0 < s1) {
            if (s0 + stages - 1 <= s1) wait_and_meet<(stages - 2) * loads>();
            else wait_and_meet<0>();
#pragma unroll
            for (int j = 0; j < fn; ++j) bf[0][j] = rb.read(tb, j, 0);
            af[0] = ra.read(ta, 0, 0);
            af[1] = ra.read(ta, 1, 0);
        }
        for (int s = s0; s < s1; ++s) {
            const int to = buf == 0 ? stages - 1 : buf - 1;    // the place of the step before this one, which all have read
            buf = buf + 1 == stages ? 0 : buf + 1;
            const unsigned na = lds0 + buf * a_bytes, nb = lds0 + stages * a_bytes + buf * b_bytes;
            const bool more = s + stages - 1 < s1;
#pragma unroll
            for (int g = 0; g < groups; ++g) {
                if (g == 0 && more) request(s + stages - 1, to);
                if (g + 2 < groups) af[(g + 2) & 3] = ra.read(ta, (g + 2) % fm, (g + 2) / fm);
                if (g < fn) bf[1][g] = rb.read(tb, g, 1);
                if (g == groups - 2 && s + 1 < s1) {
                    if (more) wait_and_meet<(stages - 2) * loads>();
                    else wait_and_meet<0>();
#pragma unroll
                    for (int j = 0; j < fn; ++j) bf[0][j] = rb.read(nb, j, 0);
                    af[0] = ra.read(na, 0, 0);
                    af[1] = ra.read(na, 1, 0);
                }
#pragma unroll
                for (int j = 0; j < fn; ++j) acc[g % fm][j] = Half<T>::mma(bf[g / fm][j], af[g & 3], acc[g % fm][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
            ta = na;
            tb = nb;
        }
    } else if constexpr (LOOSE) {
        // Through registers, as many steps ahead as otherwise, and two places in shared memory.
        constexpr int ahead = stages - 1;
        using A = Loose<a_adj, BM, threads>;
        using B = Loose<b_adj, BN, threads>;
        A la;
        B lb;
        Reader<a_adj, BM> ra;
        ra.start(wrow, lane);
        if constexpr (a_adj) la.start(q.a.ld, (int64_t)s0 * kStep, 0, tid, left_at);
        else la.start(q.a.ld, (int64_t)s0 * kStep, q.a_cols, tid, [&](int c, int64_t& col) { col = m0 + 8 * c; return pa; }, twice_a);
        auto second_half = [&](int step) { return OP == kOpInput && step >= half_steps; };
        auto begin_b = [&](int step) {
            const bool second = second_half(step);
            const int64_t k0 = (int64_t)(second ? step - half_steps : step) * kStep;
            if constexpr (b_adj) lb.start(q.b.ld, k0, 0, tid, [&](int c) { const int64_t r = n0 + c; return (second ? pb2 : pb) + (r < q.N ? r : q.N - 1) * q.b.ld; });
            else lb.start(q.b.ld, k0, q.b_cols, tid, [&](int c, int64_t& col) {
                if constexpr (OP == kOpUp) {
                    const int w = c / (wn / 8), in = c % (wn / 8);
                    col = n0 + w * (wn / 2) + (in % (wn / 16)) * 8;
                    return in >= wn / 16 ? pb2 : pb;
                } else {
                    col = n0 + 8 * c;
                    return pb;
                }
            }, OP == kOpWeight ? q.twice_b : 0);
        };
        begin_b(s0);
        auto left_b = [&](int step) { return q.K - (int64_t)(second_half(step) ? step - half_steps : step) * kStep; };
        short8v va[ahead][A::kPieces], vb[ahead][B::kPieces];
        auto request = [&](int step, int u) {
            if (OP == kOpInput && step == half_steps && step > s0) begin_b(step);
            la.request(va[u], q.a.ld, left_a(step), zeros);
            lb.request(vb[u], q.b.ld, left_b(step), zeros);
        };
        ask_word();                                            // (the compiler's waits would take it for one of the others behind these)
#pragma unroll
        for (int u = 0; u < ahead; ++u)
            if (s0 + u < s1) request(s0 + u, u);
        int buf = 0;
        for (int s = s0; s < s1; s += ahead) {
#pragma unroll
            for (int u = 0; u < ahead; ++u) {
                if (s + u >= s1) break;
                const unsigned ta = lds0 + buf * a_bytes, tb = lds0 + stages * a_bytes + buf * b_bytes;
                la.put(ta, va[u], left_a(s + u), tid);
                lb.put(tb, vb[u], left_b(s + u), tid);
                if (s + u + ahead < s1) request(s + u + ahead, u);
                // (behind it all have read the step before this one, whose place the next one takes)
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    short8v af[fm], bf[fn];
#pragma unroll
                    for (int j = 0; j < fn; ++j) bf[j] = rb.read(tb, j, h);
#pragma unroll
                    for (int i = 0; i < fm; ++i) af[i] = ra.read(ta, i, h);
#pragma unroll
                    for (int i = 0; i < fm; ++i)
#pragma unroll
                        for (int j = 0; j < fn; ++j) acc[i][j] = Half<T>::mma(bf[j], af[i], acc[i][j]);
                }
                buf ^= 1;
            }
        }
    } else {
        Mover<a_adj, BM, threads> ma;
        ma.start(q.a.ld, (int64_t)s0 * kStep, tid, [&](int r) { return left_at(a_adj ? r : 8 * r); }, twice_a);
        Reader<a_adj, BM> ra;
        ra.start(wrow, lane);
        auto request = [&](int step, int buf) {
            ma.request(lds_a + buf * a_bytes, q.a.ld, left_a(step), zeros);
            request_b(step, buf);
        };
        constexpr int loads = Mover<a_adj, BM, threads>::kPieces + Mover<b_adj, BN, threads>::kPieces;      // of a thread and step
#pragma unroll
        for (int i = 0; i < stages - 1; ++i)
            if (s0 + i < s1) request(s0 + i, i);
        ask_word();
        int buf = 0;
        for (int s = s0; s < s1; ++s) {
            const int behind = s1 - 1 - s;                         // steps behind this one
            if (stages > 2 && behind >= stages - 2) wait_and_meet<(stages - 2) * loads>();
            else if (stages > 3 && behind == 1) wait_and_meet<loads>();
            else wait_and_meet<0>();
            // (all have read the step before this one, whose place is free now)
            if (behind >= stages - 1) request(s + stages - 1, buf == 0 ? stages - 1 : buf - 1);
            const unsigned ta = lds0 + buf * a_bytes, tb = lds0 + stages * a_bytes + buf * b_bytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                short8v af[fm], bf[fn];
#pragma unroll
                for (int j = 0; j < fn; ++j) bf[j] = rb.read(tb, j, h);
#pragma unroll
                for (int i = 0; i < fm; ++i) af[i] = ra.read(ta, i, h);
#pragma unroll
                for (int i = 0; i < fm; ++i)
#pragma unroll
                    for (int j = 0; j < fn; ++j) acc[i][j] = Half<T>::mma(bf[j], af[i], acc[i][j]);
            }
            buf = buf + 1 == stages ? 0 : buf + 1;
        }
    }

    if (q.splits > 1) {
        // The parts of a tile, [split][fragment][thread] of four floats (rows behind the last one are left out).  Written, waited for, counted; the last
        // one adds them up.
        static_assert(fm * fn % 4 == 0, "");
        float4v* mine = (float4v*)q.partial + ((size_t)tile * q.splits + split) * (fm * fn) * threads + tid;
#pragma unroll
        for (int i = 0; i < fm; ++i)
            if (m0 + wrow + (lane & 15) + 16 * i < q.M) {
#pragma unroll
                for (int j = 0; j < fn; ++j) store_shared(mine + (i * fn + j) * threads, acc[i][j]);
            }
        wait_and_meet<0>();
        if (tid == 0) arrived = __hip_atomic_fetch_add(q.counter + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (arrived != (unsigned)q.splits - 1) return;
        if (tid == 0) __hip_atomic_store(q.counter + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next launch
        // Four parts at a time: a trip to what other dies wrote takes 0.8 us.
        const float4v* const first = (const float4v*)q.partial + (size_t)tile * q.splits * (fm * fn) * threads;
#pragma unroll
        for (int f = 0; f < fm * fn; f += 4) {
            float4v sum[4];
            unsigned far[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sum[k] = float4v{0.f, 0.f, 0.f, 0.f};
                far[k] = (unsigned)((f + k) * threads + tid) * 16u;
            }
#pragma unroll 1
            for (int p = 0; p < q.splits; p += 4) {
                const float4v* from[4];
                float4v v[16];
#pragma unroll
                for (int k = 0; k < 4; ++k) from[k] = uniform(first + (size_t)min(p + k, q.splits - 1) * (fm * fn) * threads);
                load_shared(from, far, v);
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] += v[k];
                if (p + 1 < q.splits) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[k] += v[4 + k];
                }
                if (p + 2 < q.splits) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[k] += v[8 + k];
                }
                if (p + 3 < q.splits) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[k] += v[12 + k];
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[(f + k) / fn][(f + k) % fn] = sum[k];
        }
    }

    // Out: a lane holds row lane % 16 and four neighbouring columns of every fragment.  They go to shared memory and come back as eight neighbouring
    // columns, so that memory is read and written in whole lines and the code for a result stands there once: code that runs once is paid for with the
    // time that its fetching takes (unrolled, these lines took 20 to 40 us at kOpDown's tiles of 128 and 256).
    constexpr int turns = tile_turns<OP, TILE>(), pitch = tile_pitch<TILE>(), wt = wm / turns;    // rows of a wavefront and turn
    float* const res = reinterpret_cast<float*>(stage);
    constexpr int cols8 = (OP == kOpUp ? BN / 2 : BN) / 8, pieces = (BM / turns) * cols8, mine = pieces / threads;
    static_assert(pieces % threads == 0, "");
    // piece i of this thread in this turn: its row and first column, and where it stands in shared memory
    auto place = [&](int turn, int i, int64_t& r, int64_t& c) {
        const int id = tid + i * threads, lr = id / cols8, lc = 8 * (id % cols8);
        r = m0 + (lr / wt) * wm + turn * wt + lr % wt;
        c = n0 + lc;
        return res + lr * pitch + lc;
    };
    auto floats8 = [](const float* from, float* v) {
        *reinterpret_cast<float4v*>(v) = *reinterpret_cast<const float4v*>(from);
        *reinterpret_cast<float4v*>(v + 4) = *reinterpret_cast<const float4v*>(from + 4);
    };
    constexpr bool pairs = BM <= 64;                           // (few rows do not come in larger tiles)
    constexpr int keep = OP == kOpDown ? mine : 1;
    short8v gk[keep], uk[keep];                                // G and U of the next turn, on their way
    short8v* const gus = reinterpret_cast<short8v*>(res + (BM / turns) * pitch) + tid;            // of this turn, a thread's own
    auto request_gu = [&](int turn) {
        if constexpr (OP == kOpDown) {
#pragma unroll
            for (int i = 0; i < mine; ++i) {
                int64_t r, c;
                place(turn, i, r, c);
                if (r < q.M && q.N >= 8) {
                    const int64_t from = min(c, q.N - 8);      // a row's last piece, and those behind it: its last eight columns, shifted later
                    gk[i] = load8(q.g, r, from);
                    uk[i] = load8(q.u, r, from);
                }
            }
        }
    };
    unsigned any = 0u;
    if constexpr (scales) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (nothing else is on its way here)
    request_gu(0);
#pragma unroll 1
    for (int turn = 0; turn < turns; ++turn) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < turns; ++t)
            if (t == turn) {
#pragma unroll
                for (int i = 0; i < fm / turns; ++i)
#pragma unroll
                    for (int j = 0; j < fn; ++j) {
                        int col = wcol + 16 * j;
                        if constexpr (OP == kOpUp) col = (j < fn / 2 ? 0 : BN / 2 - wn / 2) + (wave % S::WN) * (wn / 2) + 16 * j;      // G left, U right
                        *reinterpret_cast<float4v*>(res + ((wave / S::WN) * wt + 16 * i + (lane & 15)) * pitch + col + 4 * (lane >> 4)) =
                            acc[t * (fm / turns) + i][j];
                    }
            }
        if constexpr (OP == kOpDown) {
#pragma unroll
            for (int i = 0; i < mine; ++i) {
                int64_t r, c;
                place(turn, i, r, c);
                if (c + 8 > q.N) {                             // zeros behind the last column
                    const int left = (int)max(q.N - c, (int64_t)0);
                    gk[i] = first_of(without_first(gk[i], 8 - left), left);
                    uk[i] = first_of(without_first(uk[i], 8 - left), left);
                }
                gus[2 * i * threads] = gk[i];
                gus[(2 * i + 1) * threads] = uk[i];
            }
            if (turn + 1 < turns) request_gu(turn + 1);
        }
        __syncthreads();
        if constexpr (scales) {
            if (turn == 0) any = found[0];
            if constexpr (!makes) {
                if (any) add_scaled<T, OP, TILE>(q, res, turn, m0, n0, tid, found);
            }
        }
        unsigned again = 0u;                                   // pieces that need exponents, or have an infinity or a NaN
        static_assert(mine <= 32, "");
        auto work = [&](auto act) {
#pragma unroll 1
            for (int i = 0; i < mine; ++i) {
                int64_t r, c;
                const float* const at = place(turn, i, r, c);
                if (r >= q.M) continue;
                // (H, dG and dU have q.half columns, a multiple of 64: whole pieces, zeros behind the last column)
                const int left = (int)min(q.N - c, (int64_t)8);
                if constexpr (OP == kOpUp) {
                    if (c >= q.half) continue;
                    float g[8], u[8];
                    floats8(at, g);
                    floats8(at + BN / 2, u);
                    short8v hb, gb, ub;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        hb[k] = bits_of<T>(act_value<act.value>(g[k]) * u[k]);
                        gb[k] = bits_of<T>(g[k]);
                        ub[k] = bits_of<T>(u[k]);
                    }
                    if (left < 8) hb = first_of(hb, left);
                    const bool pair = pairs && q.pair;
                    const int64_t row = pair ? 2 * r : r;
                    if (pairs) hb = settled(hb);
                    store8(q.out, row, c, hb);
                    if (pair) {
                        short8v rest;
#pragma unroll
                        for (int k = 0; k < 8; ++k) rest[k] = rest_of<T>(act_value<act.value>(g[k]) * u[k], hb[k]);
                        store8(q.out, row + 1, c, left == 8 ? rest : first_of(rest, left));
                    }
                    if constexpr (scales) {
                        if (any) {
                            q.scale[(row * q.out.ld + c) >> 3] = 0;
                            if (pair) q.scale[((row + 1) * q.out.ld + c) >> 3] = 0;
                        }
                        if (has_no_number(hb)) again |= 1u << i;
                    }
                    if (q.g.p) {
                        store_some(q.g, r, c, q.N, gb);
                        store_some(q.u, r, c, q.N, ub);
                    }
                } else if constexpr (OP == kOpDown) {
                    if (c >= q.half) continue;
                    short8v& gs = gus[2 * i * threads];
                    short8v& us = gus[(2 * i + 1) * threads];
                    if (q.N < 8)
#pragma unroll 1
                        for (int k = 0; k < left; ++k) {
                            reinterpret_cast<short*>(&gs)[k] = *element(q.g, r, c + k);
                            reinterpret_cast<short*>(&us)[k] = *element(q.u, r, c + k);
                        }
                    float dh[8];
                    floats8(at, dh);
                    if (left < 8) {                            // (an infinity in dY times the zeros behind the last row of Wd is no number)
#pragma unroll
                        for (int k = 0; k < 8; ++k) dh[k] = k < left ? dh[k] : 0.f;
                    }
                    const short8v gb = gs, ub = us;
                    short8v hb, dgb, dub;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float slope;
                        const float u = value_of<T>(ub[k]), a = act_both<act.value>(value_of<T>(gb[k]), slope);
                        hb[k] = bits_of<T>(a * u);
                        dub[k] = bits_of<T>(dh[k] * a);
                        dgb[k] = bits_of<T>(dh[k] * u * slope);
                    }
                    const bool pair = pairs && q.pair, numberless = scales && (has_no_number(hb) || has_no_number(dgb) || has_no_number(dub));
                    const int64_t row = pair ? 2 * r : r;
                    if (pairs) {
                        hb = settled(hb);
                        dgb = settled(dgb);
                        dub = settled(dub);
                    }
                    store8(q.out, row, c, hb);
                    store8(q.out2, row, c, dgb);
                    store8(q.out2, row, c + q.half, dub);
                    if (pair) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            float slope;
                            const float u = value_of<T>(ub[k]), a = act_both<act.value>(value_of<T>(gb[k]), slope);
                            hb[k] = rest_of<T>(a * u, hb[k]);
                            dub[k] = rest_of<T>(dh[k] * a, dub[k]);
                            dgb[k] = rest_of<T>(dh[k] * u * slope, dgb[k]);
                        }
                        store8(q.out, row + 1, c, hb);
                        store8(q.out2, row + 1, c, dgb);
                        store8(q.out2, row + 1, c + q.half, dub);
                    }
                    if constexpr (scales) {
                        if (any)
                            for (int64_t at = row; at <= row + pair; ++at) {
                                unsigned char* const of_d = q.scale2 + ((at * q.out2.ld + c) >> 3);
                                q.scale[(at * q.out.ld + c) >> 3] = of_d[0] = of_d[q.half >> 3] = 0;
                            }
                        if (numberless) again |= 1u << i;
                    }
                } else {
                    // (two halves: q.half is a multiple of 64, eight columns never straddle)
                    const bool second = OP == kOpWeight && q.half && c >= q.half;
                    const GatedMat& to = second ? q.out2 : q.out;
                    const int64_t cc = second ? c - q.half : c;
                    const bool pair = OP != kOpWeight && q.pair;
                    if (pair && (r & 1)) continue;             // (with the row before it)
                    float v[8];
                    floats8(at, v);
                    if (pair) {
                        float rest[8];
                        floats8(at + pitch, rest);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] += is_number(v[k]) ? rest[k] : 0.f;        // (an infinite weight times a rest may have any sign)
                    }
                    short8v b;
#pragma unroll
                    for (int k = 0; k < 8; ++k) b[k] = bits_of<T>(v[k]);
                    store_some(to, pair ? r >> 1 : r, cc, q.N, b);
                    if (OP == kOpWeight && (q.twice_a | q.twice_b)) {
                        float most = 0.f;                      // (NaN where one of the eight is no number)
#pragma unroll
                        for (int k = 0; k < 8; ++k) most = __builtin_fmaf(v[k], 0.f, most);
                        if (!(most == 0.f)) {
#pragma unroll 1
                            for (int k = 0; k < 8; ++k)
                                if (cc + k < q.N && !is_number(at[k])) *element(to, r, cc + k) = bits_of<T>(without_rest<T>(q, r, c + k));
                        }
                    }
                }
            }
        };
        if constexpr (OP == kOpUp || OP == kOpDown) with_act(q.act, work);
        else work(std::integral_constant<int, 0>());
        if constexpr (scales && makes) {
            while (again) {
                const int i = __builtin_ctz(again);
                again &= again - 1u;
                int64_t r, c;
                const float* const at = place(turn, i, r, c);
                const int left = (int)min(q.N - c, (int64_t)8);
#pragma unroll 1
                for (int which = 0; which < (OP == kOpUp ? 1 : 3); ++which) {
                    asm volatile("" : "+s"(which));            // (one piece of code for all three)
                    store_scaled<T>(q, pairs && q.pair, which ? q.out2 : q.out, r, which == 2 ? c + q.half : c, which ? q.scale2 : q.scale, [&](int k) {
                        float v = 0.f;
                        if (k < left)
                            with_act(q.act, [&](auto act) {
                                if constexpr (OP == kOpUp) v = act_value<act.value>(at[k]) * at[BN / 2 + k];
                                else {
                                    const float u = value_of<T>(reinterpret_cast<const short*>(gus + (2 * i + 1) * threads)[k]);
                                    float slope;
                                    const float a = act_both<act.value>(value_of<T>(reinterpret_cast<const short*>(gus + 2 * i * threads)[k]), slope);
                                    v = which == 0 ? a * u : which == 1 ? at[k] * u * slope : at[k] * a;
                                }
                            });
                        return v;
                    });
                }
            }
        }
    }
}

// Workgroups go to the eight dies in turn: a die gets neighbouring tiles, whose operands its L2 then holds.
__device__ __forceinline__ int neighbours(int id, int total)
{
    const int die = id & 7, each = total >> 3, more = total & 7;
    return die * each + min(die, more) + (id >> 3);
}

template <typename T, GatedOp OP, int TILE, bool LOOSE>
__global__ void __launch_bounds__(tile_threads<TILE>(), tile_waves<TILE>()) gated_tile_kernel(GatedProduct q)
{
    tile_body<T, OP, TILE, LOOSE>(q, neighbours(blockIdx.x, gridDim.x));
}

// The products that need nothing but what kOpDown left, in one launch: dX, dWd, [dWg | dWu], as far as they are wanted.  Each begins at a multiple of
// eight workgroups.
struct GradProducts {
    GatedProduct input, down, gate;
    int input_end, down_end, gate_end;
};
template <typename T, int TILE, bool LOOSE>
__global__ void __launch_bounds__(tile_threads<TILE>(), tile_waves<TILE>()) gated_grads_kernel(GradProducts g)
{
    int id = blockIdx.x;
    if (id < g.input_end) {
        const int n = g.input.tiles_m * g.input.tiles_n * g.input.splits;
        if (id < n) tile_body<T, kOpInput, TILE, LOOSE>(g.input, neighbours(id, n));
        return;
    }
    id -= g.input_end;
    const bool down = id < g.down_end;
    const GatedProduct& q = down ? g.down : g.gate;
    if (!down) id -= g.down_end;
    const int n = q.tiles_m * q.tiles_n * q.splits;
    if (id < n) tile_body<T, kOpWeight, TILE, LOOSE>(q, neighbours(id, n));
}

template <typename K> hipError_t prepare_kernel(K kernel, unsigned lds)
{
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

// f(tile, loose) for every kind of tile, and every one that takes operands at any address, until one fails
template <typename F> hipError_t each_tile(F f)
{
    constexpr std::integral_constant<int, kTileMedium> medium{};
    constexpr std::integral_constant<int, kTileDeep> deep{};
    constexpr std::integral_constant<int, kTileSmall> small{};
    hipError_t e = f(std::integral_constant<int, kTileLarge>(), std::false_type());
    if (e == hipSuccess) e = f(medium, std::false_type());
    if (e == hipSuccess) e = f(medium, std::true_type());
    if (e == hipSuccess) e = f(deep, std::false_type());
    if (e == hipSuccess) e = f(deep, std::true_type());
    if (e == hipSuccess) e = f(small, std::false_type());
    if (e == hipSuccess) e = f(small, std::true_type());
    return e;
}
template <typename F> hipError_t each_row_tile(F f)
{
    constexpr std::integral_constant<int, kTile32> of_32{};
    constexpr std::integral_constant<int, kTile16> of_16{};
    hipError_t e = each_tile(f);
    if (e == hipSuccess) e = f(of_32, std::false_type());
    if (e == hipSuccess) e = f(of_32, std::true_type());
    if (e == hipSuccess) e = f(of_16, std::false_type());
    if (e == hipSuccess) e = f(of_16, std::true_type());
    return e;
}

template <typename T, GatedOp OP> hipError_t prepare_op()
{
    return each_row_tile([](auto t, auto loose) { return prepare_kernel(&gated_tile_kernel<T, OP, t.value, loose.value>, tile_lds<OP, t.value>()); });
}
template <typename T> hipError_t prepare_all()
{
    hipError_t e = prepare_op<T, kOpUp>();
    if (e == hipSuccess) e = prepare_op<T, kOpMul>();
    if (e == hipSuccess) e = prepare_op<T, kOpDown>();
    if (e == hipSuccess) e = each_tile([](auto t, auto loose) { return prepare_kernel(&gated_grads_kernel<T, t.value, loose.value>, tile_lds<kOpWeight, t.value>()); });
    return e;
}

template <typename T, GatedOp OP> hipError_t launch_op(const GatedProduct& q, hipStream_t stream)
{
    const dim3 grid((unsigned)(q.tiles_m * q.tiles_n * q.splits));
    return each_row_tile([&](auto t, auto loose) {
        if (q.tile != t.value || q.loose != loose.value) return hipSuccess;
        hipLaunchKernelGGL((gated_tile_kernel<T, OP, t.value, loose.value>), grid, dim3(tile_threads<t.value>()), (tile_lds<OP, t.value>()), stream, q);
        return hipGetLastError();
    });
}

template <typename T> hipError_t launch_any(const GatedProduct& q, GatedOp op, hipStream_t stream)
{
    if (op == kOpUp) return launch_op<T, kOpUp>(q, stream);
    if (op == kOpMul) return launch_op<T, kOpMul>(q, stream);
    if (op == kOpDown) return launch_op<T, kOpDown>(q, stream);
    return hipErrorInvalidValue;
}

// `input`, `down`, `gate` have one kind of tile, and are all loose or none; NULL: not wanted
template <typename T> hipError_t launch_grads(const GatedProduct* input, const GatedProduct* down, const GatedProduct* gate, hipStream_t stream)
{
    GradProducts g{};
    int tile = kTileLarge, end = 0;
    bool loose = false;
    auto add = [&](const GatedProduct* from, GatedProduct& to) {
        if (!from) return 0;
        to = *from;
        tile = from->tile;
        loose = from->loose;
        const int n = (from->tiles_m * from->tiles_n * from->splits + 7) / 8 * 8;
        end += n;
        return n;
    };
    g.input_end = add(input, g.input);
    g.down_end = add(down, g.down);
    g.gate_end = add(gate, g.gate);
    if (end == 0) return hipSuccess;
    return each_tile([&](auto t, auto any) {
        if (tile != t.value || loose != any.value) return hipSuccess;
        hipLaunchKernelGGL((gated_grads_kernel<T, t.value, any.value>), dim3((unsigned)end), dim3(tile_threads<t.value>()), (tile_lds<kOpWeight, t.value>()), stream, g);
        return hipGetLastError();
    });
}

}  // namespace
}  // namespace bmgd
