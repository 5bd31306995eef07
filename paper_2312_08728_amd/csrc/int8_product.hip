// Product in 8-bit integers: y_ij = x_scales[i] w_scales[j] sum_k x_ik w_jk, and the codes of a layer's weights.
//
// Both operands have the summed index adjacent in memory, 16 codes to a lane's operand of v_mfma_i32_16x16x64_i8 (a = A[lane % 16][16 (lane / 16) + i],
// b = B[16 (lane / 16) + i][lane % 16], c[v] = C[4 (lane / 16) + v][lane % 16]).  The instruction forms the transpose of the result, so that a lane ends with four
// neighbouring columns of a row.  Sums are exact, in whatever order parts of them are added.
//
// What bounds it (us).  8,192 x 4,096 x 8,192: 228 on codes of normal numbers (2.4 POP/s; a library's product without scales 305 and 1.8), 281 on uniform ones: the matrix units, busy 56 % of the time at
// 1.65 GHz, the clock that is left under their load.  1 x 4,096 x 8,192: 8.1, 33.6 MB of weights at 5 TB/s and a launch.  333 x 1,365 x 1,000 (rows at any byte): 7.1, a launch, a trip to
// memory and eleven steps of 0.3; with rows of 1,360 5.3.  The layout of weights, made once for a layer, is far from its bytes: see int8_quantize_kernel.
#include "lds_load.h"
#include "operator_calls.h"
#include "rows_device.h"

#include <math.h>

#include <algorithm>
#include <atomic>

using namespace bmgd;

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) int4v lds_int4;
struct __attribute__((packed)) Loose16 { int4v v; };

struct ProductArgs {
    const char *x, *w;
    char* y;
    int64_t ldx, ldw, ldy;
    const float *sx, *sw;
    int64_t rows;
    int p, out;
    int tiles_m, tiles_n;
};

__device__ __forceinline__ int4v mma(int4v w, int4v x, int4v c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, c, 0, 0, 0); }

// The 16 codes at k of a row of p, zeros behind its end
__device__ __forceinline__ int4v codes_at(const char* row, int k, int p)
{
    if (k + 16 <= p) return reinterpret_cast<const Loose16*>(row + k)->v;
    int4v v = 0;
    if (k >= p) return v;
    if (p >= 16) {
        // the row's last 16, moved down
        const unsigned __int128 last = __builtin_bit_cast(unsigned __int128, reinterpret_cast<const Loose16*>(row + p - 16)->v);
        return __builtin_bit_cast(int4v, last >> 8 * (k + 16 - p));
    }
    unsigned __int128 b = 0;
    for (int i = 0; i < p; ++i) b |= (unsigned __int128)(unsigned char)row[i] << 8 * i;
    return __builtin_bit_cast(int4v, b >> 8 * k);
}

// Four neighbouring results of a row, the first `count` of which exist
template <typename T> __device__ __forceinline__ void put_four(T* y, float4v v, int count)
{
    typedef T four __attribute__((ext_vector_type(4)));
    typedef T loose __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    four o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (T)v[i];
    if (count >= 4) *reinterpret_cast<loose*>(y) = o;
    else
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < count) y[i] = o[i];
}
// Four sums with their scales, in 32 bits whatever is done next: a product and its rounding to 16 bits could be one instruction with one rounding.
__device__ __forceinline__ float4v scaled(int4v c, float sx, const float* sw)
{
    float4v v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f = (float)c[i] * sx * sw[i];
        asm("" : "+v"(f));
        v[i] = f;
    }
    return v;
}

constexpr int kFewWaves = 8;

// 16 RF rows and 16 columns for a workgroup, whose wavefronts share the sum; every operand comes straight to registers.
template <typename T, int RF> __global__ void __launch_bounds__(64 * kFewWaves) int8_few_kernel(ProductArgs a)
{
    constexpr int U = RF > 2 ? 4 : 8;
    __shared__ int4v parts[kFewWaves][RF][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = lane & 15, q = lane >> 4;
    const int col = blockIdx.x * 16;
    const int64_t row0 = (int64_t)blockIdx.y * (16 * RF);
    const char* const w = a.w + (int64_t)min(col + in, a.out - 1) * a.ldw;
    const char* x[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) x[f] = a.x + min(row0 + 16 * f + in, a.rows - 1) * a.ldx;
    int4v sum[RF] = {};
    const int whole = a.p >> 6, each = (whole + kFewWaves - 1) / kFewWaves;
    int s = wave * each;
    const int end = min(s + each, whole);
    for (; s + U <= end; s += U) {
        int4v b[U], v[RF][U];
#pragma unroll
        for (int u = 0; u < U; ++u) b[u] = reinterpret_cast<const Loose16*>(w + 64 * (s + u) + 16 * q)->v;
#pragma unroll
        for (int f = 0; f < RF; ++f)
#pragma unroll
            for (int u = 0; u < U; ++u) v[f][u] = reinterpret_cast<const Loose16*>(x[f] + 64 * (s + u) + 16 * q)->v;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int f = 0; f < RF; ++f) sum[f] = mma(b[u], v[f][u], sum[f]);
    }
    for (; s < end; ++s) {
        const int4v b = reinterpret_cast<const Loose16*>(w + 64 * s + 16 * q)->v;
#pragma unroll
        for (int f = 0; f < RF; ++f) sum[f] = mma(b, reinterpret_cast<const Loose16*>(x[f] + 64 * s + 16 * q)->v, sum[f]);
    }
    if (wave == kFewWaves - 1 && a.p & 63) {
        const int k = 64 * whole + 16 * q;
        const int4v b = codes_at(w, k, a.p);
#pragma unroll
        for (int f = 0; f < RF; ++f) sum[f] = mma(b, codes_at(x[f], k, a.p), sum[f]);
    }
#pragma unroll
    for (int f = 0; f < RF; ++f) parts[wave][f][lane] = sum[f];
    __syncthreads();
    if (wave >= RF) return;
    int4v c = parts[0][wave][lane];
#pragma unroll
    for (int i = 1; i < kFewWaves; ++i) c += parts[i][wave][lane];
    const int64_t row = row0 + 16 * wave + in;
    const int j = col + 4 * q;
    if (row >= a.rows || j >= a.out) return;
    float sw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sw[i] = j + i < a.out ? a.sw[j + i] : 0.f;
    put_four(reinterpret_cast<T*>(a.y) + row * a.ldy + j, scaled(c, a.sx[row], sw), a.out - j);
}

constexpr int kStep = 128;          // codes of a row that a step takes

// Wait until at most N of this wavefront's loads to shared memory are on their way and its reads of shared memory are done, then for the others.
template <int N> __device__ __forceinline__ void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// A tile of BM rows and BN columns by WM x WN wavefronts.  A step of an operand lies in shared memory as rows of 128 bytes, eight pieces of 16; piece c of row r
// lies in place c ^ (r & 7), so that the rows that an instruction's lanes read at the same piece lie in different banks.
//   loose      operands at any address, through registers, AHEAD steps on their way, two places in shared memory
//   otherwise  straight to shared memory, AHEAD steps on their way
template <int BM_, int BN_, int WM_, int WN_, int AHEAD_, bool LOOSE_> struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kThreads = 64 * WM * WN, AHEAD = AHEAD_;
    static constexpr bool LOOSE = LOOSE_, kHalves = BM * BN == 256 * 256 && !LOOSE;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;                   // 16 x 16 results of a wavefront
    static constexpr int kPlaces = LOOSE ? 2 : AHEAD + 1;
    static constexpr int kBytes = (BM + BN) * kStep;                             // of a step
    static constexpr int PM = BM * 8 / kThreads, PN = BN * 8 / kThreads;         // pieces that a thread brings
    static constexpr size_t kShared = (size_t)kPlaces * kBytes;
};

// The results of a wavefront leave through its own part of shared memory, so that rows are written in whole lines, as many at a time as it holds.
template <typename T, class C> __device__ __forceinline__ void write_tile(const ProductArgs& a, const int4v (&sum)[C::FM][C::FN], char* shared, int64_t row0, int col0, int wave, int lane)
{
    constexpr int kRow = C::FN * 16 * (int)sizeof(T), kChunks = kRow / 16, kTurn = kChunks < 8 ? kChunks - 1 : 7;
    constexpr int kOnce = C::BM * C::BN * (int)sizeof(T) > (int)C::kShared ? C::FM / 2 : C::FM;
    static_assert(kOnce * 16 * kRow * C::WM * C::WN <= (int)C::kShared, "");
    typedef T four __attribute__((ext_vector_type(4)));
    const int in = lane & 15, q = lane >> 4;
    char* const own = shared + wave * (kOnce * 16 * kRow);
    float sw[C::FN][4];
#pragma unroll
    for (int g = 0; g < C::FN; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) sw[g][i] = a.sw[min(col0 + 16 * g + 4 * q + i, a.out - 1)];
    __syncthreads();
#pragma unroll
    for (int first = 0; first < C::FM; first += kOnce) {
#pragma unroll
        for (int f = 0; f < kOnce; ++f) {
            const float sx = a.sx[min(row0 + 16 * (first + f) + in, a.rows - 1)];
#pragma unroll
            for (int g = 0; g < C::FN; ++g) {
                const float4v v = scaled(sum[first + f][g], sx, sw[g]);
                four o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = (T)v[i];
                const int at = (16 * g + 4 * q) * (int)sizeof(T);
                *reinterpret_cast<four*>(own + (16 * f + in) * kRow + 16 * ((at >> 4) ^ (in & kTurn)) + (at & 15)) = o;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 2
        for (int i = lane; i < kOnce * 16 * kChunks; i += 64) {
            const int r = i / kChunks, c = i % kChunks, j = col0 + c * (16 / (int)sizeof(T));
            const int64_t row = row0 + 16 * first + r;
            const typename Piece<T>::vec v = *reinterpret_cast<const typename Piece<T>::vec*>(own + r * kRow + 16 * (c ^ (r & kTurn)));
            if (row >= a.rows) continue;
            T* const to = reinterpret_cast<T*>(a.y) + row * a.ldy;
            if (j + Piece<T>::N <= a.out) Piece<T>::store(to + j, v);
            else if (j < a.out) Piece<T>::store_part(to, j, 0, a.out, v);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

template <typename T, class C> __global__ void __launch_bounds__(C::kThreads) int8_tile_kernel(ProductArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) char shared[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), in = lane & 15, q = lane >> 4;
    const unsigned base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)shared;
    // workgroups of a die (every eighth one) have neighbouring tiles, eight rows of tiles at a time
    const int total = a.tiles_m * a.tiles_n, id = blockIdx.x;
    const int here = total / 8, more = total % 8, die = id % 8;
    const int at = die * here + min(die, more) + id / 8;
    const int band = 8 * a.tiles_n, top = at / band * 8, high = min(a.tiles_m - top, 8);
    const int tm = top + at % band % high, tn = at % band / high;
    const int64_t row0 = (int64_t)tm * C::BM;
    const int col0 = tn * C::BN;
    const int steps = (a.p + kStep - 1) / kStep;

    // what this thread brings: piece c of row r, to the place that its lane has
    const char *px[C::PM], *pw[C::PN];
    const int r0 = threadIdx.x >> 3, c0 = 16 * ((threadIdx.x & 7) ^ (r0 & 7));
#pragma unroll
    for (int i = 0; i < C::PM; ++i) px[i] = a.x + min(row0 + r0 + i * (C::kThreads / 8), a.rows - 1) * a.ldx;
#pragma unroll
    for (int i = 0; i < C::PN; ++i) pw[i] = a.w + (int64_t)min(col0 + r0 + i * (C::kThreads / 8), a.out - 1) * a.ldw;
    // piece i of x or w of a step, straight to shared memory (behind the end of a row: any, w is taken as zero there)
    auto bring_x = [&](int step, int place, int i) {
        const int k = step * kStep + c0;
        load_to_lds(reinterpret_cast<const unsigned short*>(px[i] + (k < a.p ? k : 0)), base + place * C::kBytes + wave * 1024 + i * C::kThreads * 16);
    };
    auto bring_w = [&](int step, int place, int i) {
        const int k = step * kStep + c0;
        load_to_lds(reinterpret_cast<const unsigned short*>(pw[i] + (k < a.p ? k : 0)), base + place * C::kBytes + C::BM * kStep + wave * 1024 + i * C::kThreads * 16);
    };
    const int m0 = wave / C::WN * (C::FM * 16), n0 = wave % C::WN * (C::FN * 16);
    // operands of an instruction: 16 rows (f) at half h of a step
    auto read_x = [&](int place, int f, int h) {
        return *reinterpret_cast<const int4v*>(shared + place * C::kBytes + (m0 + 16 * f + in) * kStep + 16 * ((4 * h + q) ^ (in & 7)));
    };
    auto read_w = [&](int place, int g, int h) {
        return *reinterpret_cast<const int4v*>(shared + place * C::kBytes + (C::BM + n0 + 16 * g + in) * kStep + 16 * ((4 * h + q) ^ (in & 7)));
    };
    // whether lanes of half h of this step are behind the end
    auto behind = [&](int step, int h) { return step * kStep + 64 * h + 16 * q >= a.p; };
    int4v sum[C::FM][C::FN] = {};

    if constexpr (C::kHalves) {
        // All of w's operands of a step are in registers before half of x's rows have been multiplied; so the first half of x's rows and w make room for the step
        // after the next one in the middle of a step, the second half at the next one's beginning: each is asked for a whole step before it is needed, and nothing is waited for at once.
        // A wavefront's first 64 rows are pieces 0 and 2 of its threads (rows 0-63 and 128-191 of the tile), the other 64 pieces 1 and 3.
        static_assert(C::PM == 4 && C::PN == 4 && C::FM == 8 && C::FN == 4 && C::WM == 2, "");
        constexpr int kLate = 8;                                // loads of a thread on their way at a wait: a half of x, w, a half of x
        auto bring_half = [&](int step, int half) {
            bring_x(step, step & 1, half);
            bring_x(step, step & 1, half + 2);
        };
        auto bring_all_w = [&](int step) {
#pragma unroll
            for (int i = 0; i < 4; ++i) bring_w(step, step & 1, i);
        };
        int4v xf[4], wf[2][4];
        bring_all_w(0);
        bring_half(0, 0);
        bring_half(0, 1);
        if (steps > 1) {
            bring_half(1, 0);
            bring_all_w(1);
            wait_and_meet<6>();
        } else wait_and_meet<0>();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int g = 0; g < 4; ++g) wf[h][g] = read_w(0, g, h);
        xf[0] = read_x(0, 0, 0);
        xf[1] = read_x(0, 0, 1);
        for (int s = 0; s < steps; ++s) {
            const bool next = s + 1 < steps, after = s + 2 < steps;
            if (!next && a.p % kStep) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (behind(s, h))
#pragma unroll
                        for (int g = 0; g < 4; ++g) wf[h][g] = 0;
            }
#pragma unroll
            for (int f = 0; f < 8; ++f) {
                if (f == 1 && next) bring_half(s + 1, 1);
                if (f == 3) {
                    if (next) wait_and_meet<kLate>();
                    else wait_and_meet<0>();
                }
                if (f == 4 && after) bring_half(s + 2, 0);
                if (f == 5 && after) bring_all_w(s + 2);
                if (f == 7) {
                    if (after) wait_and_meet<kLate>();
                    else wait_and_meet<0>();
                }
                if (f < 7) {
                    xf[(2 * f + 2) & 3] = read_x(s & 1, f + 1, 0);
                    xf[(2 * f + 3) & 3] = read_x(s & 1, f + 1, 1);
                } else if (next) {
                    xf[0] = read_x((s + 1) & 1, 0, 0);
                    xf[1] = read_x((s + 1) & 1, 0, 1);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) sum[f][g] = mma(wf[h][g], xf[(2 * f + h) & 3], sum[f][g]);
                    if (f == 7 && next) {
#pragma unroll
                        for (int g = 0; g < 4; ++g) wf[h][g] = read_w((s + 1) & 1, g, h);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    } else {
        auto multiply = [&](int step, int place) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int4v x[C::FM], w[C::FN];
#pragma unroll
                for (int f = 0; f < C::FM; ++f) x[f] = read_x(place, f, h);
#pragma unroll
                for (int g = 0; g < C::FN; ++g) w[g] = read_w(place, g, h);
                if (!C::LOOSE && step + 1 == steps && behind(step, h))
#pragma unroll
                    for (int g = 0; g < C::FN; ++g) w[g] = 0;
#pragma unroll
                for (int f = 0; f < C::FM; ++f)
#pragma unroll
                    for (int g = 0; g < C::FN; ++g) sum[f][g] = mma(w[g], x[f], sum[f][g]);
            }
        };
        if constexpr (C::LOOSE) {
            int4v held[C::AHEAD][C::PM + C::PN];
            auto request = [&](int step, int to) {
                const int k = step * kStep + c0;
#pragma unroll
                for (int i = 0; i < C::PM; ++i) held[to][i] = codes_at(px[i], k, a.p);
#pragma unroll
                for (int i = 0; i < C::PN; ++i) held[to][C::PM + i] = codes_at(pw[i], k, a.p);
            };
#pragma unroll
            for (int i = 0; i < C::AHEAD; ++i)
                if (i < steps) request(i, i);
            for (int first = 0; first < steps; first += C::AHEAD) {
#pragma unroll
                for (int i = 0; i < C::AHEAD; ++i) {
                    const int step = first + i;
                    if (step >= steps) break;
                    const int place = step & 1;
                    char* const to = shared + place * C::kBytes + threadIdx.x * 16;
#pragma unroll
                    for (int k = 0; k < C::PM; ++k) *reinterpret_cast<int4v*>(to + k * C::kThreads * 16) = held[i][k];
#pragma unroll
                    for (int k = 0; k < C::PN; ++k) *reinterpret_cast<int4v*>(to + C::BM * kStep + k * C::kThreads * 16) = held[i][C::PM + k];
                    __syncthreads();
                    if (step + C::AHEAD < steps) request(step + C::AHEAD, i);
                    multiply(step, place);
                }
            }
        } else {
            auto request = [&](int step, int place) {
#pragma unroll
                for (int i = 0; i < C::PM; ++i) bring_x(step, place, i);
#pragma unroll
                for (int i = 0; i < C::PN; ++i) bring_w(step, place, i);
            };
#pragma unroll
            for (int i = 0; i < C::AHEAD; ++i)
                if (i < steps) request(i, i);
            int place = 0;
            for (int step = 0; step < steps; ++step) {
                if (step + C::AHEAD <= steps) wait_and_meet<(C::AHEAD - 1) * (C::PM + C::PN)>();
                else wait_and_meet<0>();
                // (to the place of the step before this one, which all have read)
                if (step + C::AHEAD < steps) request(step + C::AHEAD, place == 0 ? C::AHEAD : place - 1);
                multiply(step, place);
                place = place == C::AHEAD ? 0 : place + 1;
            }
        }
    }
    write_tile<T, C>(a, sum, shared, row0 + m0, col0 + n0, wave, lane);
}

struct QuantArgs {
    const char* weights;
    int64_t stride;
    char* w;
    int64_t ldw;
    float* scales;
    int p, out;
};

constexpr int kQuantCols = 64;

// A workgroup has 64 outputs: their largest weights first, then the codes, 64 x 64 of them at a time turned around in shared memory.  4,096 x 8,192, bf16: 790 us for 101 MB (a copy of them
// takes 20), 8,192 x 1,000: 1,310.  What bounds it is the chain of single elements that a thread reads, p / 4 of them twice, in few workgroups; a program lays a layer out once.
template <typename T> __global__ void __launch_bounds__(256) int8_quantize_kernel(QuantArgs a)
{
#pragma clang fp contract(off)
    __shared__ unsigned tops[4][kQuantCols];
    __shared__ signed char turned[kQuantCols][kQuantCols + 4];
    const int col = threadIdx.x & 63, slice = threadIdx.x >> 6, j = blockIdx.x * kQuantCols + col;
    const T* const from = reinterpret_cast<const T*>(a.weights);
    unsigned top = 0;
    if (j < a.out)
        for (int k = slice; k < a.p; k += 4) {
            const unsigned b = __builtin_bit_cast(unsigned, (float)from[k * a.stride + j]) & 0x7fffffffu;
            top = b > top ? b : top;
        }
    tops[slice][col] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) top = tops[i][col] > top ? tops[i][col] : top;
    const float size = __builtin_bit_cast(float, top);
    const bool held = top < 0x7f800000u && size >= 0x1p-118f;
    const double inv = held ? 1.0 / (double)size * 127.0 : 0.0;
    if (slice == 0 && j < a.out) a.scales[j] = top >= 0x7f800000u ? __builtin_nanf("") : held ? size / 127.f : 0.f;
    for (int k0 = 0; k0 < a.p; k0 += 64) {
        __syncthreads();
        for (int k = slice; k < 64; k += 4)
            if (j < a.out && k0 + k < a.p) {
                const double scaled = (double)(float)from[(k0 + k) * a.stride + j] * inv;
                turned[col][k] = held ? (signed char)__builtin_bit_cast(unsigned long long, scaled + 0x1.8p52) : 0;
            }
        __syncthreads();
        for (int i = slice; i < 64; i += 4) {
            const int to = blockIdx.x * kQuantCols + i;
            if (to < a.out && k0 + col < a.p) a.w[to * a.ldw + k0 + col] = turned[i][col];
        }
    }
}

template <typename F> void with_type(int dtype, F f)
{
    if (dtype == BMGD_F32) f(float());
    else if (dtype == BMGD_BF16) f(__bf16());
    else f(_Float16());
}

template <typename T, class C> hipError_t launch_tile(ProductArgs a, hipStream_t s)
{
    a.tiles_m = (int)((a.rows + C::BM - 1) / C::BM);
    a.tiles_n = (a.out + C::BN - 1) / C::BN;
    constexpr size_t bytes = C::kShared;
    if constexpr (bytes > 65536) {
        // once per device
        static std::atomic<uint64_t> done{0};
        int device = 0;
        hipError_t e = hipGetDevice(&device);
        if (e != hipSuccess) return e;
        const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
        if (!(done.load(std::memory_order_acquire) & bit)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(&int8_tile_kernel<T, C>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
            if (e != hipSuccess) return e;
            done.fetch_or(bit, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL((int8_tile_kernel<T, C>), dim3((unsigned)(a.tiles_m * a.tiles_n)), dim3(C::kThreads), bytes, s, a);
    return hipGetLastError();
}

template <typename T> hipError_t launch_product(const ProductArgs& a, hipStream_t s)
{
    const uintptr_t all = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)a.p | (uintptr_t)a.ldx | (uintptr_t)a.ldw;
    const bool loose = all & 15;
    const int64_t units = compute_units();
    auto tiles = [&](int64_t m, int64_t n) { return (a.rows + m - 1) / m * ((a.out + n - 1) / n); };
    auto tile = [&](auto of) {
        typedef decltype(of) C;
        return launch_tile<T, C>(a, s);
    };
    // Measured, us (rows x p x out): 2,048 x 4,096 x 4,096: tiles of 256 48, of 128 two or three to a unit 36, of 128 alone with one step more on its way 48, of 64 x 128 44, of 64 63;
    //      2,000 x 2,000 x 2,000: 30, 19, 17, 20, 24;  512 x 4,096 x 4,096: 44, 23, 22, 17, 18;  256 x 4,096 x 4,096: 44, 23, 22, 16, 13.  Loose: 4,097 x 2,319 x 2,965: of 128 66, of 64 92;
    //      2,000 x 2,001 x 2,000: of 128 27, with eight wavefronts and one step more on its way 23, of 64 33.
    if (loose) {
        if (tiles(128, 128) > units) return tile(Tile<128, 128, 2, 2, 1, true>());
        if (tiles(128, 128) > units / 2) return tile(Tile<128, 128, 2, 4, 2, true>());
    } else {
        if (tiles(256, 256) >= units) return tile(Tile<256, 256, 2, 4, 1, false>());
        if (tiles(128, 128) > units) return tile(Tile<128, 128, 2, 2, 1, false>());
        if (tiles(128, 128) > units / 2) return tile(Tile<128, 128, 2, 2, 2, false>());
        if (tiles(64, 128) > units * 3 / 4) return tile(Tile<64, 128, 2, 2, 2, false>());
    }
    // Few tiles.  A step of one takes 0.17 us (32 x 32) or 0.28 (64 x 64), loose ones 0.24 and 0.42, of 32 x 64 0.31 (aligned: 0.21, but where these are no more than units
    // tiles of 32 x 32 are two to a unit at most).  Workgroups of 16 columns without steps read rows more
    // often: their operands come at 12 TB/s in all (4.4 where pieces cross lines) and 45 GB/s to a unit.  Measured, us, tiles and these: 64 x 4,096 x 4,096: 9.4 and 12;  100 x 8,192 x 1,000:
    // 15 and 13;  16 x 4,096 x 8,192: 9.4 and 10.2;  1 x 4,096 x 8,192: 9.4 and 8.1;  333 x 1,365 x 1,000, loose: 7.4 and 15.
    const bool small = tiles(32, 32) <= (loose ? units : 2 * units), flat = loose && tiles(32, 64) <= units;
    const double tile_us = 4.0 + (small ? loose ? 0.24 : 0.17 : flat ? 0.31 : loose ? 0.42 : 0.28) * ((a.p + kStep - 1) / kStep);
    auto few_us = [&](int64_t rf) {
        const double each = (16.0 + (double)std::min(16 * rf, a.rows)) * a.p, groups = (double)((a.out + 15) / 16) * (double)((a.rows + 16 * rf - 1) / (16 * rf));
        return 4.8 + std::max(each * groups / (loose ? 4.4e6 : 12e6), each / 45e3);
    };
    auto few = [&](auto rf) {
        constexpr int RF = decltype(rf)::value;
        hipLaunchKernelGGL((int8_few_kernel<T, RF>), dim3((unsigned)((a.out + 15) / 16), (unsigned)((a.rows + 16 * RF - 1) / (16 * RF))), dim3(64 * kFewWaves), 0, s, a);
        return hipGetLastError();
    };
    const double one = few_us(1), two = few_us(2), four = few_us(4), best = std::min(one, std::min(two, four));
    if (best < tile_us && a.rows < (1 << 19)) return one == best ? few(std::integral_constant<int, 1>()) : two == best ? few(std::integral_constant<int, 2>()) : few(std::integral_constant<int, 4>());
    if (loose) return small ? tile(Tile<32, 32, 2, 2, 6, true>()) : flat ? tile(Tile<32, 64, 2, 2, 4, true>()) : tile(Tile<64, 64, 2, 4, 4, true>());
    return small ? tile(Tile<32, 32, 2, 2, 4, false>()) : tile(Tile<64, 64, 2, 4, 3, false>());
}

void check(Call& q, const bmgd_product_config* cfg)
{
    if (!cfg) return q.refuse(BMGD_EINVAL, "cfg and tensors must not be NULL");
    if (cfg->p < 1 || cfg->p > 131071) q.refuse(BMGD_EINVAL, "p must be in [1, 131071]");
    if (cfg->out_n < 1 || cfg->out_n > (1 << 20)) q.refuse(BMGD_EINVAL, "out_n must be in [1, 2^20]");
    if (!known_type(cfg->dtype)) q.refuse(BMGD_EINVAL, "unknown dtype");
}

}  // namespace

#define BMGD_API __attribute__((visibility("default")))

extern "C" {

BMGD_API int bmgd_product_forward(const bmgd_product_config* cfg, int64_t rows, const bmgd_product_tensors* t, void* stream)
{
    Call q{"bmgd_product_forward"};
    check(q, cfg);
    if (!t) q.refuse(BMGD_EINVAL, "cfg and tensors must not be NULL");
    q.rows(rows);
    if (q.code != BMGD_OK) return q.code;
    const bool some = rows > 0;
    q.matrix("x", t->x, rows, cfg->p, some, 1);
    q.matrix("w", t->w, cfg->out_n, cfg->p, some, 1);
    q.matrix("y", t->y, rows, cfg->out_n, some, size_of(cfg->dtype));
    q.address("x_scales", t->x_scales, some, 4);
    q.address("w_scales", t->w_scales, some, 4);
    for (const void* in : {(const void*)t->x.data, (const void*)t->w.data, (const void*)t->x_scales, (const void*)t->w_scales}) q.apart("y", t->y.data, in);
    // (a launch has less than 2^32 threads)
    if ((rows + 127) / 128 * ((cfg->out_n + 127) / 128) >= (int64_t(1) << 23)) q.refuse(BMGD_EINVAL, "2^23 tiles of 128 x 128 or more");
    if (q.code != BMGD_OK || !some) return q.code;
    ProductArgs a{};
    a.x = static_cast<const char*>(t->x.data);
    a.w = static_cast<const char*>(t->w.data);
    a.y = static_cast<char*>(t->y.data);
    a.ldx = rows > 1 ? t->x.stride : 0;                         // (of one row: not looked at, so no reason for another path)
    a.ldw = cfg->out_n > 1 ? t->w.stride : 0;
    a.ldy = t->y.stride;
    a.sx = t->x_scales;
    a.sw = t->w_scales;
    a.rows = rows;
    a.p = (int)cfg->p;
    a.out = (int)cfg->out_n;
    hipError_t e = hipSuccess;
    with_type(cfg->dtype, [&](auto type) { e = launch_product<decltype(type)>(a, static_cast<hipStream_t>(stream)); });
    return q.hip(e, "launch");
}

BMGD_API int bmgd_product_quantize(const bmgd_product_config* cfg, const bmgd_matrix* weights, const bmgd_matrix* w, float* w_scales, void* stream)
{
    Call q{"bmgd_product_quantize"};
    check(q, cfg);
    if (!weights || !w) q.refuse(BMGD_EINVAL, "weights and w must not be NULL");
    if (q.code != BMGD_OK) return q.code;
    q.matrix("weights", *weights, cfg->p, cfg->out_n, true, size_of(cfg->dtype));
    q.matrix("w", *w, cfg->out_n, cfg->p, true, 1);
    q.address("w_scales", w_scales, true, 4);
    q.apart("w", w->data, weights->data);
    q.apart("w_scales", w_scales, weights->data);
    q.apart("w_scales", w_scales, w->data);
    if (q.code != BMGD_OK) return q.code;
    QuantArgs a{static_cast<const char*>(weights->data), cfg->p > 1 ? weights->stride : 0, static_cast<char*>(w->data), cfg->out_n > 1 ? w->stride : 0, w_scales,
                (int)cfg->p, (int)cfg->out_n};
    with_type(cfg->dtype, [&](auto type) {
        hipLaunchKernelGGL(int8_quantize_kernel<decltype(type)>, dim3((unsigned)((a.out + kQuantCols - 1) / kQuantCols)), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    });
    return q.launched();
}

}  // extern "C"
