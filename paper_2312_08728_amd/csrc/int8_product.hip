// Product in 8-bit integers: y_ij = x_scales[i] w_scales[j] sum_k x_ik w_jk, and the codes of a layer's weights.
//
// Both operands have the summed index adjacent in memory, 16 codes to a lane's operand of v_mfma_i32_16x16x64_i8 (a = A[lane % 16][16 (lane / 16) + i],
// b = B[16 (lane / 16) + i][lane % 16], c[v] = C[4 (lane / 16) + v][lane % 16]).  The instruction forms the transpose of the result, so that a lane ends with four
// neighbouring columns of a row.  Sums are exact, in whatever order parts of them are added.
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

// Up to 16 RF rows: a workgroup makes 16 columns of them, its wavefronts share the sum, every operand comes from memory once and straight to registers.
template <typename T, int RF> __global__ void __launch_bounds__(64 * kFewWaves) int8_few_kernel(ProductArgs a)
{
    constexpr int U = 8;
    __shared__ int4v parts[kFewWaves][RF][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = lane & 15, q = lane >> 4;
    const int col = blockIdx.x * 16;
    const char* const w = a.w + (int64_t)min(col + in, a.out - 1) * a.ldw;
    const char* x[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) x[f] = a.x + min((int64_t)16 * f + in, a.rows - 1) * a.ldx;
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
    const int64_t row = 16 * wave + in;
    const int j = col + 4 * q;
    if (row >= a.rows || j >= a.out) return;
    float sw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sw[i] = j + i < a.out ? a.sw[j + i] : 0.f;
    put_four(reinterpret_cast<T*>(a.y) + row * a.ldy + j, scaled(c, a.sx[row], sw), a.out - j);
}

constexpr int kStep = 128;          // codes of a row that a step takes

// A tile of BM rows and BN columns by WM x WN wavefronts.  A step of an operand lies in shared memory as rows of 128 bytes, eight pieces of 16; piece c of row r
// lies in place c ^ (r & 7), so that the rows that an instruction's lanes read at the same piece lie in different banks.  Loose: operands at any
// address, through registers.
template <int BM_, int BN_, int WM_, int WN_, bool LOOSE_> struct Tile {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, kThreads = 64 * WM * WN;
    static constexpr bool LOOSE = LOOSE_;
    static constexpr int FM = BM / WM / 16, FN = BN / WN / 16;                   // 16 x 16 results of a wavefront
    static constexpr int kBytes = (BM + BN) * kStep;                             // of a step
    static constexpr int PM = BM * 8 / kThreads, PN = BN * 8 / kThreads;         // pieces that a thread brings
};

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
    int4v held[C::LOOSE ? C::PM + C::PN : 1];
    auto request = [&](int step, int buffer) {
        const int k = step * kStep + c0;
        if constexpr (C::LOOSE) {
#pragma unroll
            for (int i = 0; i < C::PM; ++i) held[i] = codes_at(px[i], k, a.p);
#pragma unroll
            for (int i = 0; i < C::PN; ++i) held[C::PM + i] = codes_at(pw[i], k, a.p);
        } else {
            const int from = k < a.p ? k : 0;                   // (pieces behind the end: any, x is taken as zero there)
            const unsigned to = base + buffer * C::kBytes + wave * 1024;
#pragma unroll
            for (int i = 0; i < C::PM; ++i) load_to_lds(reinterpret_cast<const unsigned short*>(px[i] + from), to + i * C::kThreads * 16);
#pragma unroll
            for (int i = 0; i < C::PN; ++i) load_to_lds(reinterpret_cast<const unsigned short*>(pw[i] + from), to + C::BM * kStep + i * C::kThreads * 16);
        }
    };
    auto arrive = [&](int buffer) {
        if constexpr (C::LOOSE) {
            char* const to = shared + buffer * C::kBytes + threadIdx.x * 16;
#pragma unroll
            for (int i = 0; i < C::PM; ++i) *reinterpret_cast<int4v*>(to + i * C::kThreads * 16) = held[i];
#pragma unroll
            for (int i = 0; i < C::PN; ++i) *reinterpret_cast<int4v*>(to + C::BM * kStep + i * C::kThreads * 16) = held[C::PM + i];
        } else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    int4v sum[C::FM][C::FN] = {};
    const int m0 = wave / C::WN * (C::FM * 16), n0 = wave % C::WN * (C::FN * 16);
    auto multiply = [&](int step, int buffer) {
        const char* const xs = shared + buffer * C::kBytes + (m0 + in) * kStep;
        const char* const ws = shared + buffer * C::kBytes + C::BM * kStep + (n0 + in) * kStep;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int place = 16 * ((4 * h + q) ^ (in & 7));
            int4v x[C::FM], w[C::FN];
#pragma unroll
            for (int f = 0; f < C::FM; ++f) x[f] = *reinterpret_cast<const int4v*>(xs + f * 16 * kStep + place);
#pragma unroll
            for (int f = 0; f < C::FN; ++f) w[f] = *reinterpret_cast<const int4v*>(ws + f * 16 * kStep + place);
            if (!C::LOOSE && step * kStep + 64 * h + 16 * q >= a.p)
#pragma unroll
                for (int f = 0; f < C::FM; ++f) x[f] = 0;
#pragma unroll
            for (int f = 0; f < C::FM; ++f)
#pragma unroll
                for (int g = 0; g < C::FN; ++g) sum[f][g] = mma(w[g], x[f], sum[f][g]);
        }
    };

    request(0, 0);
    for (int step = 0; step < steps; ++step) {
        arrive(step & 1);
        if (step + 1 < steps) request(step + 1, (step + 1) & 1);
        multiply(step, step & 1);
    }

#pragma unroll
    for (int g = 0; g < C::FN; ++g) {
        const int j = col0 + n0 + 16 * g + 4 * q;
        float sw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sw[i] = j + i < a.out ? a.sw[j + i] : 0.f;
#pragma unroll
        for (int f = 0; f < C::FM; ++f) {
            const int64_t row = row0 + m0 + 16 * f + in;
            if (row < a.rows && j < a.out) put_four(reinterpret_cast<T*>(a.y) + row * a.ldy + j, scaled(sum[f][g], a.sx[row], sw), a.out - j);
        }
    }
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

// A workgroup has 64 outputs: their largest weights first, then the codes, 64 x 64 of them at a time turned around in shared memory.
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
    constexpr size_t bytes = 2 * C::kBytes;
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
    if (a.rows <= 32) {
        const dim3 grid((unsigned)((a.out + 15) / 16)), block(64 * kFewWaves);
        if (a.rows <= 16) hipLaunchKernelGGL((int8_few_kernel<T, 1>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((int8_few_kernel<T, 2>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    const uintptr_t all = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w) | (uintptr_t)a.p | (uintptr_t)a.ldx | (uintptr_t)a.ldw;
    const bool loose = all & 15;
    const int64_t units = compute_units();
    auto tiles = [&](int64_t m, int64_t n) { return (a.rows + m - 1) / m * ((a.out + n - 1) / n); };
    if (!loose && tiles(256, 256) >= units) return launch_tile<T, Tile<256, 256, 2, 4, false>>(a, s);
    if (tiles(128, 128) >= units) return loose ? launch_tile<T, Tile<128, 128, 2, 2, true>>(a, s) : launch_tile<T, Tile<128, 128, 2, 2, false>>(a, s);
    return loose ? launch_tile<T, Tile<64, 64, 2, 2, true>>(a, s) : launch_tile<T, Tile<64, 64, 2, 2, false>>(a, s);
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
