// Root-mean-square norm with the residual's addition, into 16 or 32 bits or into 8-bit codes with a scale for each row; its gradient; the values of codes.
//
//      s = x + residual, rounded;  r = (mean s^2 + eps)^(-1/2);  y = s w r;  codes = rint(s w ((1 / max|s w|) 127)), scale = max|s w| r / 127
//      dx = r (w dy - s r^2 mean(w dy s)) + dsum;  dw = sum over the rows of dy s r
//
// A row is read once: W wavefronts hold it in registers, NV pieces of 16 bytes a lane, while its sum (and largest element) is formed, and write the
// result from there.  The s that is normed is the rounded one, which the stream goes on with and a backward pass reads.  Codes come from s w alone (r
// is common to a row) in 64 bits: products of 16-bit elements are exact, so values next to the middle of two codes go where the definition says.
//
// What bounds it (us).  8,192 rows of 8,192, bf16, residual, 8 bits: 93 (470 MB, 5.0 TB/s), the values of the codes 65 (335 MB): memory.  Backward of 8,192 rows of 4,096 with dsum 52
// (268 MB, 5.3 TB/s) and 4.4 for the 512 parts of dw.  777 rows of 1,365, f16: 4.6, 1,000 rows of 512 backward, fp32: 7.5, one row: 3.5: a launch (2.8) and a trip to memory.
// Rows that registers do not hold are read a second time, mostly from cache: 4,000 rows of 40,000, bf16, with residual, 16 bits: 262 (1.28 GB, 4.9 TB/s), 8 bits: 273 (4.1 TB/s);
// backward 229 (960 MB, 4.2 TB/s), with dw 369, which reads x and dy once more.
#include "operator_calls.h"
#include "rows_device.h"

#include <math.h>

#include <algorithm>

using namespace bmgd;

namespace {

struct Side {
    char* data;
    int64_t stride;         // in elements
};
template <typename T> __device__ __forceinline__ T* row_of(const Side& m, int64_t row) { return reinterpret_cast<T*>(m.data) + row * m.stride; }

struct NormArgs {
    Side x, residual, sum, y, codes, dy, dsum, dx;
    const char* weight;
    float* scales;
    float* rstd;
    float* partial;         // of dweight: a row of n for each workgroup
    int64_t rows, first;    // first: of the launch, see kRowsOfLaunch
    int n, row_groups;      // row_groups: workgroups that go through rows, see norm_backward_kernel
    float eps, inv_n;
    char* dweight;
};

// What the largest |s w| of a row is found in: products of two 16-bit numbers are exact in 32 bits, those of 32-bit numbers in 64.
// As the bits of a number without sign, so that NaN counts as largest.
template <typename T> struct Largest {
    typedef float value;
    typedef unsigned bits;
    static constexpr bits kInfinity = 0x7f800000u;
};
template <> struct Largest<float> {
    typedef double value;
    typedef unsigned long long bits;
    static constexpr bits kInfinity = 0x7ff0000000000000ull;
};
template <typename T> __device__ __forceinline__ typename Largest<T>::bits size_bits(typename Largest<T>::value v)
{
    typedef typename Largest<T>::bits bits;
    return __builtin_bit_cast(bits, v) & (~bits(0) >> 1);
}

constexpr double kLeastRow = 0x1p-118;         // max / 127 of a row that is held stays a normal number

// Eight codes, or four, at any address.
struct __attribute__((packed)) Codes8 { unsigned long long v; };
struct __attribute__((packed)) Codes4 { unsigned v; };

// (the code is the lowest byte)
__device__ __forceinline__ unsigned code_of(double v, double inv)
{
#pragma clang fp contract(off)
    // rounded to 2^-53 first, as v inv of the definition; then, half to even, to the integer that the low bits hold
    const double scaled = v * inv;
    return (unsigned)__builtin_bit_cast(unsigned long long, scaled + 0x1.8p52);
}
// the lowest bytes of four words
__device__ __forceinline__ unsigned lowest_bytes(const unsigned* w)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u), __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
}

// Sums (and largest) of a row over its W wavefronts, in the order of the wavefronts.
template <int W> __device__ __forceinline__ float row_sum(float v, float* shared)
{
    v = wave_sum(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += shared[i];
    }
    return v;
}
template <int W, typename V> __device__ __forceinline__ V row_max(V v, V* shared)
{
    v = wave_max(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
        __syncthreads();
        v = shared[0];
#pragma unroll
        for (int i = 1; i < W; ++i) v = shared[i] > v ? shared[i] : v;
    }
    return v;
}

template <typename T> __device__ __forceinline__ typename Piece<T>::vec piece(const T* p, int j, int n)
{
    if (j + Piece<T>::N <= n) return Piece<T>::load(p + j);
    if (sizeof(T) == 4 || n < Piece<T>::N) return Piece<T>::load_part(p, j, 0, n, (T)0.f);
    // a row's last piece: its last 16 bytes, moved down, zeros behind them (element by element it takes as long as all others together)
    const unsigned __int128 last = __builtin_bit_cast(unsigned __int128, Piece<T>::load(p + n - Piece<T>::N));
    return __builtin_bit_cast(typename Piece<T>::vec, last >> 8 * (int)sizeof(T) * (j + Piece<T>::N - n));
}
template <typename T> __device__ __forceinline__ void put(T* p, int j, int n, typename Piece<T>::vec v)
{
    if (j + Piece<T>::N <= n) Piece<T>::store(p + j, v);
    else Piece<T>::store_part(p, j, 0, n, v);
}
template <int N> __device__ __forceinline__ void put_codes(char* p, int j, int n, unsigned long long v)
{
    if (j + N <= n) {
        if constexpr (N == 8) reinterpret_cast<Codes8*>(p + j)->v = v;
        else reinterpret_cast<Codes4*>(p + j)->v = (unsigned)v;
    }
    else
        for (int k = 0; j + k < n; ++k) p[j + k] = (char)(v >> 8 * k);
}

// the sums of a piece's columns
template <typename T> __device__ __forceinline__ void put_sums(float* p, int j, int n, typename Piece<T>::wide v)
{
    typedef float loose __attribute__((ext_vector_type(Piece<T>::N), aligned(4)));
    if (j + Piece<T>::N <= n) *reinterpret_cast<loose*>(p + j) = v;
    else
#pragma unroll
        for (int k = 0; k < Piece<T>::N; ++k)
            if (j + k < n) p[j + k] = v[k];
}

// s of the piece at j; `sum` receives it
template <typename T> __device__ __forceinline__ typename Piece<T>::vec summed(const NormArgs& a, int64_t row, int j)
{
    typename Piece<T>::vec v = piece(row_of<T>(a.x, row), j, a.n);
    if (a.residual.data) v = narrow<T>(widen<T>(v) + widen<T>(piece(row_of<T>(a.residual, row), j, a.n)));
    if (a.sum.data) put(row_of<T>(a.sum, row), j, a.n, v);
    return v;
}

template <typename T> __device__ __forceinline__ void write_y(const NormArgs& a, int64_t row, int j, typename Piece<T>::vec s, typename Piece<T>::vec w, float r)
{
    put(row_of<T>(a.y, row), j, a.n, narrow<T>(widen<T>(s) * widen<T>(w) * r));
}

template <typename T> __device__ __forceinline__ void write_codes(const NormArgs& a, int64_t row, int j, typename Piece<T>::vec s, typename Piece<T>::vec w, double inv)
{
    typedef typename Largest<T>::value value;
    unsigned code[Piece<T>::N];
#pragma unroll
    for (int k = 0; k < Piece<T>::N; ++k) code[k] = code_of((double)((value)s[k] * (value)w[k]), inv);
    unsigned long long c = lowest_bytes(code);
    if constexpr (Piece<T>::N == 8) c |= (unsigned long long)lowest_bytes(code + 4) << 32;
    put_codes<Piece<T>::N>(row_of<char>(a.codes, row), j, a.n, c);
}

// r of a row from its sum of squares
__device__ __forceinline__ float rstd_of(const NormArgs& a, float squares) { return 1.f / sqrtf(__builtin_fmaf(squares, a.inv_n, a.eps)); }

// (1 / largest) 127, each rounded (0 where the row is held as zeros or stands for NaN), and the row's scale
template <typename T> __device__ __forceinline__ double scale_of(typename Largest<T>::bits top, float r, float* scale)
{
    const typename Largest<T>::value v = __builtin_bit_cast(typename Largest<T>::value, top);
    if (top >= Largest<T>::kInfinity) {
        *scale = __builtin_nanf("");
        return 0.0;
    }
    if ((double)v < kLeastRow) {
        *scale = 0.f;
        return 0.0;
    }
    *scale = (float)v * r / 127.f;
    return 1.0 / (double)v * 127.0;
}

template <typename T> __device__ __forceinline__ typename Piece<T>::vec ones()
{
    typename Piece<T>::vec w;
#pragma unroll
    for (int k = 0; k < Piece<T>::N; ++k) w[k] = (T)1.f;
    return w;
}

constexpr int block_of(int w) { return w < 4 ? 256 : 64 * w; }

template <typename T, int W, int NV> __global__ void __launch_bounds__(block_of(W)) norm_forward_kernel(NormArgs a)
{
    typedef typename Largest<T>::bits bits;
    typedef typename Largest<T>::value value;
    constexpr int kLanes = 64 * W, kRows = block_of(W) / kLanes;
    __shared__ float sums[16];
    __shared__ bits tops[16];
    const int t = threadIdx.x % kLanes;
    const int64_t row = a.first + (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;
    if (row >= a.rows) return;                                  // (whole wavefronts, and none of a workgroup with barriers)
    typename Piece<T>::vec s[NV], w[NV];
    float squares = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = Piece<T>::N * (t + i * kLanes);
        if (j < a.n) {
            s[i] = piece(row_of<T>(a.x, row), j, a.n);
            w[i] = a.weight ? piece(reinterpret_cast<const T*>(a.weight), j, a.n) : ones<T>();
        }
    }
    if (a.residual.data) {
        typename Piece<T>::vec q[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = Piece<T>::N * (t + i * kLanes);
            if (j < a.n) q[i] = piece(row_of<T>(a.residual, row), j, a.n);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = Piece<T>::N * (t + i * kLanes);
            if (j < a.n) s[i] = narrow<T>(widen<T>(s[i]) + widen<T>(q[i]));
        }
    }
    bits top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = Piece<T>::N * (t + i * kLanes);
        if (j >= a.n) continue;
        if (a.sum.data) put(row_of<T>(a.sum, row), j, a.n, s[i]);
        const typename Piece<T>::wide v = widen<T>(s[i]);
#pragma unroll
        for (int k = 0; k < Piece<T>::N; ++k) squares = __builtin_fmaf(v[k], v[k], squares);
        if (a.codes.data) {
#pragma unroll
            for (int k = 0; k < Piece<T>::N; ++k) {
                const bits b = size_bits<T>((value)s[i][k] * (value)w[i][k]);
                if (j + k < a.n) top = b > top ? b : top;
            }
        }
    }
    const float r = rstd_of(a, row_sum<W>(squares, sums));
    if (a.rstd && t == 0) a.rstd[row] = r;
    if (a.y.data) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = Piece<T>::N * (t + i * kLanes);
            if (j < a.n) write_y<T>(a, row, j, s[i], w[i], r);
        }
    }
    if (a.codes.data) {
        float scale;
        const double inv = scale_of<T>(row_max<W>(top, tops), r, &scale);
        if (t == 0) a.scales[row] = scale;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = Piece<T>::N * (t + i * kLanes);
            if (j < a.n) write_codes<T>(a, row, j, s[i], w[i], inv);
        }
    }
}

constexpr int kLongWaves = 16, kLong = 64 * kLongWaves;        // rows that do not fit in registers

// The same in two passes over the row.  Each thread reads again what it has read, or written, itself.
template <typename T> __global__ void __launch_bounds__(kLong) norm_forward_long_kernel(NormArgs a)
{
    typedef typename Largest<T>::bits bits;
    typedef typename Largest<T>::value value;
    __shared__ float sums[kLongWaves];
    __shared__ bits tops[kLongWaves];
    const int64_t row = a.first + blockIdx.x;
    float squares = 0.f;
    bits top = 0;
    for (int j = Piece<T>::N * threadIdx.x; j < a.n; j += Piece<T>::N * kLong) {
        const typename Piece<T>::vec s = summed<T>(a, row, j);
        const typename Piece<T>::wide v = widen<T>(s);
#pragma unroll
        for (int k = 0; k < Piece<T>::N; ++k) squares = __builtin_fmaf(v[k], v[k], squares);
        if (a.codes.data) {
            const typename Piece<T>::vec w = a.weight ? piece(reinterpret_cast<const T*>(a.weight), j, a.n) : ones<T>();
#pragma unroll
            for (int k = 0; k < Piece<T>::N; ++k) {
                const bits b = size_bits<T>((value)s[k] * (value)w[k]);
                if (j + k < a.n) top = b > top ? b : top;
            }
        }
    }
    const float r = rstd_of(a, row_sum<kLongWaves>(squares, sums));
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = r;
    double inv = 0.0;
    if (a.codes.data) {
        float scale;
        inv = scale_of<T>(row_max<kLongWaves>(top, tops), r, &scale);
        if (threadIdx.x == 0) a.scales[row] = scale;
    }
    for (int j = Piece<T>::N * threadIdx.x; j < a.n; j += Piece<T>::N * kLong) {
        typename Piece<T>::vec s;
        if (a.sum.data) s = piece(row_of<T>(a.sum, row), j, a.n);
        else {
            s = piece(row_of<T>(a.x, row), j, a.n);
            if (a.residual.data) s = narrow<T>(widen<T>(s) + widen<T>(piece(row_of<T>(a.residual, row), j, a.n)));
        }
        const typename Piece<T>::vec w = a.weight ? piece(reinterpret_cast<const T*>(a.weight), j, a.n) : ones<T>();
        if (a.y.data) write_y<T>(a, row, j, s, w, r);
        if (a.codes.data) write_codes<T>(a, row, j, s, w, inv);
    }
}

template <typename T>
__device__ __forceinline__ typename Piece<T>::wide input_gradient(typename Piece<T>::wide d, typename Piece<T>::wide s, float r, float c, typename Piece<T>::vec dsum, bool has)
{
    typename Piece<T>::wide v = (d - s * c) * r;
    if (has) v += widen<T>(dsum);
    return v;
}

// How a backward call finds dw.
enum Weights {
    kNoWeights,
    kParts,                 // each workgroup keeps its part of dw in registers and leaves it for norm_join_kernel
    kColumns                // other workgroups of the launch, `row_groups` and following, read the same rows again, four pieces of columns each: r is given, so dw waits for nothing
};

// dw of four pieces of columns, from all rows: every kSlices-th row for a thread, then the slices in order.
template <typename T, int THREADS> __device__ __forceinline__ void column_sums(const NormArgs& a, int group, float* shared)
{
    constexpr int N = Piece<T>::N, kSlices = THREADS / 4, U = 4;
    typedef typename Piece<T>::wide wide;
    const int slice = threadIdx.x / 4, mine = threadIdx.x % 4, j = N * (4 * group + mine);
    wide dw = 0.f;
    if (j < a.n) {
        const T *const x = row_of<T>(a.x, 0), *const dy = row_of<T>(a.dy, 0);
        int64_t row = slice;
        for (; row + (U - 1) * kSlices < a.rows; row += U * kSlices) {
            typename Piece<T>::vec s[U], g[U];
            float r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                s[u] = piece(x + (row + u * kSlices) * a.x.stride, j, a.n);
                g[u] = piece(dy + (row + u * kSlices) * a.dy.stride, j, a.n);
                r[u] = a.rstd[row + u * kSlices];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) dw += widen<T>(g[u]) * (widen<T>(s[u]) * r[u]);
        }
        for (; row < a.rows; row += kSlices) dw += widen<T>(piece(dy + row * a.dy.stride, j, a.n)) * (widen<T>(piece(x + row * a.x.stride, j, a.n)) * a.rstd[row]);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) shared[slice * (4 * N + 1) + mine * N + k] = dw[k];
    __syncthreads();
    // 16 slices for a thread, then these
    constexpr int kGroups = kSlices / 16;
    const int col = threadIdx.x % (4 * N), part = threadIdx.x / (4 * N);
    float v = 0.f;
    if (part < kGroups)
#pragma unroll
        for (int i = 0; i < 16; ++i) v += shared[(part * 16 + i) * (4 * N + 1) + col];
    __syncthreads();
    if (part < kGroups) shared[part * (4 * N) + col] = v;
    __syncthreads();
    if (part == 0) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) v += shared[i * (4 * N) + col];
        const int to = N * 4 * group + col;
        if (to < a.n) reinterpret_cast<T*>(a.dweight)[to] = (T)v;
    }
}

// A workgroup goes through rows blockIdx.x, blockIdx.x + row_groups, ... (kRows at a time).
template <typename T, int W, int NV, Weights DW> __global__ void __launch_bounds__(block_of(W)) norm_backward_kernel(NormArgs a)
{
    constexpr int kLanes = 64 * W, kRows = block_of(W) / kLanes;
    __shared__ float sums[2][16];
    __shared__ float joined[DW == kParts && kRows > 1 ? kRows * NV * Piece<T>::N * kLanes : DW == kColumns ? block_of(W) / 4 * (4 * Piece<T>::N + 1) : 1];
    if constexpr (DW == kColumns)
        if ((int)blockIdx.x >= a.row_groups) return column_sums<T, block_of(W)>(a, blockIdx.x - a.row_groups, joined);
    const int t = threadIdx.x % kLanes, mine = threadIdx.x / kLanes;
    typename Piece<T>::vec w[NV];
    typename Piece<T>::wide dw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int j = Piece<T>::N * (t + i * kLanes);
        w[i] = j < a.n && a.weight ? piece(reinterpret_cast<const T*>(a.weight), j, a.n) : ones<T>();
        dw[i] = 0.f;
    }
    // rows on their way while the one before is worked on: two where registers allow it (8,192 x 2,048, bf16, with dw: 26 us, with one 29.5)
    constexpr bool kAhead = NV <= 2;
    typename Piece<T>::vec s[NV], dy[NV], ds[NV], s2[NV], dy2[NV], ds2[NV];
    float r = 0.f, r2 = 0.f;
    auto load = [&](int64_t row, typename Piece<T>::vec(&to_s)[NV], typename Piece<T>::vec(&to_dy)[NV], typename Piece<T>::vec(&to_ds)[NV], float& to_r) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = Piece<T>::N * (t + i * kLanes);
            if (j < a.n) {
                to_s[i] = piece(row_of<T>(a.x, row), j, a.n);
                to_dy[i] = piece(row_of<T>(a.dy, row), j, a.n);
                if (a.dsum.data) to_ds[i] = piece(row_of<T>(a.dsum, row), j, a.n);
            }
        }
        to_r = a.rstd[row];
    };
    int turn = 0;
    int64_t row = (int64_t)blockIdx.x * kRows + mine;
    const int64_t step = (int64_t)a.row_groups * kRows;
    if (kAhead && row < a.rows) load(row, s2, dy2, ds2, r2);
    for (; row < a.rows; row += step, turn ^= 1) {              // (one wavefront after the other where there are no barriers)
        if constexpr (kAhead) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                s[i] = s2[i];
                dy[i] = dy2[i];
                ds[i] = ds2[i];
            }
            r = r2;
            if (row + step < a.rows) load(row + step, s2, dy2, ds2, r2);
        } else load(row, s, dy, ds, r);
        float along = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = Piece<T>::N * (t + i * kLanes);
            if (j >= a.n) continue;
            const typename Piece<T>::wide v = widen<T>(s[i]), g = widen<T>(dy[i]), f = widen<T>(w[i]);
            // (a last piece has zeros behind the row's end)
#pragma unroll
            for (int k = 0; k < Piece<T>::N; ++k) along = __builtin_fmaf(g[k] * f[k], v[k], along);
            if constexpr (DW == kParts) {
#pragma unroll
                for (int k = 0; k < Piece<T>::N; ++k) dw[i][k] = __builtin_fmaf(g[k], v[k] * r, dw[i][k]);
            }
        }
        const float c = row_sum<W>(along, sums[turn]) * a.inv_n * r * r;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int j = Piece<T>::N * (t + i * kLanes);
            if (j < a.n)
                put(row_of<T>(a.dx, row), j, a.n, narrow<T>(input_gradient<T>(widen<T>(dy[i]) * widen<T>(w[i]), widen<T>(s[i]), r, c, ds[i], a.dsum.data != nullptr)));
        }
    }
    if constexpr (DW == kParts) {
        float* const to = a.partial + (int64_t)blockIdx.x * a.n;
        if constexpr (kRows == 1) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = Piece<T>::N * (t + i * kLanes);
                if (j < a.n) put_sums<T>(to, j, a.n, dw[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < Piece<T>::N; ++k) joined[((mine * NV + i) * Piece<T>::N + k) * kLanes + t] = dw[i][k];
            __syncthreads();
            for (int q = threadIdx.x; q < NV * Piece<T>::N * kLanes; q += block_of(W)) {
                const int at = q % kLanes, k = q / kLanes % Piece<T>::N, i = q / kLanes / Piece<T>::N, j = Piece<T>::N * (at + i * kLanes) + k;
                float v = 0.f;
#pragma unroll
                for (int m = 0; m < kRows; ++m) v += joined[m * NV * Piece<T>::N * kLanes + q];
                if (j < a.n) to[j] = v;
            }
        }
    }
}

// dx of rows that do not fit in registers.
template <typename T> __global__ void __launch_bounds__(kLong) norm_backward_long_kernel(NormArgs a)
{
    __shared__ float sums[kLongWaves];
    const int64_t row = a.first + blockIdx.x;
    const T *const x = row_of<T>(a.x, row), *const dy = row_of<T>(a.dy, row), *const weight = reinterpret_cast<const T*>(a.weight);
    const float r = a.rstd[row];
    float along = 0.f;
    for (int j = Piece<T>::N * threadIdx.x; j < a.n; j += Piece<T>::N * kLong) {
        const typename Piece<T>::wide v = widen<T>(piece(x, j, a.n)), g = widen<T>(piece(dy, j, a.n)), f = widen<T>(weight ? piece(weight, j, a.n) : ones<T>());
#pragma unroll
        for (int k = 0; k < Piece<T>::N; ++k) along = __builtin_fmaf(g[k] * f[k], v[k], along);
    }
    const float c = row_sum<kLongWaves>(along, sums) * a.inv_n * r * r;
    for (int j = Piece<T>::N * threadIdx.x; j < a.n; j += Piece<T>::N * kLong) {
        const typename Piece<T>::wide v = widen<T>(piece(x, j, a.n)), d = widen<T>(piece(dy, j, a.n)) * widen<T>(weight ? piece(weight, j, a.n) : ones<T>());
        typename Piece<T>::vec ds = {};
        if (a.dsum.data) ds = piece(row_of<T>(a.dsum, row), j, a.n);
        put(row_of<T>(a.dx, row), j, a.n, narrow<T>(input_gradient<T>(d, v, r, c, ds, a.dsum.data != nullptr)));
    }
}

// Their part of dw: a thread has a piece of columns and every gridDim.y-th row, four at a time.
template <typename T> __global__ void __launch_bounds__(64) norm_columns_kernel(NormArgs a)
{
    typedef typename Piece<T>::vec vec;
    constexpr int U = 4;
    const int j = Piece<T>::N * (blockIdx.x * 64 + threadIdx.x);
    if (j >= a.n) return;
    typename Piece<T>::wide dw = 0.f;
    for (int64_t row = blockIdx.y; row < a.rows; row += U * (int64_t)gridDim.y) {
        vec s[U], g[U];
        float r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = row + u * (int64_t)gridDim.y;
            if (at < a.rows) {
                s[u] = piece(row_of<T>(a.x, at), j, a.n);
                g[u] = piece(row_of<T>(a.dy, at), j, a.n);
                r[u] = a.rstd[at];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (row + u * (int64_t)gridDim.y < a.rows) dw += widen<T>(g[u]) * (widen<T>(s[u]) * r[u]);
    }
    put_sums<T>(a.partial + (int64_t)blockIdx.y * a.n, j, a.n, dw);
}

// dweight from the parts, always in the same order: a workgroup has 16 columns, 64 threads of it every 64th part of one of them; then eight and eight of these.
template <typename T> __global__ void __launch_bounds__(1024) norm_join_kernel(const float* __restrict__ partial, T* __restrict__ dweight, int parts, int n)
{
    __shared__ float sums[64][17], eights[8][16];
    const int col = threadIdx.x & 15, slice = threadIdx.x >> 4, j = blockIdx.x * 16 + col;
    float v = 0.f;
    if (j < n) {
#pragma unroll 8
        for (int g = slice; g < parts; g += 64) v += partial[(int64_t)g * n + j];
    }
    sums[slice][col] = v;
    __syncthreads();
    if (slice < 8) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += sums[8 * slice + i][col];
        eights[slice][col] = v;
    }
    __syncthreads();
    if (slice == 0 && j < n) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += eights[i][col];
        dweight[j] = (T)v;
    }
}

template <typename T> __global__ void __launch_bounds__(256) zero_weights_kernel(T* dweight, int n)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j < n) dweight[j] = (T)0.f;
}

struct ValueArgs {
    Side codes, out;
    const float* scales;
    int64_t rows;
    int n, per_row;         // pieces of Piece<T>::N
};

template <typename T> __global__ void __launch_bounds__(256) values_kernel(ValueArgs a)
{
    constexpr int N = Piece<T>::N;
    const int64_t pieces = a.rows * a.per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = pieces >> 31 ? i / a.per_row : (int64_t)((unsigned)i / (unsigned)a.per_row);
        const int j = N * (int)(i - row * a.per_row);
        const char* const from = row_of<char>(a.codes, row) + j;
        unsigned long long c = 0;
        if (j + N <= a.n) c = N == 8 ? reinterpret_cast<const Codes8*>(from)->v : reinterpret_cast<const Codes4*>(from)->v;
        else
            for (int k = 0; j + k < a.n; ++k) c |= (unsigned long long)(unsigned char)from[k] << 8 * k;
        const float scale = a.scales[row];
        typename Piece<T>::wide v;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = scale * (float)(signed char)(c >> 8 * k);
        put(row_of<T>(a.out, row), j, a.n, narrow<T>(v));
    }
}

constexpr int kRegisterPieces = 4 * 64 * 16;                    // rows up to this length are kept in registers,
constexpr int kGradientPieces = 2 * 64 * 16;                    // and these in a backward call, which has three rows at a time and dw
constexpr int kMaxParts = 512;                                  // of dweight

// f(constant T, W, NV): wavefronts for a row and pieces of eight for a lane
template <typename T, typename F> void with_shape(int n, int64_t rows, F f)
{
    const int pieces = (n + Piece<T>::N - 1) / Piece<T>::N;
#define SHAPE(W, NV) f(std::integral_constant<int, W>(), std::integral_constant<int, NV>())
    if (pieces <= 64) SHAPE(1, 1);
    else if (pieces <= 128) SHAPE(1, 2);
    else if (pieces <= 256) SHAPE(4, 1);
    else if (pieces <= 512) SHAPE(4, 2);
    else if (pieces <= 1024) SHAPE(4, 4);
    else if (pieces <= 2048) SHAPE(16, 2);
    else SHAPE(16, 4);
#undef SHAPE
}

template <typename F> void with_type(int dtype, F f)
{
    if (dtype == BMGD_F32) f(float());
    else if (dtype == BMGD_BF16) f(__bf16());
    else f(_Float16());
}

bool valid(const bmgd_norm_config& c) { return c.n >= 1 && c.n <= (1 << 20) && known_type(c.dtype) && c.eps >= 0.0 && isfinite(c.eps) && isfinite((float)c.eps); }

int64_t pieces_of(const bmgd_norm_config& c) { return (c.n * (int64_t)size_of(c.dtype) + 15) / 16; }

// Workgroups of a backward call, each of which leaves a part of dweight.
int64_t parts_of(const bmgd_norm_config& c, int64_t rows)
{
    // So many that units are busy, so few that the parts are little beside the rows.  Rows that begin inside lines want more on their way: 8,192 x 1,365, bf16: 33 us with 1,024 parts, 45 with 512;
    // 8,192 x 2,048: 27 and 26.
    const bool crossing = c.n * (int64_t)size_of(c.dtype) % 16 != 0;
    const int64_t pieces = pieces_of(c), at_once = pieces <= 128 ? 4 : 1;                                          // rows of a workgroup
    if (pieces > kGradientPieces) return std::max<int64_t>(1, std::min<int64_t>(rows / 32, kMaxParts));
    return std::max<int64_t>(1, std::min<int64_t>((rows + at_once - 1) / at_once, pieces > 1024 ? kMaxParts / 2 : crossing && pieces > 128 && pieces <= 256 ? 2 * kMaxParts : kMaxParts));
}

// Whether dw is found by workgroups of its own: no second launch, but every row is read twice, 64 bytes at a time.  Measured, us, with them and with parts that are joined (rows x n):
//      bf16 1,000 x 512: 7 and 10;  2,000 x 512: 11 and 11;  500 x 4,096: 8 and 15;  1,000 x 4,096: 12 and 16;  1,000 x 1,365 (rows that begin inside a line): 28 and 13;
//      fp32 1,000 x 512: 8 and 10;  500 x 4,096: 10 and 16;  1,000 x 4,096: 18 and 17.
bool by_columns(const bmgd_norm_config& c, int64_t rows)
{
    const int64_t bytes = c.n * (int64_t)size_of(c.dtype);
    return pieces_of(c) <= kGradientPieces && bytes % 16 == 0 && rows <= 1024 && rows * bytes <= (int64_t(8) << 20);
}

void check(Call& q, const bmgd_norm_config* cfg, int64_t rows, const void* t)
{
    if (!cfg || !t) return q.refuse(BMGD_EINVAL, "cfg and tensors must not be NULL");
    if (cfg->n < 1 || cfg->n > (1 << 20)) q.refuse(BMGD_EINVAL, "n must be in [1, 2^20]");
    if (!known_type(cfg->dtype)) q.refuse(BMGD_EINVAL, "unknown dtype");
    if (!valid(*cfg)) q.refuse(BMGD_EINVAL, "eps must be finite and >= 0");
    q.rows(rows);
}

Side side(const bmgd_matrix& m) { return Side{static_cast<char*>(m.data), m.stride}; }

NormArgs args_of(const bmgd_norm_config& c, int64_t rows, const bmgd_norm_tensors& t)
{
    NormArgs a{};
    a.x = side(t.x);
    a.weight = static_cast<const char*>(t.weight);
    a.rstd = t.rstd;
    a.rows = rows;
    a.n = (int)c.n;
    a.eps = (float)c.eps;
    a.inv_n = (float)(1.0 / (double)c.n);
    return a;
}

}  // namespace

#define BMGD_API __attribute__((visibility("default")))

extern "C" {

BMGD_API size_t bmgd_norm_workspace_bytes(const bmgd_norm_config* cfg, int64_t rows)
{
    if (!cfg || !valid(*cfg) || rows < 0 || rows > kMaxCallRows || by_columns(*cfg, rows)) return 0;
    return ((size_t)parts_of(*cfg, rows) * (size_t)cfg->n * sizeof(float) + 255) / 256 * 256;
}

BMGD_API int bmgd_norm_forward(const bmgd_norm_config* cfg, int64_t rows, const bmgd_norm_tensors* t, void* stream)
{
    Call q{"bmgd_norm_forward"};
    check(q, cfg, rows, t);
    if (q.code != BMGD_OK) return q.code;
    const size_t item = size_of(cfg->dtype);
    const bool some = rows > 0;
    q.matrix("x", t->x, rows, cfg->n, some, item);
    q.matrix("residual", t->residual, rows, cfg->n, false, item);
    q.matrix("sum", t->sum, rows, cfg->n, false, item);
    q.matrix("y", t->y, rows, cfg->n, false, item);
    q.matrix("codes", t->codes, rows, cfg->n, false, 1);
    q.address("weight", t->weight, false, item);
    q.address("scales", t->scales, some && t->codes.data, 4);
    q.address("rstd", t->rstd, false, 4);
    if (some && !t->y.data && !t->codes.data) q.refuse(BMGD_EINVAL, "y or codes is wanted");
    q.apart("sum", t->sum.data, t->y.data);
    q.apart("sum", t->sum.data, t->codes.data);
    q.apart("y", t->y.data, t->codes.data);
    for (const void* in : {t->x.data, t->residual.data}) q.apart("codes", t->codes.data, in);
    q.apart("rstd", t->rstd, t->codes.data ? t->scales : nullptr);
    for (const void* out : {t->sum.data, t->y.data, t->codes.data}) {
        q.apart("a result", out, t->weight);
        q.apart("a result", out, t->rstd);
        if (t->codes.data) q.apart("a result", out, t->scales);
    }
    for (const void* in : {(const void*)t->x.data, (const void*)t->residual.data, t->weight}) {
        q.apart("rstd", t->rstd, in);
        if (t->codes.data) q.apart("scales", t->scales, in);
    }
    // (in place means element by element)
    for (const bmgd_matrix* in : {&t->x, &t->residual})
        for (const bmgd_matrix* out : {&t->sum, &t->y})
            if (in->data && in->data == out->data && rows > 1 && in->stride != out->stride) q.refuse("sum or y", "begins where an operand does, with another stride");
    if (q.code != BMGD_OK || !some) return q.code;
    NormArgs a = args_of(*cfg, rows, *t);
    a.residual = side(t->residual);
    a.sum = side(t->sum);
    a.y = side(t->y);
    a.codes = side(t->codes);
    a.scales = t->scales;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    with_type(cfg->dtype, [&](auto type) {
        typedef decltype(type) T;
        for (a.first = 0; a.first < rows; a.first += kRowsOfLaunch) {
            const int64_t now = std::min(rows - a.first, kRowsOfLaunch);
            if (pieces_of(*cfg) > kRegisterPieces) {
                hipLaunchKernelGGL(norm_forward_long_kernel<T>, dim3((unsigned)now), dim3(kLong), 0, s, a);
                continue;
            }
            with_shape<T>(a.n, rows, [&](auto w, auto nv) {
                constexpr int W = decltype(w)::value, NV = decltype(nv)::value, kRows = block_of(W) / (64 * W);
                hipLaunchKernelGGL((norm_forward_kernel<T, W, NV>), dim3((unsigned)((now + kRows - 1) / kRows)), dim3(block_of(W)), 0, s, a);
            });
        }
    });
    return q.launched();
}

BMGD_API int bmgd_norm_backward(const bmgd_norm_config* cfg, int64_t rows, const bmgd_norm_tensors* t, void* stream)
{
    Call q{"bmgd_norm_backward"};
    check(q, cfg, rows, t);
    if (q.code != BMGD_OK) return q.code;
    const size_t item = size_of(cfg->dtype);
    const bool some = rows > 0;
    q.matrix("dy", t->dy, rows, cfg->n, some, item);
    q.matrix("x", t->x, rows, cfg->n, some, item);
    q.matrix("dsum", t->dsum, rows, cfg->n, false, item);
    q.matrix("dx", t->dx, rows, cfg->n, some, item);
    q.address("weight", t->weight, false, item);
    q.address("dweight", t->dweight, false, item);
    q.address("rstd", t->rstd, some, 4);
    for (const void* in : {(const void*)t->x.data, t->weight, (const void*)t->rstd}) q.apart("dx", t->dx.data, in);
    for (const bmgd_matrix* in : {&t->dy, &t->dsum})
        if (in->data && in->data == t->dx.data && rows > 1 && in->stride != t->dx.stride) q.refuse("dx", "begins where an operand does, with another stride");
    for (const void* in : {(const void*)t->x.data, (const void*)t->dy.data, (const void*)t->dsum.data, (const void*)t->dx.data, t->weight, (const void*)t->rstd}) q.apart("dweight", t->dweight, in);
    const size_t need = t->dweight && some ? bmgd_norm_workspace_bytes(cfg, rows) : 0;
    if (need) {
        if (!t->workspace || (reinterpret_cast<uintptr_t>(t->workspace) & 255)) q.refuse("workspace", "256-byte aligned device memory is wanted for dweight");
        else if (t->workspace_bytes < need) q.refuse(BMGD_ENOMEM, "workspace too small");
    }
    if (q.code != BMGD_OK) return q.code;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (!some) {
        if (!t->dweight) return BMGD_OK;
        with_type(cfg->dtype, [&](auto type) {
            typedef decltype(type) T;
            hipLaunchKernelGGL(zero_weights_kernel<T>, dim3((unsigned)((cfg->n + 255) / 256)), dim3(256), 0, s, static_cast<T*>(t->dweight), (int)cfg->n);
        });
        return q.launched();
    }
    NormArgs a = args_of(*cfg, rows, *t);
    a.dy = side(t->dy);
    a.dsum = side(t->dsum);
    a.dx = side(t->dx);
    a.partial = static_cast<float*>(t->workspace);
    const int64_t parts = parts_of(*cfg, rows), lasts = (pieces_of(*cfg) + 3) / 4;
    a.row_groups = (int)parts;
    a.dweight = static_cast<char*>(t->dweight);
    const bool columns = t->dweight && by_columns(*cfg, rows), at_once = columns && t->dx.data != t->dy.data;
    with_type(cfg->dtype, [&](auto type) {
        typedef decltype(type) T;
        if (pieces_of(*cfg) > kGradientPieces) {
            if (t->dweight)                                     // (first: dx may be dy)
                hipLaunchKernelGGL(norm_columns_kernel<T>, dim3((unsigned)((pieces_of(*cfg) + 63) / 64), (unsigned)parts), dim3(64), 0, s, a);
            for (a.first = 0; a.first < rows; a.first += kRowsOfLaunch)
                hipLaunchKernelGGL(norm_backward_long_kernel<T>, dim3((unsigned)std::min(rows - a.first, kRowsOfLaunch)), dim3(kLong), 0, s, a);
            return;
        }
        with_shape<T>(a.n, rows, [&](auto w, auto nv) {
            constexpr int W = decltype(w)::value, NV = decltype(nv)::value;
            if constexpr (64 * W * NV <= kGradientPieces) {
                if (at_once) hipLaunchKernelGGL((norm_backward_kernel<T, W, NV, kColumns>), dim3((unsigned)(parts + lasts)), dim3(block_of(W)), 0, s, a);
                else if (columns) {
                    // dx takes the place of dy: dw first, the same sums
                    a.row_groups = 0;
                    hipLaunchKernelGGL((norm_backward_kernel<T, W, NV, kColumns>), dim3((unsigned)lasts), dim3(block_of(W)), 0, s, a);
                    a.row_groups = (int)parts;
                    hipLaunchKernelGGL((norm_backward_kernel<T, W, NV, kNoWeights>), dim3((unsigned)parts), dim3(block_of(W)), 0, s, a);
                } else if (t->dweight) hipLaunchKernelGGL((norm_backward_kernel<T, W, NV, kParts>), dim3((unsigned)parts), dim3(block_of(W)), 0, s, a);
                else {
                    // (nothing is left behind, so as many workgroups as units take: 8,192 x 1,365, bf16, with dsum: 29 us, with 512 of them 52)
                    constexpr int kRows = block_of(W) / (64 * W);
                    a.row_groups = (int)std::min<int64_t>((rows + kRows - 1) / kRows, NV * W <= 8 ? 4 * kMaxParts : kMaxParts);
                    hipLaunchKernelGGL((norm_backward_kernel<T, W, NV, kNoWeights>), dim3((unsigned)a.row_groups), dim3(block_of(W)), 0, s, a);
                }
            }
        });
    });
    const int rc = q.launched();
    if (rc != BMGD_OK || !t->dweight || columns) return rc;
    with_type(cfg->dtype, [&](auto type) {
        typedef decltype(type) T;
        hipLaunchKernelGGL(norm_join_kernel<T>, dim3((unsigned)((cfg->n + 15) / 16)), dim3(1024), 0, s, a.partial, static_cast<T*>(t->dweight), (int)parts, a.n);
    });
    return q.launched();
}

BMGD_API int bmgd_product_values(int64_t rows, int64_t n, const bmgd_matrix* codes, const float* scales, const bmgd_matrix* out, int32_t dtype, void* stream)
{
    Call q{"bmgd_product_values"};
    if (!codes || !out) q.refuse(BMGD_EINVAL, "codes and out must not be NULL");
    if (n < 1 || n > (1 << 20)) q.refuse(BMGD_EINVAL, "n must be in [1, 2^20]");
    if (!known_type(dtype)) q.refuse(BMGD_EINVAL, "unknown dtype");
    q.rows(rows);
    if (q.code != BMGD_OK) return q.code;
    q.matrix("codes", *codes, rows, n, rows > 0, 1);
    q.matrix("out", *out, rows, n, rows > 0, size_of(dtype));
    q.address("scales", scales, rows > 0, 4);
    q.apart("out", out->data, codes->data);
    q.apart("out", out->data, scales);
    if (q.code != BMGD_OK || rows == 0) return q.code;
    ValueArgs a{side(*codes), side(*out), scales, rows, (int)n, (int)((n * (int64_t)size_of(dtype) + 15) / 16)};
    const unsigned groups = (unsigned)std::min<int64_t>((rows * a.per_row + 255) / 256, int64_t(1) << 20);
    with_type(dtype, [&](auto type) {
        typedef decltype(type) T;
        hipLaunchKernelGGL(values_kernel<T>, dim3(groups), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    });
    return q.launched();
}

}  // extern "C"
