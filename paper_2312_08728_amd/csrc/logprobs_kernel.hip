// Log probabilities of given classes, entropy and the most probable classes of rows of logits, in one pass over them; their gradient.
//
// A thread holds its largest logit m so far, s = sum 2^d and w = sum 2^d d, d = x log2 e - r with r = m log2 e rounded; where r grows by g, s becomes s 2^-g and
// w (w - g s) 2^-g.  Threads, wavefronts and parts of a row are put together the same way.  Then ln p_j = ln 2 (d_j - log2 s) and the entropy is ln 2 (log2 s - w / s).
// d is one instruction with one rounding; r's own rounding is the same for all and leaves with log2 s.  Rows whose largest logit is not below 1e37 in size (all of the
// type's lowest value, no class at all, infinity) are read once more with d = (x - m) log2 e, which does not leave the range.  -infinity adds nothing.
//
// The most probable classes.  A logit and its class are one 64-bit number, larger where the logit is larger and, of equal ones, the class lower; so no two are
// equal.  Each thread keeps its largest piece of eight; 64 groups of threads have 64 such numbers, and the top-th largest of them is not above the top-th
// largest of all.  The few threads that reach it read their logits again (from cache) and list those that do; the place of each in the list is the number of larger ones.
// Where the list would be too long, or a row has NaN, the classes are found one after the other.
#include "operator_calls.h"
#include "rows_device.h"

#include <math.h>

#include <algorithm>

using namespace bmgd;

namespace {

typedef unsigned long long Key;

constexpr float kLog2E = 1.44269504f, kLn2 = 0.693147182f;
constexpr float kLowest = -3.40282347e38f;
constexpr float kUsual = 1e37f;                  // x log2 e - r is finite, or -infinity for one far below, where m is smaller than this
constexpr float kFar = -1000.f;                  // 2^-1000 is 0, times this still 0
constexpr int kMaxTop = 64, kMaxParts = 64;
constexpr int kList = 512;                       // a segment of fewer classes than 8 top fits whole

struct LogArgs {
    const char* logits;
    int64_t stride;                              // in elements
    char* dlogits;
    int64_t dstride;
    const int* labels;
    float *logprob, *entropy, *top_logprobs, *kept;
    int* top_classes;
    const float *dlogprob, *dentropy;
    float* part_stats;                           // [row][part][3]
    Key* part_keys;                              // [row][part][top]
    int64_t rows, first;                         // first: of the launch
    int classes, top, parts, span, chunks;
};

struct Stats {
    float m, s, w;
};

// To another reference
__device__ __forceinline__ void scale_down(Stats& a, float to, float d)
{
    d = fmaxf(d, kFar);
    const float f = __builtin_amdgcn_exp2f(d);
    a.w = f * __builtin_fmaf(d, a.s, a.w);
    a.s *= f;
    a.m = to;
}
// r of m: rounded, wherever it is used
__device__ __forceinline__ float reference(float m)
{
    float r = m * kLog2E;
    asm("" : "+v"(r));
    return r;
}
__device__ __forceinline__ void refer_to(Stats& a, float to)
{
    if (fabsf(to) < kUsual) scale_down(a, to, reference(a.m) - reference(to));
    else scale_down(a, to, (a.m - to) * kLog2E);
}

__device__ __forceinline__ Stats wave_merge(Stats a)
{
    refer_to(a, wave_max(a.m));
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    return a;
}

// Larger numbers for larger logits, one for both zeros, NaN above all.
__device__ __forceinline__ unsigned ordered(float x)
{
    const int b = __builtin_bit_cast(int, x + 0.f);
    return x != x ? ~0u : (unsigned)b ^ ((unsigned)(b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(Key k)
{
    const unsigned u = (unsigned)(k >> 32);
    return __builtin_bit_cast(float, u & 0x80000000u ? u ^ 0x80000000u : ~u);           // (~0: NaN)
}
__device__ __forceinline__ Key key_of(float x, int at) { return (Key)ordered(x) << 32 | (0xffffffffu - (unsigned)at); }
__device__ __forceinline__ int class_of(Key k) { return (int)(0xffffffffu - (unsigned)k); }

// The threads of a row: all W wavefronts of a workgroup, or one wavefront of four (which waits for no other).
template <int W> __device__ __forceinline__ void together()
{
    if constexpr (W > 1) __syncthreads();
    else {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
}

// Of the wavefront's 64 numbers, which lie in shared memory too, the one with `rank` larger ones, 0 if there is none (they differ, but for zeros).
__device__ __forceinline__ Key ranked(Key v, const Key* all, int rank)
{
    int larger = 0;
#pragma unroll 16
    for (int i = 0; i < 64; ++i) larger += all[i] > v;
    const unsigned long long found = __ballot(larger == rank);
    return found ? of_lane(v, __builtin_ctzll(found)) : 0;
}

template <typename T> __device__ __forceinline__ typename Eight<T>::vec logits_at(const T* x, int j, int end)
{
    return j + 8 <= end ? Eight<T>::load(x + j) : Eight<T>::load_part(x + j, end - j, (T)-__builtin_inff());
}

__device__ __forceinline__ float largest(float8v v)
{
    return fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
}

// ENT: with w
template <int U, bool ENT> __device__ __forceinline__ void take(Stats& st, const float8v* v, const float* most)
{
    float m = st.m;
#pragma unroll
    for (int u = 0; u < U; ++u) m = fmaxf(m, most[u]);
    const float r = reference(m);
    if (m > st.m) scale_down(st, m, reference(st.m) - r);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float d = __builtin_fmaf(v[u][k], kLog2E, -r), e = __builtin_amdgcn_exp2f(d);
            st.s += e;
            if constexpr (ENT) st.w = __builtin_fmaf(e, fmaxf(d, kFar), st.w);
        }
}

// A row of unusual size: its largest, then the sums
__device__ __forceinline__ void take_unusual(Stats& st, float8v v)
{
    const float m = fmaxf(st.m, largest(v));
    if (m > st.m) scale_down(st, m, (st.m - m) * kLog2E);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float d = (v[k] - m) * kLog2E, e = __builtin_amdgcn_exp2f(d);
        st.s += e;
        st.w = __builtin_fmaf(e, fmaxf(d, kFar), st.w);
    }
}

// What is known of a row's distribution: log2 of the sum, entropy; `empty` where all logits are -infinity.
struct Row {
    float m, ls, entropy;
    bool empty;
};
__device__ __forceinline__ Row finish(const Stats& a)
{
    Row r;
    r.empty = a.s == 0.f;
    r.m = r.empty ? -__builtin_inff() : a.s != a.s ? a.s : a.m;
    r.ls = r.empty ? 0.f : log2f(a.s);
    r.entropy = r.empty ? 0.f : kLn2 * (r.ls - a.w / a.s);
    return r;
}
__device__ __forceinline__ float logprob_of(const Row& r, float x)
{
    if (r.empty) return -__builtin_inff();
    // (what r has lost of m log2 e is in log2 s)
    const float lost = fabsf(r.m) < kUsual ? __builtin_fmaf(r.m, kLog2E, -reference(r.m)) : 0.f;
    return __builtin_fmaf(lost - r.ls, kLn2, x - r.m);
}

template <typename T> __device__ __forceinline__ void write_row(const LogArgs& a, int64_t row, const T* x, const Row& r)
{
    if (a.logprob) {
        const int label = a.labels[row];
        a.logprob[row] = label < 0 ? 0.f : label >= a.classes ? __builtin_nanf("") : logprob_of(r, (float)x[label]);
    }
    if (a.entropy) a.entropy[row] = r.entropy;
    if (a.kept) {
        a.kept[3 * row] = r.m;
        a.kept[3 * row + 1] = r.ls;
        a.kept[3 * row + 2] = r.entropy;
    }
}

// One of the most probable classes: of a row, or of a part of it
__device__ __forceinline__ void write_top(const LogArgs& a, int64_t row, int part, int place, Key k, const Row& r)
{
    if (a.parts > 1) a.part_keys[(row * a.parts + part) * a.top + place] = k;
    else {
        a.top_classes[row * a.top + place] = class_of(k);
        a.top_logprobs[row * a.top + place] = logprob_of(r, value_of(k));
    }
}

constexpr int threads_of(int w) { return w < 4 ? 256 : 64 * w; }

template <typename T, int W, bool TOP, bool ENT> __global__ void __launch_bounds__(threads_of(W)) logprobs_kernel(LogArgs a)
{
    constexpr int kLanes = 64 * W, kRows = threads_of(W) / kLanes, U = 4, kTurn = 8 * kLanes * U;
    typedef typename Eight<T>::vec vec;
    __shared__ Stats parts[W > 1 ? W : 1];
    __shared__ Key keys[TOP ? kRows : 1][TOP ? kLanes : 1];
    __shared__ Key list[TOP ? kRows : 1][TOP ? kList : 1];
    __shared__ Key threshold;
    __shared__ int counts[kRows];
    const int t = threadIdx.x % kLanes, mine = threadIdx.x / kLanes;
    const int64_t row = a.first + (int64_t)blockIdx.x * kRows + mine;
    if (row >= a.rows) return;                                  // (whole wavefronts, and none of a workgroup with barriers)
    const int part = blockIdx.y, begin = part * a.span, end = a.classes - begin > a.span ? begin + a.span : a.classes;
    const T* const x = reinterpret_cast<const T*>(a.logits) + row * a.stride;

    Stats st{-kUsual, 0.f, 0.f};
    float best = -__builtin_inff();
    int best_at = begin + 8 * t < end ? begin + 8 * t : -1;
    int j = begin + 8 * t;
    {
        // turns of U pieces, the next ones on their way; those that end inside a turn have -infinity behind the end
        vec next[U];
        auto request = [&](int from) {
            if (from + kTurn - 8 * kLanes + 8 <= end) {
#pragma unroll
                for (int u = 0; u < U; ++u) next[u] = Eight<T>::load(x + from + 8 * kLanes * u);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = from + 8 * kLanes * u;
                    if (i < end) next[u] = logits_at(x, i, end);
                    else next[u] = (T)-__builtin_inff();
                }
            }
        };
        request(j);
        while (j < end) {
            float8v v[U];
            float most[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = widen<T>(next[u]);
            const int now = j;
            j += kTurn;
            if (j < end) request(j);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                most[u] = largest(v[u]);
                if constexpr (TOP)
                    if (most[u] > best) {
                        best = most[u];
                        best_at = now + 8 * kLanes * u;
                    }
            }
            take<U, ENT>(st, v, most);
        }
    }

    auto merged = [&](Stats own) {
        own = wave_merge(own);
        if constexpr (W > 1) {
            if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = own;
            __syncthreads();
            float m = parts[0].m;
#pragma unroll
            for (int i = 1; i < W; ++i) m = fmaxf(m, parts[i].m);
            Stats all{m, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < W; ++i) {
                Stats o = parts[i];
                refer_to(o, m);
                all.s += o.s;
                all.w += o.w;
            }
            return all;
        } else return own;
    };
    if constexpr (TOP) keys[mine][t] = best_at < 0 ? 0 : key_of(best, best_at + 7 < end ? best_at + 7 : end - 1);
    if (t == 0) counts[mine] = 0;
    st = merged(st);
    if (!(st.m > -kUsual && st.m < kUsual)) {
        if constexpr (W > 1) __syncthreads();                   // (`parts` has been read)
        st = Stats{kLowest, 0.f, 0.f};
        for (int i = begin + 8 * t; i < end; i += 8 * kLanes) take_unusual(st, widen<T>(logits_at(x, i, end)));
        st = merged(st);
    }
    const Row r = finish(st);
    if (t == 0) {
        if (a.parts > 1) {
            float* const to = a.part_stats + (row * a.parts + part) * 3;
            to[0] = st.m;
            to[1] = st.s;
            to[2] = st.w;
        } else write_row(a, row, x, r);
    }
    if constexpr (TOP) {
        // a number that at least `top` of the segment's are not below
        Key least;
        if constexpr (W > 1) {
            if (threadIdx.x < 64) {
                Key k = keys[0][t];
#pragma unroll
                for (int i = 1; i < W; ++i) k = keys[0][64 * i + t] > k ? keys[0][64 * i + t] : k;
                keys[0][t] = k;
                together<1>();
                k = ranked(k, keys[0], a.top - 1);
                if (t == 0) threshold = k;
            }
            __syncthreads();
            least = threshold;
        } else {
            together<1>();
            least = ranked(keys[mine][t], keys[mine], a.top - 1);
        }
        const bool plain = st.s == st.s;
        if (plain && best_at >= 0 && key_of(best, best_at) >= least) {
            auto look = [&](float8v v, int i) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const Key q = key_of(v[k], i + k);
                    if (i + k < end && q >= least) {
                        const int at = atomicAdd(&counts[mine], 1);
                        if (at < kList) list[mine][at] = q;
                    }
                }
            };
            for (int from = begin + 8 * t; from < end; from += 2 * kTurn) {
                vec v[2 * U];
#pragma unroll
                for (int u = 0; u < 2 * U; ++u) {
                    const int i = from + 8 * kLanes * u;
                    if (i < end) v[u] = logits_at(x, i, end);
                }
#pragma unroll
                for (int u = 0; u < 2 * U; ++u) {
                    const int i = from + 8 * kLanes * u;
                    if (i < end) {
                        const float8v f = widen<T>(v[u]);
                        if (ordered(largest(f)) >= (unsigned)(least >> 32)) look(f, i);
                    }
                }
            }
        }
        together<W>();
        const int count = counts[mine];
        if (plain && count <= kList) {
            for (int i = t; i < count; i += kLanes) {
                const Key q = list[mine][i];
                int place = 0;
                for (int o = 0; o < count; ++o) place += list[mine][o] > q;
                if (place < a.top) write_top(a, row, part, place, q, r);
            }
            if (t >= count && t < a.top) write_top(a, row, part, t, 0, r);       // (a part of fewer than `top` classes)
        } else {
            Key before = ~(Key)0;
            for (int place = 0; place < a.top; ++place) {
                Key k = 0;
                for (int i = begin + 8 * t; i < end; i += 8 * kLanes) {
                    const float8v v = widen<T>(logits_at(x, i, end));
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const Key q = key_of(v[c], i + c);
                        if (i + c < end && q < before && q > k) k = q;
                    }
                }
                k = wave_max(k);
                if constexpr (W > 1) {
                    __syncthreads();
                    if ((threadIdx.x & 63) == 0) keys[0][threadIdx.x >> 6] = k;
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < W; ++i) k = keys[0][i] > k ? keys[0][i] : k;
                }
                if (t == 0) write_top(a, row, part, place, k, r);
                before = k;
            }
        }
    }
}

// A row from its parts (at most 64).  Each part's classes are in falling order, so that the parts' n-th ones, n parts >= top, bound the top-th of the row from below.
template <typename T> __global__ void __launch_bounds__(256) logprobs_join_kernel(LogArgs a)
{
    extern __shared__ Key list[];
    __shared__ Key threshold;
    __shared__ int count;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63;
    const float* const from = a.part_stats + row * a.parts * 3;
    Stats st{kLowest, 0.f, 0.f};                                // (of a size that no part with classes has: adds nothing)
    if (lane < a.parts) st = Stats{from[3 * lane], from[3 * lane + 1], from[3 * lane + 2]};
    st = wave_merge(st);
    const Row r = finish(st);
    if (threadIdx.x == 0) {
        write_row(a, row, reinterpret_cast<const T*>(a.logits) + row * a.stride, r);
        count = 0;
    }
    if (!a.top) return;
    const Key* const keys = a.part_keys + row * a.parts * a.top;
    if (threadIdx.x < 64) {
        const int nth = (a.top + a.parts - 1) / a.parts;
        const Key least = ~wave_max(lane < a.parts ? ~keys[lane * a.top + nth - 1] : (Key)0);
        if (threadIdx.x == 0) threshold = least;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.parts * a.top; i += 256) {
        const Key q = keys[i];
        if (q && q >= threshold) list[atomicAdd(&count, 1)] = q;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += 256) {
        const Key q = list[i];
        int place = 0;
        for (int o = 0; o < count; ++o) place += list[o] > q;
        if (place < a.top) {
            a.top_classes[row * a.top + place] = class_of(q);
            a.top_logprobs[row * a.top + place] = logprob_of(r, value_of(q));
        }
    }
}

// dlogits: W wavefronts have a row (W = 1), or a chunk of one.
constexpr int kChunk = 8 * 4 * 256;

// What a row's gradients are made of: dlogits = 2^d (both + d of_entropy), d = x log2 e - shift, and dl more at the label.  shift is r + log2 s rounded; what that loses
// is put into the other two.
struct Slope {
    float m, shift, both, of_entropy, dl;
    int label;
    bool usual;
};
__device__ __forceinline__ Slope slope_of(float m, float ls, float entropy, float dl, float dh, int label)
{
    Slope g;
    g.m = m;
    g.usual = fabsf(m) < kUsual;
    g.shift = ls;
    float lost = 0.f;
    if (g.usual) {
        const float r = reference(m), of_ls = (g.shift = r + ls) - r;
        lost = (r - (g.shift - of_ls)) + (ls - of_ls);
    }
    const float f = __builtin_amdgcn_exp2f(-lost);
    g.of_entropy = -dh * kLn2 * f;
    g.both = -(dl + dh * (entropy - kLn2 * lost)) * f;
    g.dl = dl;
    g.label = label;
    return g;
}
template <bool DH> __device__ __forceinline__ float8v logit_gradients(float8v v, const Slope& g)
{
    float8v o;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float d = g.usual ? __builtin_fmaf(v[k], kLog2E, -g.shift) : __builtin_fmaf(v[k] - g.m, kLog2E, -g.shift);
        const float p = __builtin_amdgcn_exp2f(d);
        o[k] = DH ? p * __builtin_fmaf(fmaxf(d, kFar), g.of_entropy, g.both) : p * g.both;
    }
    return o;
}

template <typename T, int W, bool DH> __global__ void __launch_bounds__(256) logprobs_backward_kernel(LogArgs a)
{
    constexpr int kLanes = 64 * W, kRows = 4 / W, U = 4;
    typedef typename Eight<T>::vec vec;
    const int t = threadIdx.x % kLanes;
    const int64_t items = W == 1 ? a.rows : a.rows * a.chunks;
    for (int64_t item = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; item < items; item += (int64_t)gridDim.x * kRows) {
        int64_t row = item;
        int begin = 0, end = a.classes;
        if constexpr (W > 1) {
            row = items >> 31 ? item / a.chunks : (int64_t)((unsigned)item / (unsigned)a.chunks);
            begin = (int)(item - row * a.chunks) * kChunk;
            end = a.classes - begin > kChunk ? begin + kChunk : a.classes;
        }
        const T* const x = reinterpret_cast<const T*>(a.logits) + row * a.stride;
        T* const out = reinterpret_cast<T*>(a.dlogits) + row * a.dstride;
        const float m = a.kept[3 * row], entropy = a.kept[3 * row + 2], dh = DH ? a.dentropy[row] : 0.f;
        const int label = a.dlogprob ? a.labels[row] : -1;
        const Slope g = slope_of(m, a.kept[3 * row + 1], entropy, label < 0 ? 0.f : label >= a.classes ? __builtin_nanf("") : a.dlogprob[row], dh, label);
        const bool empty = m == -__builtin_inff() && g.label < a.classes;
        for (int j = begin + 8 * t; j < end; j += 8 * kLanes * U) {
            vec v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = j + 8 * kLanes * u;
                if (i < end) v[u] = logits_at(x, i, end);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = j + 8 * kLanes * u;
                if (i >= end) continue;
                float8v o = logit_gradients<DH>(widen<T>(v[u]), g);
                if ((unsigned)(g.label - i) < 8u) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) o[k] += k == g.label - i ? g.dl : 0.f;
                }
                if (empty) o = 0.f;
                const vec w = narrow<T>(o);
                if (i + 8 <= end) Eight<T>::store(out + i, w);
                else Eight<T>::store_part(out + i, w, end - i);
            }
        }
    }
}

template <typename F> void with_type(int dtype, F f)
{
    if (dtype == BMGD_F32) f(float());
    else if (dtype == BMGD_BF16) f(__bf16());
    else f(_Float16());
}

bool valid(const bmgd_logprobs_config& c)
{
    return c.classes >= 1 && c.classes <= (1 << 24) && known_type(c.dtype) && c.top >= 0 && c.top <= kMaxTop && c.top <= c.classes;
}

constexpr int kWide = 16384;                     // a part of a row has this many classes or more

// Parts of a row, where few rows would leave compute units idle.
int parts_of(int64_t classes, int64_t rows)
{
    const int64_t parts = std::min<int64_t>(std::min<int64_t>(512 / std::max<int64_t>(rows, 1), kMaxParts), classes / kWide);
    return (int)std::max<int64_t>(parts, 1);
}
// classes of a part: whole pieces of eight
int span_of(int64_t classes, int parts) { return (int)((classes + parts - 1) / parts + 7) / 8 * 8; }

size_t stats_bytes(int64_t rows, int parts) { return ((size_t)rows * parts * 3 * sizeof(float) + 255) / 256 * 256; }

void check(Call& q, const bmgd_logprobs_config* cfg, int64_t rows, const void* t)
{
    if (!cfg || !t) return q.refuse(BMGD_EINVAL, "cfg and tensors must not be NULL");
    if (cfg->classes < 1 || cfg->classes > (1 << 24)) q.refuse(BMGD_EINVAL, "classes must be in [1, 2^24]");
    if (!known_type(cfg->dtype)) q.refuse(BMGD_EINVAL, "unknown dtype");
    if (!valid(*cfg)) q.refuse(BMGD_EINVAL, "top must be in [0, 64] and not above classes");
    q.rows(rows);
}

}  // namespace

#define BMGD_API __attribute__((visibility("default")))

extern "C" {

BMGD_API size_t bmgd_logprobs_workspace_bytes(const bmgd_logprobs_config* cfg, int64_t rows)
{
    if (!cfg || !valid(*cfg) || rows < 1 || rows > kMaxCallRows) return 0;
    const int parts = parts_of(cfg->classes, rows);
    if (parts == 1) return 0;
    return stats_bytes(rows, parts) + ((size_t)rows * parts * cfg->top * sizeof(Key) + 255) / 256 * 256;
}

BMGD_API int bmgd_logprobs_forward(const bmgd_logprobs_config* cfg, int64_t rows, const bmgd_logprobs_tensors* t, void* stream)
{
    Call q{"bmgd_logprobs_forward"};
    check(q, cfg, rows, t);
    if (q.code != BMGD_OK) return q.code;
    const bool some = rows > 0;
    q.matrix("logits", t->logits, rows, cfg->classes, some, size_of(cfg->dtype));
    q.address("labels", t->labels, some && t->logprob, 4);
    q.address("logprob", t->logprob, false, 4);
    q.address("entropy", t->entropy, false, 4);
    q.address("top_classes", t->top_classes, some && cfg->top, 4);
    q.address("top_logprobs", t->top_logprobs, some && cfg->top, 4);
    q.address("kept", t->kept, false, 4);
    const void* const written[] = {t->logprob, t->entropy, cfg->top ? t->top_classes : nullptr, cfg->top ? t->top_logprobs : nullptr, t->kept};
    for (int i = 0; i < 5; ++i) {
        q.apart("a result", written[i], t->logits.data);
        q.apart("a result", written[i], t->labels);
        for (int k = 0; k < i; ++k) q.apart("a result", written[i], written[k]);
    }
    const size_t need = bmgd_logprobs_workspace_bytes(cfg, rows);
    if (need) {
        if (!t->workspace || (reinterpret_cast<uintptr_t>(t->workspace) & 255)) q.refuse("workspace", "256-byte aligned device memory is wanted");
        else if (t->workspace_bytes < need) q.refuse(BMGD_ENOMEM, "workspace too small");
    }
    if (q.code != BMGD_OK || !some) return q.code;
    LogArgs a{};
    a.logits = static_cast<const char*>(t->logits.data);
    a.stride = t->logits.stride;
    a.labels = t->labels;
    a.logprob = t->logprob;
    a.entropy = t->entropy;
    a.top_classes = t->top_classes;
    a.top_logprobs = t->top_logprobs;
    a.kept = t->kept;
    a.rows = rows;
    a.classes = (int)cfg->classes;
    a.top = cfg->top;
    a.parts = parts_of(cfg->classes, rows);
    a.span = span_of(cfg->classes, a.parts);
    if (a.parts > 1) {
        a.part_stats = static_cast<float*>(t->workspace);
        a.part_keys = reinterpret_cast<Key*>(static_cast<char*>(t->workspace) + stats_bytes(rows, a.parts));
    }
    const hipStream_t s = static_cast<hipStream_t>(stream);
    with_type(cfg->dtype, [&](auto type) {
        typedef decltype(type) T;
        auto launch = [&](auto w, auto top, auto ent) {
            constexpr int W = decltype(w)::value, kRows = threads_of(W) / (64 * W);
            constexpr bool TOP = decltype(top)::value, ENT = decltype(ent)::value;
            for (a.first = 0; a.first < rows; a.first += kRowsOfLaunch) {
                const int64_t now = std::min(rows - a.first, kRowsOfLaunch);
                hipLaunchKernelGGL((logprobs_kernel<T, W, TOP, ENT>), dim3((unsigned)((now + kRows - 1) / kRows), (unsigned)a.parts), dim3(threads_of(W)), 0, s, a);
            }
        };
        auto shaped = [&](auto top, auto ent) {
            if (a.span <= 2048) launch(std::integral_constant<int, 1>(), top, ent);
            else if (a.span <= 16384 || rows * a.parts > 512) launch(std::integral_constant<int, 4>(), top, ent);
            else launch(std::integral_constant<int, 16>(), top, ent);
        };
        auto with_top = [&](auto ent) {
            if (a.top) shaped(std::true_type(), ent);
            else shaped(std::false_type(), ent);
        };
        if (a.entropy || a.kept) with_top(std::true_type());
        else with_top(std::false_type());
        if (a.parts > 1) hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3((unsigned)rows), dim3(256), (size_t)std::max(1, a.parts * a.top) * sizeof(Key), s, a);
    });
    return q.launched();
}

BMGD_API int bmgd_logprobs_backward(const bmgd_logprobs_config* cfg, int64_t rows, const bmgd_logprobs_tensors* t, void* stream)
{
    Call q{"bmgd_logprobs_backward"};
    check(q, cfg, rows, t);
    if (q.code != BMGD_OK) return q.code;
    const bool some = rows > 0;
    q.matrix("logits", t->logits, rows, cfg->classes, some, size_of(cfg->dtype));
    q.matrix("dlogits", t->dlogits, rows, cfg->classes, some, size_of(cfg->dtype));
    q.address("kept", t->kept, some, 4);
    q.address("dlogprob", t->dlogprob, false, 4);
    q.address("dentropy", t->dentropy, false, 4);
    q.address("labels", t->labels, some && t->dlogprob, 4);
    for (const void* in : {(const void*)t->labels, (const void*)t->kept, (const void*)t->dlogprob, (const void*)t->dentropy}) q.apart("dlogits", t->dlogits.data, in);
    if (t->dlogits.data && t->dlogits.data == t->logits.data && rows > 1 && t->dlogits.stride != t->logits.stride)
        q.refuse("dlogits", "begins where logits does, with another stride");
    if (q.code != BMGD_OK || !some) return q.code;
    LogArgs a{};
    a.logits = static_cast<const char*>(t->logits.data);
    a.stride = t->logits.stride;
    a.dlogits = static_cast<char*>(t->dlogits.data);
    a.dstride = t->dlogits.stride;
    a.labels = t->labels;
    a.kept = t->kept;
    a.dlogprob = t->dlogprob;
    a.dentropy = t->dentropy;
    a.rows = rows;
    a.classes = (int)cfg->classes;
    a.chunks = (int)((cfg->classes + kChunk - 1) / kChunk);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    with_type(cfg->dtype, [&](auto type) {
        typedef decltype(type) T;
        const int64_t most = int64_t(1) << 20;
        auto launch = [&](auto dh) {
            constexpr bool DH = decltype(dh)::value;
            if (cfg->classes <= 2048) hipLaunchKernelGGL((logprobs_backward_kernel<T, 1, DH>), dim3((unsigned)std::min((rows + 3) / 4, most)), dim3(256), 0, s, a);
            else hipLaunchKernelGGL((logprobs_backward_kernel<T, 4, DH>), dim3((unsigned)std::min(rows * a.chunks, most)), dim3(256), 0, s, a);
        };
        if (a.dentropy) launch(std::true_type());
        else launch(std::false_type());
    });
    return q.launched();
}

}  // extern "C"
