// Log probabilities of given classes, entropy and the most probable classes of rows of logits, in one pass over them; their gradient.
//
// A thread holds its largest logit m so far, s = sum 2^d and w = sum 2^d d, d = x log2 e - r with r = m log2 e rounded; where r grows by g, s becomes s 2^-g and
// w (w - g s) 2^-g.  Threads, wavefronts and parts of a row are put together the same way.  Then ln p_j = ln 2 (d_j - log2 s) and the entropy is ln 2 (log2 s - w / s).
// d is one instruction with one rounding; r's own rounding is the same for all and leaves with log2 s.  Rows whose largest logit is not below 2^24 in size (masked in all
// classes with some large number or the type's lowest, no class at all, infinity) are read once more with d = (x - m) log2 e.  -infinity adds nothing.
//
// The most probable classes.  A logit and its class are one 64-bit number, larger where the logit is larger and, of equal ones, the class lower; so no two are
// equal.  Of what the threads read first (8,192 logits of 16 bits for four wavefronts), 64 groups of threads have their largest numbers; the top-th largest of these is not above the top-th
// largest of the row.  Pieces that reach it are put into shared memory as they pass by.  After 2, 4, 8, ... turns (from 64 / top on) their classes that do are counted against one another, the
// place of each being the number of larger ones; the top-th of them is what later ones have to reach, so that between two counts about as many are listed as are wanted.
// Where a list overflows (logits that rise all along a row), the row is read again with a bound that comes of all of it; where it does so again, or a row has NaN, the
// classes are found one after the other.
//
// What bounds it (us, sets of tensors in turn that are larger together than the caches).  8,192 x 32,000, bf16: 94 without classes (5.6 TB/s), 119 with eight: memory, and counting that four workgroups to a unit
// do not hide.  4,097 x 10,001, f16: 22 by itself and 25 in front of its gradient, of which memory 16, the rest a launch, the first trip and the last turn; the gradient 30 (5.5 TB/s).  16 x 100,003, fp32, twenty classes: 12, two launches.  1 x 1,000: 4.9, a launch and a chain of one trip to memory, a count and sums.
#include "operator_calls.h"
#include "rows_device.h"

#include <math.h>

#include <algorithm>

using namespace bmgd;

namespace {

typedef unsigned long long Key;

constexpr float kLog2E = 1.44269504f, kLn2 = 0.693147182f;
constexpr float kLowest = -3.40282347e38f;
constexpr float kUsual = 16777216.f;             // where m is smaller than 2^24 r is off by 1 at most, so 2^d of the largest logit is about 1 (at 1e10 it would be 2^440)
constexpr float kFar = -1000.f;                  // 2^-1000 is 0, times this still 0
constexpr int kMaxTop = 64, kMaxParts = 64;
constexpr int kList = 640;                       // classes listed between two counts at most: 64 pieces of eight and some more,
constexpr int pieces_kept(int w) { return w == 1 ? 168 : 256; }        // and pieces: with a wavefront to a row one of 660 fp32 or 1,320 16-bit logits fits whole

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
    int classes, top, parts, span;
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
// What a Stats' sums refer to: r of m, m log2 e itself, or, in parts of one row, whichever is due to the size of the part's own m.
enum Refers { kRounded, kItself, kEither };
template <Refers OF> __device__ __forceinline__ void refer_to(Stats& a, float to)
{
    const bool rounded = OF == kRounded || (OF == kEither && fabsf(a.m) < kUsual), to_rounded = OF == kRounded || (OF == kEither && fabsf(to) < kUsual);
    float d;
    if (rounded) d = to_rounded ? reference(a.m) - reference(to) : __builtin_fmaf(-to, kLog2E, reference(a.m));
    else d = to_rounded ? __builtin_fmaf(a.m, kLog2E, -reference(to)) : (a.m - to) * kLog2E;
    scale_down(a, to, d);
}

template <Refers OF> __device__ __forceinline__ Stats wave_merge(Stats a)
{
    refer_to<OF>(a, wave_max(a.m));
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    return a;
}

// Larger numbers for larger logits, one for both zeros, one for all NaN above all others.  (Not the largest of 32 bits: with class 0 that would be the largest of all 64-bit
// numbers, which stands for "nothing yet" where classes are found one after the other.)
constexpr unsigned kOrderedNan = ~1u;
__device__ __forceinline__ unsigned ordered(float x)
{
    const int b = __builtin_bit_cast(int, x + 0.f);
    return x != x ? kOrderedNan : (unsigned)b ^ ((unsigned)(b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(Key k)
{
    const unsigned u = (unsigned)(k >> 32);
    return __builtin_bit_cast(float, u & 0x80000000u ? u ^ 0x80000000u : ~u);           // (kOrderedNan: NaN)
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

// How many of `count` numbers in shared memory are larger than v, which four neighbouring lanes have: each looks at a quarter
__device__ __forceinline__ int larger_than(Key v, const Key* all, int count)
{
    int larger = 0;
#pragma unroll 4
    for (int i = threadIdx.x & 3; i < count; i += 4) larger += all[i] > v;
    larger += from_lane<kSwap1>(larger);
    return larger + from_lane<kSwap2>(larger);
}

// Pieces begin at multiples of 16 bytes: `before` elements before the row, which with those behind `end` count as -infinity.
template <typename T> __device__ __forceinline__ int before_row(const T* x) { return (int)(((uintptr_t)x & 15) / sizeof(T)); }
template <typename T> __device__ __forceinline__ typename Piece<T>::vec logits_at(const T* x, int j, int begin, int end)
{
    return j >= begin && j + Piece<T>::N <= end ? Piece<T>::load(x + j) : Piece<T>::load_part(x, j, begin, end, (T)-__builtin_inff());
}

// What is left of a segment [begin, end) beside its whole pieces: a piece that begins before it (at head), and one that ends behind it.  `whole`: where the
// whole ones begin.
struct Edges {
    int whole, before, behind;                   // (kNowhere: none)
};
constexpr int kNowhere = 0x7fffffff;
template <int N> __device__ __forceinline__ Edges edges_of(int head, int begin, int end)
{
    Edges e;
    const bool early = head < begin;
    const int last = head + (end - head) / N * N;
    e.whole = early ? head + N : head;
    e.before = early ? head : kNowhere;
    e.behind = last < end && last >= e.whole ? last : kNowhere;
    return e;
}

template <typename V> __device__ __forceinline__ float largest(V v)
{
    constexpr int N = sizeof(V) / 4;
    float m = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
    if constexpr (N == 8) m = fmaxf(m, fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    return m;
}

// ENT: with w
template <int U, bool ENT, typename V> __device__ __forceinline__ void take(Stats& st, const V* v, const float* most)
{
    float m = st.m;
#pragma unroll
    for (int u = 0; u < U; ++u) m = fmaxf(m, most[u]);
    const float r = reference(m);
    if (m > st.m) scale_down(st, m, reference(st.m) - r);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < (int)sizeof(V) / 4; ++k) {
            const float d = __builtin_fmaf(v[u][k], kLog2E, -r), e = __builtin_amdgcn_exp2f(d);
            st.s += e;
            if constexpr (ENT) st.w = __builtin_fmaf(e, fmaxf(d, kFar), st.w);
        }
}

// A row of unusual size: its largest, then the sums
template <typename V> __device__ __forceinline__ void take_unusual(Stats& st, V v)
{
    const float m = fmaxf(st.m, largest(v));
    if (m > st.m) scale_down(st, m, (st.m - m) * kLog2E);
#pragma unroll
    for (int k = 0; k < (int)sizeof(V) / 4; ++k) {
        const float d = (v[k] - m) * kLog2E, e = __builtin_amdgcn_exp2f(d);
        st.s += e;
        st.w = __builtin_fmaf(e, fmaxf(d, kFar), st.w);
    }
}

// What is known of a row's distribution: log2 of the sum (relative to what its Stats refer to), entropy; `empty` where all logits are -infinity.
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

// at_label: the logit of a label that is one of the classes
__device__ __forceinline__ void write_row(const LogArgs& a, int64_t row, int label, float at_label, const Row& r)
{
    if (a.logprob) a.logprob[row] = label < 0 ? 0.f : label >= a.classes ? __builtin_nanf("") : logprob_of(r, at_label);
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
    constexpr int kLanes = 64 * W, kRows = threads_of(W) / kLanes, N = Piece<T>::N, U = 4, kTurn = N * kLanes * U, kPieces = pieces_kept(W);
    typedef typename Piece<T>::vec vec;
    typedef typename Piece<T>::wide wide;
    __shared__ Stats parts[W > 1 ? W : 1];
    __shared__ Key groups_of[TOP ? kRows : 1][TOP ? (W > 1 ? 128 : 64) : 1];
    __shared__ Key list[TOP ? kRows : 1][TOP ? kList : 1];
    __shared__ Key sorted[TOP ? kRows : 1][2][TOP ? kMaxTop : 1];
    __shared__ vec pieces[TOP ? kRows : 1][TOP ? kPieces : 1];
    __shared__ int places[TOP ? kRows : 1][TOP ? kPieces : 1];
    __shared__ Key threshold;
    __shared__ int kept[kRows][2], listed[kRows][2];            // how many pieces and classes, in turn: one is cleared while the other is in use
    const int t = threadIdx.x % kLanes, mine = threadIdx.x / kLanes;
    const int64_t row = a.first + (int64_t)blockIdx.x * kRows + mine;
    if (row >= a.rows) return;                                  // (whole wavefronts, and none of a workgroup with barriers)
    const T* const x = reinterpret_cast<const T*>(a.logits) + row * a.stride;
    // the segment [begin, end) of this part, its pieces from `head` on
    const int part = blockIdx.y, head = part * a.span - before_row(x), begin = max(head, 0), end = part + 1 < a.parts ? min(head + a.span, a.classes) : a.classes;

    const int label = a.logprob && a.parts == 1 ? a.labels[row] : -1;
    Stats st{-kUsual, 0.f, 0.f};
    Key least = 0;                                              // at least `top` of the segment's numbers are not below
    float seen = -__builtin_inff();
    const Edges edge = edges_of<N>(head, begin, end);
    // one of the pieces that are not whole, for the first two threads
    const int edge_at = t == 0 ? edge.before : t == 1 ? edge.behind : kNowhere;
    vec edge_piece = (vec)(T)-__builtin_inff();
    if (edge_at != kNowhere) edge_piece = Piece<T>::load_part(x, edge_at, begin, end, (T)-__builtin_inff());
    vec next[U];
    // (the four threads of a group are a quarter of a turn apart: the first pieces, which win where logits are equal, are in different groups)
    int j = edge.whole + N * (W > 1 ? t % 4 * (kLanes / 4) + t / 4 : t);
    auto request = [&]() {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = j + N * kLanes * u;
            if (i + N <= end) next[u] = Piece<T>::load(x + i);
            else next[u] = (T)-__builtin_inff();
        }
    };
    int in_use = 0, have = 0;                                   // have: numbers in sorted[mine][in_use]
    bool over = false;
    auto keep = [&](vec piece, int at) {
        const int place = atomicAdd(&kept[mine][in_use], 1);
        if (place < kPieces) {
            pieces[mine][place] = piece;
            places[mine][place] = at;
        }
    };
    // The piece that begins before the segment is listed in the first turn, the one that ends behind it after the last: it has the highest classes of all, so a threshold of
    // its own would hide equal logits of the turns between.
    auto keep_edge = [&]() {
        if (key_of(largest(widen<T>(edge_piece)), max(edge_at, begin)) >= least) keep(edge_piece, edge_at);
    };
    // What is listed without the classes below a closer bound: two numbers of `nth` lanes are not below the nth largest of the lanes' second numbers.  (Of 64 lanes' largest
    // numbers the 64th leaves most of a short row.  8,192 x 600, fp32, the 64 most probable classes: 150 us without it, 42 with it.)
    auto without_lower = [&](int n) {
        Key first = 0, second = 0;
        for (int i = t; i < n; i += 64) {
            const Key q = list[mine][i], lower = q < first ? q : first;
            second = lower > second ? lower : second;
            first = q > first ? q : first;
        }
        groups_of[mine][t] = second;
        together<1>();
        int place = 0;
#pragma unroll 8
        for (int i = 0; i < 64; ++i) place += groups_of[mine][i] > second;
        const unsigned long long found = __ballot(place == (a.top + 1) / 2 - 1);
        const Key closer = found ? of_lane(second, __builtin_ctzll(found)) : 0;
        // (to places that have been read)
        int left = 0;
        for (int i = 0; i < n; i += 64) {
            const Key q = i + t < n ? list[mine][i + t] : 0;
            const bool stays = i + t < n && q >= closer;
            const unsigned long long all = __ballot(stays);
            if (stays) list[mine][left + __popcll(all & ((1ull << t) - 1))] = q;
            left += __popcll(all);
        }
        together<1>();
        return left;
    };
    auto count_kept = [&]() {
        together<W>();
        const int held = kept[mine][in_use];
        over |= held > kPieces;
        for (int i = t; i < min(held, kPieces) * N; i += kLanes) {
            const int at = places[mine][i / N] + i % N;
            const Key q = key_of((float)pieces[mine][i / N][i % N], at);
            if (at >= begin && at < end && q >= least) {
                const int place = atomicAdd(&listed[mine][in_use], 1);
                if (place < kList) list[mine][place] = q;
            }
        }
        together<W>();
        int fresh = min(listed[mine][in_use], kList);
        over |= listed[mine][in_use] > kList;
        if constexpr (W == 1)
            if (fresh > 2 * kMaxTop) fresh = without_lower(fresh);
        const Key* const old = sorted[mine][in_use];
        for (int i = t / 4; i < have + fresh; i += kLanes / 4) {
            const Key q = i < have ? old[i] : list[mine][i - have];
            const int place = larger_than(q, old, have) + larger_than(q, list[mine], fresh);
            if (t % 4 == 0 && place < a.top) sorted[mine][in_use ^ 1][place] = q;
        }
        together<W>();
        if (t == 0) kept[mine][in_use] = listed[mine][in_use] = 0;
        in_use ^= 1;
        have = min(have + fresh, a.top);
        if (have == a.top) least = sorted[mine][in_use][have - 1];
    };
    // From each thread's largest number the top-th largest of groups of them, 0 if there are fewer.  (Numbers differ but for zeros, of threads without a class.)
    auto larger = [](Key p, Key q) { return p > q ? p : q; };
    auto bound = [&](Key k) -> Key {
        if constexpr (W > 1) {
            // 64 groups of four threads; where 64 would leave many to list 128 of two, each of which is counted by four threads too
            const bool few = a.top <= 32;
            k = larger(k, from_lane<kSwap1>(k));
            if (few) k = larger(k, from_lane<kSwap2>(k));
            const int of = few ? 4 : 2;
            if (t % of == 0) groups_of[0][t / of] = k;
            if (t == 0) threshold = 0;
            __syncthreads();
            for (int i = t / 4; i < kLanes / of; i += kLanes / 4) {
                k = groups_of[0][i];
                if (larger_than(k, groups_of[0], kLanes / of) == a.top - 1) threshold = k;
            }
            __syncthreads();
            return threshold;
        } else {
            groups_of[mine][t] = k;
            together<1>();
            int place = 0;
#pragma unroll 8
            for (int i = 0; i < 64; ++i) place += groups_of[mine][i] > k;
            const unsigned long long found = __ballot(place == a.top - 1);
            return found ? of_lane(k, __builtin_ctzll(found)) : 0;
        }
    };
    // turns of U pieces, the next ones on their way
    auto turn = [&](auto first) {
        vec now[U];
        float most[U];
        const int at = j;
#pragma unroll
        for (int u = 0; u < U; ++u) now[u] = next[u];
        j += kTurn;
        request();
#pragma unroll
        for (int u = 0; u < U; ++u) most[u] = largest(widen<T>(now[u]));
        if constexpr (TOP) {
            if constexpr (decltype(first)::value) {
                float best = most[0];
                int best_at = at;
#pragma unroll
                for (int u = 1; u < U; ++u)
                    if (most[u] > best) {
                        best = most[u];
                        best_at = at + N * kLanes * u;
                    }
                // (with the last class of the piece: not above what it stands for)
                Key k = at + N <= end ? key_of(best, best_at + N - 1) : 0;
                const bool early = t == 0 && edge_at != kNowhere;
                if (early) k = larger(k, key_of(largest(widen<T>(edge_piece)), min(edge_at + N, end) - 1));
                if (t == 0) kept[mine][0] = kept[mine][1] = listed[mine][0] = listed[mine][1] = 0;
                least = bound(k);
                // (where there is no top-th, all are listed)
                if (early) keep_edge();
            }
            const float value = least ? value_of(least) : -__builtin_inff();
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = at + N * kLanes * u;
                // (later turns have higher classes than the threshold's, which is never of the piece behind the whole ones: equal logits do not reach it)
                const bool reaches = decltype(first)::value ? key_of(most[u], i) >= least : most[u] > value;
                if (reaches && i + N <= end) keep(now[u], i);
            }
        }
        wide v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (widened again, so that 16 registers and not 32 are held meanwhile)
            typedef int words __attribute__((ext_vector_type(4)));
            words raw = __builtin_bit_cast(words, now[u]);
            if constexpr (TOP) asm("" : "+v"(raw));
            v[u] = widen<T>(__builtin_bit_cast(vec, raw));
        }
        take<U, ENT>(st, v, most);
#pragma unroll
        for (int u = 0; u < U; ++u) seen = fmaxf(seen, most[u]);
    };
    request();
    const float at_label = label >= 0 && label < a.classes ? (float)x[label] : 0.f;
    turn(std::true_type());
    const int turns = (end - edge.whole + kTurn - 1) / kTurn;   // (of the row: some threads have nothing left in the last one)
    for (int n = 1; n < turns; ++n) {
        turn(std::false_type());
        // (before 64 / top turns fewer than 128 pieces are expected)
        if constexpr (TOP)
            if (!(n & (n + 1)) && a.top * (n + 1) >= 64 && n + 1 < turns) count_kept();
    }
    if (edge_at != kNowhere) {
        const wide v = widen<T>(edge_piece);
        const float most = largest(v);
        take<1, ENT>(st, &v, &most);
        seen = fmaxf(seen, most);
        if constexpr (TOP)
            if (t == 1) keep_edge();
    }

    auto merged = [&](Stats own, auto of) {
        constexpr Refers OF = decltype(of)::value;
        own = wave_merge<OF>(own);
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
                refer_to<OF>(o, m);
                all.s += o.s;
                all.w += o.w;
            }
            return all;
        } else {
            together<1>();
            return own;
        }
    };
    constexpr std::integral_constant<Refers, kRounded> rounded;
    constexpr std::integral_constant<Refers, kItself> itself;
    st = merged(st, rounded);
    if (!(st.m > -kUsual && st.m < kUsual)) {
        if constexpr (W > 1) __syncthreads();                   // (`parts` has been read)
        const bool none = st.s == 0.f && merged(Stats{seen, 0.f, 0.f}, itself).m == -__builtin_inff();
        if constexpr (W > 1) __syncthreads();
        st = Stats{kLowest, 0.f, 0.f};
        if (!none) {
            for (int i = head + N * t; i < end; i += N * kLanes) take_unusual(st, widen<T>(logits_at(x, i, begin, end)));
            st = merged(st, itself);
        }
    }
    const Row r = finish(st);
    if (t == 0) {
        if (a.parts > 1) {
            float* const to = a.part_stats + (row * a.parts + part) * 3;
            to[0] = st.m;
            to[1] = st.s;
            to[2] = st.w;
        } else write_row(a, row, label, at_label, r);
    }
    if constexpr (TOP) {
        for (bool again = false;; again = true) {
            count_kept();
            if (!over || again) break;
            // The bound again, of all that the threads have read, and everything that reaches it.
            over = false;
            have = 0;
            Key k = 0;
            for (int i = head + N * (W > 1 ? t % 4 * (kLanes / 4) + t / 4 : t); i < end; i += N * kLanes)
                k = larger(k, key_of(largest(widen<T>(logits_at(x, i, begin, end))), min(i + N, end) - 1));
            least = larger(least, bound(k));
            for (int i = head + N * t; i < end; i += N * kLanes) {
                const vec v = logits_at(x, i, begin, end);
                if (key_of(largest(widen<T>(v)), max(i, begin)) >= least) keep(v, i);
            }
        }
        if (st.s == st.s && !over) {
            if (t < a.top) write_top(a, row, part, t, t < have ? sorted[mine][in_use][t] : 0, r);          // (a part may have fewer than `top` classes)
        } else {
            Key before = ~(Key)0;                               // above every class's number
            for (int place = 0; place < a.top; ++place) {
                Key k = 0;
                for (int i = head + N * t; i < end; i += N * kLanes) {
                    const wide v = widen<T>(logits_at(x, i, begin, end));
#pragma unroll
                    for (int c = 0; c < N; ++c) {
                        const Key q = key_of(v[c], i + c);
                        if (i + c >= begin && i + c < end && q < before && q > k) k = q;
                    }
                }
                k = wave_max(k);
                if constexpr (W > 1) {
                    __syncthreads();
                    if ((threadIdx.x & 63) == 0) groups_of[0][threadIdx.x >> 6] = k;
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < W; ++i) k = groups_of[0][i] > k ? groups_of[0][i] : k;
                }
                if (t == 0) write_top(a, row, part, place, k, r);
                before = k;
            }
        }
    }
}

// A row from its parts (at most 64): all that it reads is asked for first.  Each part's classes are in falling order.  The top-th of a part is not above the top-th of the
// row, nor is the h-th largest of the parts' n-th ones, where h is half of the parts and h n >= top (half of them may have nothing but -infinity).
template <typename T> __global__ void __launch_bounds__(256) logprobs_join_kernel(LogArgs a)
{
    extern __shared__ Key list[];
    __shared__ Key bounds[64], at_half;
    __shared__ int count;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, keys_of_row = a.parts * a.top;
    const float* const from = a.part_stats + row * a.parts * 3;
    const Key* const keys = a.part_keys + row * keys_of_row;
    const int label = a.logprob ? a.labels[row] : -1;
    Key mine = (int)threadIdx.x < keys_of_row ? keys[threadIdx.x] : 0;
    Stats st{kLowest, 0.f, 0.f};                                // (of a size that no part with classes has: adds nothing)
    if (lane < a.parts) st = Stats{from[3 * lane], from[3 * lane + 1], from[3 * lane + 2]};
    const int half = a.parts / 2, nth = (a.top + half - 1) / half;
    Key bound = 0, last = 0;
    if (a.top && lane < a.parts) {
        bound = keys[lane * a.top + nth - 1];
        last = keys[lane * a.top + a.top - 1];
    }
    const T* const x = reinterpret_cast<const T*>(a.logits) + row * a.stride;
    const float at_label = label >= 0 && label < a.classes ? (float)x[label] : 0.f;
    st = wave_merge<kEither>(st);
    const Row r = finish(st);
    if (threadIdx.x == 0) {
        write_row(a, row, label, at_label, r);
        count = 0;
        at_half = 0;
    }
    if (!a.top) return;
    if (threadIdx.x < 64) bounds[lane] = bound;
    __syncthreads();
    // (parts' numbers differ but for zeros)
    const Key counted = bounds[threadIdx.x / 4];
    if (counted && larger_than(counted, bounds, 64) == half - 1) at_half = counted;
    Key least = wave_max(last);
    __syncthreads();
    least = at_half > least ? at_half : least;
    for (int i = threadIdx.x; i < keys_of_row; i += 256) {
        if (i >= 256) mine = keys[i];
        if (mine && mine >= least) list[atomicAdd(&count, 1)] = mine;
    }
    __syncthreads();
    for (int i = threadIdx.x / 4; i < count; i += 64) {
        const Key q = list[i];
        const int place = larger_than(q, list, count);
        if (threadIdx.x % 4 == 0 && place < a.top) {
            a.top_classes[row * a.top + place] = class_of(q);
            a.top_logprobs[row * a.top + place] = logprob_of(r, value_of(q));
        }
    }
}

// dlogits: W wavefronts have a row (W = 1), or a chunk of one.
constexpr int kTurns = 4;                        // pieces of a thread

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
template <bool DH> __device__ __forceinline__ float logit_gradient(float x, const Slope& g)
{
    const float d = g.usual ? __builtin_fmaf(x, kLog2E, -g.shift) : __builtin_fmaf(x - g.m, kLog2E, -g.shift);
    const float p = __builtin_amdgcn_exp2f(d);
    return DH ? p * __builtin_fmaf(fmaxf(d, kFar), g.of_entropy, g.both) : p * g.both;
}

template <typename T, int W, bool DH> __global__ void __launch_bounds__(256) logprobs_backward_kernel(LogArgs a)
{
    constexpr int kLanes = 64 * W, kRows = 4 / W, N = Piece<T>::N, U = kTurns;
    typedef typename Piece<T>::vec vec;
    typedef typename Piece<T>::wide wide;
    const int t = threadIdx.x % kLanes;
    const int64_t items = W == 1 ? a.rows : a.rows * a.parts;
    for (int64_t item = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes; item < items; item += (int64_t)gridDim.x * kRows) {
        int64_t row = item;
        int part = 0;
        if constexpr (W > 1) {
            row = items >> 31 ? item / a.parts : (int64_t)((unsigned)item / (unsigned)a.parts);
            part = (int)(item - row * a.parts);
        }
        const T* const x = reinterpret_cast<const T*>(a.logits) + row * a.stride;
        T* const out = reinterpret_cast<T*>(a.dlogits) + row * a.dstride;
        const int head = part * a.span - before_row(x), begin = max(head, 0), end = W > 1 ? min(head + a.span, a.classes) : a.classes;
        const float m = a.kept[3 * row], entropy = a.kept[3 * row + 2], dh = DH ? a.dentropy[row] : 0.f;
        const int label = a.dlogprob ? a.labels[row] : -1;
        const Slope g = slope_of(m, a.kept[3 * row + 1], entropy, label < 0 ? 0.f : label >= a.classes ? __builtin_nanf("") : a.dlogprob[row], dh, label);
        const bool empty = m == -__builtin_inff() && g.label < a.classes;
        auto gradients = [&](vec v, int i) {
            wide o = widen<T>(v);
#pragma unroll
            for (int k = 0; k < N; ++k) o[k] = logit_gradient<DH>(o[k], g);
            if (g.label >= 0 && (unsigned)(g.label - i) < (unsigned)N) {
#pragma unroll
                for (int k = 0; k < N; ++k) o[k] += k == g.label - i ? g.dl : 0.f;
            }
            if (empty) o = 0.f;
            return narrow<T>(o);
        };
        const Edges edge = edges_of<N>(head, begin, end);
        for (int j = edge.whole + N * t; j + N <= end; j += N * kLanes * U) {
            vec v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = j + N * kLanes * u;
                if (i + N <= end) v[u] = Piece<T>::load(x + i);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = j + N * kLanes * u;
                if (i + N <= end) Piece<T>::store(out + i, gradients(v[u], i));
            }
        }
        // the elements of the pieces that are not whole, one for a thread
        if (t < 2 * N) {
            const int at = t < N ? edge.before : edge.behind, i = at == kNowhere ? end : at + t % N;
            if (i >= begin && i < end) {
                const float o = logit_gradient<DH>((float)x[i], g) + (i == g.label ? g.dl : 0.f);
                out[i] = (T)(empty ? 0.f : o);
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

constexpr int kWide = 1024;                      // a part of a row has this many pieces or more: a turn

// Parts of a row, where few rows would leave compute units idle.
int parts_of(const bmgd_logprobs_config& c, int64_t rows)
{
    const int64_t parts = std::min<int64_t>(std::min<int64_t>(512 / std::max<int64_t>(rows, 1), kMaxParts), c.classes * (int64_t)size_of(c.dtype) / 16 / kWide);
    return (int)std::max<int64_t>(parts, 1);
}
// classes of a part: whole pieces of eight
int span_of(int64_t classes, int parts) { return (int)((classes + 7 + parts - 1) / parts + 7) / 8 * 8; }

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
    const int parts = parts_of(*cfg, rows);
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
    a.parts = parts_of(*cfg, rows);
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
        // A wavefront for each row, if the rows are many or short.  Measured, us, with it and with four for a row (16 bits, with entropy, sets of tensors in turn that are
        // larger together than the caches; no classes, five):
        //      8,192 x 1,000: 9 and 24, 15 and 42;  8,192 x 4,000: 17 and 29, 24 and 48;  4,097 x 10,001: 22 and 30, 30 and 39 (so that with classes too a wavefront would do for many rows
        //      of this length);  8,192 x 16,000: 56 and 53;  8,192 x 32,000: 101 and 94, eight: 130 and 119;  1,000 x 10,001, five: 16 and 13;  100 x 4,000, five: 7.9 and 6.4.
        // Of 64 groups the 64th largest leaves 300 classes to list, now and then more than the list holds.  So more than 16 only where all of a row's pieces are kept, and
        // with few rows, each of which then takes as long as the call, more than 32:
        //      8,192 x 700, the 64 most probable: 45 and 170, 20: 19 and 48;  8,192 x 1,300, 64: 51 and 75;  100 x 1,000, 64: 17 and 35, 32: 8.5 and 6.7.
        const int64_t pieces = (int64_t)a.span * (int64_t)sizeof(T) / 16;
        const bool many = rows >= 4 * compute_units(), wave = pieces <= 128 || (many && pieces <= (a.top ? 512 : 2048));
        const bool listed = a.top <= 16 || (pieces + 2 <= pieces_kept(1) && (many || a.top > 32));
        auto shaped = [&](auto top, auto ent) {
            if (wave && listed) launch(std::integral_constant<int, 1>(), top, ent);
            else launch(std::integral_constant<int, 4>(), top, ent);
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
    // parts of up to four pieces for each of 256 threads, alike but for the last one
    const int piece = 256 * (int)(16 / size_of(cfg->dtype)), pieces = (int)((cfg->classes + 7 + piece - 1) / piece);
    a.parts = (pieces + kTurns - 1) / kTurns;
    a.span = (pieces + a.parts - 1) / a.parts * piece;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    with_type(cfg->dtype, [&](auto type) {
        typedef decltype(type) T;
        const int64_t most = int64_t(1) << 20;
        auto launch = [&](auto dh) {
            constexpr bool DH = decltype(dh)::value;
            if (cfg->classes <= 2048) hipLaunchKernelGGL((logprobs_backward_kernel<T, 1, DH>), dim3((unsigned)std::min((rows + 3) / 4, most)), dim3(256), 0, s, a);
            else hipLaunchKernelGGL((logprobs_backward_kernel<T, 4, DH>), dim3((unsigned)std::min(rows * a.parts, most)), dim3(256), 0, s, a);
        };
        if (a.dentropy) launch(std::true_type());
        else launch(std::false_type());
    });
    return q.launched();
}

}  // extern "C"
