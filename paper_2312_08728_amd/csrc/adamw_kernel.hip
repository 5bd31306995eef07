// AdamW (decoupled weight decay) over many tensors in few launches, moments in 32 bits or in 8.
//
//      m <- b1 m + (1 - b1) g;  s <- b2 s + (1 - b2) g^2
//      theta <- theta (1 - lr wd) - lr (m / (1 - b1^k)) / (sqrt(s / (1 - b2^k)) + eps)
//
// Every element is read and written once.  Per element 8 bytes of theta, 2 or 4 of gradient, 2 of the 16-bit copy if there is one, and 16 of
// moments in 32 bits, 4 + 1/16 in 8: the memory bounds it, the sums of the moments stay in fp32 registers.
//
// Moments in 8 bits: 256 neighbouring elements (the last block of a tensor may be shorter) share a scale, the largest of their moments in fp32.
// m = a sgn(c) (c / 127)^2 and s = b (c / 255)^4, the code c the nearest on that scale: near the largest moment codes lie 1.6 % apart
// (in sqrt(s), which the update divides by, 0.8 %), and values down to 1.5e-5 of the largest m (of the largest sqrt(s)) keep a code.
// An s that is not zero keeps a code of at least 1, so that no update divides by eps alone.  theta is updated from the moments before they
// are rounded to codes.  A block whose largest moment is below the smallest normal fp32 number is held as zeros; a block in which a moment is not finite
// gets that as its scale and codes of zero, that is, stands for NaN in all its elements from then on: nothing hides it.
// A wavefront holds a block, four elements a lane; the largest is found with lane exchanges.
//
// Measured: 20 M elements in 160 tensors, bf16 gradients and copies, moments in 32 bits: 114 us in two launches, 4.9 TB/s; 100.7 M elements in 8 bits 289 us, 5.6
// TB/s (a copy of 1 GiB reaches 5.1, reads and writes together).  In 8 bits the instructions count as well: with exact roots and quotients throughout, 150 vector
// instructions an element, it took 387 us.  A workgroup takes 1,024 elements; with 4,096, loads of all four thousands first, it took 2 to 6 % longer.
#include "../../include/bmgd.h"
#include "bmgd_internal.h"

#include <float.h>
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>

using namespace bmgd;

namespace {

constexpr int kThreads = 256, kBlock = 256;                  // threads of a workgroup; elements that share a scale
constexpr int kPiece = 4 * kThreads;                          // elements that a workgroup takes at a time
constexpr int kMaxTensors = 108;                              // of a launch: they travel as kernel arguments

static_assert(sizeof(bmgd_adamw_tensor) == 64, "");

struct Rates {
    float b1, c1, b2, c2;           // beta1, 1 - beta1, beta2, 1 - beta2
    float m_fix, s_fix;             // 1 / (1 - beta1^k), 1 / (1 - beta2^k)
    float decay, lr, eps, grad_scale;                         // lr * weight_decay, ...
};

// The tensors of a launch.  Addresses are told as distances from the lowest of their kind, in elements (codes: in words of four), so that a tensor takes 36 bytes of
// the kernel arguments' 4 KB; tensors too far apart for that go to different launches.
enum { kTheta, kGrad, kCopy, kM, kS, kMScale, kSScale, kKinds };
struct Table {
    char* base[kKinds];
    unsigned far[kMaxTensors][kKinds];
    unsigned n[kMaxTensors];
    unsigned first[kMaxTensors];                              // first workgroup of each tensor
    int count;
};

constexpr unsigned kNone = ~0u;                               // no copy of this tensor

struct Args {
    Table t;
    int has_copy, copy_dtype;
    Rates r;
};

struct MomentArgs {                                           // kTheta: m's values, kGrad: s's
    Table t;
};
static_assert(sizeof(Args) <= 4096 && sizeof(MomentArgs) <= 4096, "kernel arguments");

typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef short short4u __attribute__((ext_vector_type(4), aligned(2)));

// Which tensor workgroup `id` works on.
__device__ __forceinline__ int tensor_of(const Table& t, unsigned id)
{
    const int lane = threadIdx.x & 63;
    int n = __popcll(__ballot(lane < t.count && t.first[min(lane, kMaxTensors - 1)] <= id));
    if (t.count > 64) n += __popcll(__ballot(64 + lane < t.count && t.first[min(64 + lane, kMaxTensors - 1)] <= id));
    return __builtin_amdgcn_readfirstlane(n - 1);
}
static_assert(kMaxTensors <= 128, "");

template <typename T> __device__ __forceinline__ float4v load_grad(const void* p, int64_t at, int64_t left);

template <> __device__ __forceinline__ float4v load_grad<float>(const void* p, int64_t at, int64_t left)
{
    const float* from = static_cast<const float*>(p) + at;
    if (left >= 4) return *reinterpret_cast<const float4u*>(from);
    float4v v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) v[i] = from[i];
    return v;
}

template <typename T> __device__ __forceinline__ float4v load_half(const void* p, int64_t at, int64_t left)
{
    const short* from = static_cast<const short*>(p) + at;
    short4u b = {0, 0, 0, 0};
    if (left >= 4) b = *reinterpret_cast<const short4u*>(from);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) b[i] = from[i];
    }
    float4v v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)__builtin_bit_cast(T, (short)b[i]);
    return v;
}
template <> __device__ __forceinline__ float4v load_grad<__bf16>(const void* p, int64_t at, int64_t left) { return load_half<__bf16>(p, at, left); }
template <> __device__ __forceinline__ float4v load_grad<_Float16>(const void* p, int64_t at, int64_t left) { return load_half<_Float16>(p, at, left); }

__device__ __forceinline__ void store_floats(float* to, int64_t left, float4v v)
{
    if (left >= 4) *reinterpret_cast<float4u*>(to) = v;
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) to[i] = v[i];
    }
}

__device__ __forceinline__ void store_copy(void* copy, int dtype, int64_t at, int64_t left, float4v v)
{
    short4u b;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        b[i] = dtype == BMGD_BF16 ? __builtin_bit_cast(short, (__bf16)v[i]) : __builtin_bit_cast(short, (_Float16)v[i]);
    short* to = static_cast<short*>(copy) + at;
    if (left >= 4) *reinterpret_cast<short4u*>(to) = b;
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) to[i] = b[i];
    }
}

// The largest of a wavefront's words, in all its lanes.
template <int CTRL> __device__ __forceinline__ unsigned dpp_max(unsigned v)
{
    return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ unsigned wave_max(unsigned v)
{
    v = dpp_max<0xB1>(v);       // quad_perm [1,0,3,2]
    v = dpp_max<0x4E>(v);       // quad_perm [2,3,0,1]
    v = dpp_max<0x141>(v);      // row_half_mirror
    v = dpp_max<0x140>(v);      // row_mirror
    // the four rows of 16 lanes
    const unsigned a = max((unsigned)__builtin_amdgcn_readlane((int)v, 0), (unsigned)__builtin_amdgcn_readlane((int)v, 16));
    const unsigned b = max((unsigned)__builtin_amdgcn_readlane((int)v, 32), (unsigned)__builtin_amdgcn_readlane((int)v, 48));
    return max(a, b);
}

// The scale of a block whose largest value has these bits (ordered as whole numbers: NaN above infinity above all others), and the factor that takes a
// moment to its share of it.
__device__ __forceinline__ float scale_of(unsigned bits, float& inv)
{
    const float top = __uint_as_float(bits);
    const bool finite = bits < 0x7F800000u, normal = bits >= 0x00800000u;
    inv = finite && normal ? 1.f / top : 0.f;
    return normal ? top : 0.f;
}

__device__ __forceinline__ float m_value(int code, float scale)
{
#pragma clang fp contract(off)
    const float t = (float)code * (1.f / 127.f);
    return scale * (t * fabsf(t));
}
__device__ __forceinline__ float s_value(unsigned code, float scale)
{
#pragma clang fp contract(off)
    float t = (float)code * (1.f / 255.f);
    t = t * t;
    return scale * (t * t);
}

// The square root to 2^-23 of its value, also of what the hardware's takes for zero.
__device__ __forceinline__ float quick_sqrt(float x)
{
    const bool small = x < 0x1p-96f;
    return __builtin_amdgcn_sqrtf(small ? x * 0x1p64f : x) * (small ? 0x1p-32f : 1.f);
}

// One element.  Products and sums are rounded one by one, so that the codes do not depend on what the compiler joins.  QUICK: the hardware's square root and
// reciprocal (with moments in 8 bits the instructions count, and what they add, 2^-22 of the step, is far below what the codes do; eps is a normal number there).
// Decay and step are added first and taken off theta with one rounding: a factor 1 - lr wd, rounded to 32 bits, is off by up to 2^-25 the same way in every step and
// element, a third of a decay of 1e-7.  (An infinite theta stays what it is: no infinity is taken off it.)
template <bool QUICK> __device__ __forceinline__ float update(const Rates& r, float theta, float g, float& m, float& s)
{
#pragma clang fp contract(off)
    g = g * r.grad_scale;
    m = r.b1 * m + r.c1 * g;
    s = r.b2 * s + r.c2 * (g * g);
    float way;
    if constexpr (QUICK) way = m * r.m_fix * __builtin_amdgcn_rcpf(quick_sqrt(s * r.s_fix) + r.eps);
    else way = m * r.m_fix / (sqrtf(s * r.s_fix) + r.eps);
    return theta - (r.decay * __builtin_amdgcn_fmed3f(theta, -FLT_MAX, FLT_MAX) + r.lr * way);
}

template <typename G, bool EIGHT>
__global__ void __launch_bounds__(kThreads) adamw_kernel(Args a)
{
    const int which = tensor_of(a.t, blockIdx.x);
    const unsigned* const far = a.t.far[which];
    float* const theta_at = reinterpret_cast<float*>(a.t.base[kTheta]) + far[kTheta];
    const char* const grad_at = a.t.base[kGrad] + sizeof(G) * (size_t)far[kGrad];
    char* const copy_at = a.t.base[kCopy] + 2 * (size_t)far[kCopy];
    char* const m_at = a.t.base[kM] + 4 * (size_t)far[kM];
    char* const s_at = a.t.base[kS] + 4 * (size_t)far[kS];
    const bool copies = a.has_copy && far[kCopy] != kNone;
    const int64_t at = (int64_t)(blockIdx.x - a.t.first[which]) * kPiece + 4 * threadIdx.x, left = (int64_t)a.t.n[which] - at;
    const float4v g = load_grad<G>(grad_at, at, left);
    float4v theta = load_grad<float>(theta_at, at, left);
    if constexpr (!EIGHT) {
        if (left <= 0) return;
        float4v m = load_grad<float>(m_at, at, left), s = load_grad<float>(s_at, at, left);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mi = m[i], si = s[i];
            theta[i] = update<false>(a.r, theta[i], g[i], mi, si);
            m[i] = mi;
            s[i] = si;
        }
        store_floats(theta_at + at, left, theta);
        store_floats(reinterpret_cast<float*>(m_at) + at, left, m);
        store_floats(reinterpret_cast<float*>(s_at) + at, left, s);
        if (copies) store_copy(copy_at, a.copy_dtype, at, left, theta);
    } else {
#pragma clang fp contract(off)
        // (a wavefront whose block lies behind the tensor's end leaves as a whole)
        if (left + 4 * (int64_t)(threadIdx.x & 63) <= 0) return;
        float* const ma_at = reinterpret_cast<float*>(a.t.base[kMScale]) + far[kMScale] + at / kBlock;
        float* const sa_at = reinterpret_cast<float*>(a.t.base[kSScale]) + far[kSScale] + at / kBlock;
        unsigned mc = 0u, sc = 0u;
        if (left >= 4) {
            mc = *reinterpret_cast<const unsigned*>(m_at + at);
            sc = *reinterpret_cast<const unsigned*>(s_at + at);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < left) {
                    mc |= (unsigned)(unsigned char)m_at[at + i] << (8 * i);
                    sc |= (unsigned)(unsigned char)s_at[at + i] << (8 * i);
                }
        }
        const float ma = *ma_at, sa = *sa_at;
        float m[4], s[4];
        unsigned m_top = 0u, s_top = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = m_value((int)(signed char)(mc >> (8 * i)), ma);
            s[i] = s_value(sc >> (8 * i) & 255u, sa);
            theta[i] = update<true>(a.r, theta[i], g[i], m[i], s[i]);
            if (i < left) {
                m_top = max(m_top, __float_as_uint(m[i]) & 0x7FFFFFFFu);
                s_top = max(s_top, __float_as_uint(s[i]) & 0x7FFFFFFFu);
            }
        }
        if (left > 0) {
            store_floats(theta_at + at, left, theta);
            if (copies) store_copy(copy_at, a.copy_dtype, at, left, theta);
        }
        float m_inv, s_inv;
        const float m_scale = scale_of(wave_max(m_top), m_inv), s_scale = scale_of(wave_max(s_top), s_inv);
        // Where the codes lie, with the hardware's square root (2^-23); the next to a middle between two codes is taken again with the exact one, so that
        // codes are those of exact roots.  255 2^-22 is the most that the two can be apart.
        float mr[4], sr[4], middle = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = fabsf(m[i]) * m_inv, y = s[i] * s_inv;
            const float mf = 127.f * __builtin_amdgcn_sqrtf(x), sf = 255.f * __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(y));
            mr[i] = rintf(mf);
            sr[i] = rintf(sf);
            middle = fmaxf(middle, fmaxf(fabsf(mf - mr[i]), fabsf(sf - sr[i])));
        }
        if (middle > 0.4999f) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                mr[i] = rintf(127.f * sqrtf(fabsf(m[i]) * m_inv));
                sr[i] = rintf(255.f * sqrtf(sqrtf(s[i] * s_inv)));
            }
        }
        unsigned mb = 0u, sb = 0u;
        if (m_inv > 0.f) {                                     // (otherwise a scale that is zero or not finite: all codes are zero)
#pragma unroll
            for (int i = 0; i < 4; ++i) mb |= ((unsigned)(int)copysignf(mr[i], m[i]) & 255u) << (8 * i);
        }
        if (s_inv > 0.f) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sb |= (unsigned)(s[i] > 0.f ? fmaxf(sr[i], 1.f) : 0.f) << (8 * i);
        }
        if (left >= 4) {
            *reinterpret_cast<unsigned*>(m_at + at) = mb;
            *reinterpret_cast<unsigned*>(s_at + at) = sb;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < left) {
                    m_at[at + i] = (char)(mb >> (8 * i));
                    s_at[at + i] = (char)(sb >> (8 * i));
                }
        }
        if ((threadIdx.x & 63) == 0) {
            *ma_at = m_scale;
            *sa_at = s_scale;
        }
    }
}

// What codes and scales stand for, in fp32: the quotients rounded once, so that a value is off by no more than 8 2^-24 (m: 4).
__device__ __forceinline__ float m_exported(int code, float scale)
{
    const float t = (float)code / 127.f;
    return scale * (t * fabsf(t));
}
__device__ __forceinline__ float s_exported(unsigned code, float scale)
{
    float t = (float)code / 255.f;
    t = t * t;
    return scale * (t * t);
}

__global__ void __launch_bounds__(kThreads) adamw_moments_kernel(MomentArgs a)
{
    const int which = tensor_of(a.t, blockIdx.x);
    const unsigned* const far = a.t.far[which];
    struct { const signed char* m; const unsigned char* s; const float* m_scale; const float* s_scale; float* m_out; float* s_out; int64_t n; } t;
    t.m = reinterpret_cast<const signed char*>(a.t.base[kM] + 4 * (size_t)far[kM]);
    t.s = reinterpret_cast<const unsigned char*>(a.t.base[kS] + 4 * (size_t)far[kS]);
    t.m_scale = reinterpret_cast<const float*>(a.t.base[kMScale]) + far[kMScale];
    t.s_scale = reinterpret_cast<const float*>(a.t.base[kSScale]) + far[kSScale];
    t.m_out = reinterpret_cast<float*>(a.t.base[kTheta]) + far[kTheta];
    t.s_out = reinterpret_cast<float*>(a.t.base[kGrad]) + far[kGrad];
    t.n = a.t.n[which];
    const int64_t at = (int64_t)(blockIdx.x - a.t.first[which]) * kPiece + 4 * threadIdx.x, left = t.n - at;
    if (left <= 0) return;
    const float ma = t.m_scale[at / kBlock], sa = t.s_scale[at / kBlock];
    float4v m = {0.f, 0.f, 0.f, 0.f}, s = {0.f, 0.f, 0.f, 0.f};
    if (left >= 4) {
        const unsigned mc = *reinterpret_cast<const unsigned*>(t.m + at), sc = *reinterpret_cast<const unsigned*>(t.s + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = m_exported((int)(signed char)(mc >> (8 * i)), ma);
            s[i] = s_exported(sc >> (8 * i) & 255u, sa);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) {
                m[i] = m_exported(t.m[at + i], ma);
                s[i] = s_exported(t.s[at + i], sa);
            }
    }
    store_floats(t.m_out + at, left, m);
    store_floats(t.s_out + at, left, s);
}

int fail(int code, const char* what)
{
    set_create_error(what);
    return code;
}

int hip_fail(hipError_t e, const char* what)
{
    char buf[256];
    snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
    (void)hipGetLastError();
    return fail(BMGD_EHIP, buf);
}

int tensor_fail(const char* call, int64_t i, const char* why)
{
    char buf[256];
    snprintf(buf, sizeof buf, "%s: tensor %lld: %s", call, (long long)i, why);
    return fail(BMGD_EINVAL, buf);
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

constexpr int64_t kMaxElements = int64_t(1) << 38;
constexpr int64_t kMaxWorkgroups = int64_t(1) << 30;

template <typename G> hipError_t launch_step(const Args& a, unsigned groups, bool eight, hipStream_t s)
{
    if (eight) hipLaunchKernelGGL((adamw_kernel<G, true>), dim3(groups), dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<G, false>), dim3(groups), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

// Collects tensors into tables of one launch each.
struct Collector {
    Table t;
    uintptr_t lo[kKinds], hi[kKinds];       // of the addresses of each kind that the table has
    uintptr_t at[kMaxTensors][kKinds];
    int64_t groups;

    void clear()
    {
        t.count = 0;
        groups = 0;
        for (int k = 0; k < kKinds; ++k) lo[k] = hi[k] = 0;
    }
    // False if the table has no place for it: close the table first.  p[k] = 0: none of this kind.
    bool add(const uintptr_t* p, const int* size, int64_t n, int64_t need)
    {
        if (t.count == kMaxTensors || (t.count > 0 && groups + need > kMaxWorkgroups)) return false;
        uintptr_t l[kKinds], h[kKinds];
        for (int k = 0; k < kKinds; ++k) {
            l[k] = lo[k];
            h[k] = hi[k];
            if (!p[k]) continue;
            if (!l[k] || p[k] < l[k]) l[k] = p[k];
            if (p[k] > h[k]) h[k] = p[k];
            // (distances are whole elements: an address is a multiple of its element's size)
            if ((h[k] - l[k]) / size[k] >= kNone) return false;
        }
        for (int k = 0; k < kKinds; ++k) {
            lo[k] = l[k];
            hi[k] = h[k];
            at[t.count][k] = p[k];
        }
        t.n[t.count] = (unsigned)n;
        t.first[t.count++] = (unsigned)groups;
        groups += need;
        return true;
    }
    const Table& close(const int* size)
    {
        for (int k = 0; k < kKinds; ++k) t.base[k] = reinterpret_cast<char*>(lo[k]);
        for (int i = 0; i < t.count; ++i)
            for (int k = 0; k < kKinds; ++k) t.far[i][k] = at[i][k] ? (unsigned)((at[i][k] - lo[k]) / size[k]) : kNone;
        return t;
    }
};

constexpr int64_t kEntry = int64_t(1) << 31;                  // elements of one entry of a table: longer tensors take several

// f(entry's addresses, elements) for the pieces of a tensor; advance[k]: bytes that 256 elements take
template <typename F> int entries_of(const uintptr_t* p, const int* advance, int64_t n, F f)
{
    for (int64_t from = 0; from < n; from += kEntry) {
        uintptr_t q[kKinds];
        for (int k = 0; k < kKinds; ++k) q[k] = p[k] ? p[k] + (uintptr_t)(from / kBlock) * advance[k] : 0;
        const int rc = f(q, n - from < kEntry ? n - from : kEntry);
        if (rc != BMGD_OK) return rc;
    }
    return BMGD_OK;
}

uintptr_t address(const void* p) { return reinterpret_cast<uintptr_t>(p); }

}  // namespace

#define BMGD_API __attribute__((visibility("default")))

extern "C" {

BMGD_API void bmgd_adamw_default_config(bmgd_adamw_config* cfg)
{
    if (!cfg) return;
    memset(cfg, 0, sizeof *cfg);
    cfg->lr = 1e-3;
    cfg->beta1 = 0.9;
    cfg->beta2 = 0.999;
    cfg->eps = 1e-8;
    cfg->weight_decay = 0.01;
    cfg->grad_scale = 1.0;
    cfg->grad_dtype = BMGD_F32;
    cfg->copy_dtype = BMGD_BF16;
    cfg->state_bits = 32;
}

BMGD_API int bmgd_adamw_step(const bmgd_adamw_config* cfg, const bmgd_adamw_tensor* tensors, int64_t count, int64_t step, void* stream)
{
    static const char call[] = "bmgd_adamw_step";
    if (!cfg) return fail(BMGD_EINVAL, "bmgd_adamw_step: cfg must not be NULL");
    if (count < 0 || (count > 0 && !tensors)) return fail(BMGD_EINVAL, "bmgd_adamw_step: tensors must hold count >= 0 entries");
    if (!(cfg->lr >= 0.0) || !isfinite(cfg->lr)) return fail(BMGD_EINVAL, "bmgd_adamw_step: lr must be finite and >= 0");
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0))
        return fail(BMGD_EINVAL, "bmgd_adamw_step: beta1 and beta2 must be in [0, 1)");
    if (!(cfg->eps >= 0.0) || !isfinite(cfg->eps)) return fail(BMGD_EINVAL, "bmgd_adamw_step: eps must be finite and >= 0");
    if (!(cfg->weight_decay >= 0.0) || !isfinite(cfg->weight_decay)) return fail(BMGD_EINVAL, "bmgd_adamw_step: weight_decay must be finite and >= 0");
    if (!isfinite(cfg->grad_scale)) return fail(BMGD_EINVAL, "bmgd_adamw_step: grad_scale must be finite");
    if (!isfinite((float)cfg->lr) || !isfinite((float)cfg->eps) || !isfinite((float)cfg->grad_scale) || !isfinite((float)(cfg->lr * cfg->weight_decay)))
        return fail(BMGD_EINVAL, "bmgd_adamw_step: lr, eps, grad_scale and lr * weight_decay must be finite in fp32");
    if (cfg->grad_dtype != BMGD_F32 && cfg->grad_dtype != BMGD_BF16 && cfg->grad_dtype != BMGD_F16)
        return fail(BMGD_EINVAL, "bmgd_adamw_step: unknown grad_dtype");
    if (cfg->copy_dtype != BMGD_BF16 && cfg->copy_dtype != BMGD_F16) return fail(BMGD_EINVAL, "bmgd_adamw_step: copy_dtype must be BMGD_BF16 or BMGD_F16");
    if (cfg->state_bits != 32 && cfg->state_bits != 8) return fail(BMGD_EINVAL, "bmgd_adamw_step: state_bits must be 32 or 8");
    const bool eight = cfg->state_bits == 8;
    if (eight && !((float)cfg->eps >= 0x1p-126f)) return fail(BMGD_EINVAL, "bmgd_adamw_step: moments in 8 bits need eps >= 2^-126");
    if (step < 1 || step > (int64_t(1) << 53)) return fail(BMGD_EINVAL, "bmgd_adamw_step: step must be in [1, 2^53]");
    for (int64_t i = 0; i < count; ++i) {
        const bmgd_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n > kMaxElements) return tensor_fail(call, i, "n must be in [0, 2^38]");
        if (t.n == 0) continue;
        if (!t.theta || !t.grad || !t.m || !t.s) return tensor_fail(call, i, "theta, grad, m and s must not be NULL");
        if (!aligned(t.theta, 4) || !aligned(t.grad, cfg->grad_dtype == BMGD_F32 ? 4 : 2) || !aligned(t.copy, 2) || !aligned(t.m, 4) || !aligned(t.s, 4))
            return tensor_fail(call, i, "an address is not a multiple of its element's size (codes: of 4)");
        if (eight && (!t.m_scale || !t.s_scale || !aligned(t.m_scale, 4) || !aligned(t.s_scale, 4)))
            return tensor_fail(call, i, "m_scale and s_scale must not be NULL and 4-byte aligned");
    }
    Args a;
    a.copy_dtype = cfg->copy_dtype;
    const double k = (double)step;
    a.r.b1 = (float)cfg->beta1;
    a.r.c1 = (float)(1.0 - cfg->beta1);
    a.r.b2 = (float)cfg->beta2;
    a.r.c2 = (float)(1.0 - cfg->beta2);
    a.r.m_fix = (float)(1.0 / (1.0 - pow(cfg->beta1, k)));
    a.r.s_fix = (float)(1.0 / (1.0 - pow(cfg->beta2, k)));
    a.r.decay = (float)(cfg->lr * cfg->weight_decay);
    a.r.lr = (float)cfg->lr;
    a.r.eps = (float)cfg->eps;
    a.r.grad_scale = (float)cfg->grad_scale;
    const int grad = cfg->grad_dtype == BMGD_F32 ? 4 : 2;
    const int size[kKinds] = {4, grad, 2, 4, 4, 4, 4}, advance[kKinds] = {4 * kBlock, grad * kBlock, 2 * kBlock, eight ? kBlock : 4 * kBlock, eight ? kBlock : 4 * kBlock, 4, 4};
    Collector c;
    c.clear();
    auto send = [&]() {
        if (c.t.count == 0) return (int)BMGD_OK;
        a.has_copy = c.lo[kCopy] != 0;
        a.t = c.close(size);
        const hipStream_t s = static_cast<hipStream_t>(stream);
        const unsigned groups = (unsigned)c.groups;
        const hipError_t e = cfg->grad_dtype == BMGD_F32 ? launch_step<float>(a, groups, eight, s)
                             : cfg->grad_dtype == BMGD_BF16 ? launch_step<__bf16>(a, groups, eight, s) : launch_step<_Float16>(a, groups, eight, s);
        c.clear();
        return e == hipSuccess ? (int)BMGD_OK : hip_fail(e, "launch of the AdamW step");
    };
    for (int64_t i = 0; i < count; ++i) {
        const bmgd_adamw_tensor& t = tensors[i];
        const uintptr_t p[kKinds] = {address(t.theta), address(t.grad), address(t.copy), address(t.m), address(t.s), eight ? address(t.m_scale) : 0, eight ? address(t.s_scale) : 0};
        const int rc = entries_of(p, advance, t.n, [&](const uintptr_t* q, int64_t n) {
            const int64_t need = (n + kPiece - 1) / kPiece;
            if (c.add(q, size, n, need)) return (int)BMGD_OK;
            const int r = send();
            c.add(q, size, n, need);
            return r;
        });
        if (rc != BMGD_OK) return rc;
    }
    return send();
}

BMGD_API int bmgd_adamw_moments(const bmgd_adamw_tensor* tensors, int64_t count, float* const* m_out, float* const* s_out, void* stream)
{
    static const char call[] = "bmgd_adamw_moments";
    if (count < 0 || (count > 0 && (!tensors || !m_out || !s_out))) return fail(BMGD_EINVAL, "bmgd_adamw_moments: tensors, m_out and s_out must hold count >= 0 entries");
    for (int64_t i = 0; i < count; ++i) {
        const bmgd_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n > kMaxElements) return tensor_fail(call, i, "n must be in [0, 2^38]");
        if (t.n == 0) continue;
        if (!t.m || !t.s || !t.m_scale || !t.s_scale || !m_out[i] || !s_out[i]) return tensor_fail(call, i, "codes, scales and results must not be NULL");
        if (!aligned(t.m, 4) || !aligned(t.s, 4) || !aligned(t.m_scale, 4) || !aligned(t.s_scale, 4) || !aligned(m_out[i], 4) || !aligned(s_out[i], 4))
            return tensor_fail(call, i, "addresses must be multiples of 4");
    }
    const int size[kKinds] = {4, 4, 2, 4, 4, 4, 4}, advance[kKinds] = {4 * kBlock, 4 * kBlock, 0, kBlock, kBlock, 4, 4};
    Collector c;
    c.clear();
    auto send = [&]() {
        if (c.t.count == 0) return (int)BMGD_OK;
        MomentArgs a;
        a.t = c.close(size);
        hipLaunchKernelGGL(adamw_moments_kernel, dim3((unsigned)c.groups), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
        c.clear();
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? (int)BMGD_OK : hip_fail(e, "launch of the moments' values");
    };
    for (int64_t i = 0; i < count; ++i) {
        const bmgd_adamw_tensor& t = tensors[i];
        const uintptr_t p[kKinds] = {address(m_out[i]), address(s_out[i]), 0, address(t.m), address(t.s), address(t.m_scale), address(t.s_scale)};
        const int rc = entries_of(p, advance, t.n, [&](const uintptr_t* q, int64_t n) {
            const int64_t need = (n + kPiece - 1) / kPiece;
            if (c.add(q, size, n, need)) return (int)BMGD_OK;
            const int r = send();
            c.add(q, size, n, need);
            return r;
        });
        if (rc != BMGD_OK) return rc;
    }
    return send();
}

}  // extern "C"
