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
#include "../../include/bmgd.h"
#include "bmgd_internal.h"

#include <math.h>
#include <stdio.h>
#include <string.h>

#include <algorithm>

using namespace bmgd;

namespace {

constexpr int kThreads = 256, kBlock = 256;                  // threads of a workgroup; elements that share a scale
constexpr int kPiece = 4 * kThreads;                          // elements that a workgroup takes at a time
constexpr int kMaxTensors = 48;                               // of a launch: they travel as kernel arguments

static_assert(sizeof(bmgd_adamw_tensor) == 64, "");

struct Rates {
    float b1, c1, b2, c2;           // beta1, 1 - beta1, beta2, 1 - beta2
    float m_fix, s_fix;             // 1 / (1 - beta1^k), 1 / (1 - beta2^k)
    float keep, lr, eps, grad_scale;
};

struct Args {
    bmgd_adamw_tensor t[kMaxTensors];
    unsigned first[kMaxTensors + 1];                          // first workgroup of each tensor; behind the last one the number of workgroups
    int count;
    int copy_dtype;
    Rates r;
};

struct MomentArgs {
    struct One { const signed char* m; const unsigned char* s; const float* m_scale; const float* s_scale; float* m_out; float* s_out; int64_t n; } t[kMaxTensors];
    unsigned first[kMaxTensors + 1];
    int count;
};
static_assert(sizeof(Args) <= 4096 && sizeof(MomentArgs) <= 4096, "kernel arguments");

typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef short short4u __attribute__((ext_vector_type(4), aligned(2)));

// Which tensor workgroup `id` works on.
__device__ __forceinline__ int tensor_of(const unsigned* first, int count, unsigned id)
{
    const int lane = threadIdx.x & 63;
    return __popcll(__ballot(lane < count && first[min(lane, count)] <= id)) - 1;
}

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

// One element.  Products and sums are rounded one by one, so that the codes do not depend on what the compiler joins.
__device__ __forceinline__ float update(const Rates& r, float theta, float g, float& m, float& s)
{
#pragma clang fp contract(off)
    g = g * r.grad_scale;
    m = r.b1 * m + r.c1 * g;
    s = r.b2 * s + r.c2 * (g * g);
    const float bottom = sqrtf(s * r.s_fix) + r.eps;
    return theta * r.keep - r.lr * (m * r.m_fix / bottom);
}

template <typename G, bool EIGHT, int U>
__global__ void __launch_bounds__(kThreads) adamw_kernel(Args a)
{
    const int which = __builtin_amdgcn_readfirstlane(tensor_of(a.first, a.count, blockIdx.x));
    const bmgd_adamw_tensor t = a.t[which];
    const int64_t start = (int64_t)(blockIdx.x - a.first[which]) * (kPiece * U) + 4 * threadIdx.x;
    float4v theta[U], g[U], m[U], s[U];
    unsigned mc[U], sc[U];
    float ma[U], sa[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t at = start + u * kPiece, left = t.n - at;
        g[u] = load_grad<G>(t.grad, at, left);
        theta[u] = load_grad<float>(t.theta, at, left);
        if constexpr (EIGHT) {
            mc[u] = sc[u] = 0u;
            ma[u] = sa[u] = 0.f;
            if (left >= 4) {
                mc[u] = *reinterpret_cast<const unsigned*>(static_cast<const char*>(t.m) + at);
                sc[u] = *reinterpret_cast<const unsigned*>(static_cast<const char*>(t.s) + at);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) {
                        mc[u] |= (unsigned)static_cast<const unsigned char*>(t.m)[at + i] << (8 * i);
                        sc[u] |= (unsigned)static_cast<const unsigned char*>(t.s)[at + i] << (8 * i);
                    }
            }
            if (left > 0) {
                ma[u] = t.m_scale[at / kBlock];
                sa[u] = t.s_scale[at / kBlock];
            }
        } else {
            m[u] = load_grad<float>(t.m, at, left);
            s[u] = load_grad<float>(t.s, at, left);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t at = start + u * kPiece, left = t.n - at;
        if constexpr (EIGHT) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m[u][i] = m_value((int)(signed char)(mc[u] >> (8 * i)), ma[u]);
                s[u][i] = s_value(sc[u] >> (8 * i) & 255u, sa[u]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mi = m[u][i], si = s[u][i];
            theta[u][i] = update(a.r, theta[u][i], g[u][i], mi, si);
            m[u][i] = mi;
            s[u][i] = si;
        }
        if (left > 0) {
            store_floats(t.theta + at, left, theta[u]);
            if (t.copy) store_copy(t.copy, a.copy_dtype, at, left, theta[u]);
            if constexpr (!EIGHT) {
                store_floats(static_cast<float*>(t.m) + at, left, m[u]);
                store_floats(static_cast<float*>(t.s) + at, left, s[u]);
            }
        }
        if constexpr (EIGHT) {
#pragma clang fp contract(off)
            unsigned m_top = 0u, s_top = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i < left) {
                    m_top = max(m_top, __float_as_uint(m[u][i]) & 0x7FFFFFFFu);
                    s_top = max(s_top, __float_as_uint(s[u][i]) & 0x7FFFFFFFu);
                }
            }
            float m_inv, s_inv;
            const float m_scale = scale_of(wave_max(m_top), m_inv), s_scale = scale_of(wave_max(s_top), s_inv);
            unsigned mb = 0u, sb = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (an inverse of zero: a scale that is zero or not finite; all codes are zero then)
                const float size = rintf(127.f * sqrtf(fabsf(m[u][i]) * m_inv));
                const int mq = m_inv > 0.f ? (int)copysignf(size, m[u][i]) : 0;
                float root = rintf(255.f * sqrtf(sqrtf(s[u][i] * s_inv)));
                if (s[u][i] > 0.f) root = fmaxf(root, 1.f);
                const unsigned sq = s_inv > 0.f ? (unsigned)root : 0u;
                mb |= ((unsigned)mq & 255u) << (8 * i);
                sb |= sq << (8 * i);
            }
            if (left >= 4) {
                *reinterpret_cast<unsigned*>(static_cast<char*>(t.m) + at) = mb;
                *reinterpret_cast<unsigned*>(static_cast<char*>(t.s) + at) = sb;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) {
                        static_cast<unsigned char*>(t.m)[at + i] = (unsigned char)(mb >> (8 * i));
                        static_cast<unsigned char*>(t.s)[at + i] = (unsigned char)(sb >> (8 * i));
                    }
            }
            if (left > 0 && (threadIdx.x & 63) == 0) {
                t.m_scale[at / kBlock] = m_scale;
                t.s_scale[at / kBlock] = s_scale;
            }
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
    const int which = __builtin_amdgcn_readfirstlane(tensor_of(a.first, a.count, blockIdx.x));
    const MomentArgs::One t = a.t[which];
    const int64_t at = (int64_t)(blockIdx.x - a.first[which]) * kPiece + 4 * threadIdx.x, left = t.n - at;
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

template <typename G, bool EIGHT, int U> hipError_t launch_step(const Args& a, hipStream_t s)
{
    hipLaunchKernelGGL((adamw_kernel<G, EIGHT, U>), dim3(a.first[a.count]), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <typename G> hipError_t launch_step(const Args& a, bool eight, int per, hipStream_t s)
{
    if (eight) return per == 1 ? launch_step<G, true, 1>(a, s) : launch_step<G, true, 4>(a, s);
    return per == 1 ? launch_step<G, false, 1>(a, s) : launch_step<G, false, 4>(a, s);
}

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
    if (cfg->grad_dtype != BMGD_F32 && cfg->grad_dtype != BMGD_BF16 && cfg->grad_dtype != BMGD_F16)
        return fail(BMGD_EINVAL, "bmgd_adamw_step: unknown grad_dtype");
    if (cfg->copy_dtype != BMGD_BF16 && cfg->copy_dtype != BMGD_F16) return fail(BMGD_EINVAL, "bmgd_adamw_step: copy_dtype must be BMGD_BF16 or BMGD_F16");
    if (cfg->state_bits != 32 && cfg->state_bits != 8) return fail(BMGD_EINVAL, "bmgd_adamw_step: state_bits must be 32 or 8");
    const bool eight = cfg->state_bits == 8;
    if (eight && (float)cfg->eps == 0.f) return fail(BMGD_EINVAL, "bmgd_adamw_step: moments in 8 bits need eps > 0");
    if (step < 1 || step > (int64_t(1) << 53)) return fail(BMGD_EINVAL, "bmgd_adamw_step: step must be in [1, 2^53]");
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) {
        const bmgd_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n > kMaxElements) return tensor_fail(call, i, "n must be in [0, 2^38]");
        if (t.n == 0) continue;
        if (!t.theta || !t.grad || !t.m || !t.s) return tensor_fail(call, i, "theta, grad, m and s must not be NULL");
        if (!aligned(t.theta, 4) || !aligned(t.grad, cfg->grad_dtype == BMGD_F32 ? 4 : 2) || !aligned(t.copy, 2) || !aligned(t.m, 4) || !aligned(t.s, 4))
            return tensor_fail(call, i, "an address is not a multiple of its element's size (codes: of 4)");
        if (eight && (!t.m_scale || !t.s_scale || !aligned(t.m_scale, 4) || !aligned(t.s_scale, 4)))
            return tensor_fail(call, i, "m_scale and s_scale must not be NULL and 4-byte aligned");
        total += t.n;
    }
    // A workgroup takes 4096 elements; 1024 where that would leave compute units without one.
    const int per = total >= (int64_t(1) << 20) ? 4 : 1;
    Args a;
    a.copy_dtype = cfg->copy_dtype;
    const double k = (double)step;
    a.r.b1 = (float)cfg->beta1;
    a.r.c1 = (float)(1.0 - cfg->beta1);
    a.r.b2 = (float)cfg->beta2;
    a.r.c2 = (float)(1.0 - cfg->beta2);
    a.r.m_fix = (float)(1.0 / (1.0 - pow(cfg->beta1, k)));
    a.r.s_fix = (float)(1.0 / (1.0 - pow(cfg->beta2, k)));
    a.r.keep = (float)(1.0 - cfg->lr * cfg->weight_decay);
    a.r.lr = (float)cfg->lr;
    a.r.eps = (float)cfg->eps;
    a.r.grad_scale = (float)cfg->grad_scale;
    a.count = 0;
    int64_t groups = 0;
    for (int64_t i = 0; i <= count; ++i) {
        const int64_t n = i < count ? tensors[i].n : 0, need = (n + kPiece * per - 1) / (kPiece * per);
        if (a.count > 0 && (i == count || a.count == kMaxTensors || groups + need > kMaxWorkgroups)) {
            a.first[a.count] = (unsigned)groups;
            const hipStream_t s = static_cast<hipStream_t>(stream);
            const hipError_t e = cfg->grad_dtype == BMGD_F32 ? launch_step<float>(a, eight, per, s)
                                 : cfg->grad_dtype == BMGD_BF16 ? launch_step<__bf16>(a, eight, per, s) : launch_step<_Float16>(a, eight, per, s);
            if (e != hipSuccess) return hip_fail(e, "launch of the AdamW step");
            a.count = 0;
            groups = 0;
        }
        if (need > 0) {
            a.t[a.count] = tensors[i];
            a.first[a.count++] = (unsigned)groups;
            groups += need;
        }
    }
    return BMGD_OK;
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
    MomentArgs a;
    a.count = 0;
    int64_t groups = 0;
    for (int64_t i = 0; i <= count; ++i) {
        const int64_t n = i < count ? tensors[i].n : 0, need = (n + kPiece - 1) / kPiece;
        if (a.count > 0 && (i == count || a.count == kMaxTensors || groups + need > kMaxWorkgroups)) {
            a.first[a.count] = (unsigned)groups;
            hipLaunchKernelGGL(adamw_moments_kernel, dim3(a.first[a.count]), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return hip_fail(e, "launch of the moments' values");
            a.count = 0;
            groups = 0;
        }
        if (need > 0) {
            const bmgd_adamw_tensor& t = tensors[i];
            a.t[a.count] = {static_cast<const signed char*>(t.m), static_cast<const unsigned char*>(t.s), t.m_scale, t.s_scale, m_out[i], s_out[i], t.n};
            a.first[a.count++] = (unsigned)groups;
            groups += need;
        }
    }
    return BMGD_OK;
}

}  // extern "C"
