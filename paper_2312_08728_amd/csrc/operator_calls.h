// What the entry points of the norm, the 8-bit product and the log probabilities share on the host: checks of arguments and errors.
#pragma once

#include "../../include/bmgd.h"
#include "bmgd_internal.h"

#include <stdio.h>

namespace bmgd {
namespace {

constexpr int64_t kMaxCallRows = (int64_t(1) << 30) - 1;
constexpr int64_t kRowsOfLaunch = int64_t(1) << 21;     // a launch has less than 2^32 threads, 1,024 or fewer of them to a row

inline size_t size_of(int dtype) { return dtype == BMGD_F32 ? 4 : 2; }
inline bool known_type(int dtype) { return dtype == BMGD_F32 || dtype == BMGD_BF16 || dtype == BMGD_F16; }

// One call's checks: the first one that fails gives the message.
struct Call {
    const char* name;
    int code = BMGD_OK;

    void refuse(int c, const char* why)
    {
        if (code != BMGD_OK) return;
        char buf[256];
        snprintf(buf, sizeof buf, "%s: %s", name, why);
        set_create_error(buf);
        code = c;
    }
    void refuse(const char* what, const char* why)
    {
        if (code != BMGD_OK) return;
        char buf[256];
        snprintf(buf, sizeof buf, "%s: %s: %s", name, what, why);
        set_create_error(buf);
        code = BMGD_EINVAL;
    }
    void rows(int64_t n)
    {
        if (n < 0 || n > kMaxCallRows) refuse(BMGD_EINVAL, "rows must be in [0, 2^30)");
    }
    void address(const char* what, const void* p, bool wanted, size_t size)
    {
        if (!p) {
            if (wanted) refuse(what, "must not be NULL");
        } else if (reinterpret_cast<uintptr_t>(p) & (size - 1)) {
            refuse(what, "the address is not a multiple of an element's size");
        }
    }
    void matrix(const char* what, const bmgd_matrix& m, int64_t rows, int64_t cols, bool wanted, size_t size)
    {
        address(what, m.data, wanted, size);
        if (m.data && rows > 1 && m.stride < cols) refuse(what, "the stride is less than the number of columns");
        if (m.data && rows > 1 && m.stride > (int64_t(1) << 40) / (rows >> 20 ? rows >> 20 : 1)) refuse(what, "the stride is too large");
    }
    // `written` must not begin where `other` does
    void apart(const char* what, const void* written, const void* other)
    {
        if (written && written == other) refuse(what, "is written, and is another matrix of the call too");
    }
    int hip(hipError_t e, const char* what)
    {
        if (e == hipSuccess) return BMGD_OK;
        char buf[256];
        snprintf(buf, sizeof buf, "%s: %s: %s", name, what, hipGetErrorString(e));
        (void)hipGetLastError();
        set_create_error(buf);
        return BMGD_EHIP;
    }
    int launched() { return hip(hipGetLastError(), "launch"); }
};

// Compute units of the current device, asked once per device.
inline int compute_units()
{
    constexpr int kDevices = 64;
    static int known[kDevices];                     // (the same value from every thread)
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) {
        (void)hipGetLastError();
        return 256;
    }
    if (device >= 0 && device < kDevices && __atomic_load_n(&known[device], __ATOMIC_RELAXED)) return __atomic_load_n(&known[device], __ATOMIC_RELAXED);
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || n < 1) {
        (void)hipGetLastError();
        return 256;
    }
    if (device >= 0 && device < kDevices) __atomic_store_n(&known[device], n, __ATOMIC_RELAXED);
    return n;
}

}  // namespace
}  // namespace bmgd
