// Checks of the arguments of the operators' C entries (abi_rows.hip, abi_losses.hip).
#pragma once

#include <cmath>
#include <string>

#include "rows.h"

namespace hbsjd {

constexpr int64_t kMaxStride = (int64_t)1 << 40;

inline bool elem_ok(int32_t e) { return e == HBSJD_ELEM_F32 || e == HBSJD_ELEM_BF16 || e == HBSJD_ELEM_F16; }
inline bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// null, or why a [rows][V] matrix cannot be taken
inline const char* matrix_problem(const void* p, int32_t elem, int64_t ld, int32_t V) {
    if (!elem_ok(elem)) return "unknown element type";
    if (!p) return "NULL buffer";
    if (!aligned(p, elem_size(elem))) return "buffer not aligned to its elements";
    if (ld < V || ld > kMaxStride) return "row stride below V or above 2^40";
    return nullptr;
}

inline const char* rows_problem(int64_t rows, int32_t V) {
    if (rows < 0 || rows > INT32_MAX) return "need 0 <= rows < 2^31";
    if (V < 1 || V > HBSJD_ROWS_MAX_VOCAB) return "need V in [1, 262144]";
    return nullptr;
}

inline const char* workspace_problem(const void* p, uint64_t bytes, uint64_t need) {
    if (need && (!p || bytes < need)) return "workspace smaller than the call needs";
    if (need && !aligned(p, 16)) return "workspace not aligned to 16 bytes";
    return nullptr;
}

inline bool temperature_ok(float t) { return t >= 1e-6f && t <= 1e6f; }

// log2 e / temperature in two parts
inline float2 log2_over(float temperature) {
    const double x = 1.4426950408889634074 / (double)temperature;
    float hi = (float)x;   // rounded down: the rest is positive
    if ((double)hi >= x) hi = std::nextafterf(hi, 0.f);
    return make_float2(hi, (float)(x - (double)hi));
}

inline hbsjd_status launched(const char* where) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return api_fail(HBSJD_EHIP, std::string(where) + ": " + hipGetErrorString(e));
    return HBSJD_OK;
}

}  // namespace hbsjd
