// Norm of a list of tensors and their scaling: host launchers (internal interface).
#pragma once

#include "rows.h"

namespace hbsjd {

struct GradArgs {
    int64_t count;
    const void* const* data;
    const int64_t* sizes;
    const int32_t* elems;
    int32_t order;        // 2, or 0: the largest magnitude
    void* const* out;     // null: the norm alone
    float limit;
    float* norm;
};
// bytes of workspace that a call needs
size_t grad_norm_workspace();
// false (and nothing queued) where the sizes cannot be those of tensors on a device
bool grad_norm(const GradArgs& a, void* workspace, hipStream_t s);

}  // namespace hbsjd
