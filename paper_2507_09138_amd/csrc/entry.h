// What the C entry points of several files share: error messages and checks of arguments (host only).
#pragma once
#include "common.h"
#include "hr_scores.h"

namespace hr {

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));     // sets hr_last_error(), returns code

#define HR_HIP(call)                                                                      \
    do {                                                                                  \
        hipError_t e_ = (call);                                                           \
        if (e_ != hipSuccess) return ::hr::fail(HR_ERR_HIP, "%s: %s", #call, hipGetErrorString(e_)); \
    } while (0)

inline int check_workspace(const void* ws, size_t bytes, size_t need)
{
    if (!ws) return fail(HR_ERR_WORKSPACE, "workspace is null");
    if (((uintptr_t)ws) % HR_WORKSPACE_ALIGN) return fail(HR_ERR_WORKSPACE, "workspace not %d-byte aligned", HR_WORKSPACE_ALIGN);
    if (bytes < need) return fail(HR_ERR_WORKSPACE, "workspace has %zu bytes, need %zu", bytes, need);
    return HR_OK;
}

inline size_t aligned(size_t bytes) { return (bytes + HR_WORKSPACE_ALIGN - 1) / HR_WORKSPACE_ALIGN * HR_WORKSPACE_ALIGN; }
inline size_t element_bytes(int32_t dtype) { return dtype == HR_F32 ? 4 : 2; }

}  // namespace hr
