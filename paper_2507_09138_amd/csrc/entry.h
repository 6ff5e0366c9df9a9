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

inline bool known_type(int32_t dtype) { return dtype == HR_F32 || dtype == HR_F16 || dtype == HR_BF16; }

inline int check_matrix(const char* name, const void* p, int64_t rows, int64_t k, int64_t ld, size_t es)
{
    if (rows > 0 && !p) return fail(HR_ERR_ARG, "%s is null", name);
    if (ld < k || ld > (1LL << 40)) return fail(HR_ERR_ARG, "rows of %s: %lld elements, %lld apart", name, (long long)k, (long long)ld);
    if ((uintptr_t)p % es) return fail(HR_ERR_ARG, "%s is not aligned to its elements", name);
    return HR_OK;
}

inline size_t aligned(size_t bytes) { return (bytes + HR_WORKSPACE_ALIGN - 1) / HR_WORKSPACE_ALIGN * HR_WORKSPACE_ALIGN; }
inline size_t element_bytes(int32_t dtype) { return dtype == HR_F32 ? 4 : 2; }

// f(type) with the C++ type of a code
template <typename F>
inline auto with_type(int dtype, F&& f)
{
    switch (dtype) {
    case HR_F32: return f(float{});
    case HR_F16: return f(_Float16{});
    default: return f(__bf16{});
    }
}

}  // namespace hr
