// fp8_host.h -- argument checks shared by the 8-bit operators' C-ABI sources.
#pragma once
#include "hv_fp8.h"
#include "hv_host.h"

namespace hvh {

static_assert(HV_BF16 == hv::kTypeBf16 && HV_F16 == hv::kTypeF16 && HV_F32 == hv::kTypeF32, "element types");

inline hv_status check_type(hv_type type) {
    if (type == HV_BF16 || type == HV_F16 || type == HV_F32) return HV_OK;
    return fail(HV_ERR_INVALID_ARG, "unknown element type %d", (int)type);
}

inline size_t size_of(hv_type type) { return type == HV_F32 ? 4 : 2; }

inline hv_status check_pointer(const char* what, const void* p, size_t alignment) {
    if (p == nullptr) return fail(HV_ERR_INVALID_ARG, "%s is NULL", what);
    if ((uintptr_t)p % alignment != 0)
        return fail(HV_ERR_INVALID_ARG, "%s is not %zu-byte aligned", what, alignment);
    return HV_OK;
}

inline hv_status check_workspace(const void* workspace, size_t bytes, size_t need) {
    if (need == 0) return HV_OK;
    if (workspace == nullptr || bytes < need)
        return fail(HV_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu%s", need, bytes, workspace ? "" : " (NULL)");
    if ((uintptr_t)workspace % kAlign != 0) return fail(HV_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    return HV_OK;
}

#define HV_TRY(call)                     \
    do {                                 \
        const hv_status st_ = (call);    \
        if (st_ != HV_OK) return st_;    \
    } while (0)

inline hv_status done(hipError_t e, const char* what) { return e == hipSuccess ? HV_OK : hip_fail(e, what); }

}  // namespace hvh
