// rlm_check.h -- host-side argument checks shared by the translation units of the C ABI.
#pragma once

#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "rlm_internal.h"

namespace rlm {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline size_t elem_size(rlm_dtype dt) { return dt == RLM_BF16 ? 2 : 4; }

inline rlm_status fail(rlm_status s, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    set_error("%s", buf);
    return s;
}

inline rlm_status cuda_fail(cudaError_t e, const char *what) {
    return fail(RLM_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const char *pa = static_cast<const char *>(a), *pb = static_cast<const char *>(b);
    return pa < pb + nb && pb < pa + na;
}

inline rlm_status check_workspace(const rlm_launch *ln, size_t need) {
    if (!ln) return fail(RLM_ERR_INVALID_ARG, "launch is NULL");
    if (need == 0) return RLM_OK;
    if (!ln->workspace) return fail(RLM_ERR_INVALID_ARG, "workspace is NULL but %zu bytes are needed", need);
    if ((reinterpret_cast<uintptr_t>(ln->workspace) & 255u) != 0)
        return fail(RLM_ERR_INVALID_ARG, "workspace is not 256-byte aligned");
    if (ln->workspace_bytes < need)
        return fail(RLM_ERR_INVALID_ARG, "workspace has %zu bytes, %zu needed", ln->workspace_bytes, need);
    return RLM_OK;
}

}  // namespace rlm
