// What the two files of entry points share: the thread's error message, checks of pointers, launch status.
#pragma once
#include "lca_internal.h"

namespace lca {

// Leaves the message for lca_last_error() and returns st.
__attribute__((format(printf, 2, 3))) lca_status fail(lca_status st, const char *fmt, ...);

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline lca_status check_ptr(const void *p, const char *name, bool required = true)
{
    if (p == nullptr) return required ? fail(LCA_ERR_INVALID_ARG, "%s is NULL", name) : LCA_OK;
    if (!aligned16(p)) return fail(LCA_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
    return LCA_OK;
}

#define LCA_TRY(expr)                      \
    do {                                   \
        lca_status _s = (expr);            \
        if (_s != LCA_OK) return _s;       \
    } while (0)

inline lca_status hip_status(hipError_t e, const char *what)
{
    if (e == hipSuccess) return LCA_OK;
    return fail(LCA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// The launch functions report hipGetLastError() after their kernels, and that call returns the calling thread's last
// error whoever caused it: one left behind by an earlier runtime call of the caller's own would be taken for a failed
// launch.  So the thread's error state is read, and thereby cleared, right before a launch function runs.
#define LCA_LAUNCH(call, what) ((void)hipGetLastError(), lca::hip_status((call), (what)))

}  // namespace lca
