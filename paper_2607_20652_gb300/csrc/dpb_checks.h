// dpb_checks.h -- host-side argument checks and launch reporting shared by
// the training-step entry points.
#pragma once

#include <cstdint>

#include "dpb_internal.h"

namespace dpb {

inline bool is_aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline dpb_status need(const void *p, const char *name, size_t align) {
    if (!p) return fail(DPB_ERR_INVALID_ARG, "%s is NULL", name);
    if (!is_aligned(p, align)) return fail(DPB_ERR_INVALID_ARG, "%s must be %zu-byte aligned", name, align);
    return DPB_OK;
}

inline dpb_status need_workspace(const void *ws, size_t bytes, size_t want) {
    if (!ws) return fail(DPB_ERR_INVALID_ARG, "workspace is NULL");
    if (!is_aligned(ws, 256)) return fail(DPB_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (bytes < want) return fail(DPB_ERR_INVALID_ARG, "workspace needs %zu bytes, got %zu", want, bytes);
    return DPB_OK;
}

// Where a call's device bits go (status_slot), and the workspace that it needs
// for them and for its scratch.
inline dpb_status place_status(int32_t slot, void *ws, size_t bytes, size_t want, int32_t **status) {
    if (slot == 0 || want > kStatusBytes) {
        const dpb_status s = need_workspace(ws, bytes, want);
        if (s != DPB_OK) return s;
    }
    *status = slot == 0 ? static_cast<int32_t *>(ws) : status_word(slot);
    return *status ? DPB_OK : fail(DPB_ERR_CUDA, "no status word %d on this device", slot);
}
inline dpb_status check_slot(int32_t slot) {
    if (slot < 0 || slot > DPB_STATUS_SLOTS) return fail(DPB_ERR_INVALID_ARG, "status_slot must lie in [0, %d]", DPB_STATUS_SLOTS);
    return DPB_OK;
}

// A failed launch is reported through the returned status; the runtime's
// last-error slot is cleared so that the caller's next CUDA check does not
// see it again.
inline dpb_status launch_status(cudaError_t e, const char *what) {
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(DPB_ERR_CUDA, "%s launch failed: %s", what, cudaGetErrorString(e));
    }
    return DPB_OK;
}

#define DPB_CHECK(expr)                         \
    do {                                        \
        const dpb_status check_s_ = (expr);     \
        if (check_s_ != DPB_OK) return check_s_; \
    } while (0)

}  // namespace dpb
