// dpb_checks.h -- host-side argument checks and launch reporting shared by
// the training-step entry points.
#pragma once

#include <cudaTypedefs.h>

#include <atomic>
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

// Multiprocessors of the current device, asked for once.
inline int sms_of_device() {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices];
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && dev < kDevices && (sms = known[dev].load(std::memory_order_relaxed)) > 0) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return 2;
    }
    if (dev < kDevices) known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

// The driver's encoder of tensor maps, or nullptr.
inline PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) !=
                cudaSuccess ||
            r != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    }();
    return fn;
}

// A kernel that may start, and set itself up, while the one before it in the
// stream runs; it waits for that one's results itself.
template <typename... K, typename... A>
cudaError_t launch_early(void (*kernel)(K...), dim3 blocks, int threads, size_t smem, cudaStream_t s, const A &...args) {
    cudaLaunchConfig_t how{};
    how.gridDim = blocks;
    how.blockDim = dim3(threads);
    how.dynamicSmemBytes = smem;
    how.stream = s;
    cudaLaunchAttribute early{};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    how.attrs = &early;
    how.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&how, kernel, args...);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

#define DPB_CHECK(expr)                         \
    do {                                        \
        const dpb_status check_s_ = (expr);     \
        if (check_s_ != DPB_OK) return check_s_; \
    } while (0)

}  // namespace dpb
