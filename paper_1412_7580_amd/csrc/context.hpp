// The handle behind the C ABI, and what its entry points share.
#pragma once
#include "../../include/fftconv.h"
#include "kernels.hpp"

constexpr int kMaxKernels = 8;
struct PlanCache;

struct fftconv_ctx {
    int device;
    fc::GemmSwitches sw;        // A/B switches of the contraction, read from the environment at creation
    PlanCache *plans;       // plans of the layer shapes seen so far
    hipStream_t stream;
    void *ws;
    size_t ws_bytes;
    void *step_ws;          // of the operators around the passes: a captured pass may hold `ws`, which they must not move
    size_t step_ws_bytes;
    void *static_scratch;   // this device's copy of fftconv_static_scratch (device address)
    int profiling;
    hipEvent_t ev[2 * kMaxKernels];   // start/stop pair per kernel of the last call
    int nk;                 // kernels of the last call that carry events
    const char *label[kMaxKernels];   // what each of them is (see fftconv_last_kernel_label)
    char last_hip_error[256];
};

namespace fc {

// Keeps the HIP error's text in the handle and returns FFTCONV_HIP_ERROR.
int hip_fail(fftconv_ctx *c, hipError_t e);
}  // namespace fc
