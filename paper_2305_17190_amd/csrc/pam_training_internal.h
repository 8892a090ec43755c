// Internal interface between pam_training_api.cpp and pam_training.hip: the
// activations' gradient, the gradients' norm and the optimizer's step.  Not
// installed; not part of the public ABI.
#pragma once

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "pam_training.h"

namespace pamk {

// Calls on more memory than the last-level cache holds take the hint: what they
// read first would have left the cache by the time it is read again.
constexpr int64_t kCacheBytes = (int64_t)256 << 20;

// ---------------------------------------------------------------------------
// The activations' gradient
// ---------------------------------------------------------------------------

constexpr int kGradThreads = 256;

// A workgroup takes `band` rows of lanes * (4 float32 or 8 bfloat16) columns:
// kGradThreads / lanes rows at a time.  Its column sums go to db where one
// band holds all rows, else to partial[band][n].
struct GradParams {
    const void *dy, *z;
    void *dz;
    float *db;        // or nullptr
    float *partial;
    int64_t lddy, ldz, lddz;
    int64_t m;
    int32_t n;
    int32_t bands, band, lanes;
    int32_t activation;
    int32_t streaming;   // loads with the non-temporal hint
    int32_t apart;       // dz lies on neither dy nor z
};
inline int grad_values(bool bf16) { return bf16 ? 8 : 4; }
hipError_t launch_activation_grad(bool bf16, bool z_bf16, const GradParams &p, hipStream_t stream);

// ---------------------------------------------------------------------------
// Many tensors at once
// ---------------------------------------------------------------------------

// A launch takes its tensors by value, in the kernel's arguments: no array in
// device memory would have to be written, kept or waited for.  A workgroup
// takes `chunk` values of one tensor: workgroup b of tensor j when first[j] <=
// b < first[j + 1].  At most 64 tensors, for a wave compares all of first at once.
constexpr int kStepThreads = 256;
constexpr int kStepTensors = 56;
constexpr int kNormTensors = 64;
constexpr int64_t kMostStepGroups = 16777215;   // below 2^32 threads

struct StepParams {
    pam_step_tensor_t tensor[kStepTensors];
    uint32_t first[kStepTensors];
    int32_t count;         // of tensors
    int32_t tensor0;       // number of the first in the whole call
    int64_t chunk;
    const float *norm;
    const int64_t *step_device;
    int64_t step;
    // beta^t = exp(t log_beta): in float64, from the host's or the device's step.
    double log_beta1, log_beta2;
    float step_size;       // lr / (1 - beta1^t); lr with step_device
    float sq_factor;       // 1 / sqrt(1 - beta2^t)
    float keep;            // 1 - lr weight_decay
    float beta1, rest1, beta2, rest2, eps, max_norm;
    uint32_t seed;
    int32_t grad_bf16;
    int32_t streaming;     // with the non-temporal hint
};
static_assert(sizeof(StepParams) <= 4096, "a kernel's arguments");
hipError_t launch_adamw(int state_bits, uint32_t groups, const StepParams &p, hipStream_t stream);

struct NormParams {
    const void *g[kNormTensors];
    int64_t n[kNormTensors];
    uint32_t first[kNormTensors];
    int32_t count;
    int32_t grad_bf16;
    int32_t streaming;     // loads with the non-temporal hint
    int64_t chunk;
    double *partial;       // one a workgroup
};
hipError_t launch_grad_squares(uint32_t groups, const NormParams &p, hipStream_t stream);
// norm = sqrt(the sum of `count` partial sums).
hipError_t launch_grad_norm(const double *partial, int64_t count, float *norm, hipStream_t stream);

}  // namespace pamk
