// The layer-and-step host layer (pam_training_api.cpp) beside dispatch_probe.cpp,
// whose launches are recorded: which product kernels a linear layer takes.
// Built by linear_probe.py.

#include "pam_training_api.cpp"

namespace pamk {
hipError_t launch_activation_grad(bool, bool, const GradParams &, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_adamw(int, uint32_t, const StepParams &, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_grad_squares(uint32_t, const NormParams &, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_grad_norm(const double *, int64_t, float *, hipStream_t) { return hipErrorNoDevice; }
}  // namespace pamk
