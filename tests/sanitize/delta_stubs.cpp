// Stand-ins for the kernel launchers of delta_api.cpp, as launch_stubs.cpp has them for api.cpp: every launch
// reports failure.  Test infrastructure only.
#include "delta.hpp"
#include "norms.hpp"

namespace pm {
hipError_t launch_delta_prep(const DeltaArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_delta_fwd(const DeltaArgs&, bool, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_delta_states(const DeltaArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_delta_rev(const DeltaArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_delta_segments(const DeltaArgs&, bool, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_delta_grads(const DeltaArgs&, bool, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_linear_group_sums(const float*, void*, const float*, void*, int64_t, int32_t, int32_t, int64_t, bool, hipStream_t) {
    return hipErrorInvalidValue;
}
hipError_t launch_delta_step(const DeltaStepArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_layernorm_fwd(const NormArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_layernorm_bwd(const NormArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_l2norm_fwd(const NormArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_l2norm_bwd(const NormArgs&, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace pm
