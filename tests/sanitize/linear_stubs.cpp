// Stand-ins for the kernel launchers of linear_api.cpp, as launch_stubs.cpp has them for api.cpp: every launch
// reports failure.  Test infrastructure only.
#include "linear.hpp"

namespace pm {
hipError_t launch_walk(const WalkArgs&, WalkMode, bool, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_walk_segments(const WalkArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_linear_ddecay(const LinDecayArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_linear_group_sum(const float*, void*, int64_t, int32_t, int32_t, int64_t, bool, hipStream_t) {
    return hipErrorInvalidValue;
}
hipError_t launch_linear_step(const LinStepArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_gated_fwd(const GatedArgs&, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_gated_bwd(const GatedArgs&, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace pm
