// The gated delta rule's walks of heads whose keys have up to 128 features: float in, float out.
#include "delta_walk.hpp"

namespace pm {
template hipError_t launch_delta_kc<float, float, 128>(const DeltaArgs&, DeltaWalk, hipStream_t);
}  // namespace pm
