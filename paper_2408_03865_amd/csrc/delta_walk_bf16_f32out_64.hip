// The gated delta rule's walks of heads whose keys have up to 64 features: bf16_t in, float out.
#include "delta_walk.hpp"

namespace pm {
template hipError_t launch_delta_kc<bf16_t, float, 64>(const DeltaArgs&, DeltaWalk, hipStream_t);
}  // namespace pm
