// The gated delta rule's walks of heads whose keys have up to 128 features: bf16_t in, bf16_t out.
#include "delta_walk.hpp"

namespace pm {
template hipError_t launch_delta_kc<bf16_t, bf16_t, 128>(const DeltaArgs&, DeltaWalk, hipStream_t);
}  // namespace pm
