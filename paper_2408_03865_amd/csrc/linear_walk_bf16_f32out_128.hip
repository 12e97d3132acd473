// The linear-attention walks of heads whose contracted features number up to 128: bf16_t in, float out.
#include "linear_walk.hpp"

namespace pm {
template hipError_t launch_walk_kc<bf16_t, float, 128>(const WalkArgs&, WalkMode, bool, hipStream_t);
}  // namespace pm
