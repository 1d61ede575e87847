// The kernels of attention with scores capped by a tanh that fall with the distance.
#include "attention_kernels.h"

namespace samo {

hipError_t launch_attention_cap_slope(int which, const AttnArgs &a, int64_t items, hipStream_t s) { return launch_form<kCapSlope>(which, a, items, s); }

}  // namespace samo
