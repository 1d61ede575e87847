// The kernels of attention with scores that fall with the distance.
#include "attention_kernels.h"

namespace samo {

hipError_t launch_attention_slope(int which, const AttnArgs &a, int64_t items, hipStream_t s) { return launch_form<kSlope>(which, a, items, s); }

}  // namespace samo
