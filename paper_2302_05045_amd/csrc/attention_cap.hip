// The kernels of attention with scores capped by a tanh.
#include "attention_kernels.h"

namespace samo {

hipError_t launch_attention_cap(int which, const AttnArgs &a, int64_t items, hipStream_t s) { return launch_form<kCap>(which, a, items, s); }

}  // namespace samo
