// The kernels of attention with scores that fall with the distance and have a learned bias by its bucket, capped or not.
#include "attention_kernels.h"

namespace samo {

hipError_t launch_attention_all(int which, const AttnArgs &a, int64_t items, hipStream_t s) { return launch_form<kAll>(which, a, items, s); }

}  // namespace samo
