// The kernels of attention with scores capped by a tanh with a learned bias by the distance's bucket.
#include "attention_kernels.h"

namespace samo {

hipError_t launch_attention_cap_table(int which, const AttnArgs &a, int64_t items, hipStream_t s) { return launch_form<kCapTable>(which, a, items, s); }

}  // namespace samo
