// The kernels of attention with scores with a learned bias by the distance's bucket.
#include "attention_kernels.h"

namespace samo {

hipError_t launch_attention_table(int which, const AttnArgs &a, int64_t items, hipStream_t s) { return launch_form<kTable>(which, a, items, s); }

}  // namespace samo
