// The kernels of attention with scores of several forms at once.
#include "attention_kernels.h"

namespace samo {

hipError_t launch_attention_all(int which, const AttnArgs &a, int64_t items, hipStream_t s) { return launch_form<kAll>(which, a, items, s); }

}  // namespace samo
