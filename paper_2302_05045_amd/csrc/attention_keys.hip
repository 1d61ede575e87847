// The kernels of attention with scores that are plain but for first keys seen from everywhere.
#include "attention_kernels.h"

namespace samo {

hipError_t launch_attention_keys(int which, const AttnArgs &a, int64_t items, hipStream_t s) { return launch_form<kKeys>(which, a, items, s); }

}  // namespace samo
