// The prefill attention kernels for heads of 82 to 94 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(3, 6, false)
}
