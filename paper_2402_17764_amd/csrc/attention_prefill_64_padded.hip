// The prefill attention kernels for heads of 50 to 62 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(2, 4, false)
}
