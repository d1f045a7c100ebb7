// The prefill attention kernels for heads of 2 to 16 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(1, 1, false)
}
