// The prefill attention kernels for heads of 194 to 254 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(8, 16, false)
}
