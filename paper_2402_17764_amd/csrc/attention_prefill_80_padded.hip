// The prefill attention kernels for heads of 66 to 80 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(3, 5, false)
}
