// The prefill attention kernels for heads of 98 to 112 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(4, 7, false)
}
