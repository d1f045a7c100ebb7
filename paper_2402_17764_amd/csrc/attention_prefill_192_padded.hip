// The prefill attention kernels for heads of 130 to 190 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(6, 12, false)
}
