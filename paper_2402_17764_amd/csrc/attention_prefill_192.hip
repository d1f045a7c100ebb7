// The prefill attention kernels for heads of 192 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(6, 12, true)
}
