// The prefill attention kernels for heads of 96 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(3, 6, true)
}
