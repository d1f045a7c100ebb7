// The prefill attention kernels for heads of 32 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(1, 2, true)
}
