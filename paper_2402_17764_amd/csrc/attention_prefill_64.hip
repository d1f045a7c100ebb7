// The prefill attention kernels for heads of 64 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(2, 4, true)
}
