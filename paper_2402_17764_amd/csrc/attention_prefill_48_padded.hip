// The prefill attention kernels for heads of 34 to 48 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(2, 3, false)
}
