// The prefill attention kernels for heads of 256 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(8, 16, true)
}
