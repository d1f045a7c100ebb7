// The prefill attention kernels for heads of 128 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
BITNET_PREFILL_UNIT(4, 8, true)
}
