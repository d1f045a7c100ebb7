// The prefill attention kernels for heads of 192 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
template hipError_t launch_prefill<6, 12, true>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t);
}
