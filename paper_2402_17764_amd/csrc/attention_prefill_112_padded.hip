// The prefill attention kernels for heads of 98 to 112 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
template hipError_t launch_prefill<4, 7, false>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t);
}
