// The prefill attention kernels for heads of 130 to 190 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
template hipError_t launch_prefill<6, 12, false>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t);
}
