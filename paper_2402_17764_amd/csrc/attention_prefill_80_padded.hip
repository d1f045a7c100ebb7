// The prefill attention kernels for heads of 66 to 80 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
template hipError_t launch_prefill<3, 5, false>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t);
}
