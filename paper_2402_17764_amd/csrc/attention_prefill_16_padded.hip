// The prefill attention kernels for heads of 2 to 16 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
template hipError_t launch_prefill<1, 1, false>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t);
}
