// The prefill attention kernels for heads of 18 to 30 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
template hipError_t launch_prefill<1, 2, false>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t);
}
