// The prefill attention kernels for heads of 64 dims.
#include "attention_prefill_kernel.hpp"

namespace bitnet {
template hipError_t launch_prefill<2, 4, true>(PrefillTile, const PrefillArgs&, const Parts&, const KvView&, bool, hipStream_t);
}
