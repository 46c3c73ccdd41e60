// kvb_scan for fp32 inputs.
#include "kvb_scan_kernel.h"

namespace kvb_impl {

template void launch_scan_typed<float, float>(int d, const ScanArgs &a, hipStream_t stream);

}  // namespace kvb_impl
