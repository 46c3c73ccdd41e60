// kvb_scan for fp16 inputs.
#include "kvb_scan_kernel.h"

namespace kvb_impl {

template void launch_scan_typed<f16_t, float>(int d, const ScanArgs &a, hipStream_t stream);
template void launch_scan_typed<f16_t, f16_t>(int d, const ScanArgs &a, hipStream_t stream);

}  // namespace kvb_impl
