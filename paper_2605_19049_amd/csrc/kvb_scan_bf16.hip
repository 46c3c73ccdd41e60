// kvb_scan for bf16 inputs.
#include "kvb_scan_kernel.h"

namespace kvb_impl {

template void launch_scan_typed<bf16_t, float>(int d, const ScanArgs &a, hipStream_t stream);
template void launch_scan_typed<bf16_t, bf16_t>(int d, const ScanArgs &a, hipStream_t stream);

}  // namespace kvb_impl
