// kvb_scan_backward for fp32 inputs.
#include "kvb_scan_grad_kernel.h"

namespace kvb_impl {

template void launch_scan_grad_typed<float, float>(int d, const GradArgs &a, hipStream_t stream);

}  // namespace kvb_impl
