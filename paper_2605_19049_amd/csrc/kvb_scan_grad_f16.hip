// kvb_scan_backward for fp16 inputs.
#include "kvb_scan_grad_kernel.h"

namespace kvb_impl {

template void launch_scan_grad_typed<f16_t, float>(int d, const GradArgs &a, hipStream_t stream);
template void launch_scan_grad_typed<f16_t, f16_t>(int d, const GradArgs &a, hipStream_t stream);

}  // namespace kvb_impl
