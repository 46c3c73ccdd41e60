// kvb_scan_backward for bf16 inputs.
#include "kvb_scan_grad_kernel.h"

namespace kvb_impl {

template void launch_scan_grad_typed<bf16_t, float>(int d, const GradArgs &a, hipStream_t stream);
template void launch_scan_grad_typed<bf16_t, bf16_t>(int d, const GradArgs &a, hipStream_t stream);

}  // namespace kvb_impl
