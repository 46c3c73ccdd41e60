// kvb_conv_backward for bf16 inputs.
#include "kvb_conv_grad_kernel.h"

namespace kvb_impl {

template void launch_conv_grad_typed<bf16_t>(int, const ConvGradArgs &, int64_t, float *, float *, float *, float *, hipStream_t);

}  // namespace kvb_impl
