// kvb_conv_backward for f16 inputs.
#include "kvb_conv_grad_kernel.h"

namespace kvb_impl {

template void launch_conv_grad_typed<f16_t>(int, const ConvGradArgs &, int64_t, float *, float *, float *, float *, hipStream_t);

}  // namespace kvb_impl
