// The bf16 kernels of kernels_cross.hip.
#include "cross_device.hpp"

namespace wmdec {
template int cross_launch<bf16_t>(const CrossLaunch&, hipStream_t);
}  // namespace wmdec
