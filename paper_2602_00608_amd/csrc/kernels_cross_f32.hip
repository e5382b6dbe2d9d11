// The fp32 kernels of kernels_cross.hip.
#include "cross_device.hpp"

namespace wmdec {
template int cross_launch<float>(const CrossLaunch&, hipStream_t);
}  // namespace wmdec
