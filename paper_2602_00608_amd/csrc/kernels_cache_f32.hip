// The f32 kernels of attention to a cache in four bits (see kernels_cache.hip).
#include "cache_device.hpp"

namespace wmdec {
template int cache_attention_launch<float>(const CacheLaunch&, hipStream_t);
}  // namespace wmdec
