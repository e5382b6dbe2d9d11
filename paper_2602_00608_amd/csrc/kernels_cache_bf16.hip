// The bf16 kernels of attention to a cache in four bits (see kernels_cache.hip).
#include "cache_device.hpp"

namespace wmdec {
template int cache_attention_launch<bf16_t>(const CacheLaunch&, hipStream_t);
}  // namespace wmdec
