// Attention over the 4-bit paged cache with a window and first tokens that stay visible: the kernels with SINKS.
#include "pop_cache_attention_kernels.h"

namespace pop {

hipError_t launch_attention_sinks(const AttentionArgs &a, const AttentionLaunch &l, hipStream_t s) { return launch_attention_as<true>(a, l, s); }

}  // namespace pop
