// Attention over the cache, many rows of each sequence, heads of 64 columns.
#include "kv_prompt.hpp"

namespace cats {
template hipError_t launch_kv_prompt_attention<64>(const KvAttentionArgs& a, bool bf16, hipStream_t s);
}  // namespace cats
