// Attention over the cache, many rows of each sequence, heads of 128 columns.
#include "kv_prompt.hpp"

namespace cats {
template hipError_t launch_kv_prompt_attention<128>(const KvAttentionArgs& a, bool bf16, hipStream_t s);
}  // namespace cats
