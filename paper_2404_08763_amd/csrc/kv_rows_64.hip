// Attention over the cache, few rows of each sequence, heads of 64 columns.
#include "kv_rows.hpp"

namespace cats {
template hipError_t launch_kv_rows_attention<64>(const KvAttentionArgs& a, int qt, bool bf16, hipStream_t s);
}  // namespace cats
