// Attention of many new items over a paged cache, bf16 rows (one translation unit per storage type: they compile in parallel).
#include "cache_wide.h"

namespace dlrm {
template int launch_cache_wide<DLRM_BF16>(const TreeArgs&, const TreeLaunch&, hipStream_t);
}  // namespace dlrm
