// Attention of many new items over a paged cache, f32 rows (one translation unit per storage type: they compile in parallel).
#include "cache_wide.h"

namespace dlrm {
template int launch_cache_wide<DLRM_F32>(const TreeArgs&, const TreeLaunch&, hipStream_t);
}  // namespace dlrm
