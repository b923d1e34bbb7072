// Attention over sequences with a learned bias, bf16 rows (one translation unit per storage type: they compile in parallel).
#include "seq_attn.h"

namespace dlrm {
template int launch_seq_fwd<DLRM_BF16, true>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
template int launch_seq_bwd<DLRM_BF16, true>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
}  // namespace dlrm
