// Attention over sequences, f32 rows (one translation unit per storage type: they compile in parallel).
#include "seq_attn.h"

namespace dlrm {
template int launch_seq_fwd<DLRM_F32>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
template int launch_seq_bwd<DLRM_F32>(const dlrm_seq_batch*, SeqArgs, hipStream_t);
}  // namespace dlrm
