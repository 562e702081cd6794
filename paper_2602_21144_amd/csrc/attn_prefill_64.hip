// Attention of prompt chunks: the tiles of heads padded to 64 values.
#include "attn_prefill_kernel.h"

namespace ssm {
SSM_ATTN_PREFILL_BF16(64)
SSM_ATTN_PREFILL_F32(64)
}  // namespace ssm
