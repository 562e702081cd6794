// Attention of prompt chunks: the tiles of heads padded to 96 values.
#include "attn_prefill_kernel.h"

namespace ssm {
SSM_ATTN_PREFILL_BF16(96)
SSM_ATTN_PREFILL_F32(96)
}  // namespace ssm
