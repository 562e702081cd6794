// Attention of prompt chunks: the tiles of heads padded to 128 values.
#include "attn_prefill_kernel.h"

namespace ssm {
SSM_ATTN_PREFILL_BF16(128)
SSM_ATTN_PREFILL_F32(128)
}  // namespace ssm
