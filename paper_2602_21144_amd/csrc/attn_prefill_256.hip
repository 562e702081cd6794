// Attention of prompt chunks: the tiles of heads padded to 256 values.
#include "attn_prefill_kernel.h"

namespace ssm {
SSM_ATTN_PREFILL_BF16(256)
SSM_ATTN_PREFILL_F32(256)
}  // namespace ssm
