// Attention of prompt chunks: the tiles of heads padded to 192 values.
#include "attn_prefill_kernel.h"

namespace ssm {
SSM_ATTN_PREFILL_BF16(192)
}  // namespace ssm
