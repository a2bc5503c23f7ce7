// The attention kernels of one storage type.
#include "attention_forward.h"

namespace lsp {
template hipError_t attention_forward_of<BF16>(const AttentionArgs& a, hipStream_t st);
}
