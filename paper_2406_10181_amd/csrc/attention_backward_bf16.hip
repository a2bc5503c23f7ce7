// The attention kernels of one storage type: backward pass.
#include "attention_backward.h"

namespace lsp {
template hipError_t attention_backward_of<BF16>(const AttentionArgs& a, hipStream_t st);
}
