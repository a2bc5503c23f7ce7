// The attention kernels of one storage type: backward pass.
#include "attention_backward.h"

namespace lsp {
template hipError_t attention_backward_of<F32>(const AttentionArgs& a, hipStream_t st);
}
