// The cross entropy's products in bf16.
#include "cross_entropy_products.h"

namespace lsp {
template hipError_t launch_loss_logits<BF16>(const LossArgs& a, hipStream_t st);
template hipError_t launch_loss_back<BF16>(const LossArgs& a, hipStream_t st);
}  // namespace lsp
