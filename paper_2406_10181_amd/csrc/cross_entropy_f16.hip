// The cross entropy's products in f16.
#include "cross_entropy_products.h"

namespace lsp {
template hipError_t launch_loss_logits<F16>(const LossArgs& a, hipStream_t st);
template hipError_t launch_loss_back<F16>(const LossArgs& a, hipStream_t st);
}  // namespace lsp
