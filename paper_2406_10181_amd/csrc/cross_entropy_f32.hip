// The cross entropy's products in f32.
#include "cross_entropy_products.h"

namespace lsp {
template hipError_t launch_loss_logits<F32>(const LossArgs& a, hipStream_t st);
template hipError_t launch_loss_back<F32>(const LossArgs& a, hipStream_t st);
}  // namespace lsp
