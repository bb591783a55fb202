// Logits of the losses, bf16 operands.
#include "loss_logits.hpp"

namespace kb {
hipError_t launch_loss_logits_bf16(bool grad, int BN, const LossLogitsArgs& a, int blocks, hipStream_t st) {
  return launch_loss_logits_t<1>(grad, BN, a, blocks, st);
}
}  // namespace kb
