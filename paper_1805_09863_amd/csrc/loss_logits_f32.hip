// Logits of the losses, float32 operands in three bf16 pieces.
#include "loss_logits.hpp"

namespace kb {
hipError_t launch_loss_logits_f32(bool grad, int BN, const LossLogitsArgs& a, int blocks, hipStream_t st) {
  return launch_loss_logits_t<6>(grad, BN, a, blocks, st);
}
}  // namespace kb
