// Logits of the losses, float32 operands in three bf16 pieces.
#include "loss_logits.hpp"

namespace kb {
hipError_t launch_loss_logits_f32(int planes, int BN, const LossLogitsArgs& a, int blocks, hipStream_t st) {
  return planes == 0 ? launch_loss_logits_p<6, 0>(BN, a, blocks, st) : launch_loss_logits_p<6, 3>(BN, a, blocks, st);
}
}  // namespace kb
