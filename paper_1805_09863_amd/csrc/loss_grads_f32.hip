// Gradients of the losses, float32 operands in three bf16 pieces.
#include "loss_grads.hpp"

namespace kb {
hipError_t launch_loss_dh_f32(int BN, const LossGradArgs& a, hipStream_t st) { return launch_loss_dh_p<6>(BN, a, st); }
hipError_t launch_loss_dw_f32(int, int BNh, const LossGradArgs& a, hipStream_t st) { return launch_loss_dw_p<6>(BNh, a, st); }
hipError_t launch_loss_both_f32(int BN, const LossGradArgs& h, const LossGradArgs& w, hipStream_t st) {
  return launch_loss_both_p<6>(BN, h, w, st);
}
}  // namespace kb
