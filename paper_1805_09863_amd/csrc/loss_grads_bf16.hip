// Gradients of the losses, bf16 operands.
#include "loss_grads.hpp"

namespace kb {
hipError_t launch_loss_dh_bf16(int BN, const LossGradArgs& a, hipStream_t st) { return launch_loss_dh_p<1>(BN, a, st); }
hipError_t launch_loss_dw_bf16(int planes, int BNh, const LossGradArgs& a, hipStream_t st) {
  return planes == 1 ? launch_loss_dw_p<1>(BNh, a, st) : launch_loss_dw_p<2>(BNh, a, st);
}
hipError_t launch_loss_both_bf16(int BN, const LossGradArgs& h, const LossGradArgs& w, hipStream_t st) {
  return launch_loss_both_p<1>(BN, h, w, st);
}
}  // namespace kb
