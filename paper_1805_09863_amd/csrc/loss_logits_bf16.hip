// Logits of the losses, bf16 operands.
#include "loss_logits.hpp"

namespace kb {
hipError_t launch_loss_logits_bf16(int planes, int BN, const LossLogitsArgs& a, int blocks, hipStream_t st) {
  switch (planes) {
    case 0: return launch_loss_logits_p<1, 0>(BN, a, blocks, st);
    case 1: return launch_loss_logits_p<1, 1>(BN, a, blocks, st);
    default: return launch_loss_logits_p<1, 2>(BN, a, blocks, st);
  }
}
}  // namespace kb
