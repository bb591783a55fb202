// Gradients of the losses, bf16 operands.
#include "loss_grads.hpp"

namespace kb {

hipError_t launch_loss_dh_bf16(int BN, const LossGradArgs& a, hipStream_t st) {
  const dim3 gr(a.splits * loss_row_tiles(a.N, BN) * a.mt), th(256);
  switch (BN) {
    case 256: loss_dh<LossT256, 1><<<gr, th, 0, st>>>(a); break;
    case 128: loss_dh<LossT128, 2><<<gr, th, 0, st>>>(a); break;
    case 64: loss_dh<LossT64, 2><<<gr, th, 0, st>>>(a); break;
    default: loss_dh<LossT32, 2><<<gr, th, 0, st>>>(a); break;
  }
  return hipGetLastError();
}

hipError_t launch_loss_dw_bf16(int BNh, const LossGradArgs& a, hipStream_t st) {
  const dim3 gr(a.splits * a.mt * a.ntn), th(256);
  switch (BNh) {
    case 256: loss_dw<LossT256, 1><<<gr, th, 0, st>>>(a); break;
    case 128: loss_dw<LossT128, 1><<<gr, th, 0, st>>>(a); break;
    default: loss_dw<LossT64, 2><<<gr, th, 0, st>>>(a); break;
  }
  return hipGetLastError();
}

// row tiles and state tiles of 256
hipError_t launch_loss_both_bf16(const LossGradArgs& h, const LossGradArgs& w, hipStream_t st) {
  const dim3 gr(h.splits * loss_row_tiles(h.N, 256) * h.mt + w.splits * w.mt * w.ntn), th(256);
  loss_both<LossT256, 1><<<gr, th, 0, st>>>(h, w);
  return hipGetLastError();
}

}  // namespace kb
