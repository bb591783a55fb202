// The parts of the losses' gradients added up.
#include "loss_grads.hpp"

namespace kb {

template <class T>
void join(bool bf16, const LossJoinArgs& a, const int32_t* inv, int N, hipStream_t st) {
  const int zero = inv ? (N < 256 ? N : 256) : 0;
  const dim3 gr(a.mt * a.ntn * T::MB * T::NB * 4 + zero), th(1024);
  if (bf16)
    loss_join<T, __bf16><<<gr, th, 0, st>>>(a, inv, N, zero);
  else
    loss_join<T, float><<<gr, th, 0, st>>>(a, inv, N, zero);
}

hipError_t launch_loss_join(bool bf16, const LossJoinArgs& a, const int32_t* inv, int N, hipStream_t st) {
  switch (a.BNt) {
    case 256: join<LossT256>(bf16, a, inv, N, st); break;
    case 128: join<LossT128>(bf16, a, inv, N, st); break;
    case 64: join<LossT64>(bf16, a, inv, N, st); break;
    default: join<LossT32>(bf16, a, inv, N, st); break;
  }
  return hipGetLastError();
}

}  // namespace kb
