// The parts of the losses' gradients added up.
#include "loss_grads.hpp"

namespace kb {

template <class T>
void join(bool bf16, const LossJoinArgs& a, const LossJoinMore& more, hipStream_t st) {
  // Fewer than 2^32 threads lie along a grid's axis: workgroups beyond 2^21 (2^21 rows of 1,024 states) in rows of 2^21.
  const int blocks = loss_join_blocks<T>(a.mt * a.ntn) + more.zero_wg + more.db_wg, row = 1 << 21;
  const dim3 gr(blocks < row ? blocks : row, (blocks + row - 1) / row), th(1024);
  if (bf16)
    loss_join<T, __bf16><<<gr, th, 0, st>>>(a, more);
  else
    loss_join<T, float><<<gr, th, 0, st>>>(a, more);
}

hipError_t launch_loss_join(bool bf16, const LossJoinArgs& a, LossJoinMore more, hipStream_t st) {
  more.zero_wg = more.inv ? (more.N < 256 ? more.N : 256) : 0;
  more.db_wg = more.db.db ? (more.db.V + 63) / 64 : 0;
  switch (a.BNt) {
    case 256: join<LossT256>(bf16, a, more, st); break;
    case 192: join<LossT192>(bf16, a, more, st); break;
    case 128: join<LossT128>(bf16, a, more, st); break;
    case 64: join<LossT64>(bf16, a, more, st); break;
    default: join<LossT32>(bf16, a, more, st); break;
  }
  return hipGetLastError();
}

}  // namespace kb
