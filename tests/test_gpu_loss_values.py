"""Values at which the output layer's losses can go wrong, against the fp64 oracle with its bounds (the bounds of the
gradients are those of test_gpu_loss.py)."""
import math

import numpy as np
import pytest
import torch

import test_gpu_loss as base
from oracle import loss_oracle as lo
from test_gpu_loss import kb  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
f64 = base.f64


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,H,V", base.PATHS)
@pytest.mark.parametrize("smoothing", [2.0 ** -149, 1e-41, 1e-30])
def test_smoothing_of_next_to_nothing(kb, dtype, N, H, V, smoothing):  # noqa: F811
    """smoothing / V is 0 in float32, or the least values there are.  Without words that are left out it makes no
    difference; where the smoothed labels name one, the loss is +inf and the gradient p - q as ever."""
    _, h, W, b, target, grad = base.make(25, dtype, N, H, V)
    target[0], target[1] = 1, -1
    for masked in (False, True):
        if masked:
            b[2] = b[V - 1] = -math.inf
            target[(target == 2) | (target == V - 1)] = 1
        hd, Wd, bd, td, gd = base.dev(h, W, b, target, grad)
        loss, lse = kb.cross_entropy(hd, Wd, bd, td, smoothing=smoothing)
        outs = kb.cross_entropy_grad(hd, Wd, bd, td, lse, gd, smoothing=smoothing)
        o = lo.cross_entropy(f64(h), f64(W), f64(b), target.numpy(), float(np.float32(smoothing)))
        what = f"smoothing {smoothing}, {'with' if masked else 'no'} words left out"
        if masked:
            assert np.isposinf(o.loss[o.used]).all()
            assert np.isposinf(f64(loss)[o.used]).all() and (f64(loss)[~o.used] == 0).all(), what
            o.loss[:] = 0.0  # compared above
            loss = torch.zeros(N)
        bnd = lo.bounds(o, f64(h), f64(W), f64(b), dtype == F32, f64(grad))
        base.check_rows(o, bnd, loss, lse, what)
        base.check_grads(o, bnd, h, W, grad, outs, dtype, what)
