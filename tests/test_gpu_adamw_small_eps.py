"""AdamW with an eps far below the roots of the smallest second moments, on the GPU against oracle/adamw_many.py."""
import numpy as np
import pytest

from oracle import adamw_many as A
from test_gpu_adamw_many import BETA1, BETA2, LR, SEED, U, Many

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -149


@pytest.mark.parametrize("eps", [1e-30, 1e-22, 1e-15, 3e-12, 1e-6])
@pytest.mark.parametrize("bits", [32, 8])
def test_second_moments_below_the_normal_numbers(bits, eps):
    """v = 5e-42 to 5e-36 of gradients of 1e-20 to 1e-17: the update is lr times a number near 1 wherever eps is below them.

    v is held in fp32, off by ULP / 2 if it is subnormal and by U v otherwise; so is v / bc2, which is larger.  The root takes half of each; beside
    it the update is off by 24 U (the terms of tests/test_gpu_adamw_many.py, m's among them: gradients of one sign, no cancellation)."""
    import torch
    import paper_2401_10241_amd as zb
    n = 1024
    q = Many(bits, [n], seed=15)
    q.decays = [False]
    q.list = zb.adamw_tensors([q._entry(0)])
    g = np.repeat(np.array([1e-20, 1e-19, 1e-18, 1e-17]), 256).astype(np.float32)
    q.set_grads()
    q.inner(q.dev[0]["grad"], n).copy_(torch.from_numpy(g))
    q.inner(q.dev[0]["theta"], n).zero_()  # so that the difference loses nothing
    config = zb.adamw_config(bits=bits, beta1=BETA1, beta2=BETA2, eps=eps, weight_decay=0.0, clip=float("inf"), seed=SEED)
    zb.adamw_grad_norm(q.list, q.sq.data_ptr(), q.bad.data_ptr(), workspace=q.space.data_ptr(), workspace_bytes=q.space.numel())
    zb.adamw_step(config, q.list, LR, q.clock.data_ptr(), q.sq.data_ptr(), q.bad.data_ptr())
    want, _, v = A.step(np.zeros(n), g.astype(np.float64), np.zeros(n), np.zeros(n), 1, lr=LR, beta1=BETA1, beta2=BETA2, eps=eps, decay=0.0, coef=1.0)
    got = q.inner(q.dev[0]["theta"], n).cpu().double().numpy()
    off = 0.5 * ((np.maximum(ULP / 2, U * v)) / v + np.maximum(ULP / 2, U * v / (1 - BETA2)) / (v / (1 - BETA2)))
    assert (np.abs(got - want) <= np.abs(want) * (off + 24 * U) + ULP).all()
