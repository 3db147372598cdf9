"""What a caller may do with a workspace between calls: everything but its first WORKSPACE_KEPT_BYTES may be overwritten, and calls of
different kinds and sizes may share one."""
import numpy as np
import pytest

from test_gpu_adamw_many import Many
from test_gpu_token_loss import Case, dev, policy_inputs

pytestmark = pytest.mark.gpu


def test_a_workspace_used_for_something_else_between_calls():
    import torch
    import paper_2401_10241_amd as zb
    shared = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")

    def calls(rows, space):
        """Loss, gradient and norm bits of calls on a workspace each, space(bytes) gives it."""
        k = Case("fp32", rows, 300, seed=rows)
        old, ref, adv, _ = policy_inputs(k)
        keep = [dev(a) for a in (old, adv, ref)]
        off = dev(np.array([0, rows // 3, rows // 2, rows // 2, rows], np.int32))
        q = Many(32, [rows * 500, 77], seed=rows)
        q.set_grads()
        out = []
        for _ in range(2):
            loss = torch.full((2,), 77.0, device="cuda")
            k.dflat.fill_(77)
            ws = space(zb.loss_workspace_bytes(rows))
            zb.policy_loss(k.x(), zb.policy(keep[0].data_ptr(), keep[1].data_ptr(), ref_logp=keep[2].data_ptr(), kl_coef=0.1), loss.data_ptr(), 0,
                           k.dflat.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())
            out.append(k.dflat.clone())
            ws = space(zb.loss_workspace_bytes(rows, 2))
            zb.preference_loss(k.x(), zb.preference(keep[2].data_ptr(), off.data_ptr(), 2), loss[1:].data_ptr(), 0, 0, k.dflat.data_ptr(),
                               workspace=ws.data_ptr(), workspace_bytes=ws.numel())
            q.sq.fill_(77)
            ws = space(zb.adamw_workspace_bytes(q.list))
            zb.adamw_grad_norm(q.list, q.sq.data_ptr(), q.bad.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())
            out += [loss, k.dflat.clone(), q.sq.clone(), q.bad.clone()]
        torch.cuda.synchronize()
        return out

    def used(n):
        assert n <= shared.numel()
        shared[zb.WORKSPACE_KEPT_BYTES:].random_(0, 256)
        return shared[:n]

    for rows in (1, 5, 256, 257, 90, 256):
        for a, b in zip(calls(rows, used), calls(rows, lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda"))):
            assert torch.equal(a, b) and not bool((a == 77).all()), rows
