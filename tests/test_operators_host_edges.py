"""Refusals and defaults at the borders of what the operators on the caller's own device memory take; host only, no address is followed."""

import ctypes as C

import numpy as np
import pytest

import paper_2401_10241_amd as zb
from test_operators_host import AT, rc_of, tensor

TINY, MOST = float(np.finfo(np.float32).tiny), float(np.finfo(np.float32).max)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("bad", [dict(eps=1e-46), dict(eps=TINY / 2), dict(eps=1e39), dict(eps=2 * MOST), dict(weight_decay=1e300), dict(weight_decay=-1e39),
                                 dict(lr=1e39), dict(lr=-1e300)], ids=str)
def test_numbers_that_leave_the_range_of_the_kernels(bits, bad):
    """lr, eps and weight_decay are 32-bit numbers in the kernels: 0 for an eps would give 0 / 0 where a value has had no gradient."""
    k = dict(bad)
    lr = k.pop("lr", 1e-3)
    assert rc_of(zb.adamw_step, zb.adamw_config(bits=bits, **k), zb.adamw_tensors([tensor()]), lr, AT, AT, AT) == zb.EINVAL


@pytest.mark.parametrize("loss", [1, 2])
def test_a_stage_of_more_tokens_than_its_loss_takes(loss):
    """Refused when the stage is set up, not by its first F."""
    def rc(loss, seq, mb_size):
        cfg = zb.binding.zb_config()
        zb.lib.zb_config_defaults(C.byref(cfg))
        for name, value in dict(layers=1, hidden=64, heads=2, ffn=64, seq=seq, mb_size=mb_size, max_microbatches=1, max_pending_b=1, max_pending_w=1,
                                max_inflight=1, role=2, vocab=2, loss=loss).items():
            setattr(cfg, name, value)
        need = C.c_size_t(0)
        return zb.lib.zb_stage_arena_bytes(C.byref(cfg), C.byref(need))

    assert rc(0, 1 << 21, 2) == rc(0, 1 << 12, 1 << 12) == zb.OK
    for seq, mb_size in ((1 << 21, 2), (1 << 12, 1 << 10), (1 << 12, 1 << 12)):
        assert rc(loss, seq, mb_size) == zb.EINVAL
    assert rc(loss, (1 << 21) - 1, 2) == rc(loss, 1 << 11, (1 << 11) - 2) == zb.OK


def test_places_of_tensors_listed_without_one():
    """Each starts where the one before it ends, so that no two share their random numbers; a given place stays as it is."""
    sizes = [1000, 0, 7, 300]
    assert [t.first for t in zb.adamw_tensors([tensor(n=n) for n in sizes])] == [0, 1000, 1000, 1007]
    assert [t.first for t in zb.adamw_tensors([tensor(n=5), tensor(n=5, first=1 << 33), tensor(n=2), tensor(n=2, first=0)])] == [0, 1 << 33, (1 << 33) + 5, 0]
    again = [t.first for t in zb.adamw_tensors([tensor(n=3), tensor(n=4)])]
    assert again == [0, 3]
