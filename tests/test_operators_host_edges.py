"""Refusals and defaults at the borders of what the operators on the caller's own device memory take; host only, no address is followed."""

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
