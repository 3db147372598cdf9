"""What 8-bit moments make of values that their codes cannot hold, through the C ABI on the GPU."""
import pytest

from test_gpu_adamw_many import Many

pytestmark = pytest.mark.gpu


def test_moments_that_codes_cannot_hold():
    import torch
    import paper_2401_10241_amd as zb
    q = Many(8, [512], seed=1)
    m, v = torch.full((512,), 0.5, device="cuda"), torch.full((512,), 0.25, device="cuda")
    m[3], m[300], m[301] = float("nan"), float("inf"), -float("inf")
    v[3], v[4], v[5], v[300] = float("nan"), -1.0, 1e-20, float("inf")
    values = zb.adamw_values([(m.data_ptr(), v.data_ptr())])
    zb.adamw_write_moments(q.list, values)
    zb.adamw_read_moments(q.list, values)
    most = torch.finfo(torch.float32).max
    assert m[3] == 0 and m[300] == most and m[301] == -most and m[0] == 0.5 and m[255] == 0.5 and m[256] == 0  # (0.5 beside 3e38)
    assert v[3] == 0 and v[4] == 0 and v[300] == most and v[0] == 0.25
    assert abs(float(v[5]) / (0.25 / 255 ** 4) - 1) <= 2.0 ** -23  # code 1
    assert bool(((v[256:300] / (most / 255.0 ** 4) - 1).abs() <= 2.0 ** -22).all())
