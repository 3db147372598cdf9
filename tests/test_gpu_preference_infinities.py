"""Preference loss of pairs in which a token that counts has the log-probability -infinity, on the GPU against oracle/losses.py.

Such a pair's difference x is infinite: -log sigma(+infinity) is 0, and a share of 0 (no label smoothing, or nothing but) takes
nothing of the other, infinite term.  Tolerances: those of tests/test_gpu_token_loss.py."""
import numpy as np
import pytest

from oracle import losses as L
from test_gpu_token_loss import U, Case, dev, host, scratch

pytestmark = pytest.mark.gpu

BETA, SCALE = 0.5, 0.25


@pytest.mark.parametrize("eps", [0.0, 0.1, 1.0])
@pytest.mark.parametrize("ruled_out", ["rejected", "chosen"])
@pytest.mark.parametrize("vocab", [100, 32003])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_pair_with_a_token_ruled_out(dtype, vocab, ruled_out, eps):
    import torch
    import paper_2401_10241_amd as zb
    k = Case(dtype, 14, vocab)
    off = np.array([0, 3, 7, 9, 14], np.int32)
    row = 4 if ruled_out == "rejected" else 1  # of the first pair; the second is an ordinary one
    k.targets[row] = 17
    k.z[row, 17] = -float("inf")
    k.place()
    lp, lse = L.logprobs(k.z64, k.targets)
    assert lp[row] == -np.inf and np.isfinite(np.delete(lp, row)).all()
    ref = (np.where(np.isfinite(lp), lp, -9.0) + k.rng.normal(0, 0.4, 14)).astype(np.float32)
    keep = dev(ref), dev(off)
    loss, rewards, ws = torch.zeros(1, device="cuda"), torch.zeros(4, device="cuda"), scratch(14, 2)
    zb.preference_loss(k.x(), zb.preference(keep[0].data_ptr(), keep[1].data_ptr(), 2, beta=BETA, label_smoothing=eps, scale=SCALE), loss.data_ptr(), 0,
                       rewards.data_ptr(), k.dflat.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    wl, _, wr, c, d = L.preference(k.z64, k.targets, ref, off, None, BETA, eps, SCALE)
    on = np.ones(14, bool)
    e, _ = k.error(on)
    bad = int(ruled_out == "rejected")
    got = host(rewards)
    assert got[bad] == wr[bad] == -np.inf
    es = np.array([e[a:b].sum() for a, b in zip(off[:-1], off[1:])])
    keep_q = np.arange(4) != bad
    assert (np.abs(got[keep_q] - wr[keep_q]) <= BETA * es[keep_q] + U * np.abs(wr[keep_q])).all()
    finite = eps == 0 if ruled_out == "rejected" else eps == 1
    assert np.isfinite(wl) == finite
    dx = BETA * (es[2] + es[3])  # of the ordinary pair; the other's loss and slope do not move
    if finite:
        assert abs(host(loss)[0] - wl) <= SCALE * dx + 2 * U * abs(wl)
    else:
        assert host(loss)[0] == wl == np.inf
    slope = np.where(np.arange(14) >= 7, SCALE * BETA / 4 * dx, 0.0) / e
    k.check_gradient(k.gradient(), d, lse, on, c, slope)
