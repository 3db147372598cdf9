"""The preference loss of a last stage against the oracle's loss itself, and a bound on how far its rewards may move its gradients.

A reward may be off by r = TOL |reward| + TOL BETA sqrt(seq) (as in tests/test_gpu_loss_stage.py: a sum of `seq` differences of
log-probabilities whose errors are independent).  x, the difference of two rewards, is then off by the sum dx of both; the loss by
|slope| dx <= dx times the larger share of the two log-sigmas, and the slope, the factor of every gradient row of the pair, by sigma'(x) dx <= dx / 4."""
import numpy as np
import pytest

from oracle.schedule import stage_order
from test_gpu_loss_stage import BETA, CASES, EPS, W, build, load, slope, values_of
from zb_testlib import TOL

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_L%d_h%d_a%d_f%d_s%d_b%d_V%d_m%d" % c)
def test_preference_loss_and_slope_of_a_stage(case):
    import paper_2401_10241_amd as zb
    dtype, layers, hidden, heads, ffn, seq, b, vocab, m = case
    p = 4
    w = W("loss", dtype, layers, hidden, heads, ffn, seq, b, p, p - 1, m, "H1", seed=81 + hidden, lr=1e-4)
    dev, orc = build(w, "preference", vocab, m)
    orc.begin_iteration(m)
    dev.begin_iteration(0, m)
    load(w, vocab, m, 0, dev, orc)
    for k in range(m):
        orc.forward(k)
    values = values_of(w, m, [orc.logp[k] for k in range(m)], 0)
    orc.begin_iteration(m)
    load(w, vocab, m, 0, dev, orc, values)
    dev.run_schedule(p, p - 1, m, "H1")
    dev.synchronize()
    orc.run(stage_order(p, p - 1, m, "H1"))
    tol = TOL[dtype]
    for k in range(m):
        r, got = orc.rewards[k], dev.get_token_values(zb.T_REWARDS, k)
        off = tol * np.abs(r) + tol * BETA * np.sqrt(seq)
        assert (np.abs(got - r) <= off).all()
        dx = off[0::2] + off[1::2]
        assert abs(dev.get_loss(k) - orc.loss[k]) <= max(EPS, 1 - EPS) * dx.mean() + 2.0 ** -23 * orc.loss[k]
        assert (np.abs(slope(got) - slope(r)) <= dx / 4 + 2.0 ** -22).all()
        print(f"[{dtype} V={vocab}] loss {dev.get_loss(k):.5f} oracle {orc.loss[k]:.5f}, x off by {np.abs((got - r)[0::2] - (got - r)[1::2]).max():.2e} of {dx.min():.2e}")
    dev.close()
