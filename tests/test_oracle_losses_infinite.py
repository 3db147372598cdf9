"""oracle/losses.py where a pair's difference is infinite: a share of 0 takes nothing of an infinite term."""
import numpy as np
import pytest

from oracle import losses as L


@pytest.mark.parametrize("eps", [0.0, 0.2, 1.0])
@pytest.mark.parametrize("row", [0, 2])
def test_preference_of_a_pair_with_a_token_ruled_out(row, eps):
    rng = np.random.default_rng(3)
    z, t = rng.normal(0, 2, (4, 9)), np.array([1, 2, 3, 4])
    off, ref = np.array([0, 2, 4]), np.zeros(4)
    z[row, t[row]] = -np.inf
    loss, _, rewards, c, d = L.preference(z, t, ref, off, None, 0.5, eps, 1.0)
    assert rewards[row // 2] == -np.inf
    # x = +infinity where the rejected answer is ruled out: log sigma(x) = 0, log sigma(-x) = -infinity
    share = eps if row == 2 else 1 - eps
    assert loss == (np.inf if share else 0.0)
    # d loss / d S = beta (eps sigma(x) - (1 - eps) sigma(-x))
    want = 0.5 * (eps if row == 2 else -(1 - eps))
    assert np.allclose(c, np.array([want, want, -want, -want]), rtol=0, atol=1e-15) and np.isfinite(d).all()
    # near the limit: a logit of -3000 instead
    z[row, t[row]] = -3000.0
    near = L.preference(z, t, ref, off, None, 0.5, eps, 1.0)
    assert np.allclose(near[3], c, atol=1e-12) and np.allclose(near[4], d, atol=1e-12)
    assert near[0] > 100 if share else near[0] < 1e-12
