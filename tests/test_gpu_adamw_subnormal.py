"""8-bit states of blocks whose largest moment is subnormal in fp32, on the GPU against oracle/adamw_many.py.

Such a scale is rounded to a whole number of 2^-149, up to a third away from the largest value, so values lie past the top code and take it.
Codes and scales are equal, as in tests/test_gpu_adamw_many.py, but for ties: the same gradient g in two steps gives m = (9 k + j) / 10 units where the
scale was k and g is j, half-way between two scales for one j in ten.  The largest value carries roundings of 2^-53 each on either side: of the unit, of
the code's square times it, of beta1 times it, of 1 - beta1 (or of the clip coefficient times it), of that times g, and of the sum; v has one more, of
g^2.  They stay below 8 * 2^-53 of the value on a side, so where it lies within 16 * 2^-53 of half-way between two scales either is right, and the codes
are those of the scale that the device took."""
import numpy as np
import pytest

from oracle import adamw_many as A
from test_gpu_adamw_many import BETA1, BETA2, DECAY, EPS, LR, SEED, Many as AnyTensors

pytestmark = pytest.mark.gpu

ULP = 2.0 ** -149
TOPS = [0.4, 0.6, 1.0, 1.4, 1.5, 2.5, 3.3, 5.4, 7.49, 10.5, 16.4, 31.5, 40.4, 49.5, 127.4, 1000.3, 65537.5, 2.0 ** 23 - 0.6, 2.0 ** 23 + 3]


class Many(AnyTensors):
    def held(self, k, x, name, most, power, least, u):
        """What the device holds of x, compared with the oracle's codes; as values."""
        d, n = self.dev[k], self.sizes[k]
        top = d[name + "_scale"].cpu().numpy()
        assert top[-1] == 55
        top = top[:-1]
        codes, own = A.encode(x, most, power, least, u, top)[0], A.encode(x, most, power, least, u)[1]
        big = np.abs(A._blocks(x)).max(axis=1)
        tie = np.abs(big - (top.astype(np.float64) + own) / 2) <= 16 * 2.0 ** -53 * big
        near = (top == np.nextafter(own, np.float32(0))) | (top == np.nextafter(own, np.float32(1)))
        assert ((top == own) | (tie & near)).all(), f"scales of {name}, tensor {k}"
        assert np.array_equal(self.inner(d[name], n).cpu().numpy(), codes), f"codes of {name}, tensor {k}"
        return A.decode(codes, top, most, power)

    def expect(self, coef):
        self.t += 1
        self.tol = getattr(self, "tol", [np.zeros(n) for n in self.sizes])
        for k, n in enumerate(self.sizes):
            old = self.theta[k].astype(np.float64)
            self.theta[k], m, v = A.step(old, self.g[k], self.m[k], self.v[k], self.t, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                                         decay=DECAY if self.decays[k] else 0.0, coef=coef)
            # theta: moments this far below eps move it by less than 1e-8 lr; the decay's three roundings, the difference's, and lr's and decay's own
            self.tol[k] += 2.0 ** -24 * (2 + 3 * LR * DECAY) * np.abs(old) + 1e-8 * LR + 2.0 ** -20 * np.abs(self.theta[k] - old)
            um, uv = A.numbers(np.arange(n) + self.first[k], self.t, SEED)
            self.m[k], self.v[k] = self.held(k, m, "m", 127, 2, 0, um), self.held(k, v, "v", 255, 4, 1, uv)


def given(q, grads):
    import torch
    q.set_grads()
    for k, g in enumerate(grads):
        g = np.asarray(g, np.float32)
        q.inner(q.dev[k]["grad"], q.sizes[k]).copy_(torch.from_numpy(g))
        q.g[k] = g.astype(np.float64)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("moment", ["m", "v"])
def test_scales_of_few_bits(moment, shift):
    """Blocks whose largest m or v is so many times 2^-149, whole and broken off."""
    rng = np.random.default_rng(11)
    for n in (256 * len(TOPS), 256 * len(TOPS) - 37):
        share = rng.uniform(-1, 1, (len(TOPS), 256))
        share[:, 5] = 1.0
        top = np.array(TOPS)[:, None] * ULP
        g = share * top / (1 - BETA1) if moment == "m" else np.sign(share) * np.sqrt(np.abs(share) * top / (1 - BETA2))
        q = Many(8, [n], seed=n, shift=shift)
        given(q, [g.reshape(-1)[:n]])
        for _ in range(3):
            q.step(float("inf"))
            q.expect(1.0)
        q.check()


def test_moments_that_fade_away():
    """No gradient after the first step: the scales fall through the subnormal numbers to 0."""
    q = Many(8, [300, 300], seed=12)
    rng = np.random.default_rng(13)
    given(q, [rng.uniform(-1e-36, 1e-36, 300), rng.uniform(-1.5e-18, 1.5e-18, 300)])  # m of the one and v of the other near 1e-37
    q.step(float("inf"))
    q.expect(1.0)
    given(q, [np.zeros(300), np.zeros(300)])
    for _ in range(400):
        q.step(float("inf"))
        q.expect(1.0)
    assert not q.dev[0]["m_scale"][:2].any() and float(q.dev[1]["v_scale"][0]) < 100 * ULP
    q.check()
