"""Pins of oracle/losses.py and oracle/adamw_many.py: differences, closed forms, statistics of the rounding."""
import numpy as np
import pytest

from oracle import adamw_many as A
from oracle import losses as L


def _rows(rng, rows, vocab):
    z = rng.normal(0, 2, (rows, vocab))
    return z, rng.integers(0, vocab, rows)


def _differences(f, z, at, h=1e-5):
    out = []
    for r, j in at:
        a, b = z.copy(), z.copy()
        a[r, j] += h
        b[r, j] -= h
        out.append((f(a) - f(b)) / (2 * h))
    return np.array(out)


@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_gradient_against_differences(kl):
    rng = np.random.default_rng(5)
    z, t = _rows(rng, 9, 11)
    logp, _ = L.logprobs(z, t)
    # ratios on both sides of the interval and inside it, none within 0.05 of a border
    old = logp - np.log(np.array([0.5, 0.9, 1.0, 1.1, 1.6, 0.5, 0.9, 1.1, 1.6]))
    adv = np.array([1.0, 0.7, -0.4, 1.2, 0.9, -1.1, -0.6, -0.8, -0.5])
    ref = logp + rng.normal(0, 0.4, 9)
    w = rng.uniform(0.2, 2, 9)
    w[3] = 0
    t[7] = -1
    f = lambda x: L.policy(x, t, old, adv, ref, w, 0.2, 0.3, kl, 0.7)[0]  # noqa: E731
    _, lp, c, d = L.policy(z, t, old, adv, ref, w, 0.2, 0.3, kl, 0.7)
    at = [(r, j) for r in range(9) for j in (0, 5, max(t[r], 0))]
    assert np.allclose(_differences(f, z, at), [d[r, j] for r, j in at], rtol=1e-6, atol=1e-8)
    assert not d[3].any() and not d[7].any() and lp[7] == 0
    if not kl:  # a clipped gain passes nothing, a clipped loss everything
        assert c[4] == 0 and c[5] == 0 and c[0] != 0 and c[8] != 0
    assert np.allclose(d.sum(axis=1), 0, atol=1e-12)


def test_preference_gradient_against_differences_and_closed_forms():
    rng = np.random.default_rng(6)
    z, t = _rows(rng, 12, 7)
    off = np.array([1, 4, 6, 6, 10])  # row 0 and rows 10, 11 belong to no sequence; sequence 2 is empty
    ref = L.logprobs(z, t)[0] + rng.normal(0, 1, 12)
    w = rng.uniform(0.5, 1.5, 12)
    w[2] = 0
    f = lambda x: L.preference(x, t, ref, off, w, 0.6, 0.1, 0.5)[0]  # noqa: E731
    _, _, rewards, c, d = L.preference(z, t, ref, off, w, 0.6, 0.1, 0.5)
    at = [(r, j) for r in range(12) for j in (0, 3, t[r])]
    assert np.allclose(_differences(f, z, at), [d[r, j] for r, j in at], rtol=1e-6, atol=1e-9)
    assert rewards[2] == 0 and not d[[0, 2, 10, 11]].any()
    # the policy equal to the reference: log 2 for each pair
    lp = L.logprobs(z, t)[0]
    assert np.isclose(L.preference(z, t, lp, off)[0], 2 * np.log(2))


def test_eight_bit_rounding_keeps_the_mean_and_the_codes():
    rng = np.random.default_rng(7)
    n = 700
    m, v = rng.normal(0, 1e-3, n), rng.normal(0, 1e-3, n) ** 2
    places = np.arange(n) + 12345
    sums = [np.zeros(n), np.zeros(n)]
    steps = 3000
    for t in range(1, steps + 1):
        um, uv = A.numbers(places, t, 99)
        for k, (x, most, power, least, u) in enumerate(((m, 127, 2, 0, um), (v, 255, 4, 1, uv))):
            c, top = A.encode(x, most, power, least, u)
            sums[k] += A.decode(c, top, most, power)
    for x, s, most, power, skip in ((m, sums[0], 127, 2, 0), (v, sums[1], 255, 4, 1)):
        top = np.repeat(np.abs(A._blocks(x)).max(axis=1), A.BLOCK)[:n]
        c = np.floor((np.abs(x) / top) ** (1 / power) * most)
        gap = (((c + 1) / most) ** power - (c / most) ** power) * top
        free = c >= skip  # (a v below its first code is held at that code)
        # a mean of `steps` two-valued numbers: standard deviation at most gap / (2 sqrt(steps)); 6 of them
        assert (np.abs(s / steps - x)[free] <= 6 * gap[free] / (2 * np.sqrt(steps)) + 1e-7 * top[free]).all()
    # values that are codes stay what they are (u above 1e-9 of the way and below 1 - 1e-9)
    c, top = A.encode(m, 127, 2, 0, np.full(n, 0.5))
    again, top2 = A.encode(A.decode(c, top, 127, 2), 127, 2, 0, np.full(n, 0.5))
    assert np.array_equal(c, again) and np.allclose(top, top2, rtol=1e-7)
    um, uv = A.numbers(np.arange(1 << 16), 3, 4)
    for u in (um, uv):
        assert 0 < u.min() and u.max() < 1 and abs(u.mean() - 0.5) < 6 * 0.289 / 256
    assert abs(np.corrcoef(um, uv)[0, 1]) < 6 / 256 and abs(np.corrcoef(um[1:], um[:-1])[0, 1]) < 6 / 256


def test_adamw_step_is_the_stages_step():
    from oracle import optimizer as O
    rng = np.random.default_rng(8)
    n = 50
    st = O.AdamState(rng.normal(size=n), rng.normal(size=n) * 0.1, rng.uniform(size=n) * 0.01, 4)
    th, m, v = st.theta.copy(), st.m.copy(), st.v.copy()
    g = rng.normal(size=n)
    hp = O.Hyper(lr=1e-3)
    O.adamw_step(st, g, hp)
    got = A.step(th, g, m, v, 5, lr=1e-3, beta1=hp.beta1, beta2=hp.beta2, eps=hp.eps, decay=hp.weight_decay, coef=1.0)
    for a, b in zip(got, (st.theta, st.m, st.v)):
        assert np.allclose(a, b, rtol=1e-12, atol=0)


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_loss_stage_gradients_against_differences(kind):
    """The head's, the final LayerNorm's and the input's gradients of the mean loss over two microbatches."""
    import zb_inputs
    w = zb_inputs.Workload("loss", "fp32", 1, 16, 2, 32, 5, 2, 2, 1, 2, "H1", seed=5)
    vocab, m = 13, 2
    rng = np.random.default_rng(9)
    X = [rng.normal(size=(10, 16)) for _ in range(m)]
    t = [rng.integers(0, vocab, 10) for _ in range(m)]
    weight = [rng.uniform(0.5, 1.5, 10) * (np.arange(10) != 3) for _ in range(m)]
    shift = [np.resize([0.0, 0.6, -0.7, 0.05], 10) for _ in range(m)]   # ratios far from the borders
    ref, adv = [rng.normal(0, 0.3, 10) for _ in range(m)], [rng.normal(size=10) for _ in range(m)]
    base = zb_inputs.end_stage_params(w, "last", vocab)
    base["w_head"] = base["w_head"] * 30
    params, logp0 = zb_inputs.stage_params(w), {}

    def run(extra, x0, backward=False):
        o = L.LossStageOracle(kind=kind, low=0.2, high=0.3, kl=0.1, beta=0.4, eps=0.1, vocab=vocab, extra_params=extra, layers=1, hidden=16, heads=2,
                              ffn=32, seq=5, mb_size=2, dtype="fp32", params=params)
        o.begin_iteration(m)
        for k in range(m):
            o.set_input(k, x0 if k == 0 else X[k])
            o.set_targets(k, t[k])
            lp = logp0.get(k, np.zeros(10))
            o.set_values(k, weight=weight[k], old=lp + shift[k], advantage=adv[k], ref=lp + ref[k])
            o.forward(k)
        if backward:
            for k in range(m):
                o.backward_input(k)
                o.backward_weight(k)
        return o

    for k, lp in run(base, X[0]).logp.items():
        logp0[k] = lp
    o = run(base, X[0], backward=True)

    def difference(change, h=1e-6):
        return (change(h) - change(-h)) / (2 * h)

    for name, at in (("w_head", (3, 4)), ("w_head", (10, int(t[0][1]))), ("lnf_g", (5,)), ("lnf_b", (2,))):
        def change(h):
            e = {k: v.astype(np.float64).copy() for k, v in base.items()}
            e[name][at] += h
            return run(e, X[0]).iteration_loss()
        assert np.isclose(difference(change), o.grads[o.nl][name][at], rtol=1e-5, atol=1e-9), name
    for at in ((0, 0), (6, 9)):
        def change(h):
            x = X[0].copy()
            x[at] += h
            return run(base, x).iteration_loss()
        assert np.isclose(difference(change), o.dX[0][at], rtol=1e-5, atol=1e-9)
