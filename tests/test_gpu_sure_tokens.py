"""Rows whose target has nearly all of the probability: log-probabilities near 0 and gradients 1 - p of the target, each to a share of itself,
on the GPU against oracle/losses.py.

Tolerances.  u = 2^-24.  1 - p is the share of the other tokens in the row's sum.  Each of their exponentials is off by u (2 |z - top| + 2) (the
subtraction, the product with log2(e), the exponential), a vector's sum of eight by 3 u, all else is in 64 bits; as fp32 numbers the share and the
factors around it add 8 u.  So 1 - p, and by it log p, is off by  r = u (2 D + 14)  of itself, D the mean of |z - top| over the others by their
probabilities."""
import numpy as np
import pytest

from oracle import losses as L
from test_gpu_token_loss import HALF, U, Case, dev, host, scratch

pytestmark = pytest.mark.gpu

SHAPES = [(5, 2, 0, 1), (6, 33, 0, 0), (6, 257, 3, 1), (9, 4099, 5, 0), (7, 8192, 0, 0), (7, 32003, 61, 3), (5, 50432, 0, 0), (3, 131073, 0, 1)]


def sure(dtype, shape):
    k = Case(dtype, *shape)
    rows, vocab = k.rows, k.vocab
    # targets in the first and last places, beside the aligned part and inside; 9 to 17 above the rest's largest
    k.targets[:] = [[0, vocab - 1, vocab // 2, min(7, vocab - 1), max(vocab - 5, 0)][r % 5] for r in range(rows)]
    for r in range(rows):
        rest = np.delete(k.z[r].double().numpy(), k.targets[r])
        k.z[r, k.targets[r]] = float(rest.max() + 9 + 8 * r / rows)
    if vocab > 40:
        k.z[rows - 1] = -float("inf")
        k.z[rows - 1, k.targets[rows - 1]] = 2.5  # nothing else: log p = 0, no gradient
    k.place()
    logp, lse, far = np.zeros(rows), np.zeros(rows), np.zeros(rows)
    miss = np.zeros(rows)
    for r in range(rows):
        x, t = k.z64[r], k.targets[r]
        others = np.exp(np.delete(x, t) - x[t])
        rest = others.sum()
        logp[r], lse[r], miss[r] = -np.log1p(rest), x[t] + np.log1p(rest), rest / (1 + rest)
        fine = others > 0
        far[r] = (others[fine] * (x[t] - np.delete(x, t)[fine])).sum() / rest if rest else 0.0
    assert miss.max() < 0.1 and miss[miss > 0].min() < 1e-2
    return k, logp, lse, miss, U * (2 * far + 14)


def at_targets(g, k):
    return g[np.arange(k.rows), k.targets]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "r%d_v%d_p%d_s%d" % s)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_sure_tokens(dtype, shape):
    import torch
    import paper_2401_10241_amd as zb
    k, want, lse, miss, r = sure(dtype, shape)
    rows = k.rows
    logp = torch.zeros(rows, device="cuda")
    zb.token_logprobs(k.x(), logp.data_ptr())
    assert (np.abs(host(logp) - want) <= (r + U) * np.abs(want)).all(), "log-probabilities"
    old, adv = want.astype(np.float32), np.linspace(-1, 2, rows).astype(np.float32)
    loss, ws = torch.zeros(1, device="cuda"), scratch(rows, 1)
    keep = [dev(a) for a in (old, adv)]
    zb.policy_loss(k.x(), zb.policy(keep[0].data_ptr(), keep[1].data_ptr()), loss.data_ptr(), logp.data_ptr(), k.dflat[k.shift:].data_ptr(),
                   workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    assert (np.abs(host(logp) - want) <= (r + U) * np.abs(want)).all(), "log-probabilities of the policy"
    c = -adv.astype(np.float64) * np.exp(want - old)
    tol = lambda c, extra: np.abs(c) * miss * (r + extra + 4 * U + HALF[dtype])  # noqa: E731  extra: of c, relative
    g = at_targets(k.gradient(), k)
    assert (np.abs(g - c * miss) <= tol(c, r * np.abs(want)) + 1e-38).all(), np.abs(g - c * miss) / (np.abs(c) * miss)
    off, ref = np.array([0, rows // 2, rows], np.int32), (want - 0.1).astype(np.float32)
    keep = [dev(a) for a in (off, ref)]
    zb.preference_loss(k.x(), zb.preference(keep[1].data_ptr(), keep[0].data_ptr(), 1, beta=0.5), loss.data_ptr(), logp.data_ptr(), 0,
                       k.dflat[k.shift:].data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    assert (np.abs(host(logp) - want) <= (r + U) * np.abs(want)).all(), "log-probabilities of the preference"
    gap = want - ref
    x = 0.5 * (gap[:rows // 2].sum() - gap[rows // 2:].sum())
    slope = -0.5 / (1 + np.exp(x))
    c = np.where(np.arange(rows) < rows // 2, slope, -slope)
    g = at_targets(k.gradient(), k)
    assert (np.abs(g - c * miss) <= tol(c, 0.5 * (r * np.abs(want)).sum()) + 1e-38).all(), np.abs(g - c * miss) / (np.abs(c) * miss)


def test_targets_among_equals():
    """All logits alike: exponentials, sums and 1 / V's numerator are exact, so a target's entry c (1 - 1 / V) carries three roundings and p's own, u / V:
    of 1 - p, of c and of their product."""
    import torch
    import paper_2401_10241_amd as zb
    rng = np.random.default_rng(21)
    rows, worst = 96, 0.0
    for vocab in (3, 5, 7, 11, 41, 100, 333, 1003, 5001, 40009):
        k = Case("fp32", rows, vocab)
        k.z[:] = 0.75
        k.place()
        want = -np.log(vocab)
        old, adv = np.full(rows, want, np.float32), rng.uniform(0.1, 1.9, rows).astype(np.float32)
        loss, ws = torch.zeros(1, device="cuda"), scratch(rows, rows // 2)
        keep = [dev(a) for a in (old, adv, np.arange(rows + 1, dtype=np.int32), (want - adv).astype(np.float32))]
        o, a, off, ref = (t.data_ptr() for t in keep)
        space = dict(workspace=ws.data_ptr(), workspace_bytes=ws.numel())
        zb.policy_loss(k.x(), zb.policy(o, a), loss.data_ptr(), 0, k.dflat.data_ptr(), **space)
        c = -adv.astype(np.float64) * np.exp(want - old.astype(np.float64))
        cases = [(at_targets(k.gradient(), k), c)]
        zb.preference_loss(k.x(), zb.preference(ref, off, rows // 2, beta=0.7), loss.data_ptr(), 0, 0, k.dflat.data_ptr(), **space)
        gap = want - (want - adv).astype(np.float32).astype(np.float64)
        slope = -0.7 / (1 + np.exp(0.7 * (gap[0::2] - gap[1::2])))
        cases.append((at_targets(k.gradient(), k), np.stack([slope, -slope], 1).reshape(-1)))
        for got, c in cases:
            off_by = np.abs(got / (c * (1 - 1 / vocab)) - 1)
            assert (off_by <= U * (3 + 2 / vocab) + 1e-10).all(), (vocab, off_by.max() / U)  # 1e-10: the series behind c
