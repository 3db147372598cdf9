"""Losses on the log-probabilities of given tokens (test infrastructure), in fp64 with numpy.

logits z [rows, vocab], targets t:  lse_r = log sum_j exp(z_rj),  logp_r = z_r,t(r) - lse_r.  A row counts if its target
lies in [0, vocab) and its weight is not zero; the others have logp 0 and no gradient, whatever they hold.

 * clipped policy loss with a KL term: rho = exp(logp - old), d = ref - logp,
   loss = scale * sum w (-min(rho A, clip(rho, 1 - low, 1 + high) A) + kl (exp(d) - d - 1));
 * preference loss: S_q = sum of w (logp - ref) over sequence q's rows, x = beta (S_2i - S_2i+1),
   loss = scale * sum_i -(1 - eps) log sigma(x) - eps log sigma(-x).

Both gradients are written out by the chain rule through c_r = d loss / d logp_r:
d loss / d z_rj = c_r ([j = t(r)] - exp(z_rj - lse_r)).  tests/test_oracle_losses.py pins them to differences.  `LossStageOracle`
puts them behind a last stage's layers."""
import numpy as np

from .endstages import EndStageOracle
from .layers import layernorm_bwd_input, layernorm_fwd
from .stage import StageOracle


def counting(targets, vocab, weight=None, offsets=None):
    t = np.asarray(targets)
    on = (t >= 0) & (t < vocab)
    if weight is not None:
        on &= np.asarray(weight) != 0
    if offsets is not None:
        r = np.arange(t.size)
        on &= (r >= offsets[0]) & (r < offsets[-1]) if len(offsets) > 1 else np.zeros(t.size, bool)
    return on


def logprobs(z, targets, on=None):
    """(logp, lse) of the rows; 0 where `on` is false."""
    rows, vocab = z.shape
    on = counting(targets, vocab) if on is None else on
    logp, lse = np.zeros(rows), np.zeros(rows)
    for r in np.flatnonzero(on):
        x = np.asarray(z[r], np.float64)
        top = x.max()
        with np.errstate(all="ignore"):
            lse[r] = top + np.log(np.exp(x - top).sum())
            logp[r] = x[targets[r]] - lse[r]
    return logp, lse


def dlogits(z, targets, lse, coef, on):
    out = np.zeros(z.shape)
    for r in np.flatnonzero(on & (coef != 0)):
        out[r] = -coef[r] * np.exp(np.asarray(z[r], np.float64) - lse[r])
        out[r, targets[r]] += coef[r]
    return out


def policy(z, targets, old, advantage, ref=None, weight=None, low=0.2, high=0.2, kl=0.0, scale=1.0):
    """(loss, logp, c, dlogits)."""
    on = counting(targets, z.shape[1], weight)
    logp, lse = logprobs(z, targets, on)
    loss, c = 0.0, np.zeros(len(targets))
    for r in np.flatnonzero(on):
        w = scale * (1.0 if weight is None else float(weight[r]))
        a, rho = float(advantage[r]), np.exp(logp[r] - float(old[r]))
        plain, held = rho * a, min(max(rho, 1 - low), 1 + high) * a
        loss -= w * min(plain, held)
        if plain <= held:  # the smaller term passes its gradient; inside the interval the two are one
            c[r] -= w * plain
        if kl:
            d = float(ref[r]) - logp[r]
            loss += w * kl * (np.expm1(d) - d)
            c[r] -= w * kl * np.expm1(d)
    return loss, logp, c, dlogits(z, targets, lse, c, on)


def preference(z, targets, ref, offsets, weight=None, beta=0.1, eps=0.0, scale=1.0):
    """(loss, logp, rewards, c, dlogits)."""
    on = counting(targets, z.shape[1], weight, offsets)
    logp, lse = logprobs(z, targets, on)
    w = np.where(on, 1.0 if weight is None else np.asarray(weight, np.float64), 0.0)
    gap = np.where(on, w * (logp - np.where(on, np.asarray(ref, np.float64), 0.0)), 0.0)
    sums = np.array([gap[a:b].sum() for a, b in zip(offsets[:-1], offsets[1:])])
    loss, c = 0.0, np.zeros(len(targets))
    for i in range(len(sums) // 2):
        x = beta * (sums[2 * i] - sums[2 * i + 1])
        for share, y in ((1 - eps, -x), (eps, x)):  # (a share of 0 takes nothing of an infinite term)
            loss += scale * share * np.logaddexp(0, y) if share else 0.0
        slope = scale * beta * (eps * np.exp(-np.logaddexp(0, -x)) - (1 - eps) * np.exp(-np.logaddexp(0, x)))
        for q, sign in ((2 * i, 1), (2 * i + 1, -1)):
            c[offsets[q]:offsets[q + 1]] = sign * slope * w[offsets[q]:offsets[q + 1]]
    return loss, logp, beta * sums, c, dlogits(z, targets, lse, c, on)


class LossStageOracle(EndStageOracle):
    """Last stage with one of the two losses: LOSS of a microbatch is the mean over its tokens (policy) or pairs (preference,
    samples 2i and 2i + 1, the preferred one first); B starts from the gradient of the mean over the m microbatches."""

    def __init__(self, *, kind, low=0.2, high=0.2, kl=0.0, beta=0.1, eps=0.0, **kw):
        assert kind in ("policy", "preference")
        self.kind, self.low, self.high, self.kl, self.beta, self.eps = kind, low, high, kl, beta, eps
        super().__init__(role="last", **kw)

    def begin_iteration(self, m):
        super().begin_iteration(m)
        self.values, self.logp, self.rewards = {}, {}, {}

    def set_values(self, mb, **values):
        """weight, ref and, for a policy, old and advantage."""
        self.values[mb] = values

    def forward(self, mb):
        StageOracle.forward(self, mb)
        ex, v, t = self.work_extra, self.values[mb], self.targets[mb]
        Z, xhat, r = layernorm_fwd(np.asarray(self.Y[mb], np.float64), ex["lnf_g"], ex["lnf_b"], self.ln_eps)
        z = Z @ ex["w_head"]
        if self.kind == "policy":
            self.loss[mb], self.logp[mb], _, d = policy(z, t, v["old"], v["advantage"], v["ref"], v["weight"], self.low, self.high, self.kl, 1.0 / t.size)
        else:
            off = np.arange(self.b + 1) * self.s
            self.loss[mb], self.logp[mb], self.rewards[mb], _, d = preference(z, t, v["ref"], off, v["weight"], self.beta, self.eps, 2.0 / self.b)
        self._head[mb] = (d / self.m, Z, xhat, r)

    def backward_input(self, mb):
        ex = self.work_extra
        d, Z, xhat, r = self._head.pop(mb)
        self._head_w[mb] = dict(Z=Z, dlogits=d)
        self.dY[mb], dg, db = layernorm_bwd_input(d @ ex["w_head"].T, xhat, r, ex["lnf_g"])
        self.grads[self.nl]["lnf_g"] += dg
        self.grads[self.nl]["lnf_b"] += db
        StageOracle.backward_input(self, mb)
