"""Token log-probabilities, policy loss and preference loss on the GPU against oracle/losses.py, through the C ABI.

Tolerances.  u = 2^-24.  The device computes exp(x - top) in fp32: the subtraction and the product with log2(e) put
2.5 u |x - top| on the exponent, the exponential itself 4 u, and a sum of K terms K u, so the sum of a row, and by it lse
and logp, is off by at most  e = u (2.5 sum_j p_j |z_j - top| + K + 68), K = vocab / 256 + 1 terms per lane (64 for
rescaling and for joining the lanes).  Storing logp and lse in fp32 adds u of their size.  A coefficient c of a row moves by
|dc/dlogp| e; an entry c ([target] - p) by  |dc| |[target] - p| + |c| p (e + u (2.5 |z - lse| + 6)) + 4 u |c|  and half a step
of the stored type, 2^-8 or 2^-24 of it."""
import numpy as np
import pytest

from oracle import losses as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "fp32": U}
GUARD = 77.0  # what the memory beside a result holds before and after


class Case:
    """Logits in rows of a wider buffer that starts `shift` elements into an allocation, with what the losses need."""

    def __init__(self, dtype, rows, vocab, pad=0, shift=0, seed=0, spread=2.0):
        import torch
        self.rng = np.random.default_rng(1000 * rows + vocab + seed)
        self.dtype, self.rows, self.vocab, self.stride, self.shift = dtype, rows, vocab, vocab + pad, shift
        self.kind = torch.bfloat16 if dtype == "bf16" else torch.float32
        z = torch.from_numpy(self.rng.normal(0, spread, (rows, vocab)).astype(np.float32)).to(self.kind)
        self.targets = self.rng.integers(0, vocab, rows).astype(np.int32)
        self.targets[rows // 2:rows // 2 + 1] = vocab - 1
        self.targets[:1] = 0
        self.z = z
        self.place()

    def place(self):
        """Puts self.z and self.targets on the device; call again after a change of self.z."""
        import torch
        flat = torch.full((self.shift + self.rows * self.stride + 64,), GUARD, dtype=self.kind)
        view = flat[self.shift:self.shift + self.rows * self.stride].view(self.rows, self.stride)
        view[:, :self.vocab] = self.z
        self.flat = flat.cuda()
        self.dflat = torch.full_like(self.flat, GUARD)
        self.t = torch.from_numpy(self.targets).cuda()
        self.z64 = self.z.double().numpy()

    def x(self):
        import paper_2401_10241_amd as zb
        return zb.logits(self.flat[self.shift:].data_ptr(), self.rows, self.vocab, self.t.data_ptr(), dtype=self.dtype,
                         row_stride=self.stride)

    def gradient(self, buf=None):
        """[rows, vocab] in fp64; the rest of the buffer must be as it was."""
        flat = (self.dflat if buf is None else buf).cpu()
        view = flat[self.shift:self.shift + self.rows * self.stride].view(self.rows, self.stride)
        assert (flat[:self.shift] == GUARD).all() and (flat[self.shift + self.rows * self.stride:] == GUARD).all()
        assert (view[:, self.vocab:] == GUARD).all()
        return view[:, :self.vocab].double().numpy()

    def error(self, on):
        """e of the module's first lines, per row; p."""
        e, p = np.zeros(self.rows), np.zeros((self.rows, self.vocab))
        for r in np.flatnonzero(on):
            x = self.z64[r]
            fine = np.isfinite(x)
            p[r][fine] = np.exp(x[fine] - x[fine].max())
            p[r] /= p[r].sum()
            e[r] = U * (2.5 * (p[r][fine] * (x[fine].max() - x[fine])).sum() + self.vocab / 256 + 69)
        return e, p

    def check_gradient(self, got, want, lse, on, coef, slope):
        """slope: |dc/dlogp| per row."""
        e, p = self.error(on)
        far = np.where(np.isfinite(self.z64), np.abs(self.z64 - lse[:, None]), 0.0)
        hot = np.zeros_like(p)
        hot[np.flatnonzero(on), self.targets[on]] = 1
        c = np.abs(coef)[:, None]
        tol = (np.abs(slope) * e)[:, None] * np.abs(hot - p) + c * p * (e[:, None] + U * (2.5 * far + 6)) + 4 * U * c + HALF[self.dtype] * np.abs(want)
        tol += 1e-38  # below the smallest normal number
        bad = np.abs(got - want) > tol
        assert not bad.any(), f"{bad.sum()} entries off, worst {np.max(np.abs(got - want)[bad] / tol[bad]):.2f} tolerances at {np.argwhere(bad)[0]}"


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host(t):
    return t.cpu().double().numpy()


def scratch(rows, pairs=0):
    import torch
    import paper_2401_10241_amd as zb
    return torch.zeros(zb.loss_workspace_bytes(rows, pairs), dtype=torch.uint8, device="cuda")


SHAPES = [  # rows, vocab, pad, shift
    (1, 1, 0, 0), (1, 2, 0, 1), (3, 7, 1, 0), (5, 8, 0, 0), (2, 63, 2, 3), (4, 64, 0, 0), (4, 65, 0, 0), (3, 255, 0, 1), (3, 256, 8, 0),
    (2, 1000, 0, 0), (3, 1023, 0, 2), (2, 1025, 0, 0), (2, 4099, 5, 0), (2, 8192, 0, 4), (3, 32003, 61, 0), (2, 50257, 0, 0),
    (2, 65536, 0, 0), (2, 65537, 0, 0), (2, 131072, 0, 0), (2, 131073, 7, 0), (2, 262144, 0, 1),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "r%d_v%d_p%d_s%d" % s)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_logprobs_and_their_backward(dtype, shape):
    import torch
    import paper_2401_10241_amd as zb
    k = Case(dtype, *shape)
    logp, lse = torch.full((k.rows + 1,), GUARD, device="cuda"), torch.full((k.rows + 1,), GUARD, device="cuda")
    zb.token_logprobs(k.x(), logp.data_ptr(), lse.data_ptr())
    d = k.rng.normal(0, 1, k.rows).astype(np.float32)
    zb.token_logprobs_backward(k.x(), lse.data_ptr(), dev(d).data_ptr(), k.dflat[k.shift:].data_ptr())
    want, wlse = L.logprobs(k.z64, k.targets)
    on = np.ones(k.rows, bool)
    e, _ = k.error(on)
    assert logp[-1] == GUARD and lse[-1] == GUARD
    assert (np.abs(host(lse)[:-1] - wlse) <= e + U * np.abs(wlse)).all()
    assert (np.abs(host(logp)[:-1] - want) <= e + U * np.abs(want)).all()
    # the backward starts from the stored lse: half a step of it on top of e
    c = d.astype(np.float64)
    wide = Case.error
    k.error = lambda rows: (wide(k, rows)[0] + U * np.abs(wlse), wide(k, rows)[1])
    k.check_gradient(k.gradient(), L.dlogits(k.z64, k.targets, wlse, c, on), wlse, on, c, np.zeros(k.rows))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_logprobs_of_rows_without_target_and_masked_vocabularies(dtype):
    import torch
    import paper_2401_10241_amd as zb
    k = Case(dtype, 9, 1003, pad=3, shift=1)
    low = torch.finfo(k.kind).min
    k.targets[[1, 3, 5]] = [-1, 1003, -100]
    k.z[1], k.z[3] = float("nan"), float("inf")
    k.z[2, 500:] = -float("inf")   # masked tokens
    k.targets[2] = 7
    k.z[4, 10:] = low              # masked by the type's lowest value
    k.targets[4] = 900             # the target among them: a finite, very low log-probability
    k.z[6] = -float("inf")         # one token left
    k.z[6, 1002] = 3.0
    k.targets[6] = 1002
    k.z[7, 400] = -float("inf")    # the target itself masked: log-probability -infinity
    k.targets[7] = 400
    k.place()
    logp, lse = torch.full((9,), GUARD, device="cuda"), torch.full((9,), GUARD, device="cuda")
    zb.token_logprobs(k.x(), logp.data_ptr(), lse.data_ptr())
    d = np.ones(9, np.float32)
    d[8] = 0
    zb.token_logprobs_backward(k.x(), lse.data_ptr(), dev(d).data_ptr(), k.dflat[k.shift:].data_ptr())
    on = L.counting(k.targets, 1003)
    want, wlse = L.logprobs(k.z64, k.targets, on)
    e, _ = k.error(on)
    got = host(logp)
    assert (got[~on] == 0).all() and (host(lse)[~on] == 0).all() and got[6] == 0 and got[7] == -np.inf
    fine = np.isfinite(want)
    assert (np.abs(got - want)[fine] <= (e + U * np.abs(want))[fine]).all()
    g = k.gradient()
    assert not g[~on].any() and not g[8].any()
    assert not g[2, 500:].any() and not g[4, 10:900].any() and not g[4, 901:].any() and g[4, 900] == 1 and not g[6].any()
    c = d.astype(np.float64)
    k.error = lambda rows: (e + U * np.abs(wlse), Case.error(k, rows)[1])
    k.check_gradient(g, L.dlogits(k.z64, k.targets, wlse, c, on), wlse, on, c, np.zeros(9))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_logprobs_of_undefined_rows_are_nan(dtype):
    import torch
    import paper_2401_10241_amd as zb
    for value, at in ((float("nan"), slice(3, 4)), (float("inf"), slice(6, 7)), (-float("inf"), slice(None))):
        for vocab in (11, 3001):
            k = Case(dtype, 3, vocab)
            k.z[1, at] = value
            k.place()
            logp = torch.zeros(3, device="cuda")
            loss, dl = torch.zeros(1, device="cuda"), k.dflat
            zb.token_logprobs(k.x(), logp.data_ptr())
            assert torch.isnan(logp).tolist() == [False, True, False]
            one = torch.ones(3, device="cuda")
            ws = scratch(3)
            zb.policy_loss(k.x(), zb.policy(one.data_ptr(), one.data_ptr()), loss.data_ptr(), 0, dl.data_ptr(), workspace=ws.data_ptr(),
                           workspace_bytes=ws.numel())
            g = k.gradient()
            assert np.isnan(host(loss)).all() and np.isnan(g[1]).all() and np.isfinite(g[[0, 2]]).all()


def policy_inputs(k, weight=True):
    """Ratios on both sides of the interval and in it, none nearer than 1e-3 to a border; signs of both kinds."""
    lp, _ = L.logprobs(k.z64, k.targets, L.counting(k.targets, k.vocab))
    lp = np.where(np.isfinite(lp), lp, 0.0)
    ratio = np.exp(k.rng.normal(0, 0.3, k.rows))
    for border in (0.8, 1.28):
        ratio = np.where(np.abs(ratio - border) < 1e-3, 1.0, ratio)
    old = (lp - np.log(ratio)).astype(np.float32)
    ref = (lp + k.rng.normal(0, 0.5, k.rows)).astype(np.float32)
    adv = k.rng.normal(0, 1, k.rows).astype(np.float32)
    w = k.rng.uniform(0.5, 2, k.rows).astype(np.float32)
    w[k.rng.random(k.rows) < 0.3] = 0
    return old, ref, adv, (w if weight else None)


def check_policy(k, kl, w, old, ref, adv, scale=0.25, in_place=False, out=None):
    import torch
    import paper_2401_10241_amd as zb
    loss, logp = torch.full((1,), GUARD, device="cuda"), torch.full((k.rows,), GUARD, device="cuda")
    keep = [dev(a) for a in (old, adv, ref)] + ([dev(w)] if w is not None else [])
    p = zb.policy(keep[0].data_ptr(), keep[1].data_ptr(), ref_logp=keep[2].data_ptr() if kl else 0,
                  weight=keep[3].data_ptr() if w is not None else 0, clip_low=0.2, clip_high=0.28, kl_coef=kl, scale=scale)
    ws = scratch(k.rows)
    buf = k.flat if in_place else k.dflat
    zb.policy_loss(k.x(), p, loss.data_ptr(), logp.data_ptr(), buf[k.shift:].data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    wl, wlp, c, d = L.policy(k.z64, k.targets, old, adv, ref, w, 0.2, 0.28, kl, scale)
    on = L.counting(k.targets, k.vocab, w)
    _, lse = L.logprobs(k.z64, k.targets, on)
    e, _ = k.error(on)
    we = np.where(on, scale * (1.0 if w is None else w.astype(np.float64)), 0.0)
    rho = np.where(on, np.exp(np.where(on, wlp - old, 0.0)), 0.0)
    gap = np.where(on, np.exp(np.where(on, ref - wlp, 0.0)), 0.0)
    adv = np.where(on, adv, 0.0)
    slope = we * (np.abs(adv) * rho + kl * gap)
    assert (np.abs(host(logp) - wlp) <= e + U * np.abs(wlp)).all()
    assert abs(host(loss)[0] - wl) <= (we * (np.abs(adv) * rho + kl * (gap + 1)) * e).sum() + 2 * U * abs(wl)
    k.check_gradient(k.gradient(buf), d, lse, on, c, slope)


@pytest.mark.parametrize("shape", [(1, 1, 0, 0), (1, 33, 0, 0), (65, 257, 3, 1), (300, 512, 0, 0), (40, 8192, 0, 0), (5, 50257, 0, 0), (3, 131073, 0, 1),
                                   (3, 262144, 0, 0)], ids=lambda s: "r%d_v%d_p%d_s%d" % s)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_policy_loss(dtype, shape):
    for kl, weight, in_place in ((0.0, False, False), (0.07, True, False), (0.07, True, True)):
        k = Case(dtype, *shape, seed=int(100 * kl))
        old, ref, adv, w = policy_inputs(k, weight)
        check_policy(k, kl, w, old, ref, adv, in_place=in_place)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_policy_loss_of_a_padded_batch(dtype):
    k = Case(dtype, 50, 3001, pad=7, shift=3)
    old, ref, adv, w = policy_inputs(k)
    k.targets[40:] = -1
    w[20:25] = 0
    k.z[40:], k.z[20:25] = float("nan"), float("inf")
    for a in (old, ref, adv):
        a[40:], a[20:25] = np.nan, np.inf
    k.place()
    check_policy(k, 0.1, w, old, ref, adv)
    w[:] = 0  # nothing counts
    k.place()
    check_policy(k, 0.1, w, old, ref, adv)


def check_preference(k, n, weight, beta=0.5, eps=0.1, scale=0.5, in_place=False):
    """n: the sequences' lengths; the first starts at row `before`."""
    import torch
    import paper_2401_10241_amd as zb
    before = k.rows - sum(n) if k.rows - sum(n) < 3 else 2
    off = (before + np.concatenate([[0], np.cumsum(n)])).astype(np.int32)
    on = L.counting(k.targets, k.vocab, weight, off)
    lp, lse = L.logprobs(k.z64, k.targets, on)
    ref = (lp + k.rng.normal(0, 0.4, k.rows)).astype(np.float32)
    ref[~on] = np.nan
    pairs = len(n) // 2
    loss, logp, rewards = torch.full((1,), GUARD, device="cuda"), torch.full((k.rows,), GUARD, device="cuda"), torch.full((2 * pairs + 1,), GUARD, device="cuda")
    keep = [dev(ref), dev(off)] + ([dev(weight)] if weight is not None else [])
    p = zb.preference(keep[0].data_ptr(), keep[1].data_ptr(), pairs, weight=keep[2].data_ptr() if weight is not None else 0, beta=beta,
                      label_smoothing=eps, scale=scale)
    ws = scratch(k.rows, pairs)
    buf = k.flat if in_place else k.dflat
    zb.preference_loss(k.x(), p, loss.data_ptr(), logp.data_ptr(), rewards.data_ptr(), buf[k.shift:].data_ptr(), workspace=ws.data_ptr(),
                       workspace_bytes=ws.numel())
    wl, wlp, wr, c, d = L.preference(k.z64, k.targets, ref, off, weight, beta, eps, scale)
    e, _ = k.error(on)
    w = np.where(on, 1.0 if weight is None else weight.astype(np.float64), 0.0)
    es = np.array([(np.abs(w) * e)[a:b].sum() for a, b in zip(off[:-1], off[1:])])  # of the sums
    got = host(rewards)
    assert got[-1] == GUARD
    assert (np.abs(host(logp) - wlp) <= e + U * np.abs(wlp)).all()
    assert (np.abs(got[:-1] - wr) <= beta * es + U * np.abs(wr)).all()
    dx = beta * (es[0::2] + es[1::2])
    assert abs(host(loss)[0] - wl) <= scale * dx.sum() + 2 * U * abs(wl)  # |d loss / d x| <= scale
    # |d slope / d x| <= scale beta / 4; dc is that times the error of x, written as slope * e for check_gradient
    dc = np.zeros(k.rows)
    for i in range(pairs):
        a, b = off[2 * i], off[2 * i + 2]
        dc[a:b] = np.abs(w[a:b]) * scale * beta / 4 * dx[i]
    slope = np.where(e > 0, dc / np.where(e > 0, e, 1), 0.0)
    k.check_gradient(k.gradient(buf), d, lse, on, c, slope)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("case", [(2, 5, [1, 1]), (12, 257, [3, 4, 0, 2]), (300, 1003, [257, 40]), (3, 64, [0, 0]), (40, 8192, [7, 9, 1, 20]),
                                  (5, 50257, [2, 3]), (4, 131073, [1, 2]), (3, 262144, [2, 1])], ids=lambda c: "r%d_v%d_%s" % (c[0], c[1], "_".join(map(str, c[2]))))
def test_preference_loss(dtype, case):
    rows, vocab, n = case
    for weighted, in_place in ((False, False), (True, False), (True, True)):
        k = Case(dtype, rows, vocab, shift=weighted, seed=weighted)
        w = None
        if weighted:
            w = k.rng.uniform(0.5, 2, rows).astype(np.float32)
            w[k.rng.random(rows) < 0.3] = 0
            k.targets[-1] = -1
            k.z[-1] = float("nan")
            k.place()
        check_preference(k, n, w, in_place=in_place)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_preference_loss_leaves_rows_outside_the_sequences_alone(dtype):
    k = Case(dtype, 20, 1003)
    k.z[:2], k.z[12:] = float("nan"), float("inf")
    k.place()
    check_preference(k, [4, 6], None)


def test_no_rows_and_no_pairs():
    import torch
    import paper_2401_10241_amd as zb
    loss, ws = torch.full((1,), GUARD, device="cuda"), scratch(4)
    empty = zb.logits(0, 0, 100, 0)
    zb.token_logprobs(empty, 0)
    zb.policy_loss(empty, zb.policy(0, 0), loss.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    assert host(loss)[0] == 0
    k = Case("bf16", 4, 100)
    loss.fill_(GUARD)
    logp = torch.full((4,), GUARD, device="cuda")
    zb.preference_loss(k.x(), zb.preference(0, 0, 0), loss.data_ptr(), logp.data_ptr(), 0, k.dflat.data_ptr(), workspace=ws.data_ptr(),
                       workspace_bytes=ws.numel())
    assert host(loss)[0] == 0 and not host(logp).any() and not k.gradient().any()


def test_large_ratios_and_far_references():
    """Ratios that overflow a 32-bit exponential: a clipped gain stays finite, an unclipped loss is what it is."""
    import torch
    import paper_2401_10241_amd as zb
    k = Case("fp32", 3, 50)
    lp, _ = L.logprobs(k.z64, k.targets)
    old = (lp - np.array([100.0, -100.0, 100.0])).astype(np.float32)
    adv = np.array([1.0, 1.0, -1.0], np.float32)
    loss, ws = torch.zeros(1, device="cuda"), scratch(3)
    keep = dev(old), dev(adv)
    zb.policy_loss(k.x(), zb.policy(keep[0].data_ptr(), keep[1].data_ptr(), clip_low=0.2, clip_high=0.3), loss.data_ptr(), 0, k.dflat.data_ptr(),
                   workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    g = k.gradient()
    assert host(loss)[0] == np.inf and not g[0].any() and np.abs(g[1]).max() < 1e-38 and g[2, k.targets[2]] == np.inf


def test_an_advantage_of_zero_asks_for_nothing():
    import torch
    import paper_2401_10241_amd as zb
    k = Case("bf16", 3, 70)
    keep = dev(np.array([-np.inf, -1e30, -3.0], np.float32)), dev(np.zeros(3, np.float32))
    loss, ws = torch.full((1,), GUARD, device="cuda"), scratch(3)
    zb.policy_loss(k.x(), zb.policy(keep[0].data_ptr(), keep[1].data_ptr()), loss.data_ptr(), 0, k.dflat.data_ptr(), workspace=ws.data_ptr(),
                   workspace_bytes=ws.numel())
    assert host(loss)[0] == 0 and not k.gradient().any()


def test_targets_that_the_policy_or_the_reference_rules_out():
    """log-probabilities of -infinity: the ratio is 0, the KL term infinite where the reference allows the token, and no NaN beside them."""
    import torch
    import paper_2401_10241_amd as zb
    k = Case("fp32", 4, 50)
    k.targets[:] = 7
    k.z[0, 7] = k.z[1, 7] = -float("inf")
    k.place()
    lp = L.logprobs(k.z64, k.targets)[0]
    old, ref = np.full(4, -3.0, np.float32), np.full(4, -3.0, np.float32)
    old[2:] = lp[2:]
    ref[3] = -np.inf
    for adv in (1.0, -1.0):
        keep = dev(old), dev(np.full(4, adv, np.float32)), dev(ref)
        for kl in (0.0, 0.1):
            loss, ws = torch.zeros(1, device="cuda"), scratch(4)
            zb.policy_loss(k.x(), zb.policy(keep[0].data_ptr(), keep[1].data_ptr(), ref_logp=keep[2].data_ptr(), clip_low=0.2, clip_high=0.3, kl_coef=kl),
                           loss.data_ptr(), 0, k.dflat.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())
            g = k.gradient()
            # rho = 0: -min(0, 0.8 A) is 0 for a gain, 0.8 |A| for a loss, neither with a gradient
            each = 0.0 if adv > 0 else 0.8
            if kl == 0:
                assert abs(host(loss)[0] - (2 * each - 2 * adv)) <= 1e-5 and not g[:2].any() and np.isfinite(g).all()
            else:
                assert host(loss)[0] == np.inf and np.isfinite(g[2:]).all() and g[0, 7] == -np.inf
                # reference -infinity: d(exp(d) - d - 1)/dlogp = 1 - exp(d) = 1
                assert abs(g[3, 7] - (kl - adv) * (1 - np.exp(lp[3]))) <= 1e-5


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_captured_losses_replay_like_eager_ones(dtype):
    """Captured on a side stream and replayed with new logits each time, eager work between the replays."""
    import torch
    import paper_2401_10241_amd as zb
    k = Case(dtype, 33, 2051)
    old, ref, adv, w = policy_inputs(k)
    off = dev(np.array([0, 9, 20, 25, 33], np.int32))
    keep = [dev(a) for a in (old, adv, ref, w)]
    p = zb.policy(keep[0].data_ptr(), keep[1].data_ptr(), ref_logp=keep[2].data_ptr(), weight=keep[3].data_ptr(), kl_coef=0.1)
    q = zb.preference(keep[2].data_ptr(), off.data_ptr(), 2, weight=keep[3].data_ptr())

    def outputs():
        return [torch.full((n,), GUARD, device="cuda") for n in (1, 33, 1, 33, 4, 33, 33)] + [torch.zeros_like(k.flat) for _ in range(3)]

    def calls(out, ws, stream):
        a = [t.data_ptr() for t in out]
        zb.policy_loss(k.x(), p, a[0], a[1], a[7], workspace=ws.data_ptr(), workspace_bytes=ws.numel(), stream_handle=stream)
        zb.preference_loss(k.x(), q, a[2], a[3], a[4], a[8], workspace=ws.data_ptr(), workspace_bytes=ws.numel(), stream_handle=stream)
        zb.token_logprobs(k.x(), a[5], a[6], stream_handle=stream)
        zb.token_logprobs_backward(k.x(), a[6], keep[1].data_ptr(), a[9], stream_handle=stream)

    side = torch.cuda.Stream()
    first, ws1, ws2 = outputs(), scratch(33, 2), scratch(33, 2)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        calls(first, ws1, torch.cuda.current_stream().cuda_stream)
    for trial in range(4):
        k.flat.copy_(torch.randn(k.flat.shape, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        second = outputs()
        calls(second, ws2, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for a, b in zip(first, second):
            assert torch.equal(a, b)


def test_two_calls_at_once_with_workspaces_of_their_own():
    import torch
    import paper_2401_10241_amd as zb
    cases = [Case("bf16", 200, 5003, seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in cases]
    inputs, outs, spaces = [], [], []
    for k in cases:
        inputs.append([dev(a) for a in policy_inputs(k)])
        outs.append((torch.zeros(1, device="cuda"), torch.zeros(200, device="cuda")))
        spaces.append(scratch(200))

    def call(i, stream):
        o, r, a, w = inputs[i]
        zb.policy_loss(cases[i].x(), zb.policy(o.data_ptr(), a.data_ptr(), ref_logp=r.data_ptr(), weight=w.data_ptr(), kl_coef=0.1),
                       outs[i][0].data_ptr(), outs[i][1].data_ptr(), cases[i].dflat.data_ptr(), workspace=spaces[i].data_ptr(),
                       workspace_bytes=spaces[i].numel(), stream_handle=stream)

    torch.cuda.synchronize()
    alone = []
    for i in range(2):
        call(i, 0)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in (*outs[i], cases[i].dflat)])
    for _ in range(5):
        for i in range(2):
            call(i, streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in zip(alone[i], (*outs[i], cases[i].dflat)):
            assert torch.equal(a, b)
