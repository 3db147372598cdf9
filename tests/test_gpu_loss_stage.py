"""A last stage with a policy or a preference loss against oracle/losses.py through the C ABI: loss, log-probabilities, gradients, the
optimizer step after them; bits that do not depend on the order of the passes; what such a stage refuses."""
import numpy as np
import pytest

import zb_inputs
from oracle import losses as L
from oracle import optimizer as O
from oracle.schedule import stage_order
from oracle.stage import PARAM_ORDER
from zb_testlib import TOL, check_tensor, hyper

pytestmark = pytest.mark.gpu

W = zb_inputs.Workload
LOW, HIGH, KL, BETA, EPS = 0.2, 0.3, 0.1, 0.4, 0.1


def build(w, kind, vocab, m, oracle=True, **kw):
    import paper_2401_10241_amd as zb
    pb, pw, fl = zb.schedule_stash_need(w.p, w.stage, m, w.kind)
    params, extra = zb_inputs.stage_params(w), zb_inputs.end_stage_params(w, "last", vocab)
    extra["w_head"] = extra["w_head"] * 3  # logits of a spread that tells tokens apart
    shape = dict(layers=w.layers, hidden=w.hidden, heads=w.heads, ffn=w.ffn, seq=w.seq, mb_size=w.mb_size, dtype=w.dtype, ln_eps=w.ln_eps)
    pools = kw.pop("pools", (pb, pw, fl))
    dev = zb.Stage(max_microbatches=m, max_pending_b=pools[0], max_pending_w=pools[1], max_inflight=pools[2], role="last", vocab=vocab, lr=w.lr,
                   loss=kind, clip_low=LOW, clip_high=HIGH, kl_coef=KL, pref_beta=BETA, label_smoothing=EPS, **shape, **kw)
    dev.set_params(params)
    dev.set_stage_params(extra)
    if not oracle:
        return dev, None
    return dev, L.LossStageOracle(kind=kind, low=LOW, high=HIGH, kl=KL, beta=BETA, eps=EPS, vocab=vocab, extra_params=extra, hyper=hyper(w), params=params,
                                  **shape)


def load(w, vocab, m, it, dev, orc=None, values=None):
    """Inputs, targets and, once known, what the loss reads."""
    import paper_2401_10241_amd as zb
    for k in range(m):
        x, t = zb_inputs.stage_input(w, it, k), zb_inputs.target_ids(w, it, k, vocab)
        dev.set_tensor(zb.T_INPUT_X, 0, k, x)
        dev.set_ids(zb.T_TARGET_IDS, k, t)
        if orc is not None:
            orc.set_input(k, x)
            orc.set_targets(k, t)
        if values is None:
            if orc is not None:
                orc.set_values(k, weight=np.ones(w.tokens), old=np.zeros(w.tokens), advantage=np.zeros(w.tokens), ref=np.zeros(w.tokens))
            continue
        v = values[k]
        for what, name in ((zb.T_LOSS_WEIGHT, "weight"), (zb.T_REF_LOGP, "ref")) + (((zb.T_OLD_LOGP, "old"), (zb.T_ADVANTAGE, "advantage")) if dev.cfg.loss == 1
                                                                                   else ()):
            dev.set_token_values(what, k, v[name])
        if orc is not None:
            orc.set_values(k, **v)


def values_of(w, m, logp, seed=0):
    """Weights with prompts and padding, ratios that rounding does not carry over a border."""
    rng = np.random.default_rng(seed)
    out = []
    for k in range(m):
        n = w.tokens
        weight = rng.uniform(0.5, 1.5, n)
        pos = np.arange(n) % w.seq
        weight[(pos < w.seq // 4) | (pos >= w.seq - 3)] = 0
        ratio = rng.choice([0.4, 0.97, 1.05, 1.9], n)
        lp = logp[k] if logp else np.full(n, -5.0)
        out.append({a: b.astype(np.float32) for a, b in dict(weight=weight, old=lp - np.log(ratio), advantage=rng.normal(0, 1, n),
                                                             ref=lp + rng.normal(0, 0.3, n)).items()})
    return out


def slope(rewards):
    """d(loss) / d(sum of log-probabilities), but for a factor, of the pairs with these rewards."""
    x = rewards[0::2].astype(np.float64) - rewards[1::2]
    return EPS / (1 + np.exp(-x)) - (1 - EPS) / (1 + np.exp(x))


CASES = [  # dtype, layers, hidden, heads, ffn, seq, b, vocab, m
    ("fp32", 1, 64, 2, 256, 32, 2, 97, 3),
    ("bf16", 1, 256, 4, 1024, 128, 2, 1024, 4),
    ("bf16", 1, 256, 4, 1024, 96, 4, 1003, 3),   # an odd vocabulary: rows of logits that start anywhere
]


@pytest.mark.parametrize("kind", ["policy", "preference"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s_L%d_h%d_a%d_f%d_s%d_b%d_V%d_m%d" % c)
def test_loss_stage_parity(kind, case):
    import paper_2401_10241_amd as zb
    dtype, layers, hidden, heads, ffn, seq, b, vocab, m = case
    p = 4
    w = W("loss", dtype, layers, hidden, heads, ffn, seq, b, p, p - 1, m, "H1", seed=81 + hidden, lr=1e-4)
    dev, orc = build(w, kind, vocab, m)
    tol = TOL[dtype]
    for it in range(2):  # the second iteration runs on the updated head
        orc.begin_iteration(m)
        dev.begin_iteration(it, m)
        load(w, vocab, m, it, dev, orc)
        for k in range(m):  # log-probabilities that the old and the reference policy are built around
            orc.forward(k)
        values = values_of(w, m, [orc.logp[k] for k in range(m)], it)
        orc.begin_iteration(m)
        load(w, vocab, m, it, dev, orc, values)
        dev.run_schedule(p, p - 1, m, "H1")
        dev.synchronize()
        orc.run(stage_order(p, p - 1, m, "H1"))
        tol = TOL[dtype]
        if kind == "preference":
            # Every gradient row of a pair has the factor slope(x), x the difference of two rewards, each the sum of some hundred
            # log-probabilities with errors of their own.  The rewards are held to their bound below; what their accepted difference does to
            # the factor, |slope(device) / slope(oracle) - 1|, comes on top of the relative error of everything that the factor multiplies.
            tol += max(np.abs(slope(dev.get_token_values(zb.T_REWARDS, k)) / slope(orc.rewards[k]) - 1).max() for k in range(m))
        for k in range(m):
            if kind == "preference":  # a function of the rewards, which are compared below; each of them rounded to fp32
                r = dev.get_token_values(zb.T_REWARDS, k).astype(np.float64)
                x = r[0::2] - r[1::2]
                want = np.mean((1 - EPS) * np.logaddexp(0, -x) + EPS * np.logaddexp(0, x))
                assert abs(dev.get_loss(k) - want) <= 2.0 ** -24 * (np.abs(r).sum() + 2 * want)
            else:
                assert dev.get_loss(k) == pytest.approx(orc.loss[k], rel=tol, abs=tol * 0.1)
            lp = dev.get_token_values(zb.T_TOKEN_LOGP, k)
            on = values[k]["weight"] != 0
            assert not lp[~on].any() and np.allclose(lp[on], orc.logp[k][on], rtol=TOL[dtype], atol=TOL[dtype])
            if kind == "preference":
                # a sum of `seq` differences of log-probabilities, whose errors are independent
                assert np.allclose(dev.get_token_values(zb.T_REWARDS, k), orc.rewards[k], rtol=TOL[dtype], atol=TOL[dtype] * BETA * np.sqrt(seq))
            check_tensor(f"dX[{k}]", dev.get_tensor(zb.T_OUTPUT_DX, 0, k), orc.dX[k], tol, dtype)
        got = dev.get_group(zb.T_GRAD)
        for l in range(layers):
            for name in PARAM_ORDER:
                check_tensor(f"grad {l} {name}", got[l][name], orc.grads[l][name], tol, "fp32")
        for name, g in dev.get_stage_group(zb.T_STAGE_GRAD).items():
            ref = orc.grads[orc.nl][name]
            if name == "w_head":
                g, ref = g.T, ref.T
            check_tensor(f"grad {name}", g, ref, tol, "fp32", by_row=(name == "w_head"))
        rep, want = dev.optimizer_step_validated(0.0, 0.0), orc.optimizer_step(O.GlobalState(0.0, 0.0))
        assert rep.outcome == want.outcome and rep.t == it + 1
        print(f"[{kind} {dtype} V={vocab}] tolerance {tol:.3f}, losses {[round(dev.get_loss(k), 5) for k in range(m)]}", flush=True)
    dev.close()


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_loss_stage_bits_do_not_depend_on_the_order(kind):
    import paper_2401_10241_amd as zb
    m, p, vocab = 4, 4, 1003
    w = W("loss_det", "bf16", 2, 256, 4, 1024, 64, 2, p, p - 1, m, "H1", seed=83)
    values = values_of(w, m, None)
    results = []
    for mode in ("H1", "flat", "1F1B fused"):
        dev, _ = build(w, kind, vocab, m, oracle=False, pools=(m, m, m), fuse_bw=mode == "1F1B fused")
        dev.begin_iteration(0, m)
        load(w, vocab, m, 0, dev, None, values)
        if mode == "flat":
            for c, k in [(0, k) for k in range(m)] + [(1, k) for k in range(m)] + [(2, k) for k in range(m)]:
                (dev.forward, dev.backward_input, dev.backward_weight)[c](k)
        else:
            dev.run_schedule(p, p - 1, m, mode.split()[0])
        dev.synchronize()
        results.append([dev.get_tensor(zb.T_FLAT_GRADS)] + [dev.get_tensor(zb.T_OUTPUT_DX, 0, k) for k in range(m)] + [np.float32(dev.get_loss(k)) for k in range(m)])
        dev.close()
    assert np.abs(results[0][0]).max() > 0
    for other in results[1:]:
        for a, b in zip(other, results[0]):
            assert a.tobytes() == b.tobytes()


def test_a_policy_stage_that_has_not_moved_from_its_old_policy():
    """F alone gives the old log-probabilities; with them and advantages A the loss is -mean(A) and no token is clipped."""
    import paper_2401_10241_amd as zb
    m, p, vocab = 1, 2, 512
    w = W("loss_same", "bf16", 1, 256, 4, 1024, 64, 2, p, p - 1, m, "H1", seed=84)
    dev, _ = build(w, "policy", vocab, m, oracle=False, pools=(1, 1, 1))
    values = values_of(w, m, None)
    values[0]["weight"][:] = 1
    dev.begin_iteration(0, m)
    load(w, vocab, m, 0, dev, None, values)
    dev.forward(0)
    lp = dev.get_token_values(zb.T_TOKEN_LOGP, 0)
    dev.set_token_values(zb.T_OLD_LOGP, 0, lp)
    dev.set_token_values(zb.T_REF_LOGP, 0, lp)
    dev.begin_iteration(1, m)
    dev.forward(0)
    # rho = exp(logp - old) with old rounded to fp32: off by half a step of |logp| <= 16, 2^-21, in each of the tokens
    a = values[0]["advantage"].astype(np.float64)
    assert abs(dev.get_loss(0) + a.mean()) <= 2.0 ** -20 * np.abs(a).mean() + 2.0 ** -23 * abs(a.mean())
    assert np.array_equal(dev.get_token_values(zb.T_TOKEN_LOGP, 0), lp)
    dev.close()


def test_loss_stage_argument_checks():
    import paper_2401_10241_amd as zb
    w = W("loss_err", "fp32", 1, 64, 2, 256, 32, 2, 2, 1, 2, "H1", seed=3)
    dev, _ = build(w, "policy", 50, 2, oracle=False)
    for f in (lambda: dev.get_token_values(zb.T_REWARDS, 0), lambda: dev.set_token_values(zb.T_TOKEN_LOGP, 0, np.zeros(64)),
              lambda: dev.set_token_values(zb.T_ADVANTAGE, 2, np.zeros(64)), lambda: dev.set_token_values(zb.T_ADVANTAGE, 0, np.zeros(63))):
        with pytest.raises(zb.ZbError) as e:
            f()
        assert e.value.status == zb.EINVAL
    dev.set_token_values(zb.T_ADVANTAGE, 1, np.arange(64))
    assert np.array_equal(dev.get_token_values(zb.T_ADVANTAGE, 1), np.arange(64, dtype=np.float32))
    assert not dev.get_token_values(zb.T_LOSS_WEIGHT, 1).any()
    dev.close()
    dev, _ = build(w, "preference", 50, 2, oracle=False)
    for what in (zb.T_ADVANTAGE, zb.T_OLD_LOGP):
        with pytest.raises(zb.ZbError):
            dev.get_token_values(what, 0)
    dev.close()
