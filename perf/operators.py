"""Performance cases of the operators behind a post-training step: log-probabilities of given tokens, the clipped
policy loss and the preference loss with the gradient of the logits, AdamW over many tensors with 32- or 8-bit states.

A case's ``kind``:

* ``logprobs`` - log-probabilities of the target tokens and the rows' log-sum-exp; with ``grad`` also the gradient of the
  logits for given gradients of the log-probabilities.
* ``policy`` - sequences of ``seq`` rows whose first ``prompt`` rows carry no weight, ``pad`` rows without a target at the end.
* ``preference`` - ``pairs`` pairs of ragged sequences, prompts without weight.
* ``adamw`` - the norm of all gradients and one step.  The tensors are those of ``layers`` decoder layers, or with
  ``rank`` the low-rank pairs of their matrices.

``run`` computes them from elementary torch operations, or with ``own`` through the library.
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 256  # values that share the two scales of an 8-bit state
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
BETA, SMOOTHING = 0.1, 0.05
LR, BETA1, BETA2, EPS, DECAY, CLIP, SEED = 1e-4, 0.9, 0.95, 1e-8, 0.01, 1.0, 1234


def listed():
    return [
        # sampling: the log-probability of the one token just drawn, fp32 logits; latency is all there is
        {"name": "logprobs_1", "kind": "logprobs", "dtype": "fp32", "rows": 1, "vocab": 32000, "stride": 32000, "grad": False},
        # the reference policy over a batch: forward only, the vocabulary of the last stage
        {"name": "logprobs_4096", "kind": "logprobs", "dtype": "bf16", "rows": 4096, "vocab": 50432, "stride": 50432, "grad": False},
        # an odd vocabulary whose rows start at any address, with gradients: an objective of the caller's own
        {"name": "logprobs_odd", "kind": "logprobs", "dtype": "bf16", "rows": 777, "vocab": 50257, "stride": 50257, "grad": True},
        # a small fp32 policy, every row of weight
        {"name": "policy_small", "kind": "policy", "dtype": "fp32", "seqs": 2, "seq": 32, "prompt": 0, "pad": 0, "vocab": 8192, "stride": 8192},
        # odd everything: a padded batch, an odd vocabulary inside wider rows, fp32
        {"name": "policy_ragged", "kind": "policy", "dtype": "fp32", "seqs": 5, "seq": 201, "prompt": 37, "pad": 18, "vocab": 32003, "stride": 32064},
        # an update of the policy at the last stage's vocabulary: four sequences of 1024 tokens, a fifth of them prompt
        {"name": "policy_4096", "kind": "policy", "dtype": "bf16", "seqs": 4, "seq": 1024, "prompt": 200, "pad": 0, "vocab": 50432, "stride": 50432},
        # two pairs of short answers
        {"name": "preference_small", "kind": "preference", "dtype": "bf16", "pairs": 2, "mean": 48, "prompt": 8, "vocab": 32000, "stride": 32000},
        # a batch of pairs of several hundred tokens each
        {"name": "preference_large", "kind": "preference", "dtype": "bf16", "pairs": 6, "mean": 512, "prompt": 100, "vocab": 50432, "stride": 50432},
        # the twelve tensors of a small layer, fp32 states and gradients: launches and latency
        {"name": "adamw32_small", "kind": "adamw", "bits": 32, "layers": 1, "hidden": 256, "ffn": 1024, "rank": 0, "grads": "fp32", "copies": True},
        # 36 tensors of the 1.5B shape with bf16 gradients, fp32 states
        {"name": "adamw32_h2304", "kind": "adamw", "bits": 32, "layers": 3, "hidden": 2304, "ffn": 9216, "rank": 0, "grads": "bf16", "copies": True},
        # adapters of odd sizes beside a frozen stage, 8-bit states
        {"name": "adamw8_adapters", "kind": "adamw", "bits": 8, "layers": 4, "hidden": 1203, "ffn": 4811, "rank": 13, "grads": "fp32", "copies": False},
        # a layer of the 14.6B shape, 8-bit states
        {"name": "adamw8_h5120", "kind": "adamw", "bits": 8, "layers": 1, "hidden": 5120, "ffn": 20480, "rank": 0, "grads": "bf16", "copies": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["logprobs", "policy", "preference", "adamw", "adamw"])
    if kind == "adamw":
        case = {"kind": kind, "bits": rng.choice([8, 32]), "layers": rng.randint(1, 4), "hidden": 0, "ffn": 0, "rank": 0,
                "grads": rng.choice(["fp32", "bf16"]), "copies": rng.random() < 0.5}
        h = _log_int(rng, 64, 4096)
        if rng.random() < 0.4:
            case["rank"] = _log_int(rng, 1, 64)
        else:
            h = 8 * max(1, h // 8)
        case["hidden"], case["ffn"] = h, 4 * h + (rng.randint(0, 7) if case["rank"] else 0)
        while sum(_sizes(case)) > 3e8:
            case["layers"] -= 1
        return case
    vocab = rng.choice([8192, 32000, 50257, 50432, _log_int(rng, 300, 100000), _log_int(rng, 300, 100000) | 1])
    case = {"kind": kind, "dtype": rng.choice(["fp32", "bf16", "bf16"]), "vocab": vocab, "stride": vocab + rng.choice([0, 0, 0, 8, 13])}
    budget = 8e8 if case["dtype"] == "bf16" else 4e8  # bytes of the logits in half
    most = max(1, int(budget // (2 * case["stride"])))
    if kind == "logprobs":
        return dict(case, rows=_log_int(rng, 1, min(8192, 1.9 * most)), grad=rng.random() < 0.5)
    if kind == "policy":
        seq = _log_int(rng, 1, min(1024, most))
        return dict(case, seq=seq, seqs=rng.randint(1, max(1, min(8, most // seq))), prompt=rng.choice([0, seq // 3]), pad=rng.choice([0, 0, rng.randint(1, 40)]))
    mean = _log_int(rng, 2, min(1024, most // 2))
    return dict(case, mean=mean, pairs=rng.randint(1, max(1, min(8, most // (2 * mean)))), prompt=rng.choice([0, mean // 4]))


def _lengths(case):
    """Lengths of the 2 * pairs sequences: ragged, now and then a single token; they belong to the case and not to the seed."""
    rng = random.Random("%d %d %d" % (case["pairs"], case["mean"], case["vocab"]))
    return [1 if rng.random() < 0.05 else max(1, int(case["mean"] * rng.uniform(0.4, 1.4))) for _ in range(2 * case["pairs"])]


def _active(case):
    """For each row whether it has weight (and a target)."""
    if case["kind"] == "logprobs":
        return [True] * case["rows"]
    if case["kind"] == "policy":
        return ([False] * case["prompt"] + [True] * (case["seq"] - case["prompt"])) * case["seqs"] + [False] * case["pad"]
    return [t >= case["prompt"] or t == n - 1 for n in _lengths(case) for t in range(n)]  # an answer has one token at least


def _sizes(case):
    h, f, r = case["hidden"], case["ffn"], case["rank"]
    if r:
        one = [h * r, r * 3 * h, h * r, r * h, h * r, r * f, f * r, r * h]
    else:
        one = [h, h, 3 * h * h, 3 * h, h * h, h, h, h, h * f, f, f * h, h]
    return one * case["layers"]


def _starts(case):
    """Every tensor starts on a whole block of one flat vector."""
    at, out = 0, []
    for n in _sizes(case):
        out.append(at)
        at += -(-n // BLOCK) * BLOCK
    return out, at


def work(case):
    if case["kind"] == "adamw":
        n = sum(_sizes(case))
        state = 8 if case["bits"] == 32 else 2 + 8 / BLOCK
        each = (4 if case["grads"] == "fp32" else 2) + 8 + 2 * state + (2 if case["copies"] else 0)
        if case["bits"] == 8:
            each += 8  # the moments as values
        return {"bytes": n * each, "flops": 16 * n}
    act = _active(case)
    es = 2 if case["dtype"] == "bf16" else 4
    rows, row = len(act), case["vocab"] * es
    read = sum(act)
    if case["kind"] == "logprobs":
        nbytes = read * (row + 12) + (rows * (row + 4) if case["grad"] else 0)
        flops = read * case["vocab"] * (9 if case["grad"] else 5)
    else:
        nbytes = read * row + rows * (row + 24)
        flops = read * case["vocab"] * 9
    return {"bytes": nbytes, "flops": flops}


class _State:
    pass


def _logits_of(gen, rows, case):
    """Logits as a head makes them: a spread of two, the target well above the rest; rows of a wider buffer."""
    vocab, dtype = case["vocab"], DTYPES[case["dtype"]]
    buf = torch.randn(rows * case["stride"], generator=gen, device="cuda", dtype=dtype).mul_(2).view(rows, case["stride"])
    logits = buf[:, :vocab]
    cdf = torch.cumsum(1.0 / (torch.arange(vocab, dtype=torch.float64, device="cuda") + 2.7), 0)
    u = torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64) * cdf[-1]
    targets = torch.searchsorted(cdf, u).clamp_(max=vocab - 1)
    at = (torch.arange(rows, device="cuda"), targets)
    logits[at] += (6 + 3 * torch.randn(rows, generator=gen, device="cuda")).to(dtype)
    if vocab > 1000:
        tail = vocab - vocab // 500  # entries that pad the vocabulary cannot be drawn
        keep = targets >= tail
        targets[keep] = targets[keep] - tail
        logits[:, tail:] = -math.inf
    return logits, targets


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    st = _State()
    st.case, st.plan = case, None
    if case["kind"] == "adamw":
        return _prepare_adamw(st, gen)
    act = torch.tensor(_active(case), device="cuda")
    rows = act.numel()
    st.logits, targets = _logits_of(gen, rows, case)
    st.targets = targets.to(torch.int32)
    st.logp = torch.empty(rows, device="cuda")
    st.lse = torch.empty(rows, device="cuda")
    st.loss = torch.empty(1, device="cuda")
    st.dbuf = torch.empty(rows * case["stride"], dtype=st.logits.dtype, device="cuda").view(rows, case["stride"])
    normal = lambda s: s * torch.randn(rows, generator=gen, device="cuda")  # noqa: E731
    if case["kind"] == "logprobs":
        st.dlogp = normal(1.0)
        return st
    logp = torch.cat([torch.log_softmax(x.float(), 1).gather(1, t[:, None])[:, 0]
                      for x, t in zip(st.logits.split(512), targets.split(512))])
    st.weight = act.float()
    st.workspace = torch.zeros(64 * rows + (1 << 16), dtype=torch.uint8, device="cuda")
    if case["kind"] == "policy":
        st.scale = 1.0 / max(1, int(sum(_active(case))))
        st.old, st.ref, st.advantage = logp + normal(0.15), logp + normal(0.3), normal(1.0)
        if case["pad"]:  # rows behind the last sequence hold no target and whatever the buffer held before
            st.targets[-case["pad"]:] = -1
            st.logits[-case["pad"]:] = math.nan
            for x in (st.old, st.ref, st.advantage):
                x[-case["pad"]:] = math.nan
        return st
    n = _lengths(case)
    st.scale = 1.0 / case["pairs"]
    st.ref = logp + normal(0.3)
    st.offsets = torch.tensor([sum(n[:k]) for k in range(len(n) + 1)], dtype=torch.int32, device="cuda")
    st.rewards = torch.empty(len(n), device="cuda")
    return st


def _nearest(x, top, power):
    return (torch.pow(x.abs() / top.clamp_min(1e-38), 1.0 / power)).nan_to_num_(0.0)


def _prepare_adamw(st, gen):
    case = st.case
    st.starts, total = _starts(case)
    st.sizes = _sizes(case)
    normal = lambda s: torch.randn(total, generator=gen, device="cuda").mul_(s)  # noqa: E731
    live = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, n in zip(st.starts, st.sizes):
        live[a:a + n] = True
    st.theta = normal(0.02) * live
    st.grad = (normal(3e-3) * live).to(DTYPES[case["grads"]])
    st.copy = st.theta.to(torch.bfloat16) if case["copies"] else None
    m, v = normal(1e-3) * live, normal(3e-3).square_() * live
    if case["bits"] == 32:
        st.m, st.v = m, v
    else:  # a state as earlier steps left it
        m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
        st.m_scale, st.v_scale = m.abs().amax(1), v.amax(1)
        st.m = (_nearest(m, st.m_scale[:, None], 2) * 127).round_().mul_(m.sign()).to(torch.int8).view(-1)
        st.v = (_nearest(v, st.v_scale[:, None], 4) * 255).ceil_().clamp_(max=255).to(torch.uint8).view(-1)
        st.m_value, st.v_value = torch.zeros(total, device="cuda"), torch.zeros(total, device="cuda")
    # one weight decay for the matrices, none for the vectors
    st.decays = [case["rank"] > 0 or n > max(case["ffn"], 3 * case["hidden"]) for n in st.sizes]
    st.clock = torch.zeros(8, dtype=torch.int64, device="cuda")
    st.clock[0] = 100  # steps taken so far
    st.sq = torch.zeros(1, dtype=torch.float64, device="cuda")
    st.nonfinite = torch.zeros(1, dtype=torch.int32, device="cuda")
    st.workspace = torch.zeros((1 << 16) + total // 64, dtype=torch.uint8, device="cuda")
    return st


# ---- plain forms ------------------------------------------------------------------------------------------------------


def _plain_logp(st, active):
    """(probabilities in fp32, log-probabilities of the targets and log-sum-exp in fp64)."""
    z = st.logits.float()
    top = z.amax(1)
    e = (z - top[:, None]).exp_()
    s = e.sum(1, dtype=torch.float64)
    lse = top.double() + s.log()
    at = st.targets.long().clamp_min(0)[:, None]
    logp = torch.where(active, (z.gather(1, at)[:, 0].double() - top.double()) - s.log(), 0.0)
    return e, s, lse, logp, at


def _plain_dlogits(st, active, e, s, coef, at):
    """coef ([j is the target] - p_j), zero in rows that do not count."""
    coef = torch.where(active, coef, 0.0)
    of_target = (coef * (1.0 - e.gather(1, at)[:, 0].double() / s)).float()
    d = e.mul_((-coef / s).float()[:, None])
    d.scatter_(1, at, of_target[:, None])
    d = torch.where(active[:, None], d, 0.0)
    return d.to(st.logits.dtype)


def _plain_policy(st):
    active = (st.weight != 0) & (st.targets >= 0)
    e, s, _, logp, at = _plain_logp(st, active)
    old, ref, adv = (torch.where(active, x, 0.0).double() for x in (st.old, st.ref, st.advantage))
    rho, d = (logp - old).exp(), ref - logp
    clipped = torch.minimum(rho * adv, rho.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * adv)
    w = st.weight.double() * st.scale
    each = torch.where(active, w * (KL * (torch.expm1(d) - d) - clipped), 0.0)
    flows = ~(((adv > 0) & (rho > 1 + CLIP_HIGH)) | ((adv < 0) & (rho < 1 - CLIP_LOW)))
    coef = w * (torch.where(flows, -adv * rho, 0.0) - KL * torch.expm1(d))
    return {"loss": each.sum().float().view(1), "logp": logp.float(), "dlogits": _plain_dlogits(st, active, e, s, coef, at)}


def _plain_preference(st):
    active = (st.weight != 0) & (st.targets >= 0)
    e, s, _, logp, at = _plain_logp(st, active)
    n = (st.offsets[1:] - st.offsets[:-1]).long()
    of_row = torch.repeat_interleave(torch.arange(n.numel(), device="cuda"), n)
    part = torch.where(active, st.weight.double() * (logp - st.ref.double()), 0.0)
    sums = torch.zeros(n.numel(), dtype=torch.float64, device="cuda").index_add_(0, of_row, part)
    x = BETA * (sums[0::2] - sums[1::2])
    soft = lambda y: torch.clamp_min(-y, 0) + torch.log1p(torch.exp(-y.abs()))  # noqa: E731  -log sigma(y)
    each = (1 - SMOOTHING) * soft(x) + SMOOTHING * soft(-x)
    slope = st.scale * BETA * (SMOOTHING / (1 + torch.exp(-x)) - (1 - SMOOTHING) / (1 + torch.exp(x)))
    coef = st.weight.double() * torch.stack([slope, -slope], 1).view(-1)[of_row]
    return {"loss": (st.scale * each.sum()).float().view(1), "logp": logp.float(), "rewards": (BETA * sums).float(),
            "dlogits": _plain_dlogits(st, active, e, s, coef, at)}


def _plain_logprobs(st):
    active = torch.ones_like(st.targets, dtype=torch.bool)
    e, s, lse, logp, at = _plain_logp(st, active)
    out = {"logp": logp.float(), "lse": lse.float()}
    if st.case["grad"]:
        out["dlogits"] = _plain_dlogits(st, active, e, s, st.dlogp.double(), at)
    return out


def _dither(total, t, device):
    """Two numbers in (0, 1) for each place, from the seed, the step and the place alone: 16 bits each of a mixed counter."""
    low = 0xFFFFFFFF
    at = torch.arange(total, device=device)
    x = ((at & low) * 0x9E3779B1 + (at >> 32) * 0x85EBCA77 + t * 0xC2B2AE3D + SEED) & low
    for shift, factor in ((16, 0x7FEB352D), (15, 0x46A2CA6B)):
        x = ((x ^ (x >> shift)) * factor) & low
    x = x ^ (x >> 16)
    return ((x & 0xFFFF).double() + 0.5) / 65536, ((x >> 16).double() + 0.5) / 65536


def _plain_encode(x, unit, power, most, u, least):
    """Codes c with c ** power * unit below or above x, taken with the probabilities that keep the mean."""
    c = (x / unit.clamp_min(1e-300)).pow_(1.0 / power).floor_().clamp_(0, most)
    c = torch.where(c.pow(power) * unit > x, c - 1, c)
    c = torch.where(((c + 1).pow(power) * unit <= x) & (c < most), c + 1, c).clamp_(0, most)
    low = c.pow(power) * unit
    up = (c < most) & (u * ((c + 1).pow(power) * unit - low) < x - low)
    c = c + up
    return torch.where((x > 0) & (unit > 0), c.clamp_min(least), torch.zeros_like(c))


def _plain_adamw(st):
    case = st.case
    g = st.grad.float()
    sq = g.double().square().sum().view(1)
    bad = (~torch.isfinite(g).all()).to(torch.int32).view(1)
    go = (bad == 0) & torch.isfinite(sq)
    t = st.clock[:1] + 1
    coef = torch.where(go, (CLIP / (sq.sqrt() + 1e-6)).clamp_max(1.0), 0.0)
    bc1, bc2 = 1 - torch.pow(BETA1, t.double()), 1 - torch.pow(BETA2, t.double())
    total = st.theta.numel()
    if case["bits"] == 32:
        g = g * coef.float()
        m = BETA1 * st.m + (1 - BETA1) * g
        v = BETA2 * st.v + (1 - BETA2) * (g * g)
        m32, v32 = m, v
    else:
        g = g.double() * coef
        sm, sv = st.m_scale.double() / 127 ** 2, st.v_scale.double() / 255 ** 4
        c = st.m.double().view(-1, BLOCK)
        m = BETA1 * (c * c.abs() * sm[:, None]) + (1 - BETA1) * g.view(-1, BLOCK)
        v = BETA2 * (st.v.double().view(-1, BLOCK).pow(4) * sv[:, None]) + (1 - BETA2) * (g * g).view(-1, BLOCK)
        m32, v32 = m.float().view(-1), v.float().view(-1)
    decay = torch.repeat_interleave(torch.tensor([DECAY * d for d in st.decays], device="cuda"),
                                    torch.tensor([b - a for a, b in zip(st.starts, st.starts[1:] + [total])], device="cuda"))
    move = decay * st.theta + (m32 / bc1.float()) / ((v32 / bc2.float()).sqrt() + EPS)
    st.theta.copy_(torch.where(go, st.theta - LR * move, st.theta))
    out = {"theta": st.theta, "sq": sq, "nonfinite": bad}
    if case["bits"] == 32:
        st.m.copy_(torch.where(go, m, st.m))
        st.v.copy_(torch.where(go, v, st.v))
        out["m"], out["v"] = st.m, st.v
    else:
        mt, vt = m.abs().amax(1).float(), v.amax(1).float()
        um, uv = (u.view(-1, BLOCK) for u in _dither(total, t, g.device))
        sm, sv = mt.double()[:, None] / 127 ** 2, vt.double()[:, None] / 255 ** 4
        c = _plain_encode(m.abs(), sm, 2, 127, um, 0) * m.sign()
        st.m.copy_(torch.where(go, c.to(torch.int8).view(-1), st.m))
        st.v.copy_(torch.where(go, _plain_encode(v, sv, 4, 255, uv, 1).to(torch.uint8).view(-1), st.v))
        st.m_scale.copy_(torch.where(go, mt, st.m_scale))
        st.v_scale.copy_(torch.where(go, vt, st.v_scale))
        c = st.m.double().view(-1, BLOCK)
        st.m_value.copy_((c * c.abs() * (st.m_scale.double()[:, None] / 127 ** 2)).view(-1))
        st.v_value.copy_((st.v.double().view(-1, BLOCK).pow(4) * (st.v_scale.double()[:, None] / 255 ** 4)).view(-1))
        out["m"], out["v"] = st.m_value, st.v_value
    if st.copy is not None:
        st.copy.copy_(st.theta)
        out["copy"] = st.copy
    st.clock[:1] += go
    return dict(out, t=st.clock[:1])


# ---- through the library ----------------------------------------------------------------------------------------------


def _own_logits(zb, st):
    return zb.logits(st.logits.data_ptr(), st.logits.shape[0], st.case["vocab"], st.targets.data_ptr(), dtype=st.case["dtype"],
                     row_stride=st.case["stride"])


def _own_logprobs(zb, st, stream):
    x = _own_logits(zb, st)
    zb.token_logprobs(x, st.logp.data_ptr(), st.lse.data_ptr(), stream_handle=stream)
    out = {"logp": st.logp, "lse": st.lse}
    if st.case["grad"]:
        zb.token_logprobs_backward(x, st.lse.data_ptr(), st.dlogp.data_ptr(), st.dbuf.data_ptr(), stream_handle=stream)
        out["dlogits"] = st.dbuf[:, :st.case["vocab"]]
    return out


def _own_policy(zb, st, stream):
    args = zb.policy(st.old.data_ptr(), st.advantage.data_ptr(), ref_logp=st.ref.data_ptr(), weight=st.weight.data_ptr(),
                     clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL, scale=st.scale)
    zb.policy_loss(_own_logits(zb, st), args, st.loss.data_ptr(), st.logp.data_ptr(), st.dbuf.data_ptr(),
                   workspace=st.workspace.data_ptr(), workspace_bytes=st.workspace.numel(), stream_handle=stream)
    return {"loss": st.loss, "logp": st.logp, "dlogits": st.dbuf[:, :st.case["vocab"]]}


def _own_preference(zb, st, stream):
    args = zb.preference(st.ref.data_ptr(), st.offsets.data_ptr(), st.case["pairs"], weight=st.weight.data_ptr(), beta=BETA,
                         label_smoothing=SMOOTHING, scale=st.scale)
    zb.preference_loss(_own_logits(zb, st), args, st.loss.data_ptr(), st.logp.data_ptr(), st.rewards.data_ptr(),
                       st.dbuf.data_ptr(), workspace=st.workspace.data_ptr(), workspace_bytes=st.workspace.numel(), stream_handle=stream)
    return {"loss": st.loss, "logp": st.logp, "rewards": st.rewards, "dlogits": st.dbuf[:, :st.case["vocab"]]}


def _own_adamw(zb, st, stream):
    if st.plan is None:  # the tensors' addresses, listed once as an optimizer does
        each = []
        for k, (a, n) in enumerate(zip(st.starts, st.sizes)):
            one = dict(theta=st.theta[a:].data_ptr(), grad=st.grad[a:].data_ptr(), n=n, grad_dtype=st.case["grads"], decay=st.decays[k],
                       m=st.m[a:].data_ptr(), v=st.v[a:].data_ptr(), first=a)
            if st.copy is not None:
                one["copy16"] = st.copy[a:].data_ptr()
            if st.case["bits"] == 8:
                one.update(m_scale=st.m_scale[a // BLOCK:].data_ptr(), v_scale=st.v_scale[a // BLOCK:].data_ptr())
            each.append(one)
        values = [(st.m_value[a:].data_ptr(), st.v_value[a:].data_ptr()) for a in st.starts] if st.case["bits"] == 8 else None
        st.plan = (zb.adamw_config(bits=st.case["bits"], beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, clip=CLIP, seed=SEED),
                   zb.adamw_tensors(each), zb.adamw_values(values) if values else None)
    config, tensors, values = st.plan
    zb.adamw_grad_norm(tensors, st.sq.data_ptr(), st.nonfinite.data_ptr(), workspace=st.workspace.data_ptr(),
                       workspace_bytes=st.workspace.numel(), stream_handle=stream)
    zb.adamw_step(config, tensors, LR, st.clock.data_ptr(), st.sq.data_ptr(), st.nonfinite.data_ptr(), stream_handle=stream)
    out = {"theta": st.theta, "sq": st.sq, "nonfinite": st.nonfinite, "m": st.m, "v": st.v, "t": st.clock[:1]}
    if st.case["bits"] == 8:
        zb.adamw_read_moments(tensors, values, stream_handle=stream)
        out["m"], out["v"] = st.m_value, st.v_value
    if st.copy is not None:
        out["copy"] = st.copy
    return out


def run(st):
    kind = st.case["kind"]
    if own:
        import paper_2401_10241_amd as zb
        call = {"logprobs": _own_logprobs, "policy": _own_policy, "preference": _own_preference, "adamw": _own_adamw}[kind]
        return call(zb, st, torch.cuda.current_stream().cuda_stream)
    return {"logprobs": _plain_logprobs, "policy": _plain_policy, "preference": _plain_preference, "adamw": _plain_adamw}[kind](st)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------


def _exact_rows(st, rows, objective):
    """Log-probabilities of the rows given and, by differentiation, objective's gradient of their logits."""
    z = st.logits[rows].double().requires_grad_(True)
    logp = torch.log_softmax(z, 1)[torch.arange(z.shape[0], device="cuda"), st.targets[rows].long()]
    if objective is None:
        return logp.detach(), None
    return logp.detach(), torch.autograd.grad(objective(logp), z)[0]


def _exact_logits(st, objective_of):
    """objective_of(logp of the counting rows, their indices) -> a scalar; None for no gradient."""
    case = st.case
    live = torch.tensor(_active(case), device="cuda").nonzero()[:, 0]
    chunks = live.split(max(1, (1 << 25) // case["vocab"]))
    rows = st.logits.shape[0]
    logp = torch.zeros(rows, dtype=torch.float64, device="cuda")
    for c in chunks:
        logp[c] = _exact_rows(st, c, None)[0]
    if objective_of is None:
        return logp, None, None
    leaf = logp[live].requires_grad_(True)
    value = objective_of(leaf, live)
    slope = torch.zeros(rows, dtype=torch.float64, device="cuda")
    slope[live] = torch.autograd.grad(value, leaf)[0]
    # rounded to 32 bits, far finer than the compared type where that is bf16 (memory)
    kept = torch.float32 if case["dtype"] == "bf16" else torch.float64
    d = torch.zeros(rows, case["vocab"], dtype=kept, device="cuda")
    for c in chunks:
        d[c] = _exact_rows(st, c, lambda lp: (slope[c] * lp).sum())[1].to(kept)
    return logp, value.detach().view(1), d


def _exact_adamw(st):
    case = st.case
    f64 = torch.float64
    old = {k: getattr(st, k).to(f64) for k in ("theta", "grad", "m", "v")}
    if case["bits"] == 8:
        per = lambda s: torch.repeat_interleave(s.to(f64), BLOCK)  # noqa: E731
        old["m"] = torch.sign(old["m"]) * (old["m"] / 127) ** 2 * per(st.m_scale)
        old["v"] = (old["v"] / 255) ** 4 * per(st.v_scale)
    sq = (old["grad"] ** 2).sum()
    g = old["grad"] * min(1.0, CLIP / (math.sqrt(float(sq)) + 1e-6))
    t = int(st.clock[0]) + 1
    m = torch.lerp(g, old["m"], BETA1)
    v = torch.lerp(g ** 2, old["v"], BETA2)
    theta = old["theta"].clone()
    for a, n, decays in zip(st.starts, st.sizes, st.decays):
        if decays:
            theta[a:a + n] *= 1 - LR * DECAY
    theta -= LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + EPS)
    if case["bits"] == 8:
        m, v = _exact_held(m, 127, 2, 0, 0, t), _exact_held(v, 255, 4, 1, 1, t)
    out = {"theta": theta, "sq": sq.view(1), "nonfinite": None, "m": m, "v": v, "t": None}
    if st.copy is not None:
        out["copy"] = theta
    return out


def _exact_held(x, most, power, least, which, t):
    """What an 8-bit state holds of x: of the values c ** power * top / most ** power around |x| the upper one where the
    place's number is below the share of the way that |x| lies up."""
    top = x.abs().view(-1, BLOCK).amax(1).float().double()
    ladder = torch.arange(most + 2, dtype=torch.float64, device="cuda") ** power / float(most) ** power
    numbers = _dither(x.numel(), t, "cuda")[which]
    out = torch.zeros_like(x)
    step = 1 << 24
    for a in range(0, x.numel(), step):
        y = x[a:a + step]
        scale = torch.repeat_interleave(top[a // BLOCK:(a + y.numel()) // BLOCK], BLOCK)
        share = torch.where(scale > 0, y.abs() / scale, 0.0)
        c = (torch.searchsorted(ladder, share, right=True) - 1).clamp_(0, most)
        way = (share - ladder[c]) / (ladder[c + 1] - ladder[c])
        c = torch.where((numbers[a:a + step] < way) & (c < most), c + 1, c)
        c = torch.where((y != 0) & (c < least), torch.full_like(c, least), c)
        out[a:a + step] = torch.sign(y) * ladder[c] * scale
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "adamw":
        return _exact_adamw(st)
    if case["kind"] == "logprobs":
        logp, _, d = _exact_logits(st, (lambda lp, live: (lp * st.dlogp[live].double()).sum()) if case["grad"] else None)
        lse = torch.cat([torch.logsumexp(z.double(), 1) for z in st.logits.split(512)])
        return {"logp": logp, "lse": lse, **({"dlogits": d} if case["grad"] else {})}
    if case["kind"] == "policy":
        def policy(lp, live):
            rho, adv, d = torch.exp(lp - st.old[live].double()), st.advantage[live].double(), st.ref[live].double() - lp
            gain = torch.minimum(rho * adv, torch.clamp(rho, 1 - CLIP_LOW, 1 + CLIP_HIGH) * adv)
            return st.scale * (KL * (torch.expm1(d) - d) - gain).sum()
        logp, loss, d = _exact_logits(st, policy)
        return {"loss": loss, "logp": logp, "dlogits": d}
    rewards = []

    def preference(lp, live):
        gap = torch.zeros(st.logits.shape[0], dtype=torch.float64, device="cuda").index_put((live,), lp - st.ref[live].double())
        sums = torch.stack([x.sum() for x in gap.split(_lengths(case))])
        rewards.append((BETA * sums).detach())
        x = rewards[0].new_tensor(BETA) * (sums[0::2] - sums[1::2])
        logsig = torch.nn.functional.logsigmoid
        return -st.scale * ((1 - SMOOTHING) * logsig(x) + SMOOTHING * logsig(-x)).sum()

    logp, loss, d = _exact_logits(st, preference)
    return {"loss": loss, "logp": logp, "rewards": rewards[0], "dlogits": d}
