"""The operators of a post-training step at counts that pass what one launch holds (2^32 lanes), on the GPU through the C ABI."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROWS = (1 << 22) - 1  # the most that a call takes


@pytest.fixture
def room():
    """Frees what torch keeps, before and after; says how many bytes there are."""
    import torch
    torch.cuda.empty_cache()
    yield torch.cuda.mem_get_info()[0]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def test_the_most_rows_of_a_short_vocabulary(room):
    """logp, policy loss and gradient of every row.  With three logits of size 9 at most a row's sum is off by u (2.5 * 18 + 69) and so is
    logp, with its own rounding u * 20; loss and coefficient follow with |A| rho <= 3 e, and the loss of all rows is in 64 bits until
    its one rounding."""
    import torch
    import paper_2401_10241_amd as zb
    rng = np.random.default_rng(5)
    z = np.clip(rng.normal(0, 2, (ROWS, 3)), -9, 9).astype(np.float32)
    targets = rng.integers(-1, 3, ROWS).astype(np.int32)
    z64, on = z.astype(np.float64), targets >= 0
    lse = np.log(np.exp(z64).sum(1))
    logp = np.where(on, z64[np.arange(ROWS), np.maximum(targets, 0)] - lse, 0.0)
    old = (logp + rng.uniform(-1, 1, ROWS)).astype(np.float32)
    adv = np.clip(rng.normal(0, 1, ROWS), -3, 3).astype(np.float32)
    rho = np.exp(logp - old)
    # rows whose ratio is within 1e-3 of a clip bound do not count: either side would be right there
    near = (np.abs(rho - 0.8) < 1e-3) | (np.abs(rho - 1.2) < 1e-3)
    targets[near], on[near], logp[near] = -1, False, 0.0
    dev = {k: torch.from_numpy(v).cuda() for k, v in dict(z=z, t=targets, old=old, adv=adv).items()}
    x = zb.logits(dev["z"].data_ptr(), ROWS, 3, dev["t"].data_ptr(), dtype="fp32")
    out, loss, d = torch.full((ROWS,), 7.0, device="cuda"), torch.zeros(1, device="cuda"), torch.full((ROWS, 3), 7.0, device="cuda")
    space = torch.zeros(zb.loss_workspace_bytes(ROWS), dtype=torch.uint8, device="cuda")
    zb.policy_loss(x, zb.policy(dev["old"].data_ptr(), dev["adv"].data_ptr(), clip_low=0.2, clip_high=0.2, scale=1.0 / ROWS), loss.data_ptr(),
                   out.data_ptr(), d.data_ptr(), workspace=space.data_ptr(), workspace_bytes=space.numel())
    e = U * (2.5 * 18 + 69 + 20)
    assert np.abs(out.double().cpu().numpy() - logp).max() <= e
    a = adv.astype(np.float64)
    moved, kept = rho * a, np.clip(rho, 0.8, 1.2) * a
    want = np.where(on, -np.minimum(moved, kept), 0.0).sum() / ROWS
    most = 3 * np.e  # of |A| rho
    assert abs(float(loss) - want) <= most * e + U * abs(want)
    coef = np.where(on & (moved <= kept), -moved, 0.0) / ROWS
    hot = np.zeros_like(z64)
    hot[np.flatnonzero(on), targets[on]] = 1
    wantd = coef[:, None] * (hot - np.exp(z64 - lse[:, None]))
    # coefficient e of itself, probability e and u (2.5 * 18 + 6) of itself, four roundings
    assert np.abs(d.double().cpu().numpy() - wantd).max() <= most / ROWS * (2 * e + U * (2.5 * 18 + 6 + 4))

    lse32, logp2 = torch.zeros(ROWS, device="cuda"), torch.full((ROWS,), 7.0, device="cuda")
    zb.token_logprobs(x, logp2.data_ptr(), lse32.data_ptr())
    assert np.abs(logp2.double().cpu().numpy() - logp).max() <= e
    dlogp = torch.from_numpy(adv).cuda()
    zb.token_logprobs_backward(x, lse32.data_ptr(), dlogp.data_ptr(), d.data_ptr())
    wantd = np.where(on, a, 0.0)[:, None] * (hot - np.exp(z64 - lse[:, None]))
    assert np.abs(d.double().cpu().numpy() - wantd).max() <= 3 * (e + U * (2.5 * 18 + 6 + 4))


def test_the_most_pairs():
    """Pairs without tokens: log 2 each, except one; 64-bit sums, one rounding."""
    import torch
    import paper_2401_10241_amd as zb
    offsets = np.zeros(2 * ROWS + 1, np.int32)
    at = 2 * (ROWS - 2)  # the last pair but one has a token each
    offsets[at + 1:] = 1
    offsets[at + 2:] = 2
    z = np.array([[0.0, 1.0], [0.5, 0.25]], np.float32)
    z64 = z.astype(np.float64)
    logp = z64[:, 0] - np.log(np.exp(z64).sum(1))
    dev = [torch.from_numpy(v).cuda() for v in (z, np.zeros(2, np.int32), offsets, np.zeros(2, np.float32))]
    x = zb.logits(dev[0].data_ptr(), 2, 2, dev[1].data_ptr(), dtype="fp32")
    loss, rewards = torch.zeros(1, device="cuda"), torch.full((2 * ROWS,), 7.0, device="cuda")
    space = torch.zeros(zb.loss_workspace_bytes(2, ROWS), dtype=torch.uint8, device="cuda")
    zb.preference_loss(x, zb.preference(dev[3].data_ptr(), dev[2].data_ptr(), ROWS, beta=0.5, scale=1.0 / ROWS), loss.data_ptr(), 0, rewards.data_ptr(),
                       0, workspace=space.data_ptr(), workspace_bytes=space.numel())
    want = ((ROWS - 1) * np.log(2.0) + np.log1p(np.exp(-0.5 * (logp[0] - logp[1])))) / ROWS
    assert abs(float(loss) - want) <= 4 * U * want  # its rounding, and the one pair's 1e-7 among four million
    got = rewards.double().cpu().numpy()
    assert np.abs(got[at:at + 2] - 0.5 * logp).max() <= U * 80
    got[at:at + 2] = 0
    assert not got.any()


def test_a_gradient_of_more_rows_than_a_launch_holds(room):
    """Rows of five workgroups, so that the last fifth of the most rows is a launch of its own; in place, a few rows with a weight."""
    import torch
    import paper_2401_10241_amd as zb
    vocab = 8400
    if room < ROWS * vocab * 4 + (16 << 30):
        pytest.skip("141 GB of logits do not fit")
    z = torch.full((ROWS, vocab), 0.5, device="cuda")
    some = sorted({0, 1, ROWS - 1, ROWS - 2} | {((1 << 24) - 1) // 5 + k for k in (-2, -1, 0, 1)})
    rng = np.random.default_rng(6)
    part = rng.normal(0, 2, (len(some), vocab)).astype(np.float32)
    for r, row in zip(some, part):
        z[r].copy_(torch.from_numpy(row))
    targets, dlogp, lse = torch.zeros(ROWS, dtype=torch.int32, device="cuda"), torch.zeros(ROWS, device="cuda"), torch.zeros(ROWS, device="cuda")
    logp = torch.zeros(ROWS, device="cuda")
    index = torch.tensor(some, device="cuda")
    targets[index], dlogp[index] = 8399, 0.75
    x = zb.logits(z.data_ptr(), ROWS, vocab, targets.data_ptr(), dtype="fp32")
    zb.token_logprobs(x, logp.data_ptr(), lse.data_ptr())
    zb.token_logprobs_backward(x, lse.data_ptr(), dlogp.data_ptr(), z.data_ptr())
    p64 = part.astype(np.float64)
    want_lse = np.log(np.exp(p64).sum(1))
    p = np.exp(p64 - want_lse[:, None])
    far = np.abs(p64 - want_lse[:, None])
    e = U * (2.5 * far.max() + vocab / 256 + 69)
    assert np.abs(lse[index].double().cpu().numpy() - want_lse).max() <= e + U * 12
    # the rows of 0.5 everywhere, all of them: log(8400) + 0.5 and its rounding
    lse[index] = float(np.log(vocab) + 0.5)
    assert float((lse.double() - (np.log(vocab) + 0.5)).abs().max()) <= U * (vocab / 256 + 69 + 10)
    hot = np.zeros_like(p)
    hot[:, 8399] = 1
    want = 0.75 * (hot - p)
    got = z[index].double().cpu().numpy()
    assert (np.abs(got - want) <= 0.75 * p * (e + U * (12 + 2.5 * far + 6)) + 4 * U * 0.75 * hot + U * np.abs(want)).all()
    z[index] = 0
    for r in range(0, ROWS, 1 << 18):
        assert not bool(z[r:r + (1 << 18)].any()), f"rows from {r} on"


def test_a_tensor_of_more_values_than_a_launch_holds(room):
    """8-bit states of 2^34 + 5000 values: what lies past the first launch has the bits that a tensor of its own in those places gets."""
    import torch
    import paper_2401_10241_amd as zb
    base, tail = 1 << 34, 5000
    n = base + tail
    if room < n * 8 + (24 << 30):
        pytest.skip("138 GB of parameters, gradients and states do not fit")

    def tensors(n):
        return dict(theta=torch.ones(n, device="cuda"), grad=torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda"),
                    m=torch.zeros(n, dtype=torch.int8, device="cuda"), v=torch.zeros(n, dtype=torch.uint8, device="cuda"),
                    m_scale=torch.zeros((n + 255) // 256, device="cuda"), v_scale=torch.zeros((n + 255) // 256, device="cuda"))

    def listed(t, first):
        return {**{k: v.data_ptr() for k, v in t.items()}, "n": t["theta"].numel(), "first": first, "grad_dtype": "bf16", "decay": True}

    from_ = base - 2048  # what is compared: the last of the first launch, too
    big, small = tensors(n), tensors(n - from_)
    g = torch.from_numpy(np.random.default_rng(7).normal(0, 1, n - from_).astype(np.float32)).cuda().bfloat16()
    big["grad"][from_:] = g
    small["grad"].copy_(g)
    sq, bad = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    one, other = zb.adamw_tensors([listed(big, 0)]), zb.adamw_tensors([listed(small, from_)])
    space = torch.zeros(zb.adamw_workspace_bytes(one), dtype=torch.uint8, device="cuda")
    zb.adamw_grad_norm(one, sq.data_ptr(), bad.data_ptr(), workspace=space.data_ptr(), workspace_bytes=space.numel())
    want = from_ * 2.0 ** -20 + float((g.double() ** 2).sum())
    assert abs(float(sq) - want) <= 1e-12 * want and int(bad) == 0
    cfg = zb.adamw_config(bits=8, clip=1.0, weight_decay=0.1, seed=3)
    for t in (one, other):
        clock = torch.zeros(8, dtype=torch.int64, device="cuda")
        zb.adamw_step(cfg, t, 1e-2, clock.data_ptr(), sq.data_ptr(), bad.data_ptr())
        assert int(clock[0]) == 1
    for k, v in small.items():
        tailed = big[k][from_ // 256:] if k.endswith("scale") else big[k][from_:]
        assert torch.equal(tailed, v), k
    # the first 2^34: one gradient everywhere is the block's largest, code 127 and 255, and theta moves alike
    assert int(big["m"][:from_].min()) == 127 and int(big["v"][:from_].min()) == 255
    for at in range(0, from_, 1 << 30):
        part = big["theta"][at:min(at + (1 << 30), from_)]
        low, high = (float(y) for y in part.aminmax())
        assert low == high and abs(low - (1 - 1e-2 * (0.1 + 1))) <= 1e-4, f"values from {at} on"

    # moments as values and back keep the codes
    del big["theta"], big["grad"]
    torch.cuda.empty_cache()
    if room < n * 10 + (24 << 30):
        return
    m, v = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    some = zb.adamw_tensors([{**{k: t.data_ptr() for k, t in big.items()}, "n": n}])
    zb.adamw_read_moments(some, zb.adamw_values([(m.data_ptr(), v.data_ptr())]))
    assert float(m[from_ - 1]) == float(big["m_scale"][from_ // 256 - 1]) and float(m[0]) == float(m[from_ - 1]) and float(v[0]) == float(v[from_ - 1])
    old = {k: t[from_ // 256 if k.endswith("scale") else from_:].clone() for k, t in big.items()}
    for t in big.values():
        t.zero_()
    zb.adamw_write_moments(some, zb.adamw_values([(m.data_ptr(), v.data_ptr())]))
    for k, t in big.items():
        assert torch.equal(t[from_ // 256 if k.endswith("scale") else from_:], old[k]), k
    assert int(big["m"][:from_].min()) == 127 and int(big["v"][:from_].min()) == 255
