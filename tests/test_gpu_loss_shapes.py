"""Every kernel that the losses choose between: vocabularies on both sides of each length at which another one takes over, gradients laid out
unlike the logits, losses without a gradient, logits too large for the caches, more pairs than one launch adds up.

Against oracle/losses.py with the tolerances of tests/test_gpu_token_loss.py, or to the bit against calls that are compared with it there."""
import numpy as np
import pytest

from oracle import losses as L
from test_gpu_token_loss import GUARD, U, Case, check_policy, check_preference, dev, policy_inputs, scratch

pytestmark = pytest.mark.gpu

VE = {"fp32": 4, "bf16": 8}
VECTORS = [256, 1024, 2048, 4096, 7168, 8192, 12800]  # of 16 bytes: the longest row of each policy kernel that holds one in registers


@pytest.mark.parametrize("vectors", VECTORS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_policy_at_the_longest_row_of_a_kernel(dtype, vectors):
    most = vectors * VE[dtype]
    for vocab, pad, shift, in_place in ((most, 0, 0, False), (most + VE[dtype] - 1, 1, 3, True), (most + VE[dtype], 0, 0, True), (most + 3 * VE[dtype] + 1, 6, 1, False)):
        k = Case(dtype, 3, vocab, pad, shift, seed=vectors)
        old, ref, adv, w = policy_inputs(k)
        w[:] = [1.5, 0.5, 1.0]
        check_policy(k, 0.07, w, old, ref, adv, in_place=in_place)


@pytest.mark.parametrize("vocab", [16400, 32000, 32771, 60000, 65500])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_policy_inside_a_kernels_range(dtype, vocab):
    for pad, shift, in_place in ((0, 0, False), (5, 1, True)):
        k = Case(dtype, 4, vocab, pad, shift, seed=3)
        old, ref, adv, w = policy_inputs(k)
        check_policy(k, 0.07, w, old, ref, adv, in_place=in_place)


class Apart:
    """A gradient buffer of its own stride and start, with guards."""

    def __init__(self, k, pad, shift):
        import torch
        self.k, self.stride, self.shift = k, k.vocab + pad, shift
        self.flat = torch.full((shift + k.rows * self.stride + 64,), GUARD, dtype=k.kind, device="cuda")

    def args(self):
        return self.flat[self.shift:].data_ptr(), self.stride

    def values(self):
        flat = self.flat.cpu()
        view = flat[self.shift:self.shift + self.k.rows * self.stride].view(self.k.rows, self.stride)
        assert (flat[:self.shift] == GUARD).all() and (flat[self.shift + self.k.rows * self.stride:] == GUARD).all()
        assert (view[:, self.k.vocab:] == GUARD).all()
        return view[:, :self.k.vocab]


@pytest.mark.parametrize("layout", [(0, 1), (3, 0), (8, 2), (1, 5)], ids=str)
@pytest.mark.parametrize("vocab", [5, 257, 8192, 33001, 131073])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradients_laid_out_unlike_the_logits(dtype, vocab, layout):
    """The same bits as in the logits' own layout, which the other tests compare with the oracle."""
    import torch
    import paper_2401_10241_amd as zb
    rows = 7
    k = Case(dtype, rows, vocab, seed=9)
    old, ref, adv, w = policy_inputs(k)
    w[:] = [1, 0.5, 0, 2, 1, 1, 0.25]  # a row without weight
    k.targets[5] = -1                  # and one without a target
    k.place()
    keep = [dev(a) for a in (old, ref, adv, w, np.array([0, 2, 4, 4, 6], np.int32))]
    o, r, a, wt, off = (t.data_ptr() for t in keep)
    ws, loss, lse, logp = scratch(rows, 2), torch.zeros(1, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    space = dict(workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    zb.token_logprobs(k.x(), logp.data_ptr(), lse.data_ptr())
    calls = (lambda d, stride: zb.policy_loss(k.x(), zb.policy(o, a, r, wt, kl_coef=0.1), loss.data_ptr(), 0, d, stride, **space),
             lambda d, stride: zb.preference_loss(k.x(), zb.preference(r, off, 2, wt), loss.data_ptr(), 0, 0, d, stride, **space),
             lambda d, stride: zb.token_logprobs_backward(k.x(), lse.data_ptr(), a, d, stride))
    for call in calls:
        own, other = Apart(k, 0, 0), Apart(k, *layout)
        call(*own.args())
        first = loss.clone()
        call(*other.args())
        assert torch.equal(own.values(), other.values()) and torch.equal(first, loss)
        assert own.values().float().abs().max() > 0


@pytest.mark.parametrize("shape", [(1, 100), (40, 1003), (300, 515), (5, 50257), (4, 131073)], ids=str)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_losses_without_a_gradient(dtype, shape):
    """Loss, log-probabilities and rewards have the bits that they have beside a gradient; the policy's loss alone against the oracle."""
    import torch
    import paper_2401_10241_amd as zb
    rows, vocab = shape
    k = Case(dtype, rows, vocab, pad=3, shift=1)
    old, ref, adv, w = policy_inputs(k)
    w[0] = 1
    if rows > 1:
        k.targets[-1] = -1
        k.place()
    cut = sorted(k.rng.integers(0, rows + 1, 3).tolist())
    keep = [dev(a) for a in (old, ref, adv, w, np.array([0, *cut, rows], np.int32))]
    o, r, a, wt, off = (t.data_ptr() for t in keep)
    ws = scratch(rows, 2)
    space = dict(workspace=ws.data_ptr(), workspace_bytes=ws.numel())

    def outputs(d):
        out = [torch.full((n,), GUARD, device="cuda") for n in (1, rows, 1, rows, 4)]
        p = [t.data_ptr() for t in out]
        zb.policy_loss(k.x(), zb.policy(o, a, r, wt, clip_low=0.2, clip_high=0.28, kl_coef=0.1, scale=0.25), p[0], p[1], d, **space)
        zb.preference_loss(k.x(), zb.preference(r, off, 2, wt), p[2], p[3], p[4], d, **space)
        return out

    alone, beside = outputs(0), outputs(k.dflat[k.shift:].data_ptr())
    for x, y in zip(alone, beside):
        assert torch.equal(x, y)
    on = L.counting(k.targets, vocab, w)
    wl, wlp, _, _ = L.policy(k.z64, k.targets, old, adv, ref, w, 0.2, 0.28, 0.1, 0.25)
    e, _ = k.error(on)
    we = np.where(on, 0.25 * w.astype(np.float64), 0.0)
    rho, gap = np.exp(np.where(on, wlp - old, 0.0)), np.exp(np.where(on, ref - wlp, 0.0))
    assert abs(float(alone[0]) - wl) <= (we * (np.abs(adv) * rho + 0.1 * (gap + 1)) * e).sum() + 2 * U * abs(wl)
    assert (np.abs(alone[1].cpu().double().numpy() - wlp) <= e + U * np.abs(wlp)).all()


@pytest.mark.parametrize("case", [("bf16", 1400, 50432), ("fp32", 1300, 32003), ("bf16", 3000, 50257)], ids=str)
def test_logits_too_large_for_the_caches(case):
    """More than 64 and 256 MB, which are read and written past the caches: the bits of the same rows in calls of 600."""
    import torch
    import paper_2401_10241_amd as zb
    dtype, rows, vocab = case
    gen = torch.Generator(device="cuda").manual_seed(3)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    z = torch.randn(rows, vocab, generator=gen, device="cuda", dtype=kind).mul_(2)
    normal = lambda: torch.randn(rows, generator=gen, device="cuda")  # noqa: E731
    t = torch.randint(-1, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    old, ref, adv, w = normal() - 11, normal() - 11, normal(), (normal() > -0.5).float()
    ws = scratch(rows, 1)
    space = dict(workspace=ws.data_ptr(), workspace_bytes=ws.numel())

    def outputs(a, b):
        n = b - a
        x = zb.logits(z[a:].data_ptr(), n, vocab, t[a:].data_ptr(), dtype=dtype)
        p = zb.policy(old[a:].data_ptr(), adv[a:].data_ptr(), ref[a:].data_ptr(), w[a:].data_ptr(), kl_coef=0.1)
        off = torch.tensor([0, n // 2, n], dtype=torch.int32, device="cuda")
        q = zb.preference(ref[a:].data_ptr(), off.data_ptr(), 1, w[a:].data_ptr())
        vectors = [torch.zeros(n, device="cuda") for _ in range(5)]
        logp, lse, lp_policy, lp_pair, lp_alone = (v.data_ptr() for v in vectors)
        loss, grads = torch.zeros(1, device="cuda"), [torch.empty(n, vocab, dtype=kind, device="cuda") for _ in range(2)]
        zb.token_logprobs(x, logp)
        zb.token_logprobs(x, lp_alone, lse)
        zb.token_logprobs_backward(x, lse, adv[a:].data_ptr(), grads[0].data_ptr())
        zb.policy_loss(x, p, loss.data_ptr(), lp_policy, grads[1].data_ptr(), **space)
        zb.preference_loss(x, q, loss.data_ptr(), lp_pair, 0, 0, **space)
        torch.cuda.synchronize()
        return vectors + grads

    whole = outputs(0, rows)
    for a in range(0, rows, 600):
        a = min(a, rows - 600)
        for x, y in zip(whole, outputs(a, a + 600)):
            assert torch.equal(x[a:a + 600], y)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_more_pairs_than_one_launch_adds_up(dtype):
    rng = np.random.default_rng(4)
    n = rng.integers(0, 5, 2 * 300).tolist()
    k = Case(dtype, sum(n) + 3, 65, pad=2, shift=1)
    w = k.rng.uniform(0.5, 2, k.rows).astype(np.float32)
    w[k.rng.random(k.rows) < 0.2] = 0
    check_preference(k, n, w)
    check_preference(Case(dtype, sum(n) + 3, 65), n, None, in_place=True)
