"""The operators of a post-training step one after the other, as a program uses them: log-probabilities of the old and the reference policy, the
policy or the preference loss and the gradient of the logits, the products that carry it to a head and its adapter (in 64 bits, outside the library),
the norm of all gradients and the step with moments in 32 or 8 bits.  Each operator is checked from what it was given: the loss from the device's
logits, the step from the device's gradients.

Tolerances: those of the operators' own tests, with u = 2^-24 and rows of 600 logits of spread 2 around the top: e = u (2.5 * 12 + 600 / 256 + 69)."""
import numpy as np
import pytest

from oracle import adamw_many as A
from oracle import losses as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
E = U * (2.5 * 12 + 600 / 256 + 69)
ROWS, H, V, RANK = 96, 40, 600, 5
LR, DECAY, CLIP = 5e-3, 0.05, 0.5


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_steps_of_a_policy_beside_its_reference(kind, bits):
    import torch
    import paper_2401_10241_amd as zb
    rng = np.random.default_rng(bits + len(kind))
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        s = stream.cuda_stream
        new = lambda *shape, dtype=torch.float32: torch.zeros(*shape, dtype=dtype, device="cuda")  # noqa: E731
        x = torch.from_numpy(rng.normal(size=(ROWS, H))).cuda()
        base = torch.from_numpy(rng.normal(size=(H, V))).cuda() / H ** 0.5 * 2
        sizes, at = {"down": H * RANK, "up": RANK * V, "bias": V}, {"down": 0, "up": 256, "bias": 256 + RANK * V // 256 * 256 + 256}
        theta, grad, m, v = new(8192), new(8192), None, None
        theta[:H * RANK] = torch.from_numpy(rng.normal(size=H * RANK).astype(np.float32)).cuda() * 0.3
        m, v = (new(8192), new(8192)) if bits == 32 else (new(8192, dtype=torch.int8), new(8192, dtype=torch.uint8))
        scales = new(2, 32)
        entry = lambda n: dict(theta=theta[at[n]:].data_ptr(), grad=grad[at[n]:].data_ptr(), m=m[at[n]:].data_ptr(), v=v[at[n]:].data_ptr(),  # noqa: E731
                               n=sizes[n], first=at[n], decay=n != "bias",
                               **({} if bits == 32 else dict(m_scale=scales[0, at[n] // 256:].data_ptr(), v_scale=scales[1, at[n] // 256:].data_ptr())))
        tensors = zb.adamw_tensors([entry(n) for n in sizes])
        config = zb.adamw_config(bits=bits, weight_decay=DECAY, clip=CLIP, seed=5)
        clock, sq, bad = new(8, dtype=torch.int64), new(1, dtype=torch.float64), new(1, dtype=torch.int32)
        part = lambda n: theta[at[n]:at[n] + sizes[n]].double()  # noqa: E731

        def logits():
            down, up = part("down").view(H, RANK), part("up").view(RANK, V)
            return (x @ base + (x @ down) @ up + part("bias")).float().contiguous()

        targets = rng.integers(0, V, ROWS).astype(np.int32)
        targets[-4:] = -1
        weight = (np.arange(ROWS) % 24 >= 5).astype(np.float32)
        dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        t, w, off = dev(targets), dev(weight), dev(np.array([0, 24, 48, 72, ROWS], np.int32))
        adv = rng.normal(size=ROWS).astype(np.float32)
        a = dev(adv)
        ref, old, lse, logp, loss, rewards = new(ROWS), new(ROWS), new(ROWS), new(ROWS), new(1), new(4)
        space = new(zb.loss_workspace_bytes(ROWS, 2), dtype=torch.uint8)
        norm_space = new(zb.adamw_workspace_bytes(tensors), dtype=torch.uint8)
        z = logits()
        zb.token_logprobs(zb.logits(z.data_ptr(), ROWS, V, t.data_ptr(), dtype="fp32"), ref.data_ptr(), lse.data_ptr(), stream_handle=s)
        want, _ = L.logprobs(z.double().cpu().numpy(), targets)
        assert (np.abs(ref.double().cpu().numpy() - want) <= E + U * np.abs(want)).all() and not ref[-4:].any()
        mo, vo = {n: np.zeros(k) for n, k in sizes.items()}, {n: np.zeros(k) for n, k in sizes.items()}
        for step in range(1, 5):
            z = logits()
            if step % 2 == 1:  # every other step draws anew
                zb.token_logprobs(zb.logits(z.data_ptr(), ROWS, V, t.data_ptr(), dtype="fp32"), old.data_ptr(), stream_handle=s)
            d = torch.empty_like(z)
            xz = zb.logits(z.data_ptr(), ROWS, V, t.data_ptr(), dtype="fp32")
            ws = dict(workspace=space.data_ptr(), workspace_bytes=space.numel(), stream_handle=s)
            if kind == "policy":
                args = zb.policy(old.data_ptr(), a.data_ptr(), ref_logp=ref.data_ptr(), weight=w.data_ptr(), kl_coef=0.2, scale=0.05)
                zb.policy_loss(xz, args, loss.data_ptr(), logp.data_ptr(), d.data_ptr(), **ws)
                o, r = old.double().cpu().numpy(), ref.double().cpu().numpy()
                wl, wlp, c, wd = L.policy(z.double().cpu().numpy(), targets, o, adv, r, weight, 0.2, 0.2, 0.2, 0.05)
                on = L.counting(targets, V, weight)
                ratio = np.exp(np.where(on, wlp - o, 0))
                # a ratio as near to a border as the device's error could fall on its other side: none here
                assert (np.abs(ratio[on][:, None] - [0.8, 1.2]) > 4 * E).all()
                slack = 0.05 * weight * (np.abs(adv) * ratio + 0.2 * (np.exp(np.where(on, r - wlp, 0)) + 1)) * E
                assert abs(float(loss) - wl) <= slack.sum() + 2 * U * abs(wl)
            else:
                args = zb.preference(ref.data_ptr(), off.data_ptr(), 2, weight=w.data_ptr(), beta=0.5, scale=0.5)
                zb.preference_loss(xz, args, loss.data_ptr(), logp.data_ptr(), rewards.data_ptr(), d.data_ptr(), **ws)
                wl, wlp, wr, c, wd = L.preference(z.double().cpu().numpy(), targets, ref.double().cpu().numpy(), [0, 24, 48, 72, ROWS], weight, 0.5, 0.0, 0.5)
                slack = 0.5 * 0.5 / 4 * 48 * E * weight  # |d slope / d x| <= scale beta / 4, x off by the errors of 48 rows at most
                assert abs(float(loss) - wl) <= 0.5 * 2 * 48 * E + 2 * U * wl
            got = d.double().cpu().numpy()
            assert (np.abs(got - wd) <= (slack + np.abs(c) * 3 * E)[:, None] + U * np.abs(wd)).all()
            dd, down, up = d.double(), part("down").view(H, RANK), part("up").view(RANK, V)
            for n, g in (("down", x.T @ (dd @ up.T)), ("up", (x @ down).T @ dd), ("bias", dd.sum(0))):
                grad[at[n]:at[n] + sizes[n]] = g.reshape(-1).float()
            before = {n: part(n).cpu().numpy() for n in sizes}
            g64 = {n: grad[at[n]:at[n] + sizes[n]].double().cpu().numpy() for n in sizes}
            zb.adamw_grad_norm(tensors, sq.data_ptr(), bad.data_ptr(), workspace=norm_space.data_ptr(), workspace_bytes=norm_space.numel(), stream_handle=s)
            zb.adamw_step(config, tensors, LR, clock.data_ptr(), sq.data_ptr(), bad.data_ptr(), stream_handle=s)
            total = sum((g * g).sum() for g in g64.values())
            assert abs(float(sq) - total) <= 1e-12 * total and int(clock[0]) == step
            for n, k in sizes.items():
                th, mo[n], vo[n] = A.step(before[n], g64[n], mo[n], vo[n], step, lr=LR, beta1=0.9, beta2=0.95, eps=1e-8, decay=DECAY * (n != "bias"),
                                          coef=A.coefficient(total, CLIP))
                after = part(n).cpu().numpy()
                # lr times 24 u for each step that m and v have been through, of an update of at most (1 + beta1 terms) 3.2 at beta2 = 0.95
                assert (np.abs(after - th) <= U * (2 * np.abs(th) + 24 * step * LR * 3.2)).all()
                if bits == 8:
                    um, uv = A.numbers(np.arange(k) + at[n], step, 5)
                    for codes, top, x64, u, most, power, least, keep in ((m, scales[0], mo, um, 127, 2, 0, mo), (v, scales[1], vo, uv, 255, 4, 1, vo)):
                        c8, t8 = A.encode(x64[n], most, power, least, u)
                        assert np.array_equal(codes[at[n]:at[n] + k].cpu().numpy(), c8)
                        keep[n] = A.decode(c8, top[at[n] // 256:at[n] // 256 + len(t8)].cpu().numpy(), most, power)
    assert torch.isfinite(theta).all()
