"""AdamW over lists whose states no cache holds: the bits of the same tensors in lists of their own, and the norm in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grads", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_states_past_the_caches(bits, grads):
    import torch
    import paper_2401_10241_amd as zb
    total = {32: 25_000_000, 8: 50_000_000}[bits]
    sizes = [total // 2 + 3, 1025, total // 2 - 256 * 1000, 77]  # ragged tails; every tensor starts on a block
    gen = torch.Generator(device="cuda").manual_seed(bits)
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // 256) * 256

    def state():
        gen.manual_seed(bits)
        kind = torch.bfloat16 if grads == "bf16" else torch.float32
        st = dict(theta=torch.randn(at, generator=gen, device="cuda"), grad=torch.randn(at, generator=gen, device="cuda").to(kind),
                  copy16=torch.zeros(at, dtype=torch.bfloat16, device="cuda"))
        if bits == 32:
            st.update(m=torch.randn(at, generator=gen, device="cuda"), v=torch.rand(at, generator=gen, device="cuda"))
        else:
            st.update(m=torch.randint(-127, 128, (at,), generator=gen, device="cuda", dtype=torch.int8),
                      v=torch.randint(0, 256, (at,), generator=gen, device="cuda", dtype=torch.uint8),
                      m_scale=torch.rand(at // 256, generator=gen, device="cuda"), v_scale=torch.rand(at // 256, generator=gen, device="cuda"))
        return st

    def listed(st, k, a=0, b=None):
        """Values a to b of tensor k."""
        b = sizes[k] if b is None else b
        s = starts[k] + a
        return {**{name: (t[s // 256:] if name.endswith("scale") else t[s:]).data_ptr() for name, t in st.items()}, "n": b - a, "first": s,
                "grad_dtype": grads, "decay": k % 2 == 0}

    sq, bad = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    one, many = state(), state()
    tensors = zb.adamw_tensors([listed(one, k) for k in range(4)])
    space = torch.zeros(zb.adamw_workspace_bytes(tensors), dtype=torch.uint8, device="cuda")
    zb.adamw_grad_norm(tensors, sq.data_ptr(), bad.data_ptr(), workspace=space.data_ptr(), workspace_bytes=space.numel())
    want = sum(float((one["grad"][s:s + n].double() ** 2).sum()) for s, n in zip(starts, sizes))
    assert abs(float(sq) - want) <= 1e-12 * want and int(bad) == 0
    cfg = zb.adamw_config(bits=bits, clip=100.0, seed=7)
    clocks = torch.zeros(8 * 100, dtype=torch.int64, device="cuda")
    for step in range(2):
        zb.adamw_step(cfg, tensors, 1e-2, clocks.data_ptr(), sq.data_ptr(), bad.data_ptr())
    parts = [(k, a, min(a + 4096 * 256, sizes[k])) for k in range(4) for a in range(0, sizes[k], 4096 * 256)]
    assert len(parts) < 99
    for i, part in enumerate(parts):
        for step in range(2):
            zb.adamw_step(cfg, zb.adamw_tensors([listed(many, *part)]), 1e-2, clocks[8 * (i + 1):].data_ptr(), sq.data_ptr(), bad.data_ptr())
    assert int(clocks[0]) == 2
    for name in one:
        assert torch.equal(one[name], many[name]), name
    assert not torch.equal(one["theta"], state()["theta"])


def test_norm_of_gradients_past_the_caches():
    import torch
    import paper_2401_10241_amd as zb
    for kind, n, dtype in ((torch.float32, 70_000_003, "fp32"), (torch.bfloat16, 140_000_003, "bf16")):
        g = torch.randn(n + 1, device="cuda").to(kind)
        for lead in (0, 1):
            t = zb.adamw_tensors([dict(grad=g[lead:].data_ptr(), n=n, grad_dtype=dtype)])
            space = torch.zeros(zb.adamw_workspace_bytes(t), dtype=torch.uint8, device="cuda")
            sq, bad = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
            for value in (None, float("inf")):
                if value is not None:
                    g[n - 2] = value
                zb.adamw_grad_norm(t, sq.data_ptr(), bad.data_ptr(), workspace=space.data_ptr(), workspace_bytes=space.numel())
                assert int(bad) == (value is not None)
                if value is None:
                    want = sum(float((p.double() ** 2).sum()) for p in g[lead:lead + n].split(1 << 25))
                    assert abs(float(sq) - want) <= 1e-12 * want
            g[n - 2] = 0.5
