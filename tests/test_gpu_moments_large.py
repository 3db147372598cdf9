"""8-bit moments of more values than a launch holds read out and written back: a test of its own, so that it is seen to be left out where the memory
is too small."""
import pytest

pytestmark = pytest.mark.gpu


def test_moments_of_a_tensor_of_more_values_than_a_launch_holds():
    """2^34 + 5000 values: those of the first launch all at the blocks' top code, a ragged end with codes of every kind."""
    import torch
    import paper_2401_10241_amd as zb
    torch.cuda.empty_cache()
    n, tail = (1 << 34) + 5000, 5000
    if torch.cuda.mem_get_info()[0] < n * 10 + (16 << 30):
        pytest.skip("172 GB of moments do not fit")
    blocks = (n + 255) // 256
    gen = torch.Generator(device="cuda").manual_seed(2)
    st = dict(m=torch.full((n,), 127, dtype=torch.int8, device="cuda"), v=torch.full((n,), 255, dtype=torch.uint8, device="cuda"),
              m_scale=torch.full((blocks,), 0.5, device="cuda"), v_scale=torch.full((blocks,), 0.25, device="cuda"))
    st["m"][-tail:] = torch.randint(-127, 128, (tail,), generator=gen, device="cuda", dtype=torch.int8)
    st["v"][-tail:] = torch.randint(0, 256, (tail,), generator=gen, device="cuda", dtype=torch.uint8)
    st["m"][-tail::256], st["v"][-tail::256] = 127, 255  # every block holds its scale, so that it comes back
    st["m"][-1], st["v"][-1] = 127, 255
    m, v = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    tensors = zb.adamw_tensors([{**{k: t.data_ptr() for k, t in st.items()}, "n": n}])
    values = zb.adamw_values([(m.data_ptr(), v.data_ptr())])
    zb.adamw_read_moments(tensors, values)
    for part, want in ((m, 0.5), (v, 0.25)):
        for a in range(0, n - tail, 1 << 31):
            low, high = part[a:min(a + (1 << 31), n - tail)].aminmax()
            assert abs(float(low) - want) <= 2.0 ** -23 and float(low) == float(high), f"values from {a} on"
    cm, cv = st["m"][-tail:].double(), st["v"][-tail:].double()
    for got, want in ((m[-tail:], cm.sign() * (cm / 127) ** 2 * 0.5), (v[-tail:], (cv / 255) ** 4 * 0.25)):
        assert bool(((got.double() - want).abs() <= 2.0 ** -23 * want.abs()).all())
    old = {k: t[-tail:].clone() for k, t in st.items()}
    for t in st.values():
        t.zero_()
    zb.adamw_write_moments(tensors, values)
    for k, t in st.items():
        if k in ("m", "v"):
            assert torch.equal(t[-tail:], old[k]), k
            full = 127 if k == "m" else 255
            for a in range(0, n - tail, 1 << 32):
                low, high = t[a:min(a + (1 << 32), n - tail)].aminmax()
                assert int(low) == int(high) == full, f"codes from {a} on"
    assert abs(float(st["m_scale"][0]) - 0.5) <= 2.0 ** -24 and abs(float(st["v_scale"][-1]) - 0.25) <= 2.0 ** -25
    del st, m, v, part
    torch.cuda.empty_cache()
