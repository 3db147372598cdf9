"""What the operators on the caller's own device memory refuse: checked on the host before anything is launched, so the
refusals need no GPU (the addresses below are never followed)."""
import ctypes as C

import pytest

import paper_2401_10241_amd as zb

AT = 1 << 20  # an address of the right alignment


def rc_of(f, *a, **k):
    try:
        f(*a, **k)
    except zb.ZbError as e:
        return e.status
    return zb.OK


def good_logits(**k):
    return zb.logits(**{**dict(logits_ptr=AT, rows=4, vocab=100, targets_ptr=AT, dtype="fp32", row_stride=104), **k})


def changed(struct, **k):
    for name, value in k.items():
        setattr(struct, name, value)
    return struct


BAD_LOGITS = [dict(logits_ptr=0), dict(targets_ptr=0), dict(logits_ptr=AT + 2), dict(targets_ptr=AT + 2), dict(rows=-1), dict(rows=(1 << 24) + 1),
              dict(vocab=0), dict(vocab=(1 << 18) + 1, row_stride=1 << 19), dict(row_stride=99), dict(row_stride=(1 << 32) + 1),
              dict(dtype="bf16", logits_ptr=AT + 1)]


@pytest.mark.parametrize("bad", BAD_LOGITS, ids=str)
def test_bad_logits(bad):
    x, ws = good_logits(**bad), dict(workspace=AT, workspace_bytes=1 << 30)
    assert rc_of(zb.token_logprobs, x, AT, AT) == zb.EINVAL
    assert rc_of(zb.token_logprobs_backward, x, AT, AT, AT) == zb.EINVAL
    assert rc_of(zb.policy_loss, x, zb.policy(AT, AT), AT, AT, AT, **ws) == zb.EINVAL
    assert rc_of(zb.preference_loss, x, zb.preference(AT, AT, 1), AT, AT, AT, AT, **ws) == zb.EINVAL


def test_bad_arguments_of_the_logprobs():
    x = good_logits()
    assert rc_of(zb.token_logprobs, changed(good_logits(), dtype=7), AT) == zb.EINVAL
    assert rc_of(zb.token_logprobs, x, 0) == zb.EINVAL
    assert rc_of(zb.token_logprobs, x, AT + 2) == zb.EINVAL
    assert rc_of(zb.token_logprobs, x, AT, AT + 1) == zb.EINVAL
    for a in ((0, AT, AT), (AT, 0, AT), (AT, AT, 0), (AT + 1, AT, AT), (AT, AT + 2, AT), (AT, AT, AT + 2)):
        assert rc_of(zb.token_logprobs_backward, x, *a) == zb.EINVAL
    assert rc_of(zb.token_logprobs_backward, x, AT, AT, AT, 99) == zb.EINVAL
    assert rc_of(zb.token_logprobs_backward, x, AT, AT, AT, -104) == zb.EINVAL
    assert rc_of(zb.token_logprobs_backward, x, AT, AT, AT, 108) == zb.EINVAL  # in place, with another stride
    assert zb.lib.zb_token_logprobs(None, AT, AT, None) == zb.EINVAL


def test_bad_arguments_of_the_losses():
    x, nan, inf = good_logits(), float("nan"), float("inf")
    need = zb.loss_workspace_bytes(4)
    ws = dict(workspace=AT, workspace_bytes=need)
    call = lambda p, loss=AT, logp=AT, d=AT, stride=0, **k: rc_of(zb.policy_loss, x, p, loss, logp, d, stride, **{**ws, **k})  # noqa: E731
    for p in (zb.policy(0, AT), zb.policy(AT, 0), zb.policy(AT, AT, kl_coef=0.1), zb.policy(AT, AT, clip_low=-0.1), zb.policy(AT, AT, clip_low=1.1),
              zb.policy(AT, AT, clip_high=-0.1), zb.policy(AT, AT, clip_high=inf), zb.policy(AT, AT, clip_low=nan), zb.policy(AT, AT, AT, kl_coef=-1.0),
              zb.policy(AT, AT, AT, kl_coef=nan), zb.policy(AT, AT, scale=nan), zb.policy(AT + 1, AT), zb.policy(AT, AT + 2), zb.policy(AT, AT, AT + 2),
              zb.policy(AT, AT, weight=AT + 2)):
        assert call(p) == zb.EINVAL
    good = zb.policy(AT, AT)
    for k in (dict(loss=0), dict(loss=AT + 2), dict(logp=AT + 2), dict(d=AT + 2), dict(stride=99), dict(workspace=0), dict(workspace=AT + 4),
              dict(workspace_bytes=need - 1)):
        assert call(good, **k) == zb.EINVAL
    need = zb.loss_workspace_bytes(4, 9)
    assert need > zb.loss_workspace_bytes(4)
    ws = dict(workspace=AT, workspace_bytes=need)
    call = lambda p, loss=AT, logp=AT, r=AT, d=AT, stride=0, **k: rc_of(zb.preference_loss, x, p, loss, logp, r, d, stride, **{**ws, **k})  # noqa: E731
    for p in (zb.preference(0, AT, 9), zb.preference(AT, 0, 9), zb.preference(AT, AT, -1), zb.preference(AT, AT, (1 << 24) + 1),
              zb.preference(AT, AT, 9, beta=nan), zb.preference(AT, AT, 9, label_smoothing=-0.1), zb.preference(AT, AT, 9, label_smoothing=1.1),
              zb.preference(AT, AT, 9, scale=inf), zb.preference(AT + 2, AT, 9), zb.preference(AT, AT + 2, 9), zb.preference(AT, AT, 9, weight=AT + 1)):
        assert call(p) == zb.EINVAL
    good = zb.preference(AT, AT, 9)
    for k in (dict(loss=0), dict(r=AT + 2), dict(logp=AT + 2), dict(d=AT + 2), dict(stride=99), dict(workspace=0), dict(workspace=AT + 4),
              dict(workspace_bytes=need - 1)):
        assert call(good, **k) == zb.EINVAL
    for rows, pairs in ((-1, 0), (0, -1), ((1 << 24) + 1, 0)):
        assert rc_of(zb.loss_workspace_bytes, rows, pairs) == zb.EINVAL


def tensor(**k):
    return {**dict(theta=AT, grad=AT, m=AT, v=AT, m_scale=AT, v_scale=AT, n=1000), **k}


def test_bad_arguments_of_the_optimizer():
    nan, inf = float("nan"), float("inf")
    cfg = {b: zb.adamw_config(bits=b) for b in (8, 32)}
    step = lambda c, t, lr=1e-3, state=AT, sq=AT, nf=AT: rc_of(zb.adamw_step, c, zb.adamw_tensors(t), lr, state, sq, nf)  # noqa: E731
    for bits in (8, 32):
        for t in (tensor(theta=0), tensor(grad=0), tensor(m=0), tensor(v=0), tensor(theta=AT + 2), tensor(grad=AT + 2), tensor(copy16=AT + 1),
                  tensor(n=-1), tensor(n=(1 << 38) + 1), tensor(first=-1), tensor(grad=AT + 1, grad_dtype="bf16")):
            assert step(cfg[bits], [tensor(), t]) == zb.EINVAL
        for k in (dict(lr=nan), dict(lr=inf), dict(state=0), dict(state=AT + 4), dict(sq=0), dict(nf=0), dict(sq=AT + 4), dict(nf=AT + 2)):
            assert step(cfg[bits], [tensor()], **k) == zb.EINVAL
        for k in (dict(beta1=0.0), dict(beta1=1.0), dict(beta2=nan), dict(eps=0.0), dict(eps=inf), dict(clip=0.0), dict(clip=nan),
                  dict(weight_decay=nan)):
            assert step(zb.adamw_config(bits=bits, **k), [tensor()]) == zb.EINVAL
    for t in (tensor(m_scale=0), tensor(v_scale=0), tensor(m_scale=AT + 2)):
        assert step(cfg[8], [t]) == zb.EINVAL
    for t in (tensor(m=AT + 2), tensor(v=AT + 1)):
        assert step(cfg[32], [t]) == zb.EINVAL
    assert step(cfg[8], [tensor()], sq=0, nf=0) == zb.EINVAL  # codes cannot hold a NaN
    assert step(zb.adamw_config(bits=16), [tensor()]) == zb.EINVAL
    assert zb.lib.zb_adamw_step(cfg[32], None, 1, 1e-3, AT, None, None, None) == zb.EINVAL
    assert zb.lib.zb_adamw_step(cfg[32], zb.adamw_tensors([tensor()]), -1, 1e-3, AT, None, None, None) == zb.EINVAL
    odd = zb.adamw_tensors([tensor()])
    odd[0].grad_dtype = 5
    assert rc_of(zb.adamw_step, cfg[32], odd, 1e-3, AT, AT, AT) == zb.EINVAL
    with pytest.raises(TypeError):
        zb.adamw_tensors([tensor(gard=AT)])


def test_bad_arguments_of_the_norm_and_of_moving_moments():
    t = zb.adamw_tensors([tensor(n=100000)])
    need = zb.adamw_workspace_bytes(t)
    norm = lambda tt=t, sq=AT, nf=AT, ws=AT, n=need: rc_of(zb.adamw_grad_norm, tt, sq, nf, workspace=ws, workspace_bytes=n)  # noqa: E731
    for k in (dict(sq=0), dict(nf=0), dict(sq=AT + 4), dict(nf=AT + 1), dict(ws=0), dict(ws=AT + 4), dict(n=need - 1),
              dict(tt=zb.adamw_tensors([tensor(grad=0)])), dict(tt=zb.adamw_tensors([tensor(grad=AT + 2)])), dict(tt=zb.adamw_tensors([tensor(n=-5)]))):
        assert norm(**k) == zb.EINVAL
    values = zb.adamw_values([(AT, AT)])
    for move in (zb.adamw_read_moments, zb.adamw_write_moments):
        for bad in (tensor(m=0), tensor(v=0), tensor(m_scale=0), tensor(v_scale=AT + 2), tensor(n=-1)):
            assert rc_of(move, zb.adamw_tensors([bad]), values) == zb.EINVAL
        for v in ((0, AT), (AT, 0), (AT + 2, AT), (AT, AT + 1)):
            assert rc_of(move, t, zb.adamw_values([v])) == zb.EINVAL
        assert rc_of(move, t, zb.adamw_values([])) == zb.EINVAL
    assert zb.lib.zb_adamw_workspace_bytes(t, 1, None) == zb.EINVAL
    assert zb.lib.zb_adamw_read_moments(t, 1, None, None) == zb.EINVAL
    assert C.sizeof(zb.binding.zb_adamw_tensor) == 80


def test_loss_configurations_of_a_stage():
    nan, inf = float("nan"), float("inf")

    def rc(**k):
        cfg = zb.binding.zb_config()
        zb.lib.zb_config_defaults(C.byref(cfg))
        assert (cfg.loss, cfg.clip_low, cfg.clip_high, cfg.kl_coef, cfg.pref_beta, cfg.label_smoothing) == (0, 0.2, 0.2, 0.0, 0.1, 0.0)
        base = dict(layers=1, hidden=64, heads=2, ffn=256, seq=32, mb_size=2, max_microbatches=2, max_pending_b=2, max_pending_w=2, max_inflight=3, role=2,
                    vocab=512)
        for name, value in {**base, **k}.items():
            setattr(cfg, name, value)
        need = C.c_size_t(0)
        return zb.lib.zb_stage_arena_bytes(C.byref(cfg), C.byref(need)), need.value

    plain, policy, pairs = rc()[1], rc(loss=1), rc(loss=2)
    assert policy[0] == pairs[0] == zb.OK
    # the gradient takes the logits' place: three stashes of [64, 512] instead of two of logits and two of gradients, beside a few floats a token
    assert policy[1] < plain and pairs[1] < plain
    for bad in (dict(loss=3), dict(loss=-1), dict(loss=1, role=0), dict(loss=2, role=1), dict(loss=2, mb_size=3), dict(loss=1, clip_low=-0.1),
                dict(loss=1, clip_low=1.5), dict(loss=1, clip_high=inf), dict(loss=1, kl_coef=-1.0), dict(loss=1, kl_coef=nan), dict(loss=2, pref_beta=inf),
                dict(loss=2, label_smoothing=1.5), dict(loss=2, label_smoothing=nan)):
        assert rc(**bad)[0] == zb.EINVAL, bad


def test_more_rows_or_pairs_than_a_launch_holds():
    """A workgroup of up to 1024 lanes a row, and a launch has less than 2^32 lanes."""
    most = (1 << 22) - 1
    x = good_logits(rows=most + 1)
    assert rc_of(zb.token_logprobs, x, AT) == zb.EINVAL
    assert rc_of(zb.token_logprobs_backward, x, AT, AT, AT) == zb.EINVAL
    ws = dict(workspace=AT, workspace_bytes=1 << 40)
    assert rc_of(zb.policy_loss, x, zb.policy(AT, AT), AT, AT, AT, **ws) == zb.EINVAL
    for pairs in (9, most + 1):
        assert rc_of(zb.preference_loss, x if pairs == 9 else good_logits(), zb.preference(AT, AT, pairs), AT, AT, AT, AT, **ws) == zb.EINVAL
    for rows, pairs in ((most + 1, 0), (0, most + 1)):
        assert rc_of(zb.loss_workspace_bytes, rows, pairs) == zb.EINVAL
    assert zb.loss_workspace_bytes(most, most) > 0
