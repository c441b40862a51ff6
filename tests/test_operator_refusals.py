"""What the stand-alone operators refuse: every check comes before any device is looked at, so no GPU is needed and no address is followed."""
import math

import pytest

from paper_2312_14227_amd import binding as et

A = 1 << 20   # an address that nothing follows


def _policy(rows=4, classes=10, logits=A, dtype=et.ET_F32, stride=10, label=A, grad=2 * A, gdtype=et.ET_F32, gstride=10, ws=A, ws_bytes=None, loss=A, **kw):
    p = et.make_policy(kw.pop("old", A), kw.pop("adv", A), **kw)
    need = et.et_policy_loss_ws_bytes(rows) if ws_bytes is None else ws_bytes
    et.et_policy_loss(rows, classes, logits, dtype, stride, label, p, grad, gdtype, gstride, ws, need, 0, loss)


def _preference(rows=4, pairs=2, classes=10, logits=A, dtype=et.ET_F32, stride=10, label=A, grad=2 * A, gdtype=et.ET_F32, gstride=10, ws=A, ws_bytes=None,
                loss=A, offsets=A, **kw):
    need = et.et_preference_loss_ws_bytes(rows, pairs) if ws_bytes is None else ws_bytes
    et.et_preference_loss(rows, pairs, classes, logits, dtype, stride, label, et.make_preference(offsets, **kw), grad, gdtype, gstride, ws, need, 0, loss)


BOTH = [dict(rows=0), dict(rows=-1), dict(classes=0), dict(classes=(1 << 28) + 1, stride=1 << 30, gstride=1 << 30), dict(logits=0), dict(label=0), dict(ws=0), dict(loss=0), dict(dtype=2), dict(gdtype=7), dict(stride=9),
        dict(gstride=9), dict(stride=-10), dict(stride=1 << 61), dict(logits=A + 2), dict(grad=2 * A + 2), dict(label=A + 1), dict(loss=A + 2), dict(ws=A + 8),
        dict(dtype=et.ET_BF16, logits=A + 1),
        dict(grad=A, gstride=11),                          # on the logits, with another stride
        dict(grad=A, gdtype=et.ET_BF16), dict(grad=A + 4), dict(grad=A - 4)]


@pytest.mark.parametrize("kw", BOTH + [dict(old=0), dict(adv=0), dict(adv=A + 2), dict(ref_logp=A, ref_logits=A, ref_stride=10), dict(ref_logits=A, ref_stride=9),
                                       dict(ref_logits=2 * A, ref_stride=10), dict(ref_logits=A + 2, ref_stride=10), dict(clip_low=-0.1), dict(clip_low=1.5),
                                       dict(clip_high=-0.1), dict(clip_high=math.inf), dict(clip_low=math.nan), dict(kl_coef=math.nan), dict(kl_coef=math.inf),
                                       dict(logp=A + 1), dict(stats=A + 2), dict(weight=A + 3)])
def test_policy_loss_refuses(kw):
    with pytest.raises(et.EtError) as e:
        _policy(**kw)
    assert e.value.status == et.ET_EINVAL


@pytest.mark.parametrize("kw", BOTH + [dict(pairs=0), dict(pairs=1 << 30), dict(offsets=0, rows=5), dict(offsets=A + 2), dict(beta=0.0), dict(beta=-1.0),
                                       dict(beta=math.inf), dict(beta=math.nan), dict(label_smoothing=-0.1), dict(label_smoothing=1.1),
                                       dict(label_smoothing=math.nan), dict(ref_logp=A + 2), dict(logp=A + 2), dict(stats=A + 1)])
def test_preference_loss_refuses(kw):
    with pytest.raises(et.EtError) as e:
        _preference(**kw)
    assert e.value.status == et.ET_EINVAL


def test_small_workspaces():
    for call, need in ((_policy, et.et_policy_loss_ws_bytes(4)), (_preference, et.et_preference_loss_ws_bytes(4, 2))):
        with pytest.raises(et.EtError) as e:
            call(ws_bytes=need - 1)
        assert e.value.status == et.ET_ENOMEM
    assert et.et_policy_loss_ws_bytes(0) == 0 and et.et_preference_loss_ws_bytes(4, 0) == 0 and et.et_preference_loss_ws_bytes(0, 4) == 0
    need = et.et_grad_norm_ws_bytes([100, 0, 7])
    with pytest.raises(et.EtError) as e:
        et.et_grad_norm([A, 0, A], [100, 0, 7], et.ET_F32, A, need - 1, 0, A)
    assert e.value.status == et.ET_ENOMEM
    assert et.et_grad_norm_ws_bytes([1 << 49]) == 0


@pytest.mark.parametrize("kw", [dict(grad=[A, 0]), dict(grad=[A, A + 2]), dict(dtype=2), dict(ws=0), dict(ws=A + 8), dict(norm=0), dict(norm=A + 2), dict(each=A + 1),
                                dict(numel=[8, 1 << 49]), dict(out=[A, 0]), dict(out=[A + 2, A]), dict(out=[A + 16, A]), dict(max_norm=-1.0), dict(max_norm=math.nan)])
def test_grad_norm_and_clip_refuse(kw):
    a = dict(grad=[A, 2 * A], out=None, numel=[8, 8], dtype=et.ET_F32, max_norm=1.0, ws=A, norm=A, each=0) | kw
    room = 1 << 20
    with pytest.raises(et.EtError) as e:
        et.et_grad_clip(a["grad"], a["out"], a["numel"], a["dtype"], a["max_norm"], a["ws"], room, 0, a["norm"], a["each"])
    assert e.value.status == et.ET_EINVAL
    if not {"out", "max_norm"} & set(kw):
        with pytest.raises(et.EtError) as e:
            et.et_grad_norm(a["grad"], a["numel"], a["dtype"], a["ws"], room, 0, a["norm"], a["each"])
        assert e.value.status == et.ET_EINVAL


@pytest.mark.parametrize("kw", [dict(grad=[A, 0]), dict(grad=[A, A + 2]), dict(dtype=2), dict(norm=0), dict(norm=A + 2), dict(numel=[8, 1 << 49]), dict(out=[A, 0]),
                                dict(out=[A + 16, A]), dict(max_norm=-1.0), dict(max_norm=math.nan)])
def test_grad_scale_refuses(kw):
    a = dict(grad=[A, 2 * A], out=None, numel=[8, 8], dtype=et.ET_F32, max_norm=1.0, norm=A) | kw
    with pytest.raises(et.EtError) as e:
        et.et_grad_scale(a["grad"], a["out"], a["numel"], a["dtype"], a["norm"], a["max_norm"], 0)
    assert e.value.status == et.ET_EINVAL


OVERLAPS = [(["a", "a"], None), (["a", "a+4"], None), (["b", "a", "a+28"], None), (["a", "b"], ["c", "c"]), (["a", "b"], ["c", "c+4"]), (["a", "b"], ["b", "c"]), (["a", "b"], ["c", "a"]),
            (["a", "b"], ["b", "a"]), (["a", "b"], ["a", "a+16"]), (["a", "b"], ["c", "a-4"]), (["c", "b", "a"], ["c", "b", "b+12"]), (["a", "a"], ["a", "c"])]


@pytest.mark.parametrize("grad,out", OVERLAPS)
def test_outputs_that_meet_another_tensor(grad, out):
    at = lambda names: None if names is None else [eval(s, {"a": A, "b": A + 4096, "c": A + 8192}) for s in names]  # noqa: E731
    n = [8] * len(grad)
    for call in (lambda: et.et_grad_clip(at(grad), at(out), n, et.ET_F32, 1.0, A, 1 << 20, 0, A), lambda: et.et_grad_scale(at(grad), at(out), n, et.ET_F32, A, 1.0, 0)):
        with pytest.raises(et.EtError) as e:
            call()
        assert e.value.status == et.ET_EINVAL


def test_lists_of_other_lengths():
    for grad, out in (([A], None), ([A, 2 * A, 3 * A], None), ([A, 2 * A], [A])):
        with pytest.raises(et.EtError):
            et.et_grad_clip(grad, out, [8, 8], et.ET_F32, 1.0, A, 1 << 20, 0, A)
        with pytest.raises(et.EtError):
            et.et_grad_scale(grad, out, [8, 8], et.ET_F32, A, 1.0, 0)
    with pytest.raises(et.EtError):
        et.et_grad_norm([A], [8, 8], et.ET_F32, A, 1 << 20, 0, A)


def test_outputs_on_the_inputs():
    B = 1 << 30
    for kw in (dict(logp=A), dict(old=B, logp=B + 12), dict(ref_logp=B, logp=B - 12), dict(weight=B, logp=B)):
        with pytest.raises(et.EtError) as e:
            _policy(**kw)
        assert e.value.status == et.ET_EINVAL
    for kw in (dict(ref_logp=B, logp=B), dict(ref_logp=B, logp=B + 12)):
        with pytest.raises(et.EtError) as e:
            _preference(**kw)
        assert e.value.status == et.ET_EINVAL


def test_more_than_any_call_takes():
    for call, kw in ((_policy, dict(rows=(1 << 30) + 1)), (_preference, dict(rows=(1 << 30) + 1)), (_preference, dict(pairs=(1 << 23) + 1, rows=1 << 25))):
        with pytest.raises(et.EtError) as e:
            call(grad=0, ws_bytes=1 << 50, **kw)
        assert e.value.status == et.ET_EINVAL
    assert et.et_policy_loss_ws_bytes((1 << 30) + 1) == 0 and et.et_preference_loss_ws_bytes(1 << 25, (1 << 23) + 1) == 0
    assert et.et_policy_loss_ws_bytes(1 << 30) > 0 and et.et_preference_loss_ws_bytes(1 << 30, 1 << 23) > 0
