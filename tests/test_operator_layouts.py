"""Which layouts of several matrices in one buffer the losses take: overlap is looked for before the workspace's size, so that a call with too small a one says which check it came to."""
import pytest

from paper_2312_14227_amd import binding as et
from test_operator_refusals import A, _policy, _preference

F32, BF16 = et.ET_F32, et.ET_BF16

# rows of 10 elements; logits of float32 at A
BESIDE = [dict(stride=20, gstride=20, grad=A + 40), dict(stride=20, gstride=20, grad=A - 40), dict(stride=23, gstride=23, grad=A + 44), dict(stride=30, gstride=30, grad=A + 80),
          dict(stride=20, gstride=40, gdtype=BF16, grad=A + 40), dict(stride=15, gstride=30, gdtype=BF16, grad=A + 40), dict(stride=20, gstride=20, grad=A - 80 * 2 + 40),
          dict(stride=20, gstride=20, grad=A + 80 * 3 + 40), dict(stride=20, gstride=21, grad=A + 80 * 3 + 40)]
ACROSS = [dict(stride=20, gstride=20, grad=A + 36), dict(stride=20, gstride=20, grad=A + 44), dict(stride=19, gstride=19, grad=A + 40), dict(stride=20, gstride=20, grad=A - 36),
          dict(stride=20, gstride=20, grad=A - 44), dict(stride=20, gstride=20, grad=A + 80), dict(stride=15, gstride=30, gdtype=BF16, grad=A + 42),
          dict(stride=20, gstride=21, grad=A + 40), dict(stride=20, gstride=20, gdtype=BF16, grad=A + 40)]


@pytest.mark.parametrize("call", [_policy, _preference])
@pytest.mark.parametrize("kw,status", [(k, et.ET_ENOMEM) for k in BESIDE] + [(k, et.ET_EINVAL) for k in ACROSS])
def test_the_gradient_beside_the_logits(kw, status, call):
    with pytest.raises(et.EtError) as e:
        call(ws_bytes=1, **kw)
    assert e.value.status == status


@pytest.mark.parametrize("kw,status", [(dict(stride=20, gstride=20, grad=A, ref_logits=A + 40, ref_stride=20), et.ET_ENOMEM),
                                       (dict(stride=30, gstride=30, grad=A + 80, ref_logits=A + 40, ref_stride=30), et.ET_ENOMEM),
                                       (dict(stride=30, gstride=30, grad=A + 76, ref_logits=A + 40, ref_stride=30), et.ET_EINVAL),
                                       (dict(stride=20, gstride=20, grad=A, ref_logits=A + 36, ref_stride=20), et.ET_EINVAL)])
def test_the_gradient_beside_the_reference(kw, status):
    with pytest.raises(et.EtError) as e:
        _policy(ws_bytes=1, **kw)
    assert e.value.status == status
