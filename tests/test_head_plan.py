"""What the head's inspection call says: on the host, no kernel is launched."""
import ctypes as C

from paper_2406_02913_amd import szo
from test_more_refusals import head


def test_plan():
    assert szo.szo_head_plan(head(rows=1, vocab=100, width=64)) == (128, 64, 1, 128, 64, 128, 64, 1, 128)
    assert szo.szo_head_plan(head(rows=4096, vocab=32000, width=4096, x_stride=4096, weight_stride=4096)) == (256, 256, 1, 256, 256, 256, 256, 1, 256)
    assert szo.szo_head_plan(head(rows=8192, vocab=131072, width=64))[2] == 8
    for nothing in (dict(rows=0, x=None), dict(vocab=0, weight=None)):
        assert szo.szo_head_plan(head(**nothing)) == (0,) * 9


def test_plan_refuses():
    plan = (C.c_int32 * 9)()
    assert szo.lib.szo_head_plan(C.byref(head()), None) == szo.EINVAL and szo.lib.szo_head_plan(None, plan) == szo.EINVAL
    assert szo.lib.szo_head_plan(C.byref(head(scale=0.0)), plan) == szo.EINVAL and szo.lib.szo_head_plan(C.byref(head(width=96)), plan) == szo.EUNSUPPORTED
