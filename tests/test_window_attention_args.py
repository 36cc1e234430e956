"""What attention over a window refuses, before anything is enqueued: no device is needed."""
import ctypes

import pytest

from paper_2401_01728_amd import _lib

INVAL, OK = -1, 0


def _work(B=2, Sq=100, Sk=100, H=4, Hkv=2, dh=64, window=40, sinks=4, backward=0):
    n = ctypes.c_size_t(0)
    return _lib.lib().rv_k_window_attention_work(B, Sq, Sk, H, Hkv, dh, window, sinks, backward, ctypes.byref(n)), n.value


def test_sizes():
    for bad in (dict(B=0), dict(Sq=0), dict(Sk=0), dict(H=0), dict(Hkv=0), dict(Hkv=3), dict(dh=96), dict(dh=32), dict(dh=256), dict(B=(1 << 20) + 1),
                dict(Sq=(1 << 24) + 1), dict(Sk=(1 << 24) + 1), dict(H=(1 << 16) + 1, Hkv=1), dict(Sq=1 << 24, Sk=1 << 24, H=1 << 10, Hkv=1), dict(window=0),
                dict(window=-1), dict(sinks=-1)):
        assert _work(**bad) == (INVAL, 0), bad
        assert _work(backward=1, **bad) == (INVAL, 0), bad
    assert _work(backward=1, Sk=101) == (INVAL, 0)
    assert _lib.lib().rv_k_window_attention_work(2, 100, 100, 4, 2, 64, 40, 4, 0, None) == INVAL
    for good in (dict(B=1, Sq=1, Sk=1, H=1, Hkv=1), dict(Sq=1 << 24, Sk=1 << 24, B=1, H=2, Hkv=2), dict(H=64, Hkv=1, dh=128), dict(window=2 ** 31 - 1, sinks=2 ** 31 - 1)):
        assert _work(**good)[0] == OK and _work(backward=1, **good)[0] == OK, good


NAMES = ["q", "ldq", "k", "ldk", "v", "ldv", "start", "length", "out", "ldo", "lse2", "B", "Sq", "Sk", "H", "Hkv", "dh", "window", "sinks", "work", "bytes",
         "stream"]
BWD = ["q", "ldq", "k", "ldk", "v", "ldv", "length", "out", "ldo", "dout", "lddo", "lse2", "dq", "lddq", "dk", "lddk", "dv", "lddv", "B", "Sq", "H", "Hkv", "dh",
       "window", "sinks", "work", "bytes", "stream"]
GOOD = dict(q=1 << 12, ldq=256, k=2 << 12, ldk=128, v=3 << 12, ldv=128, start=None, length=None, out=4 << 12, ldo=256, lse2=5 << 12, B=2, Sq=100, Sk=100, H=4,
            Hkv=2, dh=64, window=40, sinks=4, work=6 << 12, bytes=1 << 40, stream=None, dout=7 << 12, lddo=256, dq=8 << 12, lddq=256, dk=9 << 12, lddk=128,
            dv=10 << 12, lddv=128)


def _fwd(change):
    return _lib.lib().rv_k_window_attention_fwd(*(dict(GOOD, **change)[n] for n in NAMES))


def _bwd(change):
    return _lib.lib().rv_k_window_attention_bwd(*(dict(GOOD, **change)[n] for n in BWD))


@pytest.mark.parametrize("change", [
    dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(lse2=None), dict(q=4098), dict(k=8200), dict(v=12296), dict(out=16392), dict(lse2=20482),
    dict(length=2), dict(ldq=248), dict(ldq=260), dict(ldk=120), dict(ldv=132), dict(ldo=1 << 25), dict(Hkv=3), dict(dh=80), dict(B=-1), dict(Sq=0), dict(window=0),
    dict(sinks=-1)])
def test_refused(change):
    assert _fwd(change) == INVAL and _bwd(change) == INVAL


def test_refused_by_the_forward():
    assert _fwd(dict(Sk=99)) == INVAL                     # fewer rows than tokens, and no cache
    assert _fwd(dict(Sk=0)) == INVAL and _fwd(dict(start=2)) == INVAL


@pytest.mark.parametrize("change", [dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dq=8), dict(dk=24), dict(dv=1), dict(lddo=128), dict(lddq=257),
                                    dict(lddk=64), dict(lddv=129), dict(work=None), dict(work=128), dict(bytes=0)])
def test_refused_by_the_backward(change):
    assert _bwd(change) == INVAL


def test_too_little_work_memory():
    token = dict(Sq=1, Sk=5000, window=5000)              # long enough to be cut into parts
    need = _work(**token)[1]
    assert need > 0
    assert _fwd(dict(token, start=1 << 16, bytes=need - 1)) == INVAL
    assert _fwd(dict(token, start=1 << 16, work=None)) == INVAL
    need = _work(backward=1)[1]
    assert _bwd(dict(bytes=need - 1)) == INVAL


def test_work_memory_of_many_sequences():
    """What does not go into one launch is made in several that use the same memory: no more for 2^20 sequences than for those of one launch."""
    one = dict(Sq=1, Sk=1, H=16, Hkv=16, dh=64, window=7, sinks=1, backward=1)
    status, most = _work(B=1 << 20, **one)
    assert status == OK and most == _work(B=1 << 19, **one)[1]
    assert _work(B=1 << 10, **one)[1] < most < _work(B=1, **one)[1] * (1 << 19)
    # two statistics of 32 bits for 64 rows, a tile that may begin at the last of them, of 16 heads
    assert _work(B=1, **one)[1] == 2 * 64 * 4 * 16
