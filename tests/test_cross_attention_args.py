"""What cross-attention refuses, before anything is enqueued: no device is needed."""
import ctypes

import pytest

from paper_2401_01728_amd import _lib

INVAL, OK = -1, 0


def _work(B=2, Sq=10, Sk=100, H=4, Hkv=2, dh=64, backward=0):
    n = ctypes.c_size_t(0)
    return _lib.lib().rv_k_cross_attention_work(B, Sq, Sk, H, Hkv, dh, backward, ctypes.byref(n)), n.value


def test_sizes():
    for bad in (dict(B=0), dict(Sq=0), dict(Sk=0), dict(Sk=-1), dict(H=0), dict(Hkv=0), dict(Hkv=3), dict(dh=96), dict(dh=32), dict(dh=256), dict(B=(1 << 20) + 1),
                dict(Sq=(1 << 24) + 1), dict(Sk=(1 << 24) + 1), dict(H=(1 << 16) + 1, Hkv=1), dict(Sq=1 << 24, H=1 << 10, Hkv=1)):
        assert _work(**bad) == (INVAL, 0), bad
        assert _work(backward=1, **bad) == (INVAL, 0), bad
    assert _lib.lib().rv_k_cross_attention_work(2, 10, 100, 4, 2, 64, 0, None) == INVAL
    for good in (dict(B=1, Sq=1, Sk=1, H=1, Hkv=1), dict(Sk=1 << 24, B=1, Sq=1), dict(H=64, Hkv=1, dh=128)):
        assert _work(**good)[0] == OK and _work(backward=1, **good)[0] == OK, good


NAMES = ["q", "ldq", "k", "ldk", "v", "ldv", "klen", "out", "ldo", "lse2", "B", "Sq", "Sk", "H", "Hkv", "dh", "work", "bytes", "stream"]
BWD = ["q", "ldq", "k", "ldk", "v", "ldv", "klen", "out", "ldo", "dout", "lddo", "lse2", "dq", "lddq", "dk", "lddk", "dv", "lddv", "B", "Sq", "Sk", "H", "Hkv",
       "dh", "work", "bytes", "stream"]
GOOD = dict(q=1 << 12, ldq=256, k=2 << 12, ldk=128, v=3 << 12, ldv=128, klen=None, out=4 << 12, ldo=256, lse2=5 << 12, B=2, Sq=10, Sk=100, H=4, Hkv=2, dh=64,
            work=6 << 12, bytes=1 << 40, stream=None, dout=7 << 12, lddo=256, dq=8 << 12, lddq=256, dk=9 << 12, lddk=128, dv=10 << 12, lddv=128)


@pytest.mark.parametrize("change", [
    dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(lse2=None), dict(q=4098), dict(k=8200), dict(v=12296), dict(out=16392), dict(lse2=20482), dict(klen=2),
    dict(ldq=248), dict(ldq=260), dict(ldk=120), dict(ldv=132), dict(ldo=1 << 25), dict(Hkv=3), dict(dh=80), dict(Sk=0), dict(B=-1), dict(Sq=0)])
def test_refused(change):
    a = dict(GOOD, **change)
    assert _lib.lib().rv_k_cross_attention_fwd(*(a[n] for n in NAMES)) == INVAL
    assert _lib.lib().rv_k_cross_attention_bwd(*(a[n] for n in BWD)) == INVAL


@pytest.mark.parametrize("change", [dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dq=8), dict(dk=24), dict(dv=1), dict(lddo=128), dict(lddq=257),
                                    dict(lddk=64), dict(lddv=129), dict(work=None), dict(work=128), dict(bytes=0)])
def test_refused_by_the_backward(change):
    a = dict(GOOD, **change)
    assert _lib.lib().rv_k_cross_attention_bwd(*(a[n] for n in BWD)) == INVAL


def test_too_little_work_memory():
    token = dict(GOOD, Sq=1, Sk=5000)       # long enough to be cut into parts
    need = _work(Sq=1, Sk=5000)[1]
    assert need > 0
    assert _lib.lib().rv_k_cross_attention_fwd(*(dict(token, bytes=need - 1)[n] for n in NAMES)) == INVAL
    assert _lib.lib().rv_k_cross_attention_fwd(*(dict(token, work=None)[n] for n in NAMES)) == INVAL
    need = _work(backward=1)[1]
    assert _lib.lib().rv_k_cross_attention_bwd(*(dict(GOOD, bytes=need - 1)[n] for n in BWD)) == INVAL


def test_a_sequence_larger_than_a_launch():
    """Its statistics would be 2^34 threads: refused for the backward, with the size of the work memory already.  Up to 2^34 elements all is taken,
    and so are sequences that are too many for one launch."""
    large = dict(B=1, Sq=1 << 24, Sk=100, H=64, Hkv=64, dh=128)
    assert _work(**large)[0] == OK and _work(backward=1, **large) == (INVAL, 0)
    args = dict(GOOD, B=1, Sq=1 << 24, H=64, Hkv=64, dh=128, ldq=8192, ldk=8192, ldv=8192, ldo=8192, lddo=8192, lddq=8192, lddk=8192, lddv=8192, bytes=1 << 62)
    assert _lib.lib().rv_k_cross_attention_bwd(*(args[n] for n in BWD)) == INVAL
    for some in (dict(B=1, Sq=1 << 24, Sk=1 << 24, H=8, Hkv=8, dh=128), dict(B=1, Sq=1 << 11, Sk=1 << 11, H=1 << 16, Hkv=1 << 16, dh=128),
                 dict(B=1, Sq=1 << 12, Sk=1 << 12, H=1 << 16, Hkv=1 << 16, dh=64), dict(B=1 << 20, Sq=1, Sk=1, H=16, Hkv=16, dh=64),
                 dict(B=1 << 20, Sq=1, Sk=1, H=64, Hkv=8, dh=128)):
        assert _work(**some)[0] == OK and _work(backward=1, **some)[0] == OK, some
