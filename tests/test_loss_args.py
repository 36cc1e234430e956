"""What the loss refuses, before anything is enqueued: no device is needed."""
import ctypes

import pytest

from paper_2401_01728_amd import _lib

INVAL, OK = -1, 0


def _work(T=100, d=128, V=1000, ldw=128, rows=0, gradients=1):
    n = ctypes.c_size_t(0)
    return _lib.lib().rv_loss_work(T, d, V, ldw, rows, gradients, ctypes.byref(n)), n.value


def test_sizes():
    assert _lib.lib().rv_loss_work(100, 128, 1000, 128, 0, 1, None) == INVAL
    for bad in (dict(T=0), dict(T=-1), dict(T=(1 << 20) + 1), dict(ldw=(1 << 20) + 8, V=10), dict(d=0), dict(d=32), dict(d=100), dict(d=16448), dict(V=0), dict(V=(1 << 24) + 1),
                dict(ldw=64), dict(ldw=132), dict(rows=-1), dict(V=1 << 24, ldw=128), dict(d=16384, ldw=16384, V=131072)):
        assert _work(**bad)[0] == INVAL, bad
    for good in (dict(T=1), dict(T=1 << 20, V=1), dict(d=64, ldw=64), dict(d=16384, ldw=16384, V=131071), dict(V=1), dict(V=(1 << 24) - 1, ldw=128, T=64),
                 dict(ldw=136), dict(rows=1)):
        st, n = _work(**good)
        assert st == OK and n > 0, good


def test_work_memory_is_bounded():
    """A piece of rows bounds it: what grows with the tokens is the copy of x and three indices."""
    T, d, V = 1 << 16, 1024, 131072
    for rows in (256, 1024):
        small, large = _work(T, d, V, d, rows)[1], _work(2 * T, d, V, d, rows)[1]
        assert large - small <= T * (2 * d + 12) + 4096
        assert small <= 2 * V * rows + 8 * V // 64 * rows + 4 * V * d + T * (2 * d + 12) + (1 << 28)
    # without a word of the caller: 2 GiB of exponentials
    assert _work(T, d, V, d)[1] <= (2 << 30) + (2 << 30) // 16 + 4 * V * d + T * (2 * d + 12) + (1 << 28)


def _desc(**change):
    st, n = _work()
    assert st == OK
    a = dict(x=1024, ldx=128, w=2048, ldw=128, label=4096, T=100, d=128, V=1000, rows=0, scale=1.0, loss=8192, lse=16384, dx=32768, lddx=128, dw=65536,
             work=1 << 20, work_bytes=n)
    a.update(change)
    return _lib.LossDesc(**a)


@pytest.mark.parametrize("change", [
    dict(x=None), dict(w=None), dict(label=None), dict(loss=None), dict(work=None), dict(work_bytes=0), dict(x=1026), dict(w=2056), dict(label=4100),
    dict(loss=8194), dict(lse=16386), dict(work=(1 << 20) + 16), dict(ldx=120), dict(ldx=130), dict(ldx=(1 << 20) + 8), dict(ldw=130), dict(ldw=64), dict(row_scale=2),
    dict(T=0), dict(d=96), dict(V=0), dict(rows=-5)])
def test_refused_by_both(change):
    a = _desc(**change)
    assert _lib.lib().rv_loss_step(ctypes.byref(a)) == INVAL
    assert _lib.lib().rv_loss_forward(ctypes.byref(a)) == INVAL


@pytest.mark.parametrize("change", [
    dict(dx=None, dw=None), dict(dx=32770), dict(lddx=120), dict(lddx=132), dict(dw=65544), dict(master=131072, master_out=131072, version=2048),
    dict(dw=None, master=131072), dict(dw=None, master=131072, master_out=131072), dict(dw=None, master_out=131072), dict(version=131072),
    dict(dw=None, master=131080, master_out=131072, version=2048)])
def test_refused_by_the_step(change):
    a = _desc(**change)
    assert _lib.lib().rv_loss_step(ctypes.byref(a)) == INVAL


def test_too_little_work_memory():
    need = _work()[1]
    assert _lib.lib().rv_loss_step(ctypes.byref(_desc(work_bytes=need - 1))) == INVAL
    assert _work(gradients=0)[1] < need


def test_null_description():
    assert _lib.lib().rv_loss_step(None) == INVAL and _lib.lib().rv_loss_forward(None) == INVAL
