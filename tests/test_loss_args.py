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


def _documented(T, d, V, rows, gradients):
    """What rv.h says the work memory is at most, but for the rounding of each of 14 parts to 256 bytes."""
    most = max(128, (1 << 30) // max(V, d))
    r = min(most if rows == 0 else rows, T)
    r = 128 if r <= 128 else (r + 255) // 256 * 256
    n = (V + 63) // 8 * r
    if T > 256:
        n += (T + r) * (2 * d + 12)
    if gradients:
        n += (4 if T <= 256 else 2) * (V + 63) * r + (4 * d * r if T <= 256 else 0) + 4 * d * r + (5 << 28) + 128 * d + 24 * r
        n += 4 * V * d if r < T else 0
    return n + 24 * r + 14 * 256


@pytest.mark.parametrize("T,d,V,rows", [
    (1, 64, 1, 0), (3, 64, 5_000_000, 0), (256, 64, 4_000_000, 0), (200, 64, 4_000_000, 128), (130, 64, (1 << 24) - 1, 0), (256, 16384, 131071, 0), (257, 16384, 131071, 0),
    (1 << 18, 4096, 1000, 0), (1 << 20, 16384, 64, 0), (827556, 16192, 112020, 0), (5000, 2048, 128000, 1000), (1 << 20, 64, 1 << 20, 1 << 20)])
def test_work_memory_is_what_the_header_says(T, d, V, rows):
    for gradients in (0, 1):
        st, n = _work(T, d, V, d, rows, gradients)
        assert st == OK and n <= _documented(T, d, V, rows, gradients), (gradients, n, _documented(T, d, V, rows, gradients))


@pytest.mark.parametrize("T", [1, 3, 64])
def test_few_rows_do_not_take_twice_the_exponentials(T):
    """Two parts of 64 rows have room in the 128 of a tile."""
    V, d = 5_000_000, 64
    assert _work(T, d, V, d)[1] <= (2 * V + V // 8) * 128 + (5 << 28)
    n = [_work(t, d, V, d)[1] for t in (64, 128)]
    assert n[1] - n[0] >= 2 * V * 128
