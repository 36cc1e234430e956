"""Frequencies of rotary positions, and what the rotation refuses before anything is enqueued: no device is needed."""
import ctypes
import math

import pytest

from paper_2401_01728_amd import _lib, kernels

INVAL, OK = -1, 0


def test_plain_and_linear_frequencies():
    freq, amplitude = kernels.rotary_frequencies(64)
    assert amplitude == 1.0 and freq.tolist() == pytest.approx([10000.0 ** (-2.0 * c / 64) for c in range(32)], rel=1e-14)
    slow, amplitude = kernels.rotary_frequencies(64, rule="linear", factor=8.0)
    assert amplitude == 1.0 and slow.tolist() == pytest.approx([f / 8.0 for f in freq.tolist()], rel=1e-14)


def test_a_changed_base_keeps_the_fastest_and_divides_the_slowest():
    plain = kernels.rotary_frequencies(128, base=500000.0)[0]
    freq, amplitude = kernels.rotary_frequencies(128, base=500000.0, rule="base", factor=4.0)
    assert amplitude == 1.0 and freq[0] == plain[0] == 1.0
    assert float(freq[-1]) == pytest.approx(float(plain[-1]) / 4.0, rel=1e-12)
    assert all(a < b for a, b in zip(freq[1:].tolist(), plain[1:].tolist()))


def test_parts_by_turns():
    factor, context, low, high = 16.0, 4096.0, 1.0, 32.0
    plain = kernels.rotary_frequencies(128)[0]
    freq, amplitude = kernels.rotary_frequencies(128, rule="parts", factor=factor, context=context, low=low, high=high)
    assert amplitude == pytest.approx(0.1 * math.log(factor) + 1.0, rel=1e-7)
    kinds = set()
    for f, p in zip(freq.tolist(), plain.tolist()):
        turns = context * p / (2.0 * math.pi)
        if turns >= high:
            kinds.add("stay")
            assert f == p
        elif turns <= low:
            kinds.add("divided")
            assert f == pytest.approx(p / factor, rel=1e-14)
        else:
            kinds.add("between")
            g = (turns - low) / (high - low)
            assert f == pytest.approx(p * g + p / factor * (1.0 - g), rel=1e-12)
    assert kinds == {"stay", "divided", "between"}


@pytest.mark.parametrize("change", [dict(rot=0), dict(rot=3), dict(rot=1026), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(rule=4), dict(rule=-1),
                                    dict(rule=1, factor=0.5), dict(rule=2, factor=math.nan), dict(rule=2, rot=2), dict(rule=3, context=0.0),
                                    dict(rule=3, low=32.0), dict(rule=3, low=-1.0), dict(rule=3, high=math.inf), dict(freq=None), dict(amplitude=None)])
def test_refused_frequencies(change):
    room = (ctypes.c_double * 513)()
    out = ctypes.c_float(0.0)
    a = dict(rot=64, base=10000.0, rule=0, factor=2.0, context=4096.0, low=1.0, high=32.0, freq=ctypes.addressof(room), amplitude=ctypes.addressof(out))
    call = lambda a: _lib.lib().rv_k_rotary_frequencies(*(a[n] for n in ("rot", "base", "rule", "factor", "context", "low", "high", "freq", "amplitude")))  # noqa: E731
    assert call(a) == OK
    assert call(dict(a, **change)) == INVAL


GOOD = dict(B=2, S=10, n_heads=4, n_kv_heads=2, d_head=64, rot=64, layout=0, amplitude=1.0, eps=1e-6, freq=1 << 12, pos=None, start=None, length=None,
            gamma_q=2 << 12, gamma_k=3 << 12, q=4 << 12, ldq=256, k=5 << 12, ldk=128, v=6 << 12, ldv=128, q_out=7 << 12, ldq_out=256, k_out=8 << 12,
            ldk_out=128, v_out=9 << 12, ldv_out=128, rows=0, sinks=0, dq_out=10 << 12, lddq_out=256, dk_out=11 << 12, lddk_out=128, dq=12 << 12, lddq=256,
            dk=13 << 12, lddk=128, dgamma_q=14 << 12, dgamma_k=15 << 12, work=16 << 12, work_bytes=1 << 40, stream=None)


def _both(change):
    d = _lib.RotaryDesc(**dict(GOOD, **change))
    return _lib.lib().rv_k_rotary_fwd(ctypes.byref(d)), _lib.lib().rv_k_rotary_bwd(ctypes.byref(d))


@pytest.mark.parametrize("change", [
    dict(B=0), dict(S=0), dict(B=(1 << 20) + 1), dict(S=(1 << 24) + 1), dict(B=1 << 10, S=(1 << 20) + 1), dict(n_heads=-1), dict(n_heads=0, n_kv_heads=0),
    dict(n_kv_heads=(1 << 12) + 1), dict(d_head=96), dict(d_head=32), dict(d_head=256), dict(rot=8), dict(rot=80), dict(rot=-16), dict(layout=2), dict(layout=-1),
    dict(freq=None), dict(freq=4), dict(amplitude=math.nan), dict(amplitude=math.inf), dict(eps=-1e-6), dict(eps=math.nan), dict(pos=2), dict(start=1), dict(length=3),
    dict(gamma_q=8), dict(gamma_k=18)])
def test_refused(change):
    assert _both(change) == (INVAL, INVAL)


@pytest.mark.parametrize("change", [
    dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(v_out=None), dict(q=8), dict(k_out=24), dict(v=2), dict(ldq=248), dict(ldq=260), dict(ldk=64),
    dict(ldv=1 << 25), dict(ldq_out=8), dict(ldk_out=129), dict(ldv_out=120), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(sinks=-1),
    dict(n_kv_heads=0), dict(n_kv_heads=0, v=None, rows=4)])
def test_refused_by_the_forward(change):
    assert _both(change)[0] == INVAL


@pytest.mark.parametrize("change", [
    dict(dq_out=None), dict(dk_out=None), dict(dq=None), dict(dk=None), dict(q=None), dict(k=None), dict(dq=8), dict(lddq=8), dict(lddk=136 + 4), dict(lddq_out=0),
    dict(lddk_out=120), dict(dgamma_q=2), dict(dgamma_k=1), dict(gamma_q=None), dict(gamma_k=None), dict(work=None), dict(work=128), dict(work_bytes=0)])
def test_refused_by_the_backward(change):
    assert _both(change)[1] == INVAL


def test_no_description_and_work_memory():
    assert _lib.lib().rv_k_rotary_fwd(None) == INVAL and _lib.lib().rv_k_rotary_bwd(None) == INVAL
    n = ctypes.c_size_t(0)
    assert _lib.lib().rv_k_rotary_work(2, 10, 4, 2, 64, ctypes.byref(n)) == OK and n.value >= 2 * 64 * 4
    assert _both(dict(work_bytes=n.value - 1))[1] == INVAL
    assert _lib.lib().rv_k_rotary_work(2, 10, 4, 2, 96, ctypes.byref(n)) == INVAL
    assert _lib.lib().rv_k_rotary_work(2, 10, 4, 2, 64, None) == INVAL
    assert _lib.lib().rv_k_rotary_work(1 << 10, 1 << 20, 4096, 4096, 128, ctypes.byref(n)) == OK and n.value <= 1 << 21
