"""Rotary positions with norms of heads, and their gradients, against the definition in 64 bits on the same bf16 inputs.

Tolerances, element by element; u = 2^-24 is half a step of fp32, and the result is rounded to bf16 once, off by at most 2^-8 of itself.
  angle   a fraction of a turn rounded to fp32 (2^-25 turns, 2^-22.3 rad), the 64-bit product behind it (2^-51 of the angle), cosine and sine off by a
          few u and times the amplitude: `turned` = 2^-20 + 2^-51 |angle|, absolute, of either factor
  norm    a mean of dh squares, a root, a quotient, two products: `normed` = (dh + 16) u, relative
  y       turned (|a| + |b|) amplitude + normed |y's terms| + 2^-8 |y|
  dx      without a norm the same; with one dx = r (g - xh mean(g xh)), g = dn gamma: with e = turned .. of dn,
          r (e |gamma| + |xh| mean(e |gamma xh|) + 4 normed (|g| + |xh| mean(|g xh|))) + 2^-8 |dx|
  dgamma  a sum of T heads terms, of which a lane adds up to T heads / 32 one after the other and 80 additions follow:
          sum e |xh| + (2 normed + (T heads / 32 + 80) u) sum |dn xh|
"""
import math
from fractions import Fraction

import pytest
import torch

from paper_2401_01728_amd import kernels

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _inputs(seed, B, S, H, Hkv, dh, gammas=True):
    g = torch.Generator().manual_seed(seed)
    n = lambda *shape, std=1.0: (torch.randn(*shape, generator=g) * std).to(torch.bfloat16)  # noqa: E731
    q, k, v = n(B, S, H * dh, std=1.5), n(B, S, Hkv * dh, std=1.5), n(B, S, Hkv * dh)
    dq, dk = n(B, S, H * dh, std=0.02), n(B, S, Hkv * dh, std=0.02)
    gq, gk = ((1.0 + n(dh, std=0.2).float()).to(torch.bfloat16) if gammas else None for _ in range(2))
    return q, k, v, dq, dk, gq, gk


def _positions(B, S, start, pos):
    if pos is not None:
        return pos.double()
    p = torch.arange(S, dtype=torch.float64).expand(B, -1)
    return p if start is None else p + torch.tensor(start, dtype=torch.float64).clamp(min=0)[:, None]


def _halves(rot, layout):
    """Columns of the pairs' first and second members."""
    i = torch.arange(rot // 2)
    return (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)


def _turn(x, angle, amplitude, layout, back=False):
    """x [B, S, h, dh] and the absolute sum of each result's terms."""
    y, size = x.clone(), x.abs().clone()
    a, b = _halves(2 * angle.shape[-1], layout)
    c, s = amplitude * angle.cos()[:, :, None], amplitude * angle.sin()[:, :, None] * (-1.0 if back else 1.0)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = abs(amplitude) * (x[..., a].abs() + x[..., b].abs())
    return y, size


def _turned(angle, dh, layout):
    """Bound of the factors' errors for each column of a head."""
    t = torch.zeros(*angle.shape[:2], 1, dh, dtype=torch.float64)
    a, b = _halves(2 * angle.shape[-1], layout)
    t[..., a] = t[..., b] = 2.0 ** -20 + 2.0 ** -51 * angle.abs()[:, :, None]
    return t


def _live(t, length):
    if length is None:
        return torch.ones(t.shape[0], t.shape[1], dtype=torch.bool)
    return torch.arange(t.shape[1])[None, :] < torch.tensor(length)[:, None]


def _forward(x, h, angle, amplitude, layout, gamma, eps, live):
    dh = x.shape[2] // h
    x = torch.where(live[..., None], x.double(), 0.0).unflatten(-1, (h, dh))
    normed = 0.0
    if gamma is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * gamma.double()
        normed = (dh + 16) * U
    y, size = _turn(x, angle, amplitude, layout)
    bound = (_turned(angle, dh, layout) + normed + 4 * U) * size + 2.0 ** -8 * y.abs()
    zero = lambda t: torch.where(live[..., None, None], t, 0.0).flatten(-2)  # noqa: E731
    return zero(y), zero(bound * (1 + 2.0 ** -7))


def _backward(x, d, h, angle, amplitude, layout, gamma, eps, live):
    dh = d.shape[2] // h
    d = torch.where(live[..., None], d.double(), 0.0).unflatten(-1, (h, dh))
    dn, size = _turn(d, angle, amplitude, layout, back=True)
    e = (_turned(angle, dh, layout) + 4 * U) * size
    if gamma is None:
        dx, bound, dgamma, e_gamma = dn, e, None, None
    else:
        w = gamma.double()
        x = torch.where(live[..., None], x.double(), 0.0).unflatten(-1, (h, dh))
        r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
        xh, g = x * r, dn * w
        normed = (dh + 16) * U
        m = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
        dx = r * (g - xh * m(g * xh))
        bound = r * (e * w.abs() + xh.abs() * m(e * (w * xh).abs()) + 4 * normed * (g.abs() + xh.abs() * m((g * xh).abs())))
        dgamma = (dn * xh).sum((0, 1, 2))
        terms = x.shape[0] * x.shape[1] * h
        e_gamma = (e * xh.abs()).sum((0, 1, 2)) + (2 * normed + (terms / 32 + 80) * U) * (dn * xh).abs().sum((0, 1, 2)) + 1e-30
    bound = (bound + 2.0 ** -8 * dx.abs()) * (1 + 2.0 ** -7)
    zero = lambda t: torch.where(live[..., None, None], t, 0.0).flatten(-2)  # noqa: E731
    return zero(dx), zero(bound), dgamma, e_gamma


def _near(got, ref, bound):
    got = got.cpu().double()
    assert got.shape == ref.shape and bool(torch.isfinite(got).all())
    over = (got - ref).abs() / (bound + 1e-30)
    assert bool((over <= 1.0).all()), "off by %.3g of the bound at %s" % (float(over.max()), int(over.argmax()))


def _gpu(*tensors):
    return [t.cuda() if t is not None else None for t in tensors]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda() if v is not None else None


def _check(B, S, H, Hkv, dh, rot, layout, norms, length=None, start=None, pos=None, amplitude=1.0, base=10000.0, seed=0):
    q, k, v, dq, dk, gq, gk = _inputs(seed, B, S, H, Hkv, dh)
    gq, gk = gq if "q" in norms else None, gk if "k" in norms else None
    live = _live(q, length)
    for t in (q, k, v, dq, dk):
        t[~live] = float("nan")
    freq = kernels.rotary_frequencies(rot, base)[0] if rot else None
    angle = _positions(B, S, start, pos)[..., None] * (freq if rot else torch.zeros(0, dtype=torch.float64))
    how = dict(layout=layout, amplitude=amplitude, gamma_q=gq.cuda() if gq is not None else None, gamma_k=gk.cuda() if gk is not None else None, eps=1e-5,
               pos=pos.cuda() if pos is not None else None, start=_ints(start), length=_ints(length))
    f = freq.cuda() if rot else None
    Q, K, V, dQ, dK = _gpu(q, k, v, dq, dk)
    got = kernels.rotary_fwd(Q if H else None, K if Hkv else None, f, H, Hkv, v=V if Hkv else None, **how)
    for t, x, h, w in ((got[0], q, H, gq), (got[1], k, Hkv, gk)):
        if h:
            _near(t, *_forward(x, h, angle, amplitude, layout, w, 1e-5, live))
    if Hkv:
        assert torch.equal(got[2].cpu(), torch.where(live[..., None], v, 0.0))
    grads = kernels.rotary_bwd(dQ if H else None, dK if Hkv else None, f, H, Hkv, q=Q if gq is not None else None, k=K if gk is not None else None, **how)
    for t, w_got, x, d, h, w in ((grads[0], grads[2], q, dq, H, gq), (grads[1], grads[3], k, dk, Hkv, gk)):
        if h:
            dx, bound, dw, e_w = _backward(x, d, h, angle, amplitude, layout, w, 1e-5, live)
            _near(t, dx, bound)
            assert (w_got is None) == (w is None)
            if w is not None:
                _near(w_got, dw, e_w)


# one token and many, odd numbers of tokens and heads, one of the two norms, all, part and nothing of a head turned, one side alone
@pytest.mark.parametrize("B,S,H,Hkv,dh,rot,layout,norms", [
    (1, 1, 1, 1, 64, 64, "half", ""), (1, 1, 1, 1, 128, 128, "pairs", "qk"), (3, 1, 12, 12, 64, 64, "pairs", ""), (2, 7, 5, 1, 128, 128, "half", "qk"),
    (2, 33, 25, 25, 64, 32, "pairs", "q"), (2, 33, 25, 5, 64, 32, "half", "k"), (1, 100, 3, 3, 128, 48, "half", "qk"), (1, 100, 3, 3, 128, 112, "pairs", "qk"),
    (2, 50, 8, 2, 128, 16, "half", ""), (2, 50, 8, 2, 64, 48, "half", "qk"), (2, 9, 4, 2, 64, 0, "half", "qk"), (2, 9, 4, 2, 128, 0, "pairs", ""),
    (2, 300, 4, 0, 64, 64, "half", "q"), (2, 300, 0, 3, 128, 64, "pairs", "k"), (1, 2500, 2, 1, 64, 64, "half", "qk"), (5, 1003, 1, 1, 128, 128, "half", ""),
    (1, 3, 130, 70, 128, 128, "half", "qk"), (3, 1111, 3, 2, 64, 64, "pairs", "qk")])
def test_forward_and_backward(B, S, H, Hkv, dh, rot, layout, norms):
    _check(B, S, H, Hkv, dh, rot, layout, norms)


@pytest.mark.parametrize("norms", ["", "qk"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("length,start", [([0, 40, 7], None), (None, [5, 1000000, 0]), ([1, 39, 0], [100, 2 ** 31 - 41, 3]), ([-3, 100, 40], [-7, 2, -1])])
def test_lengths_and_starts(length, start, layout, norms):
    """What lies behind a sequence is not a number on the way in and zero on the way out."""
    _check(3, 40, 4, 2, 64, 64, layout, norms, length=length, start=start, seed=1)


@pytest.mark.parametrize("layout,dh,rot", [("half", 128, 64), ("pairs", 64, 64)])
def test_positions_of_their_own(layout, dh, rot):
    """Packed sequences, far, repeated and negative positions, an amplitude and a large base."""
    g = torch.Generator().manual_seed(3)
    pos = torch.randint(-2 ** 31, 2 ** 31, (2, 77), generator=g, dtype=torch.int64).to(torch.int32)
    pos[0, :30] = torch.arange(30)
    pos[0, 30:60] = torch.arange(30)
    pos[1, 0], pos[1, 1] = 2 ** 31 - 1, -2 ** 31
    _check(2, 77, 3, 1, dh, rot, layout, "qk", length=[77, 50], start=[3, 9], pos=pos, amplitude=1.35, base=500000.0, seed=2)


def _turns(freq, pos):
    """freq pos / (2 pi) less the nearest whole number, [positions, frequencies], in whole numbers with 1 / (2 pi) to 75 digits."""
    turn = Fraction(10 ** 75, 6283185307179586476925286766559005768394338798750211641949889184615632812572)
    t = [[Fraction(f) * p * turn for f in freq] for p in pos]
    return torch.tensor([[float(x - round(x)) for x in row] for row in t], dtype=torch.float64)


@pytest.mark.parametrize("layout,dh,amplitude", [("half", 64, 1.0), ("pairs", 128, -1.5)])
def test_angles_of_far_positions_and_fast_frequencies(layout, dh, amplitude):
    """Frequencies up to 2^40 and the ends of 32-bit positions.  Every pair is one that its angle turns to nearly (0, r) or, going back, (r, 0): the small
    result, next to which a bf16 rounding is nothing, is off by the angle, 2^-25 turns, by a cosine and a sine (4 u, of which a step next to 1 is one),
    their products with the amplitude (u) and the pair's product (u), times the pair's own size."""
    g = torch.Generator().manual_seed(17)
    half, S = dh // 2, 40
    freq = torch.exp2(torch.linspace(-20.0, 40.0, half, dtype=torch.float64)) * (1.0 - 0.5 * torch.rand(half, generator=g, dtype=torch.float64))
    freq[half // 2] = 500000.0 ** (-2.0 / 128)
    freq[3] = -freq[3]
    pos = torch.randint(-2 ** 31, 2 ** 31, (S,), generator=g, dtype=torch.int64)
    pos[:6] = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2147311945])
    turns = _turns(freq.tolist(), pos.tolist())
    c, s = torch.cos(2 * math.pi * turns), torch.sin(2 * math.pi * turns)
    # whole numbers of 8 bits (bf16) whose quotient is nearest to the angle's tangent
    size = torch.arange(128, 256, dtype=torch.float64)[:, None, None]
    a, b = torch.round(size * s), torch.round(size * c)
    best = (a * c - b * s).abs().argmin(0, keepdim=True)
    a, b = a.gather(0, best)[0], b.gather(0, best)[0]
    first, second = _halves(dh, layout)
    at = pos.to(torch.int32)[None].cuda()

    def matrix(x, y):
        m = torch.zeros(1, S, dh, dtype=torch.bfloat16)
        m[0, :, first], m[0, :, second] = x.to(torch.bfloat16), y.to(torch.bfloat16)
        return m.cuda()

    how = dict(layout=layout, amplitude=amplitude, pos=at)
    # in front: (a c - b s, b c + a s); back: (b c + a s, a c - b s) of (b, a)
    there = kernels.rotary_fwd(matrix(a, b), None, freq.cuda(), 1, 0, **how)[0]
    back = kernels.rotary_bwd(matrix(b, a), None, freq.cuda(), 1, 0, **how)[0]
    bound = (2 * math.pi * 2.0 ** -25 + 6 * U) * abs(amplitude) * (a.abs() + b.abs())
    for got, columns, ref in ((there, first, a * c - b * s), (there, second, b * c + a * s), (back, first, b * c + a * s), (back, second, a * c - b * s)):
        got, ref = got[0].cpu().double()[:, columns], amplitude * ref
        over = (got - ref).abs() / (bound + 2.0 ** -8 * ref.abs() + 1e-30)
        assert bool((over <= 1.0).all()), "off by %.3g of the bound at (position, frequency) %d" % (float(over.max()), int(over.argmax()))


def test_zeros_and_extremes():
    """A head of zeros has a norm of eps alone; values whose squares are near the ends of fp32."""
    q, k, _, dq, dk, gq, gk = _inputs(4, 1, 6, 2, 1, 64)
    q[0, 0] = 0.0
    k[0, 1] = 0.0
    q[0, 2] *= 1e15
    q[0, 3] *= 1e-15
    live = _live(q, None)
    freq = kernels.rotary_frequencies(64)[0]
    angle = _positions(1, 6, None, None)[..., None] * freq
    got = kernels.rotary_fwd(*_gpu(q, k, freq), 2, 1, gamma_q=gq.cuda(), gamma_k=gk.cuda(), eps=1e-5)
    _near(got[0], *_forward(q, 2, angle, 1.0, "half", gq, 1e-5, live))
    _near(got[1], *_forward(k, 1, angle, 1.0, "half", gk, 1e-5, live))
    grads = kernels.rotary_bwd(*_gpu(dq, dk, freq), 2, 1, q=q.cuda(), k=k.cuda(), gamma_q=gq.cuda(), gamma_k=gk.cuda(), eps=1e-5)
    for i, (x, d, h, w) in enumerate(((q, dq, 2, gq), (k, dk, 1, gk))):
        dx, bound, dw, e_w = _backward(x, d, h, angle, 1.0, "half", w, 1e-5, live)
        _near(grads[i], dx, bound)
        _near(grads[2 + i], dw, e_w)


def test_a_token_that_is_not_a_number_stays_alone():
    q, k, v, dq, dk, gq, gk = _gpu(*_inputs(5, 2, 20, 4, 2, 128))
    freq = kernels.rotary_frequencies(128)[0].cuda()
    how = dict(gamma_q=gq, gamma_k=gk)
    ref = kernels.rotary_fwd(q, k, freq, 4, 2, v=v, **how)
    grads = kernels.rotary_bwd(dq, dk, freq, 4, 2, q=q, k=k, **how)
    q[1, 3, 5], k[0, 7, 200] = math.nan, math.inf
    got = kernels.rotary_fwd(q, k, freq, 4, 2, v=v, **how)
    back = kernels.rotary_bwd(dq, dk, freq, 4, 2, q=q, k=k, **how)
    for a, b, at, col in ((got[0], ref[0], (1, 3), slice(0, 128)), (got[1], ref[1], (0, 7), slice(128, 256)), (back[0], grads[0], (1, 3), slice(0, 128)),
                          (back[1], grads[1], (0, 7), slice(128, 256))):
        a, b = a.clone(), b.clone()
        assert bool(torch.isnan(a[at][col]).any())
        a[at][col] = b[at][col] = 0.0
        assert torch.equal(a, b)


# rows, sinks, tokens a call, starts and lengths: rings that are not full, that a call goes round once and several times, of one row, sinks that are
# more than the rows
@pytest.mark.parametrize("rows,sinks,S,start,length", [
    (64, 0, 1, [0, 63, 64], None), (68, 4, 1, [3, 68, 100000], None), (10, 2, 25, [0, 1, 40], [25, 0, 13]), (9, 1, 9, [0, 8, 1000], [9, 1, 8]), (1, 0, 5, [0, 0, 7], [5, 1, 0]),
    (5, 4, 12, [0, 2, 900], [12, 3, 12]), (3, 100, 7, [0, 1, 2], [3, 2, 7]), (100, 4, 70, None, [70, 0, 1]), (33, 32, 64, [0, 31, 2 ** 31 - 65], [64, 64, 64])])
@pytest.mark.parametrize("values", [True, False])
def test_cache(rows, sinks, S, start, length, values):
    """Against tokens written one after the other; rows that no token takes keep what they held, bit for bit."""
    B, H, Hkv, dh = 3, 4, 2, 64
    q, k, v, _, _, gq, gk = _inputs(6, B, S, H, Hkv, dh)
    freq = kernels.rotary_frequencies(dh)[0].cuda()
    how = dict(gamma_q=gq.cuda(), gamma_k=gk.cuda(), start=_ints(start), length=_ints(length), v=v.cuda() if values else None)
    ref = kernels.rotary_fwd(q.cuda(), k.cuda(), freq, H, Hkv, **how)
    g = torch.Generator().manual_seed(7)
    keys, held = (torch.randn(B, rows, Hkv * dh, generator=g).to(torch.bfloat16) for _ in range(2))
    cache = keys.cuda(), held.cuda() if values else None
    got = kernels.rotary_fwd(q.cuda(), k.cuda(), freq, H, Hkv, cache=cache, sinks=sinks, **how)
    assert torch.equal(got[0], ref[0]) and got[1] is cache[0]
    first = min(sinks, rows - 1)
    for b in range(B):
        for i in range(length[b] if length else S):
            p = (start[b] if start else 0) + i
            row = p if p < first else first + (p - first) % (rows - first)
            keys[b, row] = ref[1][b, i].cpu()
            held[b, row] = v[b, i]
    assert torch.equal(cache[0].cpu(), keys)
    if values:
        assert got[2] is cache[1] and torch.equal(cache[1].cpu(), held)


@pytest.mark.parametrize("sinks", [2 ** 31, 2 ** 32, 2 ** 40 + 1])
def test_sinks_behind_32_bits(sinks):
    """Any number of sinks counts as rows - 1 at most, as the attention that reads the cache takes it."""
    q, k, v, *_ = _gpu(*_inputs(16, 2, 6, 2, 2, 64))
    freq = kernels.rotary_frequencies(64)[0].cuda()
    out = []
    for n in (sinks, 3):
        cache = [torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        out.append(kernels.rotary_fwd(q, k, freq, 2, 2, v=v, cache=cache, sinks=n, start=_ints([0, 70])))
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_a_cache_of_lengths_out_of_range():
    """Lengths above S and below 0 are S and 0, for the rows too."""
    q, k, v, *_ = _gpu(*_inputs(8, 2, 6, 2, 2, 64))
    freq = kernels.rotary_frequencies(64)[0].cuda()
    out = []
    for length in ([100, -5], [6, 0]):
        cache = [torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        out.append(kernels.rotary_fwd(q, k, freq, 2, 2, v=v, cache=cache, sinks=1, length=_ints(length)))
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_columns_of_one_matrix_in_place():
    B, S, H, Hkv, dh = 2, 37, 5, 5, 64
    q, k, v, dq, dk, gq, gk = _inputs(9, B, S, H, Hkv, dh)
    freq = kernels.rotary_frequencies(dh)[0].cuda()
    how = dict(gamma_q=gq.cuda(), gamma_k=gk.cuda(), length=_ints([37, 11]), layout="pairs")
    ref = kernels.rotary_fwd(q.cuda(), k.cuda(), freq, H, Hkv, **how)
    grads = kernels.rotary_bwd(dq.cuda(), dk.cuda(), freq, H, Hkv, q=q.cuda(), k=k.cuda(), **how)
    qkv = torch.cat([torch.full((B, S, 8), 3.0, dtype=torch.bfloat16), q, k, v], -1).cuda()
    cut = lambda t: (t[..., 8:8 + H * dh], t[..., 8 + H * dh:8 + (H + Hkv) * dh])  # noqa: E731
    Q, K = cut(qkv)
    got = kernels.rotary_fwd(Q, K, freq, H, Hkv, q_out=Q, k_out=K, **how)
    assert got[0] is Q and torch.equal(Q, ref[0]) and torch.equal(K, ref[1])
    assert bool((qkv[..., :8] == 3.0).all()) and torch.equal(qkv[..., 8 + (H + Hkv) * dh:].cpu(), v)
    dqkv = torch.cat([torch.full((B, S, 8), 3.0, dtype=torch.bfloat16), dq, dk, v], -1).cuda()
    dQ, dK = cut(dqkv)
    back = kernels.rotary_bwd(dQ, dK, freq, H, Hkv, q=q.cuda(), k=k.cuda(), dq=dQ, dk=dK, **how)
    assert torch.equal(dQ, grads[0]) and torch.equal(dK, grads[1]) and torch.equal(back[2], grads[2]) and torch.equal(back[3], grads[3])
    assert bool((dqkv[..., :8] == 3.0).all()) and torch.equal(dqkv[..., 8 + (H + Hkv) * dh:].cpu(), v)
    # the gradients over the inputs, no dgamma
    Q, K = q.cuda(), k.cuda()
    back = kernels.rotary_bwd(dq.cuda(), dk.cuda(), freq, H, Hkv, q=Q, k=K, dq=Q, dk=K, weights=False, **how)
    assert torch.equal(Q, grads[0]) and torch.equal(K, grads[1]) and back[2] is None and back[3] is None


def test_gradient_against_differences():
    B, S, H, Hkv, dh, rot = 2, 5, 2, 1, 64, 32
    q, k, _, dq, dk, gq, gk = _inputs(10, B, S, H, Hkv, dh)
    freq = kernels.rotary_frequencies(rot)[0]
    grads = kernels.rotary_bwd(*_gpu(dq, dk, freq), H, Hkv, q=q.cuda(), k=k.cuda(), gamma_q=gq.cuda(), gamma_k=gk.cuda(), eps=1e-5, start=_ints([3, 11]))
    angle = _positions(B, S, [3, 11], None)[..., None] * freq
    live = _live(q, None)
    g = torch.Generator().manual_seed(11)

    def total(x, d, h, w):
        return float((_forward(x, h, angle, 1.0, "half", w, 1e-5, live)[0] * d.double()).sum())

    for x, d, h, w, dx, dw in ((q, dq, H, gq, grads[0], grads[2]), (k, dk, Hkv, gk, grads[1], grads[3])):
        for grad, at in ((dx, 0), (dw, 1)):
            base = [x.double(), w.double()]
            u = torch.randn(base[at].shape, generator=g, dtype=torch.float64)
            plus, minus = ([t + e * u if i == at else t for i, t in enumerate(base)] for e in (1e-5, -1e-5))
            num = (total(plus[0], d, h, plus[1]) - total(minus[0], d, h, minus[1])) / 2e-5
            terms = grad.cpu().double() * u
            assert abs(float(terms.sum()) - num) <= 2.0 ** -7 * float(terms.abs().sum())


def test_backward_turns_back():
    """Without norms the gradient of a forward's own result is its input, but for the roundings of both: 2^-8 each of what a pair holds."""
    q, k, *_ = _gpu(*_inputs(12, 3, 100, 4, 2, 128))
    freq = kernels.rotary_frequencies(128)[0].cuda()
    out = kernels.rotary_fwd(q, k, freq, 4, 2, start=_ints([0, 70000, 5]))
    back = kernels.rotary_bwd(*out, freq, 4, 2, start=_ints([0, 70000, 5]))
    for a, b in zip(back, (q, k)):
        x = b.double().unflatten(-1, (-1, 2, 64))
        pair = x.abs().sum(-2, keepdim=True).expand_as(x).flatten(-3)
        assert bool(((a.double() - b.double()).abs() <= 2.0 ** -8 * (b.double().abs() + 2 * pair) * 1.01).all())


def test_many_tokens():
    """More than the workgroups that add up dgamma take at once, and a long sum; on the card, against 64 bits there."""
    B, S, H, Hkv, dh = 3, 70001, 2, 1, 64
    q, k, _, dq, dk, gq, gk = _inputs(13, B, S, H, Hkv, dh)
    length = [70001, 33333, 60000]
    live = _live(q, length)
    freq = kernels.rotary_frequencies(dh)[0]
    how = dict(gamma_q=gq.cuda(), gamma_k=gk.cuda(), eps=1e-5, length=_ints(length))
    got = kernels.rotary_fwd(*_gpu(q, k, freq), H, Hkv, **how)
    grads = kernels.rotary_bwd(*_gpu(dq, dk, freq), H, Hkv, q=q.cuda(), k=k.cuda(), **how)
    angle = _positions(B, S, None, None)[..., None] * freq
    for i, (x, d, h, w) in enumerate(((q, dq, H, gq), (k, dk, Hkv, gk))):
        _near(got[i], *_forward(x, h, angle, 1.0, "half", w, 1e-5, live))
        dx, bound, dw, e_w = _backward(x, d, h, angle, 1.0, "half", w, 1e-5, live)
        _near(grads[i], dx, bound)
        _near(grads[2 + i], dw, e_w)


def test_offsets_behind_32_bits():
    """Tokens 2^24 elements apart, in and out, and a cache whose rows are: bit for bit what matrices without gaps give."""
    B, S, H, Hkv, dh = 2, 100, 2, 1, 128
    q, k, v, dq, dk, gq, gk = _inputs(14, B, S, H, Hkv, dh)
    freq = kernels.rotary_frequencies(dh)[0].cuda()
    how = dict(gamma_q=gq.cuda(), gamma_k=gk.cuda())
    ref = kernels.rotary_fwd(q.cuda(), k.cuda(), freq, H, Hkv, v=v.cuda(), **how)
    grads = kernels.rotary_bwd(dq.cuda(), dk.cuda(), freq, H, Hkv, q=q.cuda(), k=k.cuda(), **how)
    room = torch.empty(2, B, S, 1 << 24, dtype=torch.bfloat16, device="cuda")
    cut = lambda at, which=0: room[which, ..., at:at + H * dh]  # noqa: E731
    Q, K, V = cut(0), room[0, ..., 1000:1000 + dh], room[0, ..., 2000:2000 + dh]
    for a, b in ((Q, q), (K, k), (V, v)):
        a.copy_(b)
    out, cache = cut(0, 1), (room[1, ..., 1000:1000 + dh], room[1, ..., 2000:2000 + dh])
    got = kernels.rotary_fwd(Q, K, freq, H, Hkv, v=V, q_out=out, cache=cache, **how)
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    out.copy_(dq)
    cache[0].copy_(dk)
    back = kernels.rotary_bwd(out, cache[0], freq, H, Hkv, q=Q, k=K, dq=out, dk=cache[0], **how)
    for a, b in zip(back, grads):
        assert torch.equal(a, b)


def test_same_bits_other_streams_and_captured_graph():
    B, S, H, Hkv, dh = 2, 300, 6, 3, 64
    tensors = _gpu(*_inputs(15, B, S, H, Hkv, dh))
    q, k, v, dq, dk, gq, gk = tensors
    freq = kernels.rotary_frequencies(dh)[0].cuda()
    start, length = _ints([5, 100000]), _ints([300, 123])
    cache = [torch.zeros(B, 64, Hkv * dh, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def both(cache, stream=None):
        how = dict(gamma_q=gq, gamma_k=gk, start=start, length=length, stream=stream)
        return (*kernels.rotary_fwd(q, k, freq, H, Hkv, v=v, **how), *kernels.rotary_fwd(q, k, freq, H, Hkv, v=v, cache=cache, sinks=3, **how),
                *kernels.rotary_bwd(dq, dk, freq, H, Hkv, q=q, k=k, **how))

    ref = both([t.clone() for t in cache])
    torch.cuda.synchronize()
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    caches = [[t.clone() for t in cache] for _ in range(2)]
    torch.cuda.synchronize()
    runs = [both(c, st) for c, st in zip(caches, (first, second))]
    torch.cuda.synchronize()
    for got in runs:
        for a, b in zip(got, ref):
            assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    mine = [t.clone() for t in cache]
    with torch.cuda.graph(graph):
        got = both(mine)
    for seed in range(4):
        for t, fresh in zip(tensors, _inputs(40 + seed, B, S, H, Hkv, dh)):
            t.copy_(fresh)
        start.copy_(torch.tensor([7 * seed, 1000 + seed], dtype=torch.int32))
        length.copy_(torch.tensor([300 - seed, 77 * seed], dtype=torch.int32))
        for t in mine:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, both([t.clone() for t in cache])):
            assert torch.equal(a, b)
