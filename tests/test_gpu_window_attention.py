"""Attention over a window and the first tokens, and its gradients, against the definition in 64 bits on the same bf16 operands.

Tolerances, element by element; a bf16 rounding is off by at most 2^-8 of the value, and the fp32 steps in front of it (scores of dh
products, an exponential, sums over the keys) are kept together as `slack`, relative to a probability:
  out   each probability is rounded once, the result once:       (2^-8 + slack) sum p |v| + 2^-8 |out|
  dv    the same over the rows:                                  (2^-8 + slack) sum p |do| + 2^-8 |dv|
  dq    ds = p (dp - D), rounded once; D = rowsum(do o) with the o given, rounded when it was written, so off by 2^-8 sum |do o|, and dp
        by fp32 alone: per element of ds (2^-8 + slack) |ds| + p (2^-8 sum |do o| + slack sum |do| |v|), through |k|, then 2^-8 |dq|
  dk    the same through |q|
`slack` is (dh + 8) 2^-24 of the largest score's absolute products, twice (in the forward's lse and in the backward), and (keys / 32 + 64) 2^-24 for the
exponential and the sums; lse2 is off by 2^-12 at most for scores of tens.
"""
import math

import pytest
import torch

from paper_2401_01728_amd import kernels

pytestmark = pytest.mark.gpu


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda() if v is not None else None


def _inputs(seed, B, S, H, Hkv, dh, length=None):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(B, S, (H + 2 * Hkv) * dh, generator=g).to(torch.bfloat16)
    qkv[..., :H * dh] *= 1.25
    do = (torch.randn(B, S, H * dh, generator=g) * 0.02).to(torch.bfloat16)
    n = [S] * B if length is None else [max(0, min(S, x)) for x in length]
    for b in range(B):
        qkv[b, n[b]:] = float("nan")
        do[b, n[b]:] = float("nan")
    return qkv, do, n


def _split(qkv, H, Hkv, dh):
    return qkv[..., :H * dh], qkv[..., H * dh:(H + Hkv) * dh], qkv[..., (H + Hkv) * dh:]


def _reference(q, k, v, do, n, H, Hkv, window, sinks, see=None):
    """Keys are the tokens' own, or k and v [B, keys, ..] in order of positions, with see(b) the mask [tokens, keys]."""
    B, Sq, _ = q.shape
    dh = q.shape[2] // H
    f64 = dict(dtype=torch.float64, device=q.device)
    out, lse2 = torch.zeros(q.shape, **f64), torch.full((B, H, Sq), -math.inf, **f64)
    dq, dk, dv = torch.zeros(q.shape, **f64), torch.zeros(k.shape, **f64), torch.zeros(k.shape, **f64)
    e_out, e_dq, e_dk, e_dv = (torch.zeros_like(t) for t in (out, dq, dk, dv))
    for b in range(B):
        m = n[b]
        if m == 0:
            continue
        if see is None:
            p, j = torch.arange(m, device=q.device)[:, None], torch.arange(m, device=q.device)[None, :]
            sees, keys = (j <= p) & ((j > p - window) | (j < sinks)), slice(0, m)
        else:
            sees, keys = see(b)
        for h in range(H):
            c, kc = slice(h * dh, (h + 1) * dh), slice(h // (H // Hkv) * dh, (h // (H // Hkv) + 1) * dh)
            qh, kh, vh = q[b, :m, c].double(), k[b, keys, kc].double(), v[b, keys, kc].double()
            s = (qh @ kh.T / math.sqrt(dh)).masked_fill(~sees, -math.inf)
            lse = torch.logsumexp(s, 1, keepdim=True)
            p = torch.where(lse == -math.inf, 0.0, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)))
            out[b, :m, c], lse2[b, h, :m] = p @ vh, lse[:, 0] / math.log(2.0)
            slack = (dh + 8) * 2.0 ** -24 * float((qh.abs() @ kh.abs().T).max()) / math.sqrt(dh) * 2 + (kh.shape[0] / 32 + 64) * 2.0 ** -24
            r = 2.0 ** -8 + slack
            e_out[b, :m, c] = r * (p @ vh.abs()) + 2.0 ** -8 * out[b, :m, c].abs()
            if do is None:
                continue
            doh = do[b, :m, c].double()
            dp = doh @ vh.T
            D = (doh * out[b, :m, c]).sum(1, keepdim=True)
            ds = p * (dp - D)
            e_ds = r * ds.abs() + p * (2.0 ** -8 * (doh * out[b, :m, c]).abs().sum(1, keepdim=True) + slack * (doh.abs() @ vh.abs().T))
            dq[b, :m, c] = ds @ kh / math.sqrt(dh)
            e_dq[b, :m, c] = e_ds @ kh.abs() / math.sqrt(dh) + 2.0 ** -8 * dq[b, :m, c].abs()
            dk[b, keys, kc] += ds.T @ qh / math.sqrt(dh)
            e_dk[b, keys, kc] += e_ds.T @ qh.abs() / math.sqrt(dh)
            dv[b, keys, kc] += p.T @ doh
            e_dv[b, keys, kc] += r * (p.T @ doh.abs())
    e_dk += 2.0 ** -8 * dk.abs()
    e_dv += 2.0 ** -8 * dv.abs()
    # second order: a rounding of what is already off
    return (out, lse2, dq, dk, dv), tuple(e * (1 + 2.0 ** -7) + 1e-30 for e in (e_out, e_dq, e_dk, e_dv))


def _near(got, ref, bound):
    got = got.to(ref.device).double()
    assert got.shape == ref.shape and bool(torch.isfinite(got).all())
    over = (got - ref).abs() / bound
    assert bool((over <= 1.0).all()), "off by %.3g of the bound at %s" % (float(over.max()), int(over.argmax()))


def _near_lse(got, ref, off=2.0 ** -12):
    got = got.to(ref.device).double()
    assert torch.equal(got == -math.inf, ref == -math.inf)
    there = ref != -math.inf
    assert float((got - ref)[there].abs().max() if there.any() else 0.0) <= off


def _both(qkv, do, H, Hkv, dh, window, sinks, length=None, stream=None):
    q, k, v = _split(qkv, H, Hkv, dh)
    out, lse2 = kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, length=length, stream=stream)
    return (out, lse2) + kernels.window_attention_bwd(q, k, v, out, do, lse2, H, Hkv, window, sinks, length=length, stream=stream)


def _check(B, S, H, Hkv, dh, window, sinks, length=None, seed=0, on_gpu=False):
    qkv, do, n = _inputs(seed, B, S, H, Hkv, dh, length)
    if on_gpu:
        qkv, do = qkv.cuda(), do.cuda()
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(*_split(qkv, H, Hkv, dh), do, n, H, Hkv, window, sinks)
    got = _both(qkv.cuda(), do.cuda(), H, Hkv, dh, window, sinks, _ints(length))
    _near(got[0], out, e_out)
    _near_lse(got[1], lse2)
    for a, ref, bound in zip(got[2:], (dq, dk, dv), (e_dq, e_dk, e_dv)):
        _near(a, ref, bound)


# one token and few, windows and sinks around tiles of 32 and 64 and a workgroup's 128 rows, windows of one token and wider than the sequence, sinks that
# the window has not left, that fill tiles, and that are more than the sequence; shared heads whose rows are several tokens' and not a divisor of 32
@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks", [
    (1, 1, 1, 1, 64, 1, 0), (1, 1, 2, 1, 128, 5, 4), (2, 2, 3, 3, 64, 1, 0), (1, 7, 4, 1, 128, 3, 1), (2, 31, 1, 1, 64, 7, 0), (1, 33, 2, 2, 128, 33, 0),
    (1, 63, 2, 1, 64, 100, 0), (1, 64, 2, 2, 64, 64, 64), (1, 65, 3, 1, 128, 64, 1), (2, 127, 2, 2, 64, 32, 3), (1, 128, 4, 2, 128, 1, 4), (1, 129, 5, 1, 64, 63, 4),
    (1, 200, 6, 2, 64, 65, 65), (2, 257, 2, 2, 128, 16, 130), (1, 300, 8, 1, 64, 100, 4), (1, 300, 7, 1, 128, 1, 0), (1, 300, 3, 3, 64, 2, 1000),
    (1, 500, 12, 12, 64, 128, 4), (1, 511, 25, 5, 64, 200, 1), (1, 700, 2, 2, 128, 2 ** 31 - 1, 0), (1, 700, 2, 2, 128, 300, 2 ** 31 - 1), (2, 1000, 4, 2, 128, 256, 16),
    (1, 1500, 2, 1, 64, 3, 5), (1, 900, 20, 4, 64, 90, 100), (3, 150, 33, 3, 64, 40, 2)])
def test_forward_and_backward(B, S, H, Hkv, dh, window, sinks):
    _check(B, S, H, Hkv, dh, window, sinks)


@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,length", [
    (3, 200, 4, 2, 64, 30, 4, [200, 0, 65]), (4, 130, 4, 1, 128, 64, 0, [1, 130, 0, 64]), (4, 130, 2, 2, 64, 200, 3, [0, 63, 64, 129]), (2, 90, 3, 3, 64, 10, 1, [0, 0]),
    (3, 100, 2, 1, 128, 33, 100, [-5, 1000, 32]), (2, 2000, 2, 2, 64, 100, 4, [1999, 3]), (5, 300, 16, 2, 128, 128, 130, [300, 129, 128, 1, 0])])
def test_lengths(B, S, H, Hkv, dh, window, sinks, length):
    """Sequences of their own lengths, none among them; what lies behind is not a number, and zero in the results."""
    _check(B, S, H, Hkv, dh, window, sinks, length, seed=1)


# grids of many workgroups, rows and keys that end inside all blocks, long walks, sinks that thousands of rows see
@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,length", [
    (4, 2000, 16, 16, 128, 300, 4, None), (9, 777, 40, 10, 128, 500, 20, [777, 0, 1, 63, 500, 129, 64, 65, 128]), (8, 1030, 24, 12, 64, 1000, 0, [1030, 1, 700, 0, 9, 64, 333, 1]),
    (1, 9000, 8, 1, 128, 700, 5, None), (1, 7001, 3, 3, 64, 2 ** 31 - 1, 0, None), (2, 5000, 4, 4, 64, 64, 300, [5000, 4321])])
def test_many_workgroups(B, S, H, Hkv, dh, window, sinks, length):
    _check(B, S, H, Hkv, dh, window, sinks, length, seed=2, on_gpu=True)


def _cache(k, v, end, Sk, sinks):
    """Rows of sequences whose keys 0 .. end[b] - 1 were written in order; what was not written is not a number.  Which key each row holds."""
    B = k.shape[0]
    first = min(sinks, Sk - 1)
    kc, vc = (torch.full((B, Sk, k.shape[2]), float("nan"), dtype=torch.bfloat16) for _ in range(2))
    holds = []
    for b in range(B):
        j = torch.arange(end[b])
        row = torch.where(j < first, j, first + (j - first) % (Sk - first))
        held = torch.full((Sk,), -1)
        for lo in range(0, end[b], 1 << 12):               # (index_put with repeats keeps none in particular: one round of the ring at a time)
            for x in range(lo, min(end[b], lo + (1 << 12))):
                held[row[x]] = x
        there = held >= 0
        kc[b, there], vc[b, there] = k[b, held[there]], v[b, held[there]]
        holds.append(held)
    return kc, vc, holds


# single tokens and few, in one walk and in parts; chunks; rings that end inside tiles, that several sequences have gone round differently often, with rows
# for the window and one more, and fewer than the window has keys; of one row; sequences that are shorter than the sinks
CACHES = [
    (1, 1, 1024, 12, 12, 64, 1000, 0, [900], None), (3, 1, 68, 8, 2, 128, 64, 4, [0, 67, 1000], None), (3, 1, 64, 4, 1, 64, 64, 0, [5000, 63, 64], None),
    (4, 1, 4100, 8, 1, 64, 4096, 4, [4099, 4100, 9000, 3], None), (2, 1, 3001, 4, 4, 128, 3000, 1, [2500, 7001], None), (3, 1, 33, 4, 2, 64, 100, 3, [10, 32, 500], None),
    (2, 1, 1, 2, 2, 64, 5, 0, [0, 7], None), (2, 1, 3, 2, 1, 128, 5, 100, [1, 7], None), (3, 4, 40, 8, 1, 64, 16, 2, [0, 30, 100], None),
    (2, 8, 50, 4, 1, 128, 41, 2, [700, 13], [8, 5]), (3, 100, 203, 4, 2, 64, 100, 4, [0, 150, 2000], [100, 37, 99]), (2, 70, 100, 2, 2, 128, 20, 0, [33, 1000], None),
    (2, 70, 50, 2, 2, 64, 20, 0, [0, 1000], None), (2, 70, 50, 4, 2, 128, 200, 3, [0, 1000], [70, 60]), (1, 300, 1303, 8, 2, 128, 1000, 4, [1100], None),
    (2, 30, 17, 1, 1, 64, 4, 0, [3, 0], [30, 17]), (3, 5, 2000, 32, 4, 64, 1900, 7, [1994, 1995, 6000], [5, 5, 4])]


@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh,window,sinks,start,length", CACHES)
def test_cache(B, Sq, Sk, H, Hkv, dh, window, sinks, start, length):
    n = length or [Sq] * B
    end = [s + m for s, m in zip(start, n)]
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(B, max(end), Hkv * dh, generator=g).to(torch.bfloat16) for _ in range(2))
    q = (torch.randn(B, Sq, H * dh, generator=g) * 1.3).to(torch.bfloat16)
    for b in range(B):
        q[b, n[b]:] = float("nan")
    kc, vc, holds = _cache(k, v, end, Sk, sinks)

    def see(b):
        p, j = start[b] + torch.arange(n[b])[:, None], torch.arange(end[b])[None, :]
        still = torch.zeros(end[b], dtype=torch.bool)
        still[holds[b][holds[b] >= 0]] = True
        return (j <= p) & ((j > p - window) | (j < sinks)) & still, slice(0, end[b])

    (out, lse2, *_), (e_out, *_) = _reference(q, k, v, None, n, H, Hkv, window, sinks, see)
    got = kernels.window_attention_fwd(q.cuda(), kc.cuda(), vc.cuda(), H, Hkv, window, sinks, _ints(start), _ints(length))
    _near(got[0], out, e_out)
    _near_lse(got[1], lse2)


def test_positions_near_the_end():
    """start + length = 2^31 - 1 and the rows that this is: the same bits as a ring at the same phase."""
    B, Sk, H, Hkv, dh, window, sinks = 2, 103, 4, 2, 64, 99, 4
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(B, s, h * dh, generator=g).to(torch.bfloat16).cuda() for s, h in ((1, H), (Sk, Hkv), (Sk, Hkv)))
    far = 2 ** 31 - 2
    near = 10 * (Sk - sinks) + sinks + (far - sinks) % (Sk - sinks)
    a = kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, _ints([far, near]))
    b = kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, _ints([near, far]))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, _ints([-3, 0]))[0],
                       kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, _ints([0, -9]))[0])


@pytest.mark.parametrize("dh", [64, 128])
def test_a_window_of_all_is_causal_attention(dh):
    """Against the stage's own kernel: both are within the bounds of the definition, so within their sum."""
    B, S, H = 2, 192, 2
    qkv, do, n = _inputs(5, B, S, H, H, dh)
    (out, *_), (e_out, *_) = _reference(*_split(qkv, H, H, dh), do, n, H, H, S, 0)
    got = _both(qkv.cuda(), do.cuda(), H, H, dh, S, 0)
    theirs, lse2 = kernels.attention_fwd(qkv.reshape(B * S, -1).cuda(), B, S, H * dh, H)
    assert bool(((got[0].cpu().double() - theirs.reshape(B, S, -1).cpu().double()).abs() <= 2 * e_out).all())
    assert float((got[1] - lse2.view(B, H, S)).abs().max()) <= 2.0 ** -11


def test_same_bits_every_time():
    qkv, do, _ = _inputs(7, 3, 700, 8, 4, 128)
    length = _ints([700, 123, 511])
    ref = None
    for _ in range(4):
        got = _both(qkv.cuda(), do.cuda(), 8, 4, 128, 150, 4, length)
        if ref is not None:
            for a, b in zip(got, ref):
                assert torch.equal(a, b)
        ref = got


def test_strides_and_what_lies_beside():
    B, S, H, Hkv, dh = 2, 170, 4, 2, 64
    qkv, do, _ = _inputs(2, B, S, H, Hkv, dh)
    q, k, v = _split(qkv, H, Hkv, dh)
    length = _ints([170, 37])
    ref = _both(qkv.cuda(), do.cuda(), H, Hkv, dh, 50, 3, length)

    def within(t, extra, fill):
        w = torch.full((*t.shape[:2], t.shape[2] + extra), fill, dtype=torch.bfloat16, device="cuda")
        w[..., 8:8 + t.shape[2]] = t.cuda()
        return w, w[..., 8:8 + t.shape[2]]

    nan = float("nan")
    qs, ks, vs, dos = (within(t, e, nan)[1] for t, e in ((q, 24), (k, 16), (v, 40), (do, 8)))
    wide, out = within(torch.zeros_like(q), 32, 5.0)
    got = kernels.window_attention_fwd(qs, ks, vs, H, Hkv, 50, 3, length=length, out=out)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    assert bool((wide[..., :8] == 5.0).all()) and bool((wide[..., 8 + H * dh:] == 5.0).all())
    # the gradients as columns of one matrix
    dqkv = torch.full((B, S, (H + 2 * Hkv) * dh + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    cols = _split(dqkv[..., 8:-8], H, Hkv, dh)
    got = kernels.window_attention_bwd(qs, ks, vs, out, dos, ref[1], H, Hkv, 50, 3, length, *cols)
    for a, b in zip(got, ref[2:]):
        assert torch.equal(a, b)
    assert bool((dqkv[..., :8] == 5.0).all()) and bool((dqkv[..., -8:] == 5.0).all())


@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,at,by", [
    (1, 500, 2, 2, 64, 80, 4, 411, 400.0), (2, 700, 4, 1, 128, 200, 0, 300, 400.0), (1, 300, 2, 2, 64, 300, 0, 0, 300.0), (1, 600, 4, 2, 128, 100, 8, 3, 300.0)])
def test_scores_without_bounds(B, S, H, Hkv, dh, window, sinks, at, by):
    """Scores of thousands: the running maximum moves late and far, out of the window again, and the backward's accumulators begin with as much of the
    other sign.  `slack` holds the score's own error, in the forward's lse and in the backward."""
    qkv, do, n = _inputs(8, B, S, H, Hkv, dh)
    qkv[:, at, H * dh:(H + Hkv) * dh] *= by
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(*_split(qkv, H, Hkv, dh), do, n, H, Hkv, window, sinks)
    got = _both(qkv.cuda(), do.cuda(), H, Hkv, dh, window, sinks)
    for a, ref, bound in zip(got[:1] + got[2:], (out, dq, dk, dv), (e_out, e_dq, e_dk, e_dv)):
        _near(a, ref, bound)
    assert float(lse2.abs().max()) > 200.0
    q, k, _ = _split(qkv.double(), H, Hkv, dh)
    most = float((q.abs().view(B, S, H, dh).amax((0, 1, 2)) * k.abs().view(B, S, Hkv, dh).amax((0, 1, 2))).sum())
    _near_lse(got[1], lse2, 2.0 ** -12 + (dh + 8) * 2.0 ** -24 * most * math.log2(math.e) / math.sqrt(dh))


def test_gradient_against_differences():
    B, S, H, Hkv, dh, window, sinks, n = 1, 60, 2, 1, 64, 12, 3, 50
    qkv, do, _ = _inputs(9, B, S, H, Hkv, dh, [n])
    grads = _both(qkv.cuda(), do.cuda(), H, Hkv, dh, window, sinks, _ints([n]))[2:]
    q, k, v = (t[0, :n].double() for t in _split(qkv, H, Hkv, dh))
    p, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
    hide = ~((j <= p) & ((j > p - window) | (j < sinks)))

    def total(t):
        o = torch.cat([torch.softmax((t[0][:, h * dh:(h + 1) * dh] @ t[1].T / math.sqrt(dh)).masked_fill(hide, -math.inf), -1) @ t[2] for h in range(H)], -1)
        return float((o * do[0, :n].double()).sum())

    base = [q, k, v]
    g = torch.Generator().manual_seed(10)
    for i, grad in enumerate(grads):
        u = torch.randn(base[i].shape, generator=g, dtype=torch.float64)
        plus, minus = ([t + e * u if x == i else t for x, t in enumerate(base)] for e in (1e-5, -1e-5))
        num = (total(plus) - total(minus)) / 2e-5
        terms = grad[0, :n].cpu().double() * u
        assert abs(float(terms.sum()) - num) <= 2.0 ** -6 * float(terms.abs().sum())
        assert not grad[0, n:].any()


# workgroups' borders, sinks apart and not, shared heads, lengths; what is not a number lies in the middle, in a sink, in the last token
BROKEN = [(2, 200, 2, 2, 64, 40, 0, None, 70), (2, 300, 4, 1, 128, 90, 4, [300, 250], 140), (1, 500, 2, 1, 64, 64, 3, None, 1), (1, 260, 2, 2, 128, 30, 2, None, 259),
          (1, 1100, 3, 3, 64, 100, 0, None, 512), (1, 64, 8, 1, 64, 5, 1, None, 31), (1, 8, 4, 1, 128, 3, 0, None, 4)]


@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,length,at", BROKEN)
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_key_that_is_not_a_number_reaches_who_sees_it(B, S, H, Hkv, dh, window, sinks, length, at, value):
    """One token's key, value and output gradient are infinite or no numbers.  Who does not see it has what it has without; who does has no number in
    the heads that read it.  In the backward: dk and dv of the keys that the token sees, and dq of the tokens that see it."""
    qkv, do, n = _inputs(11, B, S, H, Hkv, dh, length)
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(*_split(qkv, H, Hkv, dh), do, n, H, Hkv, window, sinks)
    share, bad = H // Hkv, slice(0, H // Hkv * dh)
    qkv, do = qkv.clone(), do.clone()
    qkv[0, at, H * dh:H * dh + dh] = value                 # key and value of the first key/value head
    qkv[0, at, (H + Hkv) * dh:(H + Hkv) * dh + dh] = value
    got = _both(qkv.cuda(), do.cuda(), H, Hkv, dh, window, sinks, _ints(length))
    p = torch.arange(n[0])
    sees = (p >= at) & ((p < at + window) | (at < sinks))
    mine = torch.zeros(B, S, dtype=torch.bool)
    mine[0, :n[0]] = sees

    def clean(t, ref, bound, rows, cols):
        t = t.cpu().double()
        where = torch.ones(t.shape, dtype=torch.bool)
        where[..., cols] = ~rows[..., None]
        assert bool(torch.isfinite(t[where]).all())
        assert bool(((t - ref).abs() <= bound)[where].all())
        return t[~where]

    assert bool((~torch.isfinite(clean(got[0], out, e_out, mine, bad))).all())
    lse = got[1][0].cpu().double()
    assert float((lse - lse2[0])[share:, :n[0]].abs().max() if share < H else 0.0) <= 2.0 ** -12
    assert float((lse - lse2[0])[:, :n[0]][:, ~sees].abs().max() if (~sees).any() else 0.0) <= 2.0 ** -12
    assert bool(torch.isnan(lse[:share, :n[0]][:, sees]).all())
    clean(got[2], dq, e_dq, mine, bad)
    # keys that share a token with it
    seen_with = torch.zeros(B, S, dtype=torch.bool)
    for t in p[sees].tolist():
        j = torch.arange(t + 1)
        seen_with[0, :t + 1] |= (j > t - window) | (j < sinks)
    clean(got[3], dk, e_dk, seen_with, slice(0, dh))
    clean(got[4], dv, e_dv, seen_with, slice(0, dh))


@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,length,at", BROKEN)
def test_an_output_gradient_that_is_not_a_number(B, S, H, Hkv, dh, window, sinks, length, at):
    """It reaches its own dq and the keys that its token sees."""
    qkv, do, n = _inputs(12, B, S, H, Hkv, dh, length)
    (_, _, dq, dk, dv), (_, e_dq, e_dk, e_dv) = _reference(*_split(qkv, H, Hkv, dh), do, n, H, Hkv, window, sinks)
    q, k, v = _split(qkv.cuda(), H, Hkv, dh)
    out, lse2 = kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, length=_ints(length))
    do = do.clone()
    do[0, at, :dh] = math.nan
    got = kernels.window_attention_bwd(q, k, v, out, do.cuda(), lse2, H, Hkv, window, sinks, _ints(length))
    j = torch.arange(S)
    seen = (j <= at) & ((j > at - window) | (j < sinks))
    for t, ref, bound, rows in ((got[0], dq, e_dq, j == at), (got[1], dk, e_dk, seen), (got[2], dv, e_dv, seen)):
        t = t.cpu().double()
        where = torch.ones(t.shape, dtype=torch.bool)
        where[0, :, :dh] = ~rows[:, None]
        assert bool(((t - ref).abs() <= bound)[where].all()) and bool(torch.isnan(t[~where]).all())


# sinks that fill whole workgroups of the backward, and one that does not
MANY_SINKS = [(1, 400, 2, 2, 64, 30, 128, None, 5), (1, 500, 4, 1, 128, 70, 200, None, 140), (2, 600, 2, 1, 64, 100, 260, [600, 300], 259), (1, 450, 3, 3, 128, 1, 130, None, 300)]


@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,length,at", MANY_SINKS)
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_broken_key_of_many_sinks(B, S, H, Hkv, dh, window, sinks, length, at, value):
    test_a_key_that_is_not_a_number_reaches_who_sees_it(B, S, H, Hkv, dh, window, sinks, length, at, value)


@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,length,at", MANY_SINKS)
def test_a_broken_output_gradient_over_many_sinks(B, S, H, Hkv, dh, window, sinks, length, at):
    test_an_output_gradient_that_is_not_a_number(B, S, H, Hkv, dh, window, sinks, length, at)


@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh,window,sinks,start,length", [c for c in CACHES if c[1] > 1])
def test_a_broken_row_of_a_cache(B, Sq, Sk, H, Hkv, dh, window, sinks, start, length):
    """The newest key's value is no number: the tokens in front of it do not see it."""
    n = length or [Sq] * B
    g = torch.Generator().manual_seed(13)
    q, k, v = (torch.randn(B, s, h * dh, generator=g).to(torch.bfloat16).cuda() for s, h in ((Sq, H), (Sk, Hkv), (Sk, Hkv)))
    ref, lse2 = kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, _ints(start), _ints(length))
    first = min(sinks, Sk - 1)
    p = start[0] + n[0] - 1
    row = p if p < first else first + (p - first) % (Sk - first)
    v[0, row] = math.nan
    got, lse = kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, _ints(start), _ints(length))
    assert torch.equal(lse, lse2)
    assert bool(torch.isnan(got[0, n[0] - 1]).all())
    got[0, n[0] - 1] = ref[0, n[0] - 1] = 0.0
    # formed again in fp32, with probabilities that are not rounded: each off by 2^-8 of sum p |v| and of itself, as the plain walk's are; values are below 6
    assert bool(((got.double() - ref.double()).abs() <= 2.0 ** -6 * 6.0).all()) and bool(torch.isfinite(got).all())


# chunks whose own keys lie on both sides of the ring's end, `before` of the first sequence's in front of it, rings gone round 1 to 50 times; in one walk and in
# parts, by few rows and by workgroups of 128; with sinks and without, windows as long as the ring allows and shorter
WRAPPED = [(2, 40, 104, 4, 2, 64, 60, 4, 20), (2, 3, 68, 8, 1, 64, 60, 4, 2), (3, 16, 333, 2, 1, 128, 300, 0, 5), (2, 100, 1507, 4, 2, 128, 1400, 4, 37),
           (1, 4, 3000, 8, 2, 64, 2900, 7, 3), (2, 130, 2003, 1, 1, 64, 1800, 3, 65), (1, 300, 700, 8, 2, 128, 350, 0, 150), (2, 33, 45, 3, 3, 64, 10, 2, 1)]


@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh,window,sinks,before", WRAPPED)
@pytest.mark.parametrize("which", ["key", "value"])
def test_a_broken_row_where_the_ring_has_wrapped(B, Sq, Sk, H, Hkv, dh, window, sinks, before, which):
    """One of the last keys of a call, or its value, is no number.  Tokens in front of it, and behind its window, have
    what the definition gives without it.  Keys in the rows next to the ring's end, on both of its sides, have a score of 4 more: one of them left out or taken
    twice is several times the bound."""
    ring = Sk - sinks
    start = [sinks + (1, 50, 7)[b] * ring + ring - before - 9 * b for b in range(B)]
    end = [s + Sq for s in start]
    g = torch.Generator().manual_seed(25)
    k, v = (torch.randn(B, max(end), Hkv * dh, generator=g).to(torch.bfloat16) for _ in range(2))
    q = (torch.randn(B, Sq, H * dh, generator=g) * 1.3).to(torch.bfloat16)
    q[..., ::dh] = math.sqrt(dh)
    k[..., ::dh] = 0.0
    for b in range(B):
        phase = (torch.arange(end[b]) - sinks) % ring
        k[b, :end[b], ::dh] = torch.where((phase >= ring - 10) | (phase < 10), 4.0, 0.0).to(torch.bfloat16)[:, None]
    kc, vc, holds = _cache(k, v, end, Sk, sinks)

    def see(b):
        p, j = start[b] + torch.arange(Sq)[:, None], torch.arange(end[b])[None, :]
        still = torch.zeros(end[b], dtype=torch.bool)
        still[holds[b][holds[b] >= 0]] = True
        return (j <= p) & ((j > p - window) | (j < sinks)) & still, slice(0, end[b])

    (out, lse2, *_), (e_out, *_) = _reference(q, k, v, None, [Sq] * B, H, Hkv, window, sinks, see)
    whole = torch.zeros(B, Sq, dtype=torch.bool)
    for b in range(B):
        at = end[b] - 1 - Sq // 8
        (kc if which == "key" else vc)[b, sinks + (at - sinks) % ring] = math.nan
        whole[b] = ~see(b)[0][:, at]
    assert bool(whole.any()) and not bool(whole.all())
    got, lse = kernels.window_attention_fwd(q.cuda(), kc.cuda(), vc.cuda(), H, Hkv, window, sinks, _ints(start))
    got = got.cpu()
    _near(got[whole], out[whole], e_out[whole])
    assert bool(torch.isnan(got[~whole]).all())
    by_token = lambda t: t.cpu().double().transpose(1, 2)  # noqa: E731
    clear = whole if which == "key" else torch.ones_like(whole)
    _near_lse(by_token(lse)[clear], by_token(lse2)[clear])
    assert bool(torch.isnan(by_token(lse)[~clear]).all())


@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,length", [(2, 100, 4, 2, 64, 20, 0, [100, 60]), (1, 300, 2, 1, 128, 300, 2, None)])
def test_a_row_of_scores_of_minus_infinity(B, S, H, Hkv, dh, window, sinks, length):
    """It has no softmax: NaN, for itself and, in the backward, for the keys it shares with others; other rows and heads are what they were."""
    qkv, do, n = _inputs(14, B, S, H, Hkv, dh, length)
    qkv[0, :, H * dh + 5] = -qkv[0, :, H * dh + 5].abs() - 0.125
    r = 57
    qkv[0, r, 5] = 0.0
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(*_split(qkv, H, Hkv, dh), do, n, H, Hkv, window, sinks)
    qkv[0, r, 5] = math.inf
    got = _both(qkv.cuda(), do.cuda(), H, Hkv, dh, window, sinks, _ints(length))
    j = torch.arange(S)
    seen = (j <= r) & ((j > r - window) | (j < sinks))
    for t, ref, bound, rows in ((got[0], out, e_out, j == r), (got[2], dq, e_dq, j == r), (got[3], dk, e_dk, seen), (got[4], dv, e_dv, seen)):
        t = t.cpu().double()
        where = torch.ones(t.shape, dtype=torch.bool)
        where[0, :, :dh] = ~rows[:, None]
        assert bool(((t - ref).abs() <= bound)[where].all()) and bool(torch.isnan(t[~where]).all())
    assert bool(torch.isnan(got[1][0, 0, r]))


@pytest.mark.parametrize("Sq,Sk,H,dh,broken", [(2, 300, 1, 64, 100), (3, 700, 2, 128, 65), (16, 90, 2, 64, 32), (40, 1200, 1, 64, 400), (33, 1300, 2, 128, 300)])
def test_keys_of_scores_of_minus_infinity_beside_rows_without_numbers(Sq, Sk, H, dh, broken):
    """The first keys' scores are -inf for even tokens, whose results are those without these keys, and +inf for odd ones, who have none."""
    g = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn(1, n, cols, generator=g).to(torch.bfloat16) for n, cols in ((Sq, H * dh), (Sk, dh), (Sk, dh)))
    for h in range(H):
        q[0, 0::2, h * dh + 3], q[0, 1::2, h * dh + 3] = 1.0, -1.0
    bad = k.clone()
    bad[0, :broken, 3] = -math.inf
    start = Sk - Sq
    out, lse2 = kernels.window_attention_fwd(q.cuda(), bad.cuda(), v.cuda(), H, 1, Sk, 0, start=_ints([start]))
    see = lambda b: ((torch.arange(Sk) <= torch.arange(Sq)[:, None] + start) & (torch.arange(Sk) >= broken), slice(0, Sk))  # noqa: E731
    (ref, ref_lse, *_), (e_out, *_) = _reference(q, k, v, None, [Sq], H, 1, Sk, 0, see)
    _near(out[:, 0::2], ref[:, 0::2], e_out[:, 0::2])
    _near_lse(lse2[:, :, 0::2], ref_lse[:, :, 0::2])
    assert bool(torch.isnan(out[:, 1::2]).all()) and bool(torch.isnan(lse2[:, :, 1::2]).all())


@pytest.mark.parametrize("rise", [0.02, 0.05, 0.12, -0.05])
@pytest.mark.parametrize("S,dh,window", [(700, 64, 500), (700, 64, 650), (1400, 64, 1300), (600, 128, 300), (900, 128, 700)])
def test_scores_that_rise_from_key_to_key(S, dh, window, rise):
    """By 1 to 11 powers of two in 64 keys, and falling: a row's largest score is another one in each tile."""
    qkv, do, n = _inputs(11, 1, S, 2, 1, dh)
    q, k, _ = _split(qkv, 2, 1, dh)
    q[..., 0] = q[..., dh] = math.sqrt(dh)
    k[..., 0] = torch.arange(S) * rise
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(*_split(qkv, 2, 1, dh), do, n, 2, 1, window, 2)
    got = _both(qkv.cuda(), do.cuda(), 2, 1, dh, window, 2)
    _near(got[0], out, e_out)
    _near_lse(got[1], lse2)
    for a, ref, bound in zip(got[2:], (dq, dk, dv), (e_dq, e_dk, e_dv)):
        _near(a, ref, bound)


@pytest.mark.parametrize("Sq,dh", [(1, 64), (1, 128), (3, 64), (40, 128)])
@pytest.mark.parametrize("rise", [0.03, -0.03])
def test_scores_that_rise_in_a_cache(Sq, dh, rise):
    """Likewise for single tokens, whose waves and parts have references of their own, and for parts of more rows."""
    Sk = 3000
    g = torch.Generator().manual_seed(12)
    q, k, v = (torch.randn(1, rows, cols, generator=g).to(torch.bfloat16) for rows, cols in ((Sq, 2 * dh), (Sk, dh), (Sk, dh)))
    q[..., 0] = q[..., dh] = math.sqrt(dh)
    k[..., 0] = torch.arange(Sk) * rise
    start = Sk - Sq
    out, lse2 = kernels.window_attention_fwd(q.cuda(), k.cuda(), v.cuda(), 2, 1, Sk, 0, start=_ints([start]))
    see = lambda b: (torch.arange(Sk) <= torch.arange(Sq)[:, None] + start, slice(0, Sk))  # noqa: E731
    (ref, ref_lse, *_), (e_out, *_) = _reference(q, k, v, None, [Sq], 2, 1, Sk, 0, see)
    _near(out, ref, e_out)
    _near_lse(lse2, ref_lse)


@pytest.mark.parametrize("window,sinks", [(2 ** 32 + 5, 0), (2 ** 63, 2 ** 32), (10, 2 ** 40)])
def test_windows_and_sinks_behind_32_bits_see_all(window, sinks):
    qkv, do, _ = _inputs(2, 1, 100, 2, 2, 64)
    for a, b in zip(_both(qkv.cuda(), do.cuda(), 2, 2, 64, window, sinks), _both(qkv.cuda(), do.cuda(), 2, 2, 64, 100 if window > 100 else window, 100 if sinks else 0)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,S,H,Hkv,dh,length", [(2, 200, 4, 2, 64, None), (2, 70, 2, 2, 128, [70, 1]), (1, 1, 2, 1, 64, None)])
def test_a_window_of_one_token(B, S, H, Hkv, dh, length):
    """Its probability is 1 whatever the score: the value itself, dq and dk exactly zero, dv the sum over the heads."""
    qkv, do, n = _inputs(15, B, S, H, Hkv, dh, length)
    got = _both(qkv.cuda(), do.cuda(), H, Hkv, dh, 1, 0, _ints(length))
    for b in range(B):
        v = qkv[b, :n[b], (H + Hkv) * dh:].unflatten(-1, (Hkv, 1, dh)).expand(-1, -1, H // Hkv, -1).flatten(-3)
        assert torch.equal(got[0][b, :n[b]].cpu(), v)
    assert not got[2].any() and not got[3].any()


def test_other_stream_and_captured_graph():
    B, S, H, Hkv, dh, window, sinks = 2, 300, 4, 2, 64, 70, 4
    qkv, do, _ = _inputs(16, B, S, H, Hkv, dh)
    qkv, do = qkv.cuda(), do.cuda()
    length, start = _ints([300, 111]), _ints([299, 5000])
    q, k, v = _split(qkv, H, Hkv, dh)
    token = lambda st=None: kernels.window_attention_fwd(q[:, :1].contiguous(), k, v, H, Hkv, 290, sinks, start, stream=st)  # noqa: E731
    ref = _both(qkv, do, H, Hkv, dh, window, sinks, length)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = _both(qkv, do, H, Hkv, dh, window, sinks, length, stream=side)
    side.synchronize()
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = (*_both(qkv, do, H, Hkv, dh, window, sinks, length), *token())
    for seed in range(4):
        for t, fresh in zip((qkv, do), _inputs(30 + seed, B, S, H, Hkv, dh)):
            t.copy_(fresh)
        length.copy_(torch.tensor([300 - seed, 64 * seed], dtype=torch.int32))
        start.copy_(torch.tensor([299 + seed, 123456 * seed], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, (*_both(qkv, do, H, Hkv, dh, window, sinks, length), *token())):
            assert torch.equal(a, b)


def test_two_calls_at_once():
    """A long backward beside single tokens on another stream."""
    H, Hkv, dh = 8, 4, 128
    qkv, do, _ = _inputs(17, 4, 1500, H, Hkv, dh)
    qkv, do = qkv.cuda(), do.cuda()
    q, k, v = _split(qkv, H, Hkv, dh)
    one, start = q[:, :1].contiguous(), _ints([1499, 0, 70000, 1024])
    ref = _both(qkv, do, H, Hkv, dh, 300, 4)
    token = kernels.window_attention_fwd(one, k, v, H, Hkv, 1400, 4, start)
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got.append((kernels.window_attention_bwd(q, k, v, ref[0], do, ref[1], H, Hkv, 300, 4, stream=first),
                    kernels.window_attention_fwd(one, k, v, H, Hkv, 1400, 4, start, stream=second)))
    torch.cuda.synchronize()
    for a, b in got:
        for x, y in zip((*a, *b), (*ref[2:], *token)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("Sq,dh", [(1, 64), (80, 128)])
def test_a_cache_behind_32_bits(Sq, dh):
    """Keys and values as columns of a cache of 6 G elements whose ring ends inside a tile, tokens 2^24 elements apart: bit for bit what matrices without
    gaps give."""
    B, Sk, H, Hkv, window, sinks = 2, 200000, 4, 2, 199000, 4
    g = torch.Generator(device="cuda").manual_seed(18)
    q, k, v = (torch.randn(B, s, h * dh, generator=g, device="cuda", dtype=torch.bfloat16) for s, h in ((Sq, H), (Sk, Hkv), (Sk, Hkv)))
    start = _ints([777777, 199000])

    def apart(t, ld, at=0):
        w = torch.empty(*t.shape[:2], ld, dtype=torch.bfloat16, device="cuda")[..., at:at + t.shape[2]]
        w.copy_(t)
        return w

    ref = kernels.window_attention_fwd(q, k, v, H, Hkv, window, sinks, start)
    got = kernels.window_attention_fwd(apart(q, 1 << 24), apart(k, 16384), apart(v, 16384, 16000), H, Hkv, window, sinks, start, out=apart(torch.zeros_like(q), 1 << 24))
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_training_behind_32_bits():
    """Tokens 2^24 elements apart."""
    B, S, H, Hkv, dh = 1, 300, 2, 1, 64
    qkv, do, _ = _inputs(19, B, S, H, Hkv, dh)
    ref = _both(qkv.cuda(), do.cuda(), H, Hkv, dh, 90, 4)
    room = torch.empty(2, S, 1 << 24, dtype=torch.bfloat16, device="cuda")
    wide = room[:1, :, :256]
    wide.copy_(qkv)
    far = lambda at, cols: room[1:, :, at:at + cols]  # noqa: E731
    d, o = far(0, 128), far(200, 128)
    d.copy_(do)
    q, k, v = _split(wide, H, Hkv, dh)
    out, lse2 = kernels.window_attention_fwd(q, k, v, H, Hkv, 90, 4, out=o)
    assert torch.equal(out, ref[0]) and torch.equal(lse2, ref[1])
    got = kernels.window_attention_bwd(q, k, v, out, d, lse2, H, Hkv, 90, 4, None, far(400, 128), far(600, 64), far(700 + 4, 64))
    for a, b in zip(got, ref[2:]):
        assert torch.equal(a, b)


def test_more_sequences_than_a_launch_takes():
    """2^20 sequences of one key and 16 heads are 2^32 threads and more: values come out, dv is the output's gradient, dq and dk are zero, bit for bit."""
    B, H, dh = 1 << 20, 16, 64
    g = torch.Generator(device="cuda").manual_seed(24)
    q, k, v, do = (torch.randn(B, 1, H * dh, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    n = torch.randint(0, 2, (B,), generator=g, device="cuda", dtype=torch.int32)
    out, lse2 = kernels.window_attention_fwd(q, k, v, H, H, 7, 1, length=n)
    dq, dk, dv = kernels.window_attention_bwd(q, k, v, out, do, lse2, H, H, 7, 1, length=n)
    step = 1 << 16
    for b in range(0, B, step):
        part = slice(b, b + step)
        keep = (n[part] > 0)[:, None, None]
        assert torch.equal(out[part], torch.where(keep, v[part], 0.0)), b
        assert torch.equal(dv[part], torch.where(keep, do[part], 0.0)), b
        assert not dq[part].any() and not dk[part].any(), b
        assert torch.equal(lse2[part] == -math.inf, ~keep.expand(-1, H, 1)), b
