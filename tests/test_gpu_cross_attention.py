"""Cross-attention and its gradients against the definition in 64 bits on the same bf16 operands.

Tolerances, element by element; a bf16 rounding is off by at most 2^-8 of the value, and the fp32 steps in front of it (scores of dh
products, an exponential, sums over the keys) are kept together as `slack`, relative to a probability:
  out   each probability is rounded once, the result once:       (2^-8 + slack) sum p |v| + 2^-8 |out|
  dv    the same over the rows:                                  (2^-8 + slack) sum p |do| + 2^-8 |dv|
  dq    ds = p (dp - D), rounded once; D = rowsum(do o) with the o given, rounded when it was written, so off by 2^-8 sum |do o|, and dp
        by fp32 alone: per element of ds (2^-8 + slack) |ds| + p (2^-8 sum |do o| + slack sum |do| |v|), through |k|, then 2^-8 |dq|
  dk    the same through |q|
"""
import math

import pytest
import torch

from paper_2401_01728_amd import kernels

pytestmark = pytest.mark.gpu


def _inputs(seed, B, Sq, Sk, H, Hkv, dh, klen):
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn(B, Sq, H * dh, generator=g) * 1.3).to(torch.bfloat16)
    kv = torch.randn(B, Sk, 2 * Hkv * dh, generator=g).to(torch.bfloat16)
    do = (torch.randn(B, Sq, H * dh, generator=g) * 0.02).to(torch.bfloat16)
    n = [Sk] * B if klen is None else [max(0, min(Sk, x)) for x in klen]
    for b in range(B):
        kv[b, n[b]:] = float("nan")
    return q, kv[..., :Hkv * dh], kv[..., Hkv * dh:], do, n


def _reference(q, k, v, do, n, H, Hkv, o_given=None):
    B, Sq, _ = q.shape
    Sk = k.shape[1]
    dh = q.shape[2] // H
    f64 = dict(dtype=torch.float64, device=q.device)
    out, lse2 = torch.zeros(q.shape, **f64), torch.full((B, H, Sq), -math.inf, **f64)
    dq, dk, dv = torch.zeros(q.shape, **f64), torch.zeros(k.shape, **f64), torch.zeros(k.shape, **f64)
    e_out, e_dq, e_dk, e_dv = (torch.zeros_like(t) for t in (out, dq, dk, dv))
    for b in range(B):
        if n[b] == 0:
            continue
        for h in range(H):
            c, kc = slice(h * dh, (h + 1) * dh), slice(h // (H // Hkv) * dh, (h // (H // Hkv) + 1) * dh)
            qh, kh, vh, doh = q[b, :, c].double(), k[b, :n[b], kc].double(), v[b, :n[b], kc].double(), do[b, :, c].double()
            s = qh @ kh.T / math.sqrt(dh)
            lse = torch.logsumexp(s, 1, keepdim=True)
            p = torch.exp(s - lse)
            out[b, :, c], lse2[b, h] = p @ vh, lse[:, 0] / math.log(2.0)
            slack = (dh + 8) * 2.0 ** -24 * float((qh.abs() @ kh.abs().T).max()) / math.sqrt(dh) * 2 + (n[b] / 32 + 64) * 2.0 ** -24
            r = 2.0 ** -8 + slack
            e_out[b, :, c] = r * (p @ vh.abs()) + 2.0 ** -8 * out[b, :, c].abs()
            dp = doh @ vh.T
            D = (doh * out[b, :, c]).sum(1, keepdim=True)
            ds = p * (dp - D)
            e_ds = r * ds.abs() + p * (2.0 ** -8 * (doh * out[b, :, c]).abs().sum(1, keepdim=True) + slack * (doh.abs() @ vh.abs().T))
            dq[b, :, c] = ds @ kh / math.sqrt(dh)
            e_dq[b, :, c] = e_ds @ kh.abs() / math.sqrt(dh) + 2.0 ** -8 * dq[b, :, c].abs()
            dk[b, :n[b], kc] += ds.T @ qh / math.sqrt(dh)
            e_dk[b, :n[b], kc] += e_ds.T @ qh.abs() / math.sqrt(dh)
            dv[b, :n[b], kc] += p.T @ doh
            e_dv[b, :n[b], kc] += r * (p.T @ doh.abs())
    e_dk += 2.0 ** -8 * dk.abs()
    e_dv += 2.0 ** -8 * dv.abs()
    # second order: a rounding of what is already off
    return (out, lse2, dq, dk, dv), tuple(e * (1 + 2.0 ** -7) + 1e-30 for e in (e_out, e_dq, e_dk, e_dv))


def _near(got, ref, bound):
    got = got.to(ref.device).double()
    assert bool(torch.isfinite(got).all())
    over = (got - ref).abs() / bound
    assert bool((over <= 1.0).all()), "off by %.3g of the bound at %s" % (float(over.max()), int(over.argmax()))


def _check(B, Sq, Sk, H, Hkv, dh, klen, seed=0):
    q, k, v, do, n = _inputs(seed, B, Sq, Sk, H, Hkv, dh, klen)
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(q, k, v, do, n, H, Hkv)
    # k and v stay columns of one matrix
    kv = torch.cat([k, v], -1).cuda()
    kd, vd = kv[..., :Hkv * dh], kv[..., Hkv * dh:]
    length = torch.tensor(klen, dtype=torch.int32).cuda() if klen is not None else None
    got_out, got_lse = kernels.cross_attention_fwd(q.cuda(), kd, vd, H, Hkv, length)
    _near(got_out, out, e_out)
    got_lse = got_lse.cpu().double()
    assert torch.equal(got_lse == -math.inf, lse2 == -math.inf)
    there = lse2 != -math.inf
    assert float((got_lse - lse2)[there].abs().max() if there.any() else 0.0) <= 2.0 ** -12
    got = kernels.cross_attention_bwd(q.cuda(), kd, vd, got_out, do.cuda(), got_lse.float().cuda(), H, Hkv, length)
    for a, ref, bound in zip(got, (dq, dk, dv), (e_dq, e_dk, e_dv)):
        _near(a, ref, bound)


# single tokens and few rows (one wave's worth and one more), lengths around a tile of 32 and 64 and a workgroup's 128, long walks that are cut
# into parts on either side, shared heads, both widths of a head
@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh", [
    (1, 1, 1, 1, 1, 64), (1, 1, 1, 1, 1, 128), (2, 1, 31, 2, 1, 64), (1, 1, 33, 8, 1, 128), (3, 1, 700, 4, 4, 64), (1, 4, 1000, 8, 1, 128),
    (1, 1, 5000, 3, 3, 128), (2, 3, 65, 33, 3, 64), (1, 2, 97, 32, 2, 64), (1, 33, 64, 1, 1, 64), (2, 32, 63, 1, 1, 128), (1, 63, 129, 2, 2, 64),
    (2, 65, 31, 2, 1, 128), (1, 128, 128, 1, 1, 64), (1, 129, 257, 3, 1, 128), (2, 200, 1, 2, 2, 64), (1, 40, 1500, 6, 2, 64), (1, 300, 77, 12, 12, 64),
    (1, 1030, 70, 2, 2, 128), (1, 7, 400, 20, 4, 128), (8, 70, 200, 16, 16, 64)])
def test_forward_and_backward(B, Sq, Sk, H, Hkv, dh):
    _check(B, Sq, Sk, H, Hkv, dh, None)


@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh,klen", [
    (3, 1, 200, 4, 2, 64, [200, 0, 65]), (4, 1, 130, 4, 1, 128, [1, 130, 0, 64]), (4, 70, 130, 2, 1, 64, [0, 63, 64, 129]),
    (3, 150, 300, 4, 2, 128, [1, 257, 300]), (2, 40, 90, 3, 3, 64, [0, 0]), (3, 33, 100, 2, 2, 128, [-5, 1000, 32]), (2, 20, 2000, 2, 2, 64, [1999, 3])])
def test_lengths(B, Sq, Sk, H, Hkv, dh, klen):
    """Sequences of their own lengths, none among them; what lies behind is not a number."""
    _check(B, Sq, Sk, H, Hkv, dh, klen, seed=1)


# grids of many workgroups: eight waves to one in the backward of heads of 128; parts on both sides; rows and keys that end inside all blocks
@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh,klen", [
    (8, 700, 700, 32, 32, 128, None), (9, 333, 1001, 40, 20, 128, [1001, 0, 1, 63, 500, 1000, 777, 64, 65]), (4, 513, 1030, 24, 12, 64, [1030, 1, 700, 0])])
def test_many_workgroups(B, Sq, Sk, H, Hkv, dh, klen):
    q, k, v, do, n = _inputs(6, B, Sq, Sk, H, Hkv, dh, klen)
    q, k, v, do = q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), do.cuda()
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(q, k, v, do, n, H, Hkv)
    length = torch.tensor(klen, dtype=torch.int32).cuda() if klen is not None else None
    got_out, got_lse = kernels.cross_attention_fwd(q, k, v, H, Hkv, length)
    _near(got_out, out, e_out)
    for a, ref, bound in zip(kernels.cross_attention_bwd(q, k, v, got_out, do, got_lse, H, Hkv, length), (dq, dk, dv), (e_dq, e_dk, e_dv)):
        _near(a, ref, bound)


def test_same_bits_every_time():
    q, k, v, do, _ = _inputs(7, 3, 300, 500, 8, 4, 128, None)
    q, k, v, do = q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), do.cuda()
    length = torch.tensor([500, 123, 311], dtype=torch.int32).cuda()
    ref = None
    for _ in range(4):
        o = kernels.cross_attention_fwd(q, k, v, 8, 4, length)
        got = (*o, *kernels.cross_attention_bwd(q, k, v, o[0], do, o[1], 8, 4, length))
        if ref is not None:
            for a, b in zip(got, ref):
                assert torch.equal(a, b)
        ref = got


def test_strides_and_what_lies_beside():
    B, Sq, Sk, H, Hkv, dh = 2, 70, 100, 4, 2, 64
    q, k, v, do, _ = _inputs(2, B, Sq, Sk, H, Hkv, dh, None)
    length = torch.tensor([100, 37], dtype=torch.int32).cuda()
    ref = kernels.cross_attention_fwd(q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), H, Hkv, length)
    grads = kernels.cross_attention_bwd(q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), ref[0], do.cuda(), ref[1], H, Hkv, length)

    def within(t, extra, fill):
        w = torch.full((*t.shape[:2], t.shape[2] + extra), fill, dtype=torch.bfloat16, device="cuda")
        w[..., 8:8 + t.shape[2]] = t.cuda()
        return w, w[..., 8:8 + t.shape[2]]

    nan = float("nan")
    qs, ks, vs, dos = (within(t, e, nan)[1] for t, e in ((q, 24), (k, 16), (v, 40), (do, 8)))
    wide, out = within(torch.zeros_like(q), 32, 5.0)
    got = kernels.cross_attention_fwd(qs, ks, vs, H, Hkv, length, out=out)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    assert bool((wide[..., :8] == 5.0).all()) and bool((wide[..., 8 + H * dh:] == 5.0).all())
    wides = [within(torch.zeros_like(t), 16, 5.0) for t in (q, k, v)]
    got = kernels.cross_attention_bwd(qs, ks, vs, out, dos, ref[1], H, Hkv, length, *(t for _, t in wides))
    for a, b, (w, t) in zip(got, grads, wides):
        assert a is t and torch.equal(a, b)
        assert bool((w[..., :8] == 5.0).all()) and bool((w[..., -8:] == 5.0).all())


def test_scores_without_bounds():
    """Scores of thousands: the running maximum moves late and far; a key that nobody else comes near takes all."""
    B, Sq, Sk, H, dh = 1, 50, 500, 2, 64
    q, k, v, do, n = _inputs(3, B, Sq, Sk, H, H, dh, None)
    k = k.clone()
    k[:, 411] *= 600.0
    k[:, 70] *= 100.0
    (out, _, _, _, _), _ = _reference(q, k, v, do, n, H, H)
    got, lse2 = kernels.cross_attention_fwd(q.cuda(), k.cuda(), v.cuda().contiguous(), H, H)
    # a probability next to another may be off by the error of a score of thousands: (dh + 8) 2^-24 sum |q k| / sqrt(dh)
    err = (dh + 8) * 2.0 ** -24 * float((q.double().abs().max() ** 2 * 0 + (q[0].double().abs() @ k[0].double().abs().T).max())) / math.sqrt(dh)
    assert float((got.cpu().double() - out).abs().max()) <= (2.0 ** -7 + 2 * err) * float(v.double().abs().max())
    assert bool(torch.isfinite(lse2).all())


def test_gradient_against_differences():
    B, Sq, Sk, H, Hkv, dh = 1, 10, 70, 2, 1, 64
    q, k, v, do, n = _inputs(4, B, Sq, Sk, H, Hkv, dh, [50])
    length = torch.tensor([50], dtype=torch.int32).cuda()
    out, lse2 = kernels.cross_attention_fwd(q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), H, Hkv, length)
    grads = kernels.cross_attention_bwd(q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), out, do.cuda(), lse2, H, Hkv, length)

    def total(t):
        o = torch.cat([torch.softmax(t[0][0, :, h * dh:(h + 1) * dh] @ t[1][0, :50].T / math.sqrt(dh), -1) @ t[2][0, :50] for h in range(H)], -1)
        return float((o * do[0].double()).sum())

    base = [q.double(), k.double(), v.double()]
    g = torch.Generator().manual_seed(8)
    for i, grad in enumerate(grads):
        u = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        if i:
            u[:, 50:] = 0.0
        plus, minus = ([t + e * u if x == i else t for x, t in enumerate(base)] for e in (1e-5, -1e-5))
        plus, minus = ([torch.nan_to_num(t) for t in s] for s in (plus, minus))
        num = (total(plus) - total(minus)) / 2e-5
        terms = grad.cpu().double() * u
        assert abs(float(terms.sum()) - num) <= 2.0 ** -6 * float(terms.abs().sum())


def test_other_stream_and_captured_graph():
    B, Sq, Sk, H, Hkv, dh = 2, 40, 900, 4, 2, 64
    q, k, v, do, _ = _inputs(5, B, Sq, Sk, H, Hkv, dh, None)
    q, k, v, do = q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), do.cuda()
    length = torch.tensor([900, 411], dtype=torch.int32).cuda()
    both = lambda st=None: (lambda o: (*o, *kernels.cross_attention_bwd(q, k, v, o[0], do, o[1], H, Hkv, length, stream=st)))(  # noqa: E731
        kernels.cross_attention_fwd(q, k, v, H, Hkv, length, stream=st))
    ref = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(side)
    side.synchronize()
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
        token = kernels.cross_attention_fwd(q[:, :1].contiguous(), k, v, H, Hkv, length)
    for seed in range(4):
        for t, fresh in zip((q, k, v, do), _inputs(30 + seed, B, Sq, Sk, H, Hkv, dh, None)):
            t.copy_(fresh)
        length.copy_(torch.tensor([900 - seed, 64 * seed], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*got, *token), (*both(), *kernels.cross_attention_fwd(q[:, :1].contiguous(), k, v, H, Hkv, length))):
            assert torch.equal(a, b)


@pytest.mark.parametrize("Sq,dh", [(1, 64), (80, 128)])
def test_offsets_behind_32_bits(Sq, dh):
    """Keys and values as columns of a cache of 6 G elements, tokens 2^24 elements apart: bit for bit what matrices without gaps give, and near 64 bits."""
    B, Sk, H, Hkv = 2, 200000, 4, 2
    q, k, v, do, n = _inputs(9, B, Sq, Sk, H, Hkv, dh, [Sk, Sk - 70])
    q, k, v, do = q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), do.cuda()
    length = torch.tensor(n, dtype=torch.int32).cuda()

    def apart(t, ld, at=0):
        w = torch.empty(*t.shape[:2], ld, dtype=torch.bfloat16, device="cuda")[..., at:at + t.shape[2]]
        w.copy_(t)
        return w

    ref = kernels.cross_attention_fwd(q, k, v, H, Hkv, length)
    grads = kernels.cross_attention_bwd(q, k, v, ref[0], do, ref[1], H, Hkv, length)
    kw, vw, qw, dow, out = apart(k, 16384), apart(v, 16384, 16000), apart(q, 1 << 24), apart(do, 1 << 24), apart(torch.zeros_like(q), 1 << 24)
    got = kernels.cross_attention_fwd(qw, kw, vw, H, Hkv, length, out=out)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    both = torch.empty(B, Sk, 16384, dtype=torch.bfloat16, device="cuda")
    got = kernels.cross_attention_bwd(qw, kw, vw, out, dow, ref[1], H, Hkv, length, apart(torch.zeros_like(q), 1 << 24), both[..., 8:8 + Hkv * dh],
                                      both[..., 16384 - Hkv * dh:])
    for a, b in zip(got, grads):
        assert torch.equal(a, b)
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(q, k, v, do, n, H, Hkv)
    _near(ref[0], out, e_out)
    assert float((ref[1].double() - lse2).abs().max()) <= 2.0 ** -10
    for a, r, bound in zip(grads, (dq, dk, dv), (e_dq, e_dk, e_dv)):
        _near(a, r, bound)


def test_two_calls_at_once():
    """A long backward beside single tokens on another stream."""
    q, k, v, do, _ = _inputs(11, 4, 600, 1500, 8, 4, 128, None)
    q, k, v, do = q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), do.cuda()
    one = q[:, :1].contiguous()
    length = torch.tensor([1500, 0, 77, 1024], dtype=torch.int32).cuda()
    ref = kernels.cross_attention_fwd(q, k, v, 8, 4, length)
    grads, token = kernels.cross_attention_bwd(q, k, v, ref[0], do, ref[1], 8, 4, length), kernels.cross_attention_fwd(one, k, v, 8, 4, length)
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        got.append((kernels.cross_attention_bwd(q, k, v, ref[0], do, ref[1], 8, 4, length, stream=first),
                    kernels.cross_attention_fwd(one, k, v, 8, 4, length, stream=second)))
    torch.cuda.synchronize()
    for a, b in got:
        for x, y in zip((*a, *b), (*grads, *token)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("B,Sq,Sk,dh,klen", [(2, 20, 1, 128, None), (1, 300, 1, 64, None), (3, 40, 2000, 64, [1, 2000, 1]), (2, 1000, 70, 128, [1, 1])])
def test_one_key(B, Sq, Sk, dh, klen):
    """Its probability is 1 whatever the score: dq and dk are exactly zero."""
    q, k, v, do, n = _inputs(13, B, Sq, Sk, 4, 2, dh, klen)
    q, k, v, do = q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), do.cuda()
    q[0, 3] = float("nan")
    length = torch.tensor(klen, dtype=torch.int32).cuda() if klen is not None else None
    out, lse2 = kernels.cross_attention_fwd(q, k, v, 4, 2, length)
    dq, dk, dv = kernels.cross_attention_bwd(q, k, v, out, do, lse2, 4, 2, length)
    rows = torch.ones(B, Sq, dtype=torch.bool)
    rows[0, 3] = False
    for b in range(B):
        if n[b] == 1:
            assert not dq[b][rows[b].cuda()].any()
            assert not dk[b, 1:].any()
            if b:
                assert not dk[b].any()
    assert bool(torch.isnan(dq[0, 3]).all()) and bool(torch.isnan(dk[0, 0]).all())
    assert bool(torch.isfinite(dv[1:]).all())


def _near_where_finite(got, ref, bound):
    got = got.to(ref.device).double()
    there = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), there)
    assert bool(((got - ref).abs() <= bound)[there].all())


def _run(q, k, v, do, H, Hkv, klen):
    q, k, v, do = q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), do.cuda()
    length = torch.tensor(klen, dtype=torch.int32).cuda() if klen is not None else None
    out, lse2 = kernels.cross_attention_fwd(q, k, v, H, Hkv, length)
    return (out, lse2) + kernels.cross_attention_bwd(q, k, v, out, do, lse2, H, Hkv, length)


# single tokens in one walk and in parts; few and many rows, in parts and not; both widths of a head
INFINITE = [(2, 1, 40, 4, 2, 64), (2, 1, 40, 4, 2, 128), (2, 1, 3000, 4, 2, 64), (2, 2, 3000, 4, 2, 128), (2, 50, 200, 4, 2, 64), (2, 50, 200, 4, 2, 128),
            (2, 70, 3000, 4, 2, 64), (2, 300, 1500, 4, 2, 128)]


@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh", INFINITE)
@pytest.mark.parametrize("at", ["first", "middle", "last"])
def test_a_key_of_scores_of_minus_infinity(B, Sq, Sk, H, Hkv, dh, at):
    """Every score of one key of the first head is -inf: what is finite is what it is without that key."""
    klen = [Sk - 3, Sk]
    q, k, v, do, n = _inputs(21, B, Sq, Sk, H, Hkv, dh, klen)
    j, share = {"first": 0, "middle": n[0] // 2, "last": n[0] - 1}[at], H // Hkv
    q, k = q.clone(), k.clone()
    for h in range(share):
        q[0, :, h * dh + 5] = q[0, :, h * dh + 5].abs() + 0.125
    others = [x for x in range(Sk) if x != j]
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(q[:1], k[:1, others], v[:1, others], do[:1], [n[0] - 1], H, Hkv)
    k[0, j, 5] = -math.inf
    got_out, got_lse, got_dq, got_dk, got_dv = _run(q, k, v, do, H, Hkv, klen)
    first = slice(0, share * dh)                         # (the other heads have that key)
    _near_where_finite(got_out[:1, :, first], out[..., first], e_out[..., first])
    assert float((got_lse[:1, :share].cpu().double() - lse2[:, :share]).abs().max()) <= 2.0 ** -12
    for h in range(share):
        dq[..., h * dh + 5] = math.nan                  # 0 times -inf
    _near_where_finite(got_dq[:1, :, first], dq[..., first], e_dq[..., first])
    for got, ref, bound in ((got_dk, dk, e_dk), (got_dv, dv, e_dv)):
        _near_where_finite(got[:1, others, :dh], ref[..., :dh], bound[..., :dh])
        assert not got[0, j, :dh].any()


@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh", INFINITE)
def test_a_row_of_scores_of_minus_infinity(B, Sq, Sk, H, Hkv, dh):
    """It has no softmax: NaN, for itself and, in the backward, for the keys it shares with others; other rows, heads and sequences are what they were."""
    klen = [Sk - 3, Sk]
    q, k, v, do, n = _inputs(22, B, Sq, Sk, H, Hkv, dh, klen)
    q, k = q.clone(), k.clone()
    k[0, :, 5] = -k[0, :, 5].abs() - 0.125
    r = Sq // 2
    q[0, r, 5] = 0.0
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(q, k, v, do, n, H, Hkv)
    q[0, r, 5] = math.inf
    got_out, got_lse, got_dq, got_dk, got_dv = _run(q, k, v, do, H, Hkv, klen)
    out[0, r, :dh], lse2[0, 0, r], dq[0, r, :dh] = math.nan, math.nan, math.nan
    for t in (dk, dv):
        t[0, :n[0], :dh] = math.nan
    _near_where_finite(got_out, out, e_out)
    _near_where_finite(got_lse, lse2, torch.full_like(lse2, 2.0 ** -12))
    for got, ref, bound in ((got_dq, dq, e_dq), (got_dk, dk, e_dk), (got_dv, dv, e_dv)):
        _near_where_finite(got, ref, bound)
    assert bool(torch.isnan(got_out[0, r, :dh]).all()) and bool(torch.isnan(got_lse[0, 0, r])) and bool(torch.isnan(got_dq[0, r, :dh]).all())


@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh", INFINITE)
def test_an_infinite_value(B, Sq, Sk, H, Hkv, dh):
    """Its column is not finite, for all rows of its heads; the others are what they were."""
    klen = [Sk - 3, Sk]
    q, k, v, do, n = _inputs(23, B, Sq, Sk, H, Hkv, dh, klen)
    v = v.clone()
    j = n[0] - 1
    # (not so far behind that its probability is zero in fp32)
    (out, lse2, _, _, _), (e_out, _, _, _) = _reference(q, k, v, do, n, H, Hkv)
    v[0, j, dh + 9] = math.inf
    got, got_lse = _run(q, k, v, do, H, Hkv, klen)[:2]
    for h in range(H // Hkv, 2 * (H // Hkv)):
        out[0, :, h * dh + 9] = math.inf
    _near_where_finite(got, out, e_out)
    assert float((got_lse.cpu().double() - lse2).abs().max()) <= 2.0 ** -12


@pytest.mark.parametrize("lengths", [False, True])
def test_more_sequences_than_a_launch_takes(lengths):
    """2^20 sequences of one key and 16 heads are 2^32 threads and more.  A probability of 1 makes out the values, dv the output's gradient, dq and dk
    zero, bit for bit; a score is off by (dh + 8) 2^-24 of its products' absolute sum, and by two roundings more in base 2."""
    B, H, dh = 1 << 20, 16, 64
    g = torch.Generator(device="cuda").manual_seed(24)
    q, k, v, do = (torch.randn(B, 1, H * dh, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    n = torch.randint(0, 2, (B,), generator=g, device="cuda", dtype=torch.int32) if lengths else None
    out, lse2 = kernels.cross_attention_fwd(q, k, v, H, H, n)
    dq, dk, dv = kernels.cross_attention_bwd(q, k, v, out, do, lse2, H, H, n)
    step = 1 << 16
    for b in range(0, B, step):
        part = slice(b, b + step)
        here = torch.ones(step, dtype=torch.bool, device="cuda") if n is None else n[part] > 0
        keep = here[:, None, None]
        assert torch.equal(out[part], torch.where(keep, v[part], 0.0)), b
        assert torch.equal(dv[part], torch.where(keep, do[part], 0.0)), b
        assert not dq[part].any() and not dk[part].any(), b
        x = (q[part].double() * k[part].double()).view(step, H, dh)
        c2 = math.log2(math.e) / math.sqrt(dh)
        ref, off = x.sum(-1) * c2, x.abs().sum(-1) * c2 * (dh + 8) * 2.0 ** -24 + 2.0 ** -22
        got = lse2[part, :, 0].double()
        assert bool(((got - ref).abs() <= off)[here].all()) and bool((got[~here] == -math.inf).all()), b


@pytest.mark.parametrize("B,Sq,Sk,H,Hkv,dh,klen", [
    (1, 50, 500, 2, 2, 64, None), (2, 1, 700, 4, 1, 128, [700, 412]), (2, 150, 900, 4, 2, 64, [500, 900]), (1, 300, 600, 4, 4, 128, None), (2, 64, 2000, 2, 1, 128, [2000, 413])])
def test_gradients_of_scores_without_bounds(B, Sq, Sk, H, Hkv, dh, klen):
    """Scores of thousands, where the backward's accumulators begin with as much of the other sign.  The bounds are those of ordinary scores: `slack` has
    (dh + 8) 2^-24 of the largest sum of a score's absolute products, twice - of the score in the forward's lse and in the backward - which the
    rounding of lse / c2 and of what begins with it, two of the sums' own, are inside."""
    q, k, v, do, n = _inputs(25, B, Sq, Sk, H, Hkv, dh, klen)
    k = k.clone()
    k[:, 411] *= 400.0
    k[:, 70] *= 100.0
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(q, k, v, do, n, H, Hkv)
    got = _run(q, k, v, do, H, Hkv, klen)
    for a, ref, bound in zip(got[:1] + got[2:], (out, dq, dk, dv), (e_out, e_dq, e_dk, e_dv)):
        _near(a, ref, bound)
    assert float(lse2.abs().max()) > 300.0
    qh, kh = q.double().view(B, Sq, H, dh).transpose(1, 2), k.double().nan_to_num().reshape(B, Sk, Hkv, dh).transpose(1, 2).repeat_interleave(H // Hkv, 1)
    off = (dh + 8) * 2.0 ** -24 * float((qh.abs() @ kh.abs().transpose(-1, -2)).max()) * math.log2(math.e) / math.sqrt(dh)
    assert float((got[1].cpu().double() - lse2).abs().max()) <= 2.0 ** -12 + off


# eight waves to a workgroup of the backward of heads of 128 (2400 of them and more; 1536 are enough): lengths that end everywhere, none, shared heads, rows that
# end inside a wave's
@pytest.mark.parametrize("Sq,Sk,H,Hkv", [(300, 1200, 32, 16), (777, 600, 24, 24), (90, 700, 160, 20)])
def test_eight_waves_over_lengths(Sq, Sk, H, Hkv):
    klen = [Sk, 0, 1, 63, 64, 65, 127, 128, 129, 255, 256, 257, Sk - 1, Sk // 2, 31, 32, 33, 2, Sk - 255, 511]
    B, dh = len(klen), 128
    share = H // Hkv
    assert share * Sq > 128 and B * Hkv * (-(-Sk // 256) + -(-share * Sq // 256)) >= 2400
    q, k, v, do, n = _inputs(26, B, Sq, Sk, H, Hkv, dh, klen)
    q, k, v, do = q.cuda(), k.cuda().contiguous(), v.cuda().contiguous(), do.cuda()
    (out, lse2, dq, dk, dv), (e_out, e_dq, e_dk, e_dv) = _reference(q, k, v, do, n, H, Hkv)
    got = _run(q, k, v, do, H, Hkv, klen)
    for a, ref, bound in zip(got[:1] + got[2:], (out, dq, dk, dv), (e_out, e_dq, e_dk, e_dv)):
        _near(a, ref, bound)
