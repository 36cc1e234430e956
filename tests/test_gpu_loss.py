"""The loss at a chain's end and its gradients against the definition in 64 bits on the same bf16 operands.

Tolerances, element by element, from the roundings that the kernels make (a bf16 rounding is off by at most 2^-8 of the value):
  logits    fp32 accumulation of d products: (d + 8) 2^-24 sum |x w| at most
  loss, lse that of the logits, and a softmax sum of exp2 (2 ulp) in up to 64 + V / 64 additions of a chain, and their log
  dx, dw    the exponential is rounded to fp16 (2^-11, and 2^-40 of a row's weight where it is subnormal), dz to bf16 (2^-8), together below
            2^-8 + 2^-10, and an error of the logits, of the lse and of an exponential, `slack`, moves dz by a factor of
            exp(slack) < 1 + 2 slack; through a product of absolute values; then the result's own rounding.  The label's column has p - 1
            from fp32: its error is that of z, absolute.
"""
import math

import numpy as np
import pytest
import torch

import paper_2401_01728_amd as rv

pytestmark = pytest.mark.gpu


def _inputs(seed, T, d, V, out=0.0, sure=6.0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(V, d, generator=g) * 0.05
    label = torch.randint(0, V, (T,), generator=g)
    x = torch.randn(T, d, generator=g) + torch.rand(T, 1, generator=g) * sure / (0.05 * d) * (w[label] / 0.05)
    gone = torch.randperm(T, generator=g)[:int(T * out)]
    label[gone] = torch.tensor([-1, V, -100, 1 << 40])[torch.arange(len(gone)) % 4]
    x = x.to(torch.bfloat16)
    x[gone] = float("nan")
    return x, w.to(torch.bfloat16), label, w


def _reference(x, w, label, g):
    """loss, lse, dz [T, V], and the bound of the logits' error, in 64 bits (where the operands are); rows out of the batch are zero"""
    T, d = x.shape
    V = w.shape[0]
    takes = (label >= 0) & (label < V)
    x64, w64 = torch.where(takes[:, None], x.double(), 0.0), w.double()
    z = x64 @ w64.T
    lse = torch.logsumexp(z, 1)
    y = torch.where(takes, label, 0)
    at = z.gather(1, y[:, None])[:, 0]
    p = torch.exp(z - lse[:, None])
    hot = torch.zeros_like(z)
    hot.scatter_(1, y[:, None], 1.0)
    gt = torch.where(takes, g.double(), 0.0)[:, None]
    dz = (p - hot) * gt
    zerr = (d + 8) * 2.0 ** -24 * float((x64.abs() @ w64.abs().T).max())
    zero = torch.zeros_like(lse)
    return torch.where(takes, lse - at, zero), torch.where(takes, lse, zero), dz, zerr, x64, w64, y, takes


def _check(x, w, label, g, got_loss, got_lse, dx=None, dw=None, master=None, eta=0.0, new=None, version=None):
    loss, lse, dz, zerr, x64, w64, y, takes = _reference(x, w, label, g)
    V, here = w.shape[0], x.device
    slack = 2 * zerr + (80 + V / 64) * 2.0 ** -24 + 2.0 ** -22 * float(lse.abs().max())
    for got, ref in ((got_loss, loss), (got_lse, lse)):
        if got is not None:
            assert float((got.to(here).double() - ref).abs().max()) <= slack
    # what dz may be off by: relative, but absolute (times the row's weight) at the label
    weight = torch.where(takes, g.double().abs(), 0.0)[:, None]
    off = dz.abs() * (2.0 ** -8 + 2.0 ** -10 + 2 * slack) + weight * 2.0 ** -40
    rows = torch.arange(len(y), device=here)
    off[rows, y] = dz[rows, y].abs() * 2.0 ** -8 + torch.where(takes, g.double().abs(), 0.0) * slack
    fp32 = 2.0 ** -24 * (x.shape[0] + V)      # accumulation of the products of dz, relative to the sums of absolute values
    if dx is not None:
        ref = dz @ w64
        bound = (off + dz.abs() * fp32) @ w64.abs()
        assert bool(((dx.to(here).double() - ref).abs() <= bound * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs() + 1e-38).all())
        assert not dx.to(here)[~takes].any()
    ref = dz.T @ x64
    bound = (off + dz.abs() * fp32).T @ x64.abs()
    if dw is not None:
        assert bool(((dw.to(here).double() - ref).abs() <= bound * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs() + 1e-38).all())
    if new is not None:
        want = master.to(here).double() - eta * ref
        assert bool(((new.to(here).double() - want).abs() <= eta * bound + 2.0 ** -23 * (want.abs() + eta * ref.abs())).all())
        assert torch.equal(version, new.to(torch.bfloat16))


# one row, one token of vocabulary, less than a strip, ends inside a strip and a tile, more than one tile each way, rows that end inside
# a tile of 32, widths of one and of several tiles; few and many rows
SIZES = [(1, 64, 1), (1, 64, 5), (2, 128, 33), (3, 128, 63), (31, 64, 64), (33, 192, 65), (65, 64, 1000), (130, 448, 257), (257, 128, 2049),
         (300, 320, 4097), (129, 192, 513), (513, 256, 1031), (96, 1024, 5000), (700, 1600, 777)]


@pytest.mark.parametrize("T,d,V", SIZES)
@pytest.mark.parametrize("out", [0.0, 0.4])
def test_loss_and_gradients(T, d, V, out):
    x, w, label, _ = _inputs(T + d + V, T, d, V, out)
    g = torch.full((T,), 1.0 / T)
    loss, lse = rv.loss_forward(x.cuda(), w.cuda(), label.cuda())
    _check(x, w, label, g, loss, lse)
    loss2, dx, dw = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=1.0 / T)
    _check(x, w, label, g, loss2, None, dx, dw)


# tiles of 256 for dx (many rows of a wide state), half of the rows out; rows that a workgroup's label count walks over in more than one turn
@pytest.mark.parametrize("T,d,V,out", [(4096, 4096, 1000, 0.5), (2048, 8192, 600, 0.0), (20000, 64, 100, 0.3),
                                         (140001, 64, 40, 0.3)])
def test_many_rows(T, d, V, out):
    x, w, label, master = (t.cuda() for t in _inputs(2, T, d, V, out))
    g = torch.full((T,), 1.0, device="cuda")
    loss, dx, dw = rv.loss_step(x, w, label)
    _check(x, w, label, g, loss, None, dx, dw)
    got = rv.loss_step(x, w, label, master=master, eta=0.1)
    assert torch.equal(got[0], loss) and torch.equal(got[1], dx)
    _check(x, w, label, g, loss, None, dx, None, master, 0.1, got[2], got[3])
    # in place
    again = rv.loss_step(x, w, label, master=master, eta=0.1, master_out=master, version=w)
    for a, b in zip(again, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,d,V,rows", [(300, 128, 777, 64), (300, 320, 1031, 128), (1100, 192, 513, 512), (65, 64, 100, 1)])
@pytest.mark.parametrize("out", [0.0, 0.6])
def test_pieces_of_rows(T, d, V, rows, out):
    x, w, label, master = _inputs(7, T, d, V, out)
    g = torch.full((T,), 0.25)
    loss, lse = rv.loss_forward(x.cuda(), w.cuda(), label.cuda(), rows=rows)
    _check(x, w, label, g, loss, lse)
    loss, dx, dw = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=0.25, rows=rows)
    _check(x, w, label, g, loss, None, dx, dw)
    loss, dx, new, version = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=0.25, rows=rows, master=master.cuda(), eta=0.1)
    _check(x, w, label, g, loss, None, dx, None, master, 0.1, new, version)


@pytest.mark.parametrize("T,d,V", [(1, 64, 3), (40, 128, 130), (300, 320, 4097), (200, 1024, 16500)])
def test_update_and_row_weights(T, d, V):
    x, w, label, master = _inputs(11, T, d, V, 0.25)
    row = torch.rand(T, generator=torch.Generator().manual_seed(5)) - 0.3
    takes = (label >= 0) & (label < V)
    row[~takes] = float("nan")
    xs, ws, m = x.cuda(), w.cuda(), master.cuda()
    loss, dx, new, version = rv.loss_step(xs, ws, label.cuda(), scale=0.5, row_scale=row.cuda(), master=m, eta=0.3)
    _check(x, w, label, torch.where(takes, row, 0.0) * 0.5, loss, None, dx, None, master, 0.3, new, version)
    # in place: the same values
    loss2, dx2, m2, w2 = rv.loss_step(xs, ws, label.cuda(), scale=0.5, row_scale=row.cuda(), master=m, eta=0.3, master_out=m, version=ws, dx=xs)
    assert dx2 is xs and m2 is m and w2 is ws
    for a, b in ((loss2, loss), (dx2, dx), (m2, new), (w2, version)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,d,V", [(1, 64, 1000), (5, 192, 333), (200, 128, 700)])
def test_update_of_few_rows_is_as_exact_as_its_master(T, d, V):
    """A step as large as the weights.  Of dz the label's entry has 16 bits (two roundings to bf16, 2^-16), the others those of their
    exponential, 2^-11; `slack` (see _check) moves both."""
    x, w, label, master = _inputs(19, T, d, V, 0.2 if T > 1 else 0.0)
    _, _, new, _ = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=0.37, master=master.cuda(), eta=2.0)
    loss, lse, dz, zerr, x64, w64, y, takes = _reference(x, w, label, torch.full((T,), 0.37))
    slack = 2 * zerr + (80 + V / 64) * 2.0 ** -24 + 2.0 ** -22 * float(lse.abs().max())
    off = dz.abs() * (2.0 ** -11 + 2.0 ** -16 + 2 * slack) + 2.0 ** -40
    rows = torch.arange(T)
    off[rows, y] = dz[rows, y].abs() * 2.0 ** -16 + torch.where(takes, 0.37, 0.0) * slack
    step = dz.T @ x64
    bound = 2.0 * ((off + dz.abs() * (T + 8) * 2.0 ** -23).T @ x64.abs()) + 2.0 ** -22 * (master.double().abs() + 2.0 * step.abs())
    assert bool(((new.cpu().double() - (master.double() - 2.0 * step)).abs() <= bound).all())


def test_a_scale_is_no_bias():
    """1 / 7783 rounded to bf16 is off by 2^-9: a gradient that carried the rounding of its scale would be off by that everywhere."""
    x, w, label, _ = _inputs(21, 300, 128, 2000)
    _, dx, dw = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=1.0)
    _, dx2, dw2 = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=1.0 / 7783)
    for a, b in ((dx, dx2), (dw, dw2)):
        a, b = a.double().cpu(), b.double().cpu() * 7783
        assert abs(float((a * b).sum() / (a * a).sum()) - 1.0) < 2.0 ** -12      # (the roundings of 10^5 results, averaged)


def test_no_row_takes_part():
    T, d, V = 70, 128, 300
    x, w, label, master = _inputs(3, T, d, V, 1.0)
    loss, lse = rv.loss_forward(x.cuda(), w.cuda(), label.cuda())
    assert not loss.any() and not lse.any()
    for rows in (0, 64):
        loss, dx, dw = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), rows=rows)
        assert not loss.any() and not dx.any() and not dw.any()
        _, _, new, version = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), rows=rows, master=master.cuda(), eta=0.5)
        assert torch.equal(new, master.cuda()) and torch.equal(version, master.cuda().to(torch.bfloat16))


def test_strides_and_one_gradient_alone():
    T, d, V = 150, 192, 515
    x, w, label, _ = _inputs(4, T, d, V, 0.2)
    xs = torch.full((T, d + 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((V, d + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    dxs = torch.full((T, d + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    xs[:, 64:] = x.cuda()
    ws[:, :d] = w.cuda()
    ref = rv.loss_step(x.cuda(), w.cuda(), label.cuda())
    got = rv.loss_step(xs[:, 64:], ws[:, :d], label.cuda(), dx=dxs[:, :d])
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    assert bool((dxs[:, d:] == 7.0).all())
    only = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), want_dw=False)
    assert only[2] is None and torch.equal(only[1], ref[1])
    only = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), want_dx=False)
    assert only[1] is None and torch.equal(only[2], ref[2])


def test_large_and_infinite_values():
    """Logits of +-1e4 (their exponentials span the whole range), a column of weights that gives -inf, a row that gives NaN alone."""
    T, d, V = 40, 64, 200
    x, w, label, _ = _inputs(6, T, d, V)
    label[:] = torch.arange(T) % 100
    w[:, 1:] *= 4e4
    w[:, 0] = 0.0
    w[150, 0] = -3e38
    x[:, 0] = 1.0
    x[7] = float("nan")
    x[8, 0] = 100.0        # -3e40: -inf in fp32
    loss, lse = rv.loss_forward(x.cuda(), w.cuda(), label.cuda())
    z = x.double() @ w.double().T
    ref_lse = torch.logsumexp(z, 1)
    ref = ref_lse - z[torch.arange(T), label]
    keep = torch.arange(T) != 7
    tol = 80 * 2.0 ** -24 * float((x[keep].double()[:, 1:].abs() @ w.double()[:, 1:].abs().T).max())
    assert bool(torch.isnan(loss.cpu()[7])) and bool(torch.isnan(lse.cpu()[7]))
    assert float((loss.cpu().double() - ref)[keep].abs().max()) <= tol
    assert float((lse.cpu().double() - ref_lse)[keep].abs().max()) <= tol
    _, dx, _ = rv.loss_step(x.cuda(), w.cuda(), label.cuda())
    assert bool(torch.isfinite(dx.cpu()[keep & (torch.arange(T) != 8)].float()).all())


def test_gradient_against_differences():
    """dx . u and dw . u against central differences of the summed loss, formed in 64 bits by the definition: the directions are whole
    tensors, so the roundings of single elements average out; 2^-7 of the sum of absolute terms bounds them."""
    T, d, V = 20, 128, 90
    x, w, label, _ = _inputs(9, T, d, V, 0.2)
    _, dx, dw = rv.loss_step(x.cuda(), w.cuda(), label.cuda())
    takes = label >= 0
    takes &= label < V
    x64, w64 = torch.where(takes[:, None], x.double(), 0.0), w.double()

    def total(xx, ww):
        z = xx @ ww.T
        at = z.gather(1, torch.where(takes, label, 0)[:, None])[:, 0]
        return float(torch.where(takes, torch.logsumexp(z, 1) - at, 0.0).sum())

    g = torch.Generator().manual_seed(1)
    for which, grad in (("x", dx), ("w", dw)):
        u = torch.randn(grad.shape, generator=g, dtype=torch.float64)
        if which == "x":
            u[~takes] = 0.0
        h = 1e-5
        num = (total(x64 + h * u, w64) - total(x64 - h * u, w64)) / (2 * h) if which == "x" else (total(x64, w64 + h * u) - total(x64, w64 - h * u)) / (2 * h)
        terms = grad.cpu().double() * u
        assert abs(float(terms.sum()) - num) <= 2.0 ** -6 * float(terms.abs().sum())


def test_other_stream_and_captured_graph():
    T, d, V = 200, 128, 700
    x, w, label, master = _inputs(12, T, d, V, 0.3)
    x, w, label, master = x.cuda(), w.cuda(), label.cuda(), master.cuda()
    ref = rv.loss_step(x, w, label, master=master, eta=0.1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = rv.loss_step(x, w, label, master=master, eta=0.1, stream=side)
    side.synchronize()
    for a, b in zip(got, ref):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = rv.loss_step(x, w, label, master=master, eta=0.1)
        fwd = rv.loss_forward(x, w, label)
    for k in range(4):
        fresh, _, fresh_label, _ = _inputs(20 + k, T, d, V, 0.2 * k)
        x.copy_(fresh)
        label.copy_(fresh_label)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got + fwd, rv.loss_step(x, w, label, master=master, eta=0.1) + rv.loss_forward(x, w, label)):
            assert torch.equal(a, b)


def test_same_bits_every_time():
    x, w, label, _ = _inputs(15, 900, 512, 3001, 0.1)
    x, w, label = x.cuda(), w.cuda(), label.cuda()
    ref = rv.loss_step(x, w, label)
    for _ in range(3):
        for a, b in zip(rv.loss_step(x, w, label), ref):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T,d,V", [(3, 16384, 131071), (130, 64, (1 << 24) - 1)])
def test_offsets_behind_31_bits(T, d, V):
    """The widest weights, 4 GiB of them, and the longest vocabulary, whose exponentials of a piece of rows are 4 GiB, against 64 bits a range of
    the vocabulary at a time.  Of the additions of a softmax sum a chain has 16 + 2 in a strip, V / 4096 strips and 6 lanes, three roundings
    each: 80 + V / 1024.  Most of the weights are zero, whose products dx adds without a rounding: only the others count."""
    g = torch.Generator(device="cuda").manual_seed(21)
    w = torch.randn(V, d, generator=g, device="cuda", dtype=torch.bfloat16)
    w *= d ** -0.5
    w[4096:V // 2] = 0.0
    w[V // 2 + 4096:V - 4096] = 0.0
    x = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
    label = torch.tensor([V - 1, 0, V - 40], device="cuda").repeat(T // 3 + 1)[:T].contiguous()
    loss, dx, dw = rv.loss_step(x, w, label)
    only, lse = rv.loss_forward(x, w, label)
    step = (1 << 26) // d
    parts = [(v, min(v + step, V)) for v in range(0, V, step)]
    x64 = x.double()
    ref_lse, at, zmax = torch.full((T,), -math.inf, dtype=torch.float64, device="cuda"), torch.zeros(T, dtype=torch.float64, device="cuda"), 0.0
    for a, b in parts:
        w64 = w[a:b].double()
        z = x64 @ w64.T
        ref_lse = torch.logaddexp(ref_lse, torch.logsumexp(z, 1))
        zmax = max(zmax, float((x64.abs() @ w64.abs().T).max()))
        here = (label >= a) & (label < b)
        at[here] = z[here, label[here] - a]
    slack = 2 * (d + 8) * 2.0 ** -24 * zmax + (80 + V / 1024) * 2.0 ** -24 + 2.0 ** -22 * float(ref_lse.abs().max())
    for got, ref in ((loss, ref_lse - at), (only, ref_lse - at), (lse, ref_lse)):
        assert float((got.double() - ref).abs().max()) <= slack
    ref_dx, off_dx = torch.zeros_like(x64), torch.zeros_like(x64)
    for a, b in parts:
        w64 = w[a:b].double()
        dz = torch.exp(x64 @ w64.T - ref_lse[:, None])
        off = dz * (2.0 ** -8 + 2.0 ** -10 + 2 * slack) + 2.0 ** -40
        rows = torch.nonzero((label >= a) & (label < b))[:, 0]
        dz[rows, label[rows] - a] -= 1.0
        off[rows, label[rows] - a] = dz[rows, label[rows] - a].abs() * 2.0 ** -8 + slack
        ref_dx += dz @ w64
        off_dx += (off + dz.abs() * 2.0 ** -24 * 3 * 4096) @ w64.abs()
        ref = dz.T @ x64
        bound = (off + dz.abs() * 2.0 ** -24 * T).T @ x64.abs()
        assert bool(((dw[a:b].double() - ref).abs() <= bound * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs() + 1e-38).all()), (a, b)
    assert bool(((dx.double() - ref_dx).abs() <= off_dx * (1 + 2.0 ** -8) + 2.0 ** -8 * ref_dx.abs() + 1e-38).all())


@pytest.mark.parametrize("T,rows", [(5, 0), (200, 0), (700, 0), (700, 256)])
def test_input_gradient_over_its_input(T, rows):
    x, w, label, _ = _inputs(31, T, 256, 1500, 0.2)
    x, w, label = x.cuda(), w.cuda(), label.cuda()
    ref = rv.loss_step(x, w, label, rows=rows)
    got = rv.loss_step(x, w, label, rows=rows, dx=x)
    assert got[1] is x
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


def test_two_calls_at_once():
    cases = []
    for T, seed in ((1500, 32), (60, 33)):
        x, w, label, master = (t.cuda() for t in _inputs(seed, T, 512, 20000, 0.1))
        cases.append(dict(x=x, w=w, label=label, master=master, eta=0.1))
    ref = [rv.loss_step(**c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for i, c in enumerate(cases):
            got[i].append(rv.loss_step(**c, stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for one in got[i]:
            for a, b in zip(one, ref[i]):
                assert torch.equal(a, b)


# more tiles of 256x256 than CUs, a few left for a last round: of the logits, and of dW; the last tile row and column end in their upper half
@pytest.mark.parametrize("T,d,V", [(5200, 64, 6400), (300, 4096, 4400)])
def test_last_round_in_halves(T, d, V):
    x, w, label, master = (t.cuda() for t in _inputs(41, T, d, V))
    g = torch.full((T,), 0.5, device="cuda")
    loss, lse = rv.loss_forward(x, w, label)
    _check(x, w, label, g, loss, lse)
    loss, dx, dw = rv.loss_step(x, w, label, scale=0.5)
    _check(x, w, label, g, loss, None, dx, dw)
    loss, dx, new, version = rv.loss_step(x, w, label, scale=0.5, master=master, eta=0.1)
    _check(x, w, label, g, loss, None, dx, None, master, 0.1, new, version)
    loss, dx, dw = rv.loss_step(x, w, label, scale=0.5, rows=128)
    _check(x, w, label, g, loss, None, dx, dw)


def _exact_logits(level, T, V, d, seed):
    """Operands whose logits fp32 holds exactly, of about the size `level`: x is zero but for +-A and +-B, powers of two, and a row of w has 1 or 1/2
    against A and a whole number up to 127 against B.  Labels: a third are a row's largest logit, a third close to it, a third any."""
    g = torch.Generator().manual_seed(seed)
    A = 2.0 ** math.ceil(math.log2(level))
    B = max(2.0 ** -2, A * 2.0 ** -23)
    w = torch.randn(V, d, generator=g)
    w[:, 0] = torch.where(torch.rand(V, generator=g) < 0.5, 1.0, 0.5)
    w[:, 40] = torch.randint(-127, 128, (V,), generator=g).float()
    x = torch.zeros(T, d)
    x[:, 0] = A * (torch.randint(0, 2, (T,), generator=g) * 2 - 1)
    x[:, 40] = B * (torch.randint(0, 2, (T,), generator=g) * 2 - 1)
    x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
    z = x.double() @ w.double().T
    assert torch.equal(z.float().double(), z)
    order = torch.argsort(z, 1, descending=True)
    rank = torch.where(torch.arange(T) % 3 == 0, 0, torch.where(torch.arange(T) % 3 == 1, torch.arange(T) % 7 % V, torch.randint(0, V, (T,), generator=g)))
    return x, w, order.gather(1, rank[:, None])[:, 0], z


@pytest.mark.parametrize("level", [30.0, 1e3, 1e5, 1e6, 1.2e7, 1e8])
@pytest.mark.parametrize("T,V", [(70, 1), (70, 330), (400, 3001)])
def test_logits_of_any_size(level, T, V):
    """Where the logits are exact only the softmax is off, whatever their size.  Per row, relative to the exponential of its largest logit, `rest` the sum of the others':
      an exponential's argument, up to 16, is rounded once (2^-21, times ln 2) behind a difference of two logits that is rounded with its product by log2 e (2^-23 of it;
        what is 2^-40 or less counts as a whole), and exp2 is off by 2^-23: together below 2^-20 of the term, and the largest itself is exact;
      a sum is a chain of 16 + 2 additions in a strip and 1 + 6 joins of three roundings each, 39 at most, of which one that adds t is off by t at most;
      the log by 2^-23, top - at and the last addition by 2^-24 of themselves."""
    d = 64
    x, w, label, z = _exact_logits(level, T, V, d, 51)
    top, at = z.max(1).values, z.gather(1, label[:, None])[:, 0]
    rest = torch.exp(z - top[:, None]).sum(1) - 1.0
    loss = (top - at) + torch.log1p(rest)
    tol = rest * 2.0 ** -20 + torch.minimum(39 * 2.0 ** -24 * (1 + rest), rest) + 2.0 ** -22 * loss
    got, lse = rv.loss_forward(x.cuda(), w.cuda(), label.cuda())
    got2, dx, dw = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=0.5)
    assert torch.equal(got, got2)
    got, lse = got.cpu().double(), lse.cpu().double()
    assert bool((got >= 0).all())
    assert bool(((got - loss).abs() <= tol).all()), float(((got - loss).abs() - tol).max())
    assert bool(((lse - (top + torch.log1p(rest))).abs() <= tol + 2.0 ** -23 * (top.abs() + 16)).all())
    p = torch.exp(z - top[:, None]) / (1 + rest)[:, None]
    dz = p.clone()
    rows = torch.arange(T)
    dz[rows, label] = torch.expm1(-loss)
    # fp16 and bf16, and the sum and the factor of a strip: below 2^-10 with them; the label's entry: bf16 alone, of the loss above
    off = dz.abs() * (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -12) + 2.0 ** -40
    off[rows, label] = dz[rows, label].abs() * (2.0 ** -8 + 2.0 ** -20) + tol
    x64, w64 = x.double(), w.double()
    fp32 = 2.0 ** -24 * (T + V)
    for a, ref, bound in ((dx, dz @ w64, (off + dz.abs() * fp32) @ w64.abs()), (dw, dz.T @ x64, (off + dz.abs() * fp32).T @ x64.abs())):
        ref, bound = 0.5 * ref, 0.5 * bound
        assert bool(((a.cpu().double() - ref).abs() <= bound * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs() + 1e-38).all())


def test_losses_of_certain_tokens():
    """Logits as a model has them: no loss is negative, and where the label has all but 2^-30 of the probability the loss is below 2^-22, its gradient, too."""
    g = torch.Generator().manual_seed(52)
    T, d, V = 300, 128, 900
    w = torch.randn(V, d, generator=g)
    label = torch.randint(0, V, (T,), generator=g)
    x = torch.rand(T, 1, generator=g) * 1.2 * w[label]
    x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
    loss, dx, _ = rv.loss_step(x.cuda(), w.cuda(), label.cuda())
    z = x.double() @ w.double().T
    ref = torch.logsumexp(z, 1) - z.gather(1, label[:, None])[:, 0]
    sure = ref < 2.0 ** -30
    assert int(sure.sum()) > 100
    assert bool((loss >= 0).all())
    assert float(loss.cpu()[sure].max()) < 2.0 ** -22
    # of dz in such a row: the label's entry is the loss, all others together as much again
    assert float(dx.cpu()[sure].double().abs().max()) <= 2.0 ** -20 * float(w.double().abs().max())


@pytest.mark.parametrize("T,d,V,rows", [(200, 128, 700, 128), (129, 64, 5000, 1), (256, 1024, 3000, 128), (130, 64, 1000, 64), (200, 192, 333, 0),
                                         (140, 64, (1 << 22) + 100, 0), (3, 64, (1 << 24) - 1, 0)])
def test_update_is_as_exact_however_it_is_cut(T, d, V, rows):
    """The same bound as of few rows in one piece (test_update_of_few_rows_is_as_exact_as_its_master) where the rows are cut into pieces, by the caller or for
    a long vocabulary; the chains of the softmax sum as in test_offsets_behind_31_bits, of the pieces' sums one addition more."""
    g = torch.Generator(device="cuda").manual_seed(61)
    master = torch.randn(V, d, generator=g, device="cuda") * 0.05
    w = master.to(torch.bfloat16)
    label = torch.randint(0, V, (T,), generator=g, device="cuda")
    x = (torch.randn(T, d, generator=g, device="cuda") + torch.rand(T, 1, generator=g, device="cuda") * 6.0 / (0.05 * d) * (master[label] / 0.05)).to(torch.bfloat16)
    label[T // 2], x[T // 2] = -1, float("nan")
    loss, dx, new, version = rv.loss_step(x, w, label, scale=0.37, master=master, eta=2.0, rows=rows)
    assert torch.equal(version, new.to(torch.bfloat16))
    takes = label >= 0
    x64 = torch.where(takes[:, None], x.double(), 0.0)
    parts = [(v, min(v + (1 << 18), V)) for v in range(0, V, 1 << 18)]
    lse, zmax = torch.full((T,), -math.inf, dtype=torch.float64, device="cuda"), 0.0
    for a, b in parts:
        w64 = w[a:b].double()
        lse = torch.logaddexp(lse, torch.logsumexp(x64 @ w64.T, 1))
        zmax = max(zmax, float((x64.abs() @ w64.abs().T).max()))
    slack = 2 * (d + 8) * 2.0 ** -24 * zmax + (80 + V / 1024) * 2.0 ** -24 + 2.0 ** -22 * float(lse.abs().max())
    weight = torch.where(takes, 0.37, 0.0).double()
    ref_dx = torch.zeros_like(x64)
    for a, b in parts:
        z = x64 @ w[a:b].double().T
        dz = torch.exp(z - lse[:, None])
        rows_here = torch.nonzero((label >= a) & (label < b))[:, 0]
        off = dz * (2.0 ** -11 + 2.0 ** -16 + 2 * slack) + 2.0 ** -40
        dz[rows_here, label[rows_here] - a] -= 1.0
        off[rows_here, label[rows_here] - a] = dz[rows_here, label[rows_here] - a].abs() * 2.0 ** -16 + slack
        dz *= weight[:, None]
        off *= weight[:, None]
        step = dz.T @ x64
        bound = 2.0 * ((off + dz.abs() * (T + 8) * 2.0 ** -23).T @ x64.abs()) + 2.0 ** -22 * (master[a:b].double().abs() + 2.0 * step.abs())
        assert bool(((new[a:b].double() - (master[a:b].double() - 2.0 * step)).abs() <= bound).all()), (a, b)
        ref_dx += dz @ w[a:b].double()
    assert not dx[~takes].any() and not loss[~takes].any()
    # dx has one rounding of dz and of itself: normwise far below 2^-7 of the terms
    assert float((dx.double() - ref_dx).norm()) <= 2.0 ** -7 * float(ref_dx.norm())


@pytest.mark.parametrize("T,d,V", [(256, 128, 700), (241, 320, 1300), (97, 64, 300), (65, 192, 1000)])
def test_room_for_two_parts(T, d, V):
    """Blocks of as many rows as two parts need (192 and more), an update whose walk over them is cut and the gradient alone, whose is not."""
    x, w, label, master = _inputs(71, T, d, V, 0.2)
    g = torch.full((T,), 0.5)
    loss, dx, dw = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=0.5)
    _check(x, w, label, g, loss, None, dx, dw)
    loss, dx, new, version = rv.loss_step(x.cuda(), w.cuda(), label.cuda(), scale=0.5, master=master.cuda(), eta=0.1)
    _check(x, w, label, g, loss, None, dx, None, master, 0.1, new, version)


@pytest.mark.parametrize("T,rows", [(200, 128), (130, 1), (256, 0), (600, 256)])
def test_everything_over_its_input(T, rows):
    """dx over x, the new master over the old and the version over w, the rows in one piece and in several."""
    x, w, label, master = (t.cuda() for t in _inputs(81, T, 192, 1300, 0.2))
    ref = rv.loss_step(x, w, label, master=master, eta=0.3, rows=rows)
    got = rv.loss_step(x, w, label, master=master, eta=0.3, rows=rows, dx=x, master_out=master, version=w)
    assert got[1] is x and got[2] is master and got[3] is w
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


def test_no_row_of_a_few_takes_part():
    """A batch that is not gathered, in two pieces, and one whose second piece alone takes part."""
    T, d, V = 200, 64, 500
    x, w, label, master = (t.cuda() for t in _inputs(82, T, d, V, 1.0))
    loss, dx, new, version = rv.loss_step(x, w, label, master=master, eta=0.5, rows=128)
    assert not loss.any() and not dx.any()
    assert torch.equal(new, master) and torch.equal(version, master.to(torch.bfloat16))
    x[150:] = 1.0
    label[150:] = 7
    ref = rv.loss_step(x, w, label, master=master, eta=0.5)
    got = rv.loss_step(x, w, label, master=master, eta=0.5, rows=128)
    assert torch.equal(got[0], ref[0]) and not got[1][:150].any() and bool(got[1][150:].any())
    assert float((got[2] - ref[2]).abs().max()) <= 2.0 ** -20 * float(ref[2].abs().max())


# tiles of 256 and, where they are a last round, of 128; walks over the rows that are cut; several pieces; more labels of a tile than are looked up at a time;
# one label for all; rows that take no part
@pytest.mark.parametrize("T,d,V,rows,labels,out", [
    (257, 128, 700, 0, "any", 0.0), (300, 64, 5000, 0, "any", 0.4), (600, 192, 9000, 256, "any", 0.1), (2000, 128, 300, 0, "few", 0.0), (5000, 64, 300, 0, "one", 0.0),
    (10000, 64, 5000, 0, "any", 0.3), (10000, 64, 5000, 4500, "any", 0.0), (400, 4096, 4400, 0, "any", 0.2), (9000, 128, 600, 1024, "few", 0.0), (700, 64, 20, 0, "any", 0.0)])
def test_labels_of_an_update_have_16_bits(T, d, V, rows, labels, out):
    """Every row of x has one entry, 4, at a column that T / d rows share: logits are single products, and an element of the step has so many terms that are not zero.
    Of dz an entry of a label is off by 2^-16 (two roundings to bf16) and what the loss is (39 additions of 2^-24 and 2^-20, see
    test_logits_of_any_size), the others by 2^-8 and 2^-10 (bf16 behind fp16, with sum and factor); the weights of the rows are no powers of two."""
    g = torch.Generator(device="cuda").manual_seed(91)
    master = torch.randn(V, d, generator=g, device="cuda") * 0.5
    w = master.to(torch.bfloat16)
    x = torch.zeros(T, d, device="cuda")
    t = torch.arange(T, device="cuda")
    x[t, t * 7 % d] = 4.0
    label = {"any": torch.randint(0, V, (T,), generator=g, device="cuda"), "few": t * 5 % 3 * (V // 4) + V // 8, "one": t * 0 + 7}[labels]
    gone = torch.rand(T, generator=g, device="cuda") < out
    label, x = torch.where(gone, -1, label), torch.where(gone[:, None], math.nan, x).to(torch.bfloat16)
    weight = torch.rand(T, generator=g, device="cuda") + 0.5
    _, _, new, version = rv.loss_step(x, w, label, scale=0.5, row_scale=weight, master=master, eta=2.0, rows=rows)
    assert torch.equal(version, new.to(torch.bfloat16))
    x64 = torch.where(gone[:, None], 0.0, x.double())
    dz = torch.softmax(x64 @ w.double().T, 1)
    off = dz * (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -12) + 2.0 ** -40
    kept = torch.nonzero(~gone)[:, 0]
    dz[kept, label[kept]] -= 1.0
    off[kept, label[kept]] = dz[kept, label[kept]].abs() * 2.0 ** -16 + 39 * 2.0 ** -24 + 2.0 ** -20
    r = torch.where(gone, 0.0, weight.double())[:, None]
    dz, off = dz * r, off * r
    step = dz.T @ x64
    bound = (off + dz.abs() * (T // d + 40) * 2.0 ** -23).T @ x64.abs() + 2.0 ** -22 * (master.double().abs() + step.abs())
    assert bool(((new.double() - (master.double() - step)).abs() <= bound).all()), float(((new.double() - (master.double() - step)).abs() / bound).max())


@pytest.mark.parametrize("T", [40, 300])
def test_a_row_of_infinite_logits(T):
    """+inf among them: the row is not a number, the others are what they were; of dw, which every row is in, nothing is."""
    x, w, label, _ = (t.cuda() for t in _inputs(95, T, 128, 900))
    loss, lse = rv.loss_forward(x, w, label)
    ref = rv.loss_step(x, w, label)
    x[17, 3] = math.inf
    bad, bad_lse = rv.loss_forward(x, w, label)
    got = rv.loss_step(x, w, label)
    other = torch.arange(T, device="cuda") != 17
    for a, b in ((bad, loss), (bad_lse, lse), (got[0], ref[0]), (got[1], ref[1])):
        assert torch.equal(a[other], b[other]) and bool(torch.isnan(a[17]).all())
    assert bool(torch.isnan(got[2]).all())


@pytest.mark.parametrize("T,d,V,rows", [(300, 128, 700, 0), (300, 128, 700, 128), (2000, 64, 300, 0), (5000, 64, 70000, 256)])
def test_none_or_one_of_many_rows_takes_part(T, d, V, rows):
    """Gathered rows: none, in one piece and in several and with walks that are cut, and the last one alone."""
    x, w, label, master = (t.cuda() for t in _inputs(96, T, d, V, 1.0))
    loss, dx, dw = rv.loss_step(x, w, label, rows=rows)
    assert not loss.any() and not dx.any() and not dw.any()
    _, _, new, version = rv.loss_step(x, w, label, rows=rows, master=master, eta=0.5)
    assert torch.equal(new, master) and torch.equal(version, master.to(torch.bfloat16))
    x[T - 1], label[T - 1] = 0.5, V - 1
    g = torch.ones(T, device="cuda")
    loss, dx, new, version = rv.loss_step(x, w, label, rows=rows, master=master, eta=0.5)
    _check(x, w, label, g, loss, None, dx, None, master, 0.5, new, version)
